// Layer norm over a row of C elements, and its backward pass:
//   m = mean(x), v = mean((x - m)^2), r = 1 / sqrt(v + eps), xh = (x - m) r, y = xh w + b
//   g = dy w, dx = r (g - mean(g) - xh mean(g xh)), dw = sum over rows of dy xh, db = sum over rows of dy
//
// Both passes are bound by memory: forward reads x and writes y, backward reads x and dy and writes dx.
// So a row is read once and held in registers (in its own type) by the threads that share it, a warp or a
// block; the backward pass keeps each thread's column sums in registers over all rows that its block
// takes, and a second kernel adds up the blocks' sums (in a fixed order: the same bits every time).
#include "net.h"
#include "rows.cuh"
#include "types.cuh"

namespace ndvm {
namespace {

// A row in the registers of kRow threads, N packs of V elements each: pack j of thread t holds the
// columns (j kRow + t) V ...  kResident: blocks an SM should hold (registers a thread are cut to that).
template <typename T, int V, int N, int kRow, int kResident>
__global__ void __launch_bounds__(kBlock<kRow>, kResident) k_forward(NormArgs a, int w_f32) {
  using P = Pairs<V>;
  constexpr int H = kPairs<V>;
  __shared__ float part[2][32];
  const int t = threadIdx.x % kRow;
  const int64_t row = (int64_t)blockIdx.x * (kBlock<kRow> / kRow) + threadIdx.x / kRow;
  if (row >= a.rows) return;  // (whole groups; with a block a row, no block)
  const int cols = (int)a.cols;
  const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
  Pack<T, V> px[N];
  P sum = both(0.0f, P());
#pragma unroll
  for (int j = 0; j < N; j++) {
    const int c = (j * kRow + t) * V;
    if (c < cols) px[j] = load_pack<T, V>(x + c);
  }
#pragma unroll
  for (int j = 0; j < N; j++) {
    if ((j * kRow + t) * V >= cols) continue;
    P v[H];
    widen<T, V>(px[j], v);
#pragma unroll
    for (int e = 0; e < H; e++) sum = add(sum, v[e]);
  }
  const float mean = row_sum<kRow>(total(sum), part[0]) / (float)cols;
  const P off = both(-mean, P());
  sum = both(0.0f, P());
#pragma unroll
  for (int j = 0; j < N; j++) {
    if ((j * kRow + t) * V >= cols) continue;
    P v[H];
    widen<T, V>(px[j], v);
#pragma unroll
    for (int e = 0; e < H; e++) {
      const P d = add(v[e], off);
      sum = fma(d, d, sum);
    }
  }
  const float rstd = 1.0f / sqrtf(row_sum<kRow>(total(sum), part[1]) / (float)cols + a.eps);
  const P scale = both(rstd, P());
  T* y = static_cast<T*>(a.y) + row * a.y_stride;
#pragma unroll
  for (int j = 0; j < N; j++) {
    const int c = (j * kRow + t) * V;
    if (c >= cols) continue;
    P v[H], w[H], b[H];
    widen<T, V>(px[j], v);
    load_weight<T, V>(w, a.weight, w_f32, c, 1.0f);
    load_weight<T, V>(b, a.bias, w_f32, c, 0.0f);
#pragma unroll
    for (int e = 0; e < H; e++) narrow<T, V>(px[j], e, fma(mul(add(v[e], off), scale), w[e], b[e]));
    store_pack(y + c, px[j]);
  }
  if (t == 0 && a.stats) {
    a.stats[row] = mean;
    a.stats[a.rows + row] = rstd;
  }
}

// Rows longer than the registers of a block hold: three passes over the row, the later ones from L2.
template <typename T>
__global__ void __launch_bounds__(kLong) k_forward_long(NormArgs a, int w_f32) {
  __shared__ float part[2][32];
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
  float s = 0.0f;
  for (int64_t c = threadIdx.x; c < a.cols; c += kLong) s += to_f32(x[c]);
  const float mean = row_sum<kLong>(s, part[0]) / (float)a.cols;
  s = 0.0f;
  for (int64_t c = threadIdx.x; c < a.cols; c += kLong) {
    const float d = to_f32(x[c]) - mean;
    s += d * d;
  }
  const float rstd = 1.0f / sqrtf(row_sum<kLong>(s, part[1]) / (float)a.cols + a.eps);
  T* y = static_cast<T*>(a.y) + row * a.y_stride;
  for (int64_t c = threadIdx.x; c < a.cols; c += kLong) {
    float w[1], b[1];
    load_weight<T, 1>(w, a.weight, w_f32, c, 1.0f);
    load_weight<T, 1>(b, a.bias, w_f32, c, 0.0f);
    y[c] = from_f32<T>(fmaf((to_f32(x[c]) - mean) * rstd, w[0], b[0]));
  }
  if (threadIdx.x == 0 && a.stats) {
    a.stats[row] = mean;
    a.stats[a.rows + row] = rstd;
  }
}

// Backward: a group of kRow threads takes every so-manieth row; the next row's loads are in flight while
// the present one is worked on.  partial[block][0][c] = the block's sum of dy xh, [1][c] = of dy.

template <typename T, int V, int N, int kRow, int kResident>
__global__ void __launch_bounds__(kBackBlock<kRow>, kResident) k_backward(NormArgs a, int w_f32) {
  using P = Pairs<V>;
  constexpr int H = kPairs<V>, kBlockRows = kBackBlock<kRow> / kRow;
  __shared__ float2 part[2][kBlockRows][kRow > 32 ? kRow / 32 : 1];
  const int t = threadIdx.x % kRow, group = threadIdx.x / kRow, cols = (int)a.cols;
  const float inv = 1.0f / (float)cols;
  P dw[N][H], db[N][H];
#pragma unroll
  for (int j = 0; j < N; j++)
#pragma unroll
    for (int e = 0; e < H; e++) dw[j][e] = db[j][e] = both(0.0f, P());
  Pack<T, V> nx[N], nd[N];
  float nmean = 0.0f, nrstd = 0.0f;
  const auto fetch = [&](int64_t row) {
    if (row >= a.rows) return;
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    const T* d = static_cast<const T*>(a.dy) + row * a.dy_stride;
    nmean = a.stats[row];
    nrstd = a.stats[a.rows + row];
#pragma unroll
    for (int j = 0; j < N; j++) {
      const int c = (j * kRow + t) * V;
      if (c < cols) {
        nx[j] = load_pack<T, V>(x + c);
        nd[j] = load_pack<T, V>(d + c);
      }
    }
  };
  const int64_t step = (int64_t)gridDim.x * kBlockRows;
  int64_t row = (int64_t)blockIdx.x * kBlockRows + group;
  fetch(row);
  for (int turn = 0; row < a.rows; row += step, turn ^= 1) {
    const float rstd = nrstd;
    const P off = both(-nmean, P()), scale = both(rstd, P());
    P xh[N][H], g[N][H], sg = both(0.0f, P()), sgx = both(0.0f, P());
#pragma unroll
    for (int j = 0; j < N; j++) {
      const int c = (j * kRow + t) * V;
      if (c >= cols) continue;
      P w[H];
      load_weight<T, V>(w, a.weight, w_f32, c, 1.0f);
      widen<T, V>(nx[j], xh[j]);
      widen<T, V>(nd[j], g[j]);
#pragma unroll
      for (int e = 0; e < H; e++) {
        xh[j][e] = mul(add(xh[j][e], off), scale);
        db[j][e] = add(db[j][e], g[j][e]);
        dw[j][e] = fma(g[j][e], xh[j][e], dw[j][e]);
        g[j][e] = mul(g[j][e], w[e]);
        sg = add(sg, g[j][e]);
        sgx = fma(g[j][e], xh[j][e], sgx);
      }
    }
    fetch(row + step);
    if (!a.dx) continue;
    const float2 s = group_sum<kRow>(total(sg), total(sgx), part[turn][group], group);
    const P less = both(-s.x * inv, P()), slope = both(-s.y * inv, P());
    T* dx = static_cast<T*>(a.dx) + row * a.dx_stride;
#pragma unroll
    for (int j = 0; j < N; j++) {
      const int c = (j * kRow + t) * V;
      if (c >= cols) continue;
      Pack<T, V> out;
#pragma unroll
      for (int e = 0; e < H; e++) narrow<T, V>(out, e, mul(scale, fma(xh[j][e], slope, add(g[j][e], less))));
      store_pack(dx + c, out);
    }
  }
  if (!a.partial) return;
  float* out = a.partial + (int64_t)blockIdx.x * 2 * cols;
  if constexpr (kBlockRows == 1) {
#pragma unroll
    for (int j = 0; j < N; j++) {
      const int c = (j * kRow + t) * V;
      if (c >= cols) continue;
#pragma unroll
      for (int e = 0; e < H; e++) {
        *reinterpret_cast<P*>(out + c + e * (V / H)) = dw[j][e];
        *reinterpret_cast<P*>(out + cols + c + e * (V / H)) = db[j][e];
      }
    }
  } else {  // the groups' sums one after another
    __shared__ __align__(16) float all[2][N * V * kRow];
    for (int q = 0; q < kBlockRows; q++) {
      if (q == group) {
#pragma unroll
        for (int j = 0; j < N; j++)
#pragma unroll
          for (int e = 0; e < H; e++) {
            const int c = (j * kRow + t) * V + e * (V / H);
            P *w = reinterpret_cast<P*>(&all[0][c]), *b = reinterpret_cast<P*>(&all[1][c]);
            *w = q ? add(*w, dw[j][e]) : dw[j][e];
            *b = q ? add(*b, db[j][e]) : db[j][e];
          }
      }
      __syncthreads();
    }
    for (int i = threadIdx.x; i < cols; i += kBackBlock<kRow>) {
      out[i] = all[0][i];
      out[cols + i] = all[1][i];
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kLong) k_backward_long(NormArgs a, int w_f32) {
  __shared__ float part[2][32];
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
  const T* dy = static_cast<const T*>(a.dy) + row * a.dy_stride;
  const float mean = a.stats[row], rstd = a.stats[a.rows + row];
  float sg = 0.0f, sgx = 0.0f, w[1];
  for (int64_t c = threadIdx.x; c < a.cols; c += kLong) {
    load_weight<T, 1>(w, a.weight, w_f32, c, 1.0f);
    const float g = to_f32(dy[c]) * w[0];
    sg += g;
    sgx += g * ((to_f32(x[c]) - mean) * rstd);
  }
  const float mg = row_sum<kLong>(sg, part[0]) / (float)a.cols, mgx = row_sum<kLong>(sgx, part[1]) / (float)a.cols;
  T* dx = static_cast<T*>(a.dx) + row * a.dx_stride;
  for (int64_t c = threadIdx.x; c < a.cols; c += kLong) {
    load_weight<T, 1>(w, a.weight, w_f32, c, 1.0f);
    dx[c] = from_f32<T>(rstd * (to_f32(dy[c]) * w[0] - mg - (to_f32(x[c]) - mean) * rstd * mgx));
  }
}

// column sums of every gridDim.y-th row, for rows that k_backward does not hold
template <typename T>
__global__ void k_columns_long(NormArgs a) {
  const int64_t c = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (c >= a.cols) return;
  float sw = 0.0f, sb = 0.0f;
  for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y) {
    const float dy = to_f32(static_cast<const T*>(a.dy)[row * a.dy_stride + c]);
    sw += dy * ((to_f32(static_cast<const T*>(a.x)[row * a.x_stride + c]) - a.stats[row]) * a.stats[a.rows + row]);
    sb += dy;
  }
  a.partial[(int64_t)blockIdx.y * 2 * a.cols + c] = sw;
  a.partial[((int64_t)blockIdx.y * 2 + 1) * a.cols + c] = sb;
}

template <typename T>
cudaError_t forward(const NormArgs& a, int w_f32, cudaStream_t s) {
  if (a.rows == 0) return cudaSuccess;
  const int width = load_width<T>(a.rows, a.cols, w_f32, {a.weight, a.bias}, {{a.x, a.x_stride}, {a.y, a.y_stride}});
  const bool held = forward_variant<T>(width, a.cols, [&](auto v, auto n, auto r, auto b) {
    constexpr int kRow = decltype(r)::value, kRows = kBlock<kRow> / kRow;
    k_forward<T, decltype(v)::value, decltype(n)::value, kRow, decltype(b)::value>
        <<<(unsigned)((a.rows + kRows - 1) / kRows), kBlock<kRow>, 0, s>>>(a, w_f32);
  });
  if (!held) k_forward_long<T><<<(unsigned)a.rows, kLong, 0, s>>>(a, w_f32);
  return cudaGetLastError();
}

template <typename T>
cudaError_t backward(NormArgs a, int w_f32, cudaStream_t s) {
  const bool sums = a.dweight || a.dbias;
  if (!sums) a.partial = nullptr;
  int blocks = 0;
  if (a.rows > 0 && (a.dx || sums)) {
    const int width = load_width<T>(a.rows, a.cols, w_f32, {a.weight, a.bias}, {{a.x, a.x_stride}, {a.dy, a.dy_stride}, {a.dx, a.dx ? a.dx_stride : 0}});
    const bool held = backward_variant<T>(width, a.rows, a.cols, [&](auto v, auto n, auto r, auto b) {
      constexpr int kRow = decltype(r)::value, kThreads = kBackBlock<kRow>, kRows = kThreads / kRow;
      // as many blocks as stay resident, or a block a group of rows where there are fewer
      static const int resident = [] {
        int fit = 0;
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&fit, k_backward<T, decltype(v)::value, decltype(n)::value, kRow, decltype(b)::value>,
                                                      kThreads, 0);
        return std::clamp(fit * kSms, kSms, kMostBlocks);
      }();
      blocks = (int)std::min<int64_t>(resident, (a.rows + kRows - 1) / kRows);
      k_backward<T, decltype(v)::value, decltype(n)::value, kRow, decltype(b)::value><<<blocks, kThreads, 0, s>>>(a, w_f32);
    });
    if (!held) {
      if (a.dx) k_backward_long<T><<<(unsigned)a.rows, kLong, 0, s>>>(a, w_f32);
      blocks = (int)std::min<int64_t>(kLongBlocks, a.rows);
      if (sums) k_columns_long<T><<<dim3((unsigned)((a.cols + 255) / 256), blocks), 256, 0, s>>>(a);
    }
  }
  if (sums) {
    const dim3 grid((unsigned)((a.cols + 31) / 32), 2), block(32, 32);
    if (w_f32) k_columns_join<<<grid, block, 0, s>>>(a.partial, blocks, 2, a.cols, static_cast<float*>(a.dweight), static_cast<float*>(a.dbias));
    else k_columns_join<<<grid, block, 0, s>>>(a.partial, blocks, 2, a.cols, static_cast<T*>(a.dweight), static_cast<T*>(a.dbias));
  }
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_norm_forward(const NormArgs& a, ndvm_dtype t, ndvm_dtype wt, cudaStream_t s) {
  const int f = wt == NDVM_F32;
  return t == NDVM_F32 ? forward<float>(a, f, s) : t == NDVM_F16 ? forward<__half>(a, f, s) : forward<__nv_bfloat16>(a, f, s);
}
cudaError_t launch_norm_backward(const NormArgs& a, ndvm_dtype t, ndvm_dtype wt, cudaStream_t s) {
  const int f = wt == NDVM_F32;
  return t == NDVM_F32 ? backward<float>(a, f, s) : t == NDVM_F16 ? backward<__half>(a, f, s) : backward<__nv_bfloat16>(a, f, s);
}
size_t norm_workspace(int64_t rows, int64_t cols) {
  return (size_t)std::clamp<int64_t>(rows, 1, cols > kHeld ? kLongBlocks : kMostBlocks) * (size_t)cols * 2 * sizeof(float);
}

}  // namespace ndvm
