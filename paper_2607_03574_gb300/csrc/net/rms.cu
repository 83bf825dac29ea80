// Root-mean-square norm over a row of C elements with the residual stream's sum, and its backward pass:
//   s = round(x + residual) (s = x without one), r = 1 / sqrt(mean(s^2) + eps), y = s r w
//   g = dy w, sh = s r: dx = dresidual = dsum + r (g - sh mean(g sh)), dw = sum over rows of dy sh
// and 8-bit blocks (blocks.cuh): of y instead of y, or of any rows.
//
// All of it is bound by memory: forward reads x and the residual and writes s and y, backward reads s, dy and dsum and
// writes dx.  A row is read once and held in the registers of the threads that share it, as in the layer norm; the stream
// is rounded to its type before it is normalised, so that the backward pass sees from s alone what the forward pass saw.
#include "blocks.cuh"
#include "net.h"
#include "rows.cuh"
#include "types.cuh"

namespace ndvm {
namespace {

// What 8-bit blocks of `rows` rows leave unwritten: scales behind a row's last block, or of a row behind the last one.
__device__ __forceinline__ void clear_scales(const RmsArgs& a, int64_t row, int64_t from, int t, int threads) {
  const int64_t chunks = (a.cols + 127) / 128;
  for (int64_t b = from + t; b < chunks * 4; b += threads) a.scales[scale_at(row, b, chunks)] = 0;
}
__device__ __forceinline__ int64_t whole(int64_t rows) { return (rows + 127) / 128 * 128; }

template <typename T, int V, int N, int kRow, int kResident, bool kBlocks>
__global__ void __launch_bounds__(kBlock<kRow>, kResident) k_rms_forward(RmsArgs a, int w_f32) {
  using P = Pairs<V>;
  constexpr int H = kPairs<V>;
  __shared__ float part[32];
  const int t = threadIdx.x % kRow;
  const int64_t row = (int64_t)blockIdx.x * (kBlock<kRow> / kRow) + threadIdx.x / kRow;
  if (row >= a.rows) {  // (whole groups; with a block a row, whole blocks)
    if (kBlocks && row < whole(a.rows)) clear_scales(a, row, 0, t, kRow);
    return;
  }
  const int cols = (int)a.cols;
  const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
  Pack<T, V> px[N];
#pragma unroll
  for (int j = 0; j < N; j++) {
    const int c = (j * kRow + t) * V;
    if (c < cols) px[j] = load_pack<T, V>(x + c);
  }
  if (a.residual) {
    const T* residual = static_cast<const T*>(a.residual) + row * a.r_stride;
    T* sum = static_cast<T*>(a.sum) + row * a.sum_stride;
    Pack<T, V> pr[N];
#pragma unroll
    for (int j = 0; j < N; j++) {
      const int c = (j * kRow + t) * V;
      if (c < cols) pr[j] = load_pack<T, V>(residual + c);
    }
#pragma unroll
    for (int j = 0; j < N; j++) {
      const int c = (j * kRow + t) * V;
      if (c >= cols) continue;
      P v[H], r[H];
      widen<T, V>(px[j], v);
      widen<T, V>(pr[j], r);
#pragma unroll
      for (int e = 0; e < H; e++) narrow<T, V>(px[j], e, add(v[e], r[e]));
      if (a.sum) store_pack(sum + c, px[j]);
    }
  }
  P sum = both(0.0f, P());
#pragma unroll
  for (int j = 0; j < N; j++) {
    if ((j * kRow + t) * V >= cols) continue;
    P v[H];
    widen<T, V>(px[j], v);
#pragma unroll
    for (int e = 0; e < H; e++) sum = fma(v[e], v[e], sum);
  }
  const float rstd = 1.0f / sqrtf(row_sum<kRow>(total(sum), part) / (float)cols + a.eps);
  const P scale = both(rstd, P());
  const int64_t chunks = (cols + 127) / 128;
#pragma unroll
  for (int j = 0; j < N; j++) {
    const int c = (j * kRow + t) * V;
    P v[H], w[H];
    if (c < cols) {
      widen<T, V>(px[j], v);
      load_weight<T, V>(w, a.weight, w_f32, c, 1.0f);
    }
    if constexpr (kBlocks) {
#pragma unroll
      for (int e = 0; e < H; e++) v[e] = c < cols ? mul(mul(v[e], scale), w[e]) : both(0.0f, P());
      store_block<V>(v, group_lanes<kRow>() & (0xffffffffu >> (32 - 32 / V)) << (threadIdx.x % 32 / (32 / V) * (32 / V)),
                     a.values + row * a.v_stride + c, c < a.v_cols, c / 32 * 32 < cols ? a.scales + scale_at(row, c / 32, chunks) : nullptr);
    } else {
      if (c >= cols) continue;
#pragma unroll
      for (int e = 0; e < H; e++) narrow<T, V>(px[j], e, mul(mul(v[e], scale), w[e]));
      store_pack(static_cast<T*>(a.y) + row * a.y_stride + c, px[j]);
    }
  }
  if (kBlocks) clear_scales(a, row, (cols + 31) / 32, t, kRow);
  if (!kBlocks && t == 0 && a.rstd) a.rstd[row] = rstd;
}

// Rows longer than the registers of a block hold: two passes over the row, the later one from L2.  (The sum's rounded
// values are made again where they are not stored.)
template <typename T, bool kBlocks>
__global__ void __launch_bounds__(kLong) k_rms_forward_long(RmsArgs a, int w_f32) {
  __shared__ float part[32];
  const int64_t row = blockIdx.x, chunks = (a.cols + 127) / 128;
  if (row >= a.rows) {
    clear_scales(a, row, 0, threadIdx.x, kLong);
    return;
  }
  const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
  const T* residual = static_cast<const T*>(a.residual) + row * a.r_stride;
  // (y may be x or the residual: a thread reads the elements that it writes, in both passes)
  const auto at = [&](int64_t c) {
    return a.residual ? from_f32<T>(to_f32(x[c]) + to_f32(residual[c])) : x[c];
  };
  float s = 0.0f;
  for (int64_t c = threadIdx.x; c < a.cols; c += kLong) {
    const float v = to_f32(at(c));
    s += v * v;
  }
  const float rstd = 1.0f / sqrtf(row_sum<kLong>(s, part) / (float)a.cols + a.eps);
  for (int64_t c = threadIdx.x; c < (kBlocks ? chunks * 128 : a.cols); c += kLong) {
    float w[1], v[1] = {0.0f};
    if (c < a.cols) {
      const T stream = at(c);
      load_weight<T, 1>(w, a.weight, w_f32, c, 1.0f);
      v[0] = to_f32(stream) * rstd * w[0];
      if (a.residual && a.sum) static_cast<T*>(a.sum)[row * a.sum_stride + c] = stream;
    }
    if constexpr (kBlocks) store_block<1>(v, ~0u, a.values + row * a.v_stride + c, c < a.v_cols, a.scales + scale_at(row, c / 32, chunks));
    else static_cast<T*>(a.y)[row * a.y_stride + c] = from_f32<T>(v[0]);
  }
  if (!kBlocks && threadIdx.x == 0 && a.rstd) a.rstd[row] = rstd;
}

// Backward, as the layer norm's: a group of kRow threads takes every so-manieth row, the next row's loads in flight while the
// present one is worked on.  partial[block][c] = the block's sum of dy sh.
template <typename T, int V, int N, int kRow, int kResident>
__global__ void __launch_bounds__(kBackBlock<kRow>, kResident) k_rms_backward(RmsArgs a, int w_f32) {
  using P = Pairs<V>;
  constexpr int H = kPairs<V>, kBlockRows = kBackBlock<kRow> / kRow;
  __shared__ float2 part[2][kBlockRows][kRow > 32 ? kRow / 32 : 1];
  const int t = threadIdx.x % kRow, group = threadIdx.x / kRow, cols = (int)a.cols;
  const float inv = 1.0f / (float)cols;
  P dw[N][H];
#pragma unroll
  for (int j = 0; j < N; j++)
#pragma unroll
    for (int e = 0; e < H; e++) dw[j][e] = both(0.0f, P());
  Pack<T, V> nx[N], nd[N], ns[N];
  float nrstd = 0.0f;
  const auto fetch = [&](int64_t row) {
    if (row >= a.rows) return;
    const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
    const T* d = static_cast<const T*>(a.dy) + row * a.dy_stride;
    const T* s = static_cast<const T*>(a.dsum) + row * a.dsum_stride;
    nrstd = a.rstd[row];
#pragma unroll
    for (int j = 0; j < N; j++) {
      const int c = (j * kRow + t) * V;
      if (c < cols) {
        nx[j] = load_pack<T, V>(x + c);
        nd[j] = load_pack<T, V>(d + c);
        if (a.dsum) ns[j] = load_pack<T, V>(s + c);
      }
    }
  };
  const int64_t step = (int64_t)gridDim.x * kBlockRows;
  int64_t row = (int64_t)blockIdx.x * kBlockRows + group;
  fetch(row);
  for (int turn = 0; row < a.rows; row += step, turn ^= 1) {
    const float rstd = nrstd;
    const P scale = both(rstd, P());
    P sh[N][H], g[N][H], sgs = both(0.0f, P());
    Pack<T, V> ds[N];
#pragma unroll
    for (int j = 0; j < N; j++) {
      const int c = (j * kRow + t) * V;
      if (c >= cols) continue;
      P w[H];
      load_weight<T, V>(w, a.weight, w_f32, c, 1.0f);
      widen<T, V>(nx[j], sh[j]);
      widen<T, V>(nd[j], g[j]);
      ds[j] = ns[j];
#pragma unroll
      for (int e = 0; e < H; e++) {
        sh[j][e] = mul(sh[j][e], scale);
        dw[j][e] = fma(g[j][e], sh[j][e], dw[j][e]);
        g[j][e] = mul(g[j][e], w[e]);
        sgs = fma(g[j][e], sh[j][e], sgs);
      }
    }
    fetch(row + step);
    if (!a.dx) continue;
    const float2 s = group_sum<kRow>(total(sgs), 0.0f, part[turn][group], group);
    const P slope = both(-s.x * inv, P());
    T* dx = static_cast<T*>(a.dx) + row * a.dx_stride;
#pragma unroll
    for (int j = 0; j < N; j++) {
      const int c = (j * kRow + t) * V;
      if (c >= cols) continue;
      Pack<T, V> out;
      P d[H];
      if (a.dsum) {
        widen<T, V>(ds[j], d);
      } else {
#pragma unroll
        for (int e = 0; e < H; e++) d[e] = both(0.0f, P());
      }
#pragma unroll
      for (int e = 0; e < H; e++) narrow<T, V>(out, e, fma(scale, fma(sh[j][e], slope, g[j][e]), d[e]));
      store_pack(dx + c, out);
    }
  }
  if (!a.partial) return;
  float* out = a.partial + (int64_t)blockIdx.x * cols;
  if constexpr (kBlockRows == 1) {
#pragma unroll
    for (int j = 0; j < N; j++) {
      const int c = (j * kRow + t) * V;
      if (c >= cols) continue;
#pragma unroll
      for (int e = 0; e < H; e++) *reinterpret_cast<P*>(out + c + e * (V / H)) = dw[j][e];
    }
  } else {  // the groups' sums one after another
    __shared__ __align__(16) float all[N * V * kRow];
    for (int q = 0; q < kBlockRows; q++) {
      if (q == group) {
#pragma unroll
        for (int j = 0; j < N; j++)
#pragma unroll
          for (int e = 0; e < H; e++) {
            P* w = reinterpret_cast<P*>(&all[(j * kRow + t) * V + e * (V / H)]);
            *w = q ? add(*w, dw[j][e]) : dw[j][e];
          }
      }
      __syncthreads();
    }
    for (int i = threadIdx.x; i < cols; i += kBackBlock<kRow>) out[i] = all[i];
  }
}

template <typename T>
__global__ void __launch_bounds__(kLong) k_rms_backward_long(RmsArgs a, int w_f32) {
  __shared__ float part[32];
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
  const T* dy = static_cast<const T*>(a.dy) + row * a.dy_stride;
  const float rstd = a.rstd[row];
  float sgs = 0.0f, w[1];
  for (int64_t c = threadIdx.x; c < a.cols; c += kLong) {
    load_weight<T, 1>(w, a.weight, w_f32, c, 1.0f);
    sgs += to_f32(dy[c]) * w[0] * (to_f32(x[c]) * rstd);
  }
  const float m = row_sum<kLong>(sgs, part) / (float)a.cols;
  T* dx = static_cast<T*>(a.dx) + row * a.dx_stride;
  for (int64_t c = threadIdx.x; c < a.cols; c += kLong) {
    load_weight<T, 1>(w, a.weight, w_f32, c, 1.0f);
    const float d = a.dsum ? to_f32(static_cast<const T*>(a.dsum)[row * a.dsum_stride + c]) : 0.0f;
    dx[c] = from_f32<T>(fmaf(rstd, to_f32(dy[c]) * w[0] - to_f32(x[c]) * rstd * m, d));
  }
}

// column sums of every gridDim.y-th row, for rows that k_rms_backward does not hold
template <typename T>
__global__ void k_rms_columns_long(RmsArgs a) {
  const int64_t c = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (c >= a.cols) return;
  float s = 0.0f;
  for (int64_t row = blockIdx.y; row < a.rows; row += gridDim.y)
    s += to_f32(static_cast<const T*>(a.dy)[row * a.dy_stride + c]) * (to_f32(static_cast<const T*>(a.x)[row * a.x_stride + c]) * a.rstd[row]);
  a.partial[(int64_t)blockIdx.y * a.cols + c] = s;
}

// ------------------------------------------------------------------------------------- 8-bit blocks
// A warp a row (gridDim.y warps, each its share of whole 128s of the columns), V elements a lane.
template <typename T, int V>
__global__ void __launch_bounds__(256) k_quantize(RmsArgs a, int64_t share) {
  using P = Pairs<V>;
  constexpr int H = kPairs<V>, kUnroll = 4;
  const int lane = threadIdx.x % 32;
  const int64_t row = (int64_t)blockIdx.x * 8 + threadIdx.x / 32, chunks = (a.cols + 127) / 128;
  const int64_t from = blockIdx.y * share, to = min(from + share, chunks * 128);
  if (row >= whole(a.rows)) return;
  const bool real = row < a.rows;
  const T* x = static_cast<const T*>(a.x) + (real ? row : 0) * a.x_stride;
  const uint32_t lanes = (0xffffffffu >> (32 - 32 / V)) << (lane / (32 / V) * (32 / V));
  for (int64_t c0 = from + lane * V; c0 < to; c0 += kUnroll * 32 * V) {
    Pack<T, V> p[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; u++) {
      const int64_t c = c0 + u * 32 * V;
      if (real && c < to && c < a.cols) p[u] = load_pack<T, V>(x + c);
    }
#pragma unroll
    for (int u = 0; u < kUnroll; u++) {
      const int64_t c = c0 + u * 32 * V;
      if (c >= to) break;  // (whole blocks of lanes)
      P v[H];
      if (real && c < a.cols) {
        widen<T, V>(p[u], v);
      } else {
#pragma unroll
        for (int e = 0; e < H; e++) v[e] = both(0.0f, P());
      }
      store_block<V>(v, lanes, a.values + row * a.v_stride + c, real && c < a.v_cols, a.scales + scale_at(row, c / 32, chunks));
    }
  }
}

template <typename T, bool kVectors>
__global__ void __launch_bounds__(256) k_dequantize(RmsArgs a, int64_t share) {
  const int lane = threadIdx.x % 32;
  const int64_t row = (int64_t)blockIdx.x * 8 + threadIdx.x / 32, chunks = (a.cols + 127) / 128;
  const int64_t from = blockIdx.y * share, to = min(from + share, a.cols);
  if (row >= a.rows) return;
  T* y = static_cast<T*>(a.y) + row * a.y_stride;
#pragma unroll 4
  for (int64_t c = from + lane * 8; c < to; c += 256) {
    const uint2 q = *reinterpret_cast<const uint2*>(a.values + row * a.v_stride + c);
    const float scale = block_scale(a.scales[scale_at(row, c / 32, chunks)]);
    const uint16_t pairs[4] = {(uint16_t)q.x, (uint16_t)(q.x >> 16), (uint16_t)q.y, (uint16_t)(q.y >> 16)};
    Pack<T, 8> out;
#pragma unroll
    for (int e = 0; e < 4; e++) {
      const float2 v = from_e4m3(pairs[e]);
      narrow(out.v + 2 * e, make_float2(held<T>(v.x, scale), held<T>(v.y, scale)));
    }
    if (kVectors && c + 8 <= a.cols) {
      if constexpr (sizeof(T) == 2) {
        store_pack(y + c, out);
      } else {
        *reinterpret_cast<float4*>(y + c) = make_float4(out.v[0], out.v[1], out.v[2], out.v[3]);
        *reinterpret_cast<float4*>(y + c + 4) = make_float4(out.v[4], out.v[5], out.v[6], out.v[7]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; e++)
        if (c + e < a.cols) y[c + e] = out.v[e];
    }
  }
}

// ---------------------------------------------------------------------------------------- launches
template <typename T, bool kBlocks>
cudaError_t rms_forward(const RmsArgs& a, int w_f32, cudaStream_t s) {
  if (a.rows == 0) return cudaSuccess;
  const int64_t rows = kBlocks ? (a.rows + 127) / 128 * 128 : a.rows;
  const int width = load_width<T>(a.rows, a.cols, w_f32, {a.weight},
                                  {{a.x, a.x_stride}, {a.residual, a.residual ? a.r_stride : 0}, {a.sum, a.sum ? a.sum_stride : 0},
                                   {kBlocks ? nullptr : a.y, kBlocks ? 0 : a.y_stride}});
  const bool held = forward_variant<T>(width, a.cols, [&](auto v, auto n, auto r, auto b) {
    constexpr int V = decltype(v)::value, R = decltype(r)::value;
    // (8-bit blocks want 32 consecutive elements in one turn of a row's threads)
    constexpr int kRow = kBlocks && R * V < 32 ? 32 : R, kRows = kBlock<kRow> / kRow;
    k_rms_forward<T, V, decltype(n)::value, kRow, decltype(b)::value, kBlocks>
        <<<(unsigned)((rows + kRows - 1) / kRows), kBlock<kRow>, 0, s>>>(a, w_f32);
  });
  if (!held) k_rms_forward_long<T, kBlocks><<<(unsigned)rows, kLong, 0, s>>>(a, w_f32);
  return cudaGetLastError();
}

template <typename T>
cudaError_t rms_backward(RmsArgs a, int w_f32, cudaStream_t s) {
  if (!a.dweight) a.partial = nullptr;
  int blocks = 0;
  if (a.rows > 0 && (a.dx || a.dweight)) {
    const int width = load_width<T>(a.rows, a.cols, w_f32, {a.weight},
                                    {{a.x, a.x_stride}, {a.dy, a.dy_stride}, {a.dsum, a.dsum ? a.dsum_stride : 0}, {a.dx, a.dx ? a.dx_stride : 0}});
    const bool held = backward_variant<T>(width, a.rows, a.cols, [&](auto v, auto n, auto r, auto b) {
      constexpr int kRow = decltype(r)::value, kThreads = kBackBlock<kRow>, kRows = kThreads / kRow;
      // as many blocks as stay resident, or a block a group of rows where there are fewer
      static const int resident = [] {
        int fit = 0;
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&fit, k_rms_backward<T, decltype(v)::value, decltype(n)::value, kRow, decltype(b)::value>,
                                                      kThreads, 0);
        return std::clamp(fit * kSms, kSms, kMostBlocks);
      }();
      blocks = (int)std::min<int64_t>(resident, (a.rows + kRows - 1) / kRows);
      k_rms_backward<T, decltype(v)::value, decltype(n)::value, kRow, decltype(b)::value><<<blocks, kThreads, 0, s>>>(a, w_f32);
    });
    if (!held) {
      if (a.dx) k_rms_backward_long<T><<<(unsigned)a.rows, kLong, 0, s>>>(a, w_f32);
      blocks = (int)std::min<int64_t>(kLongBlocks, a.rows);
      if (a.dweight) k_rms_columns_long<T><<<dim3((unsigned)((a.cols + 255) / 256), blocks), 256, 0, s>>>(a);
    }
  }
  if (a.dweight) {
    const dim3 grid((unsigned)((a.cols + 31) / 32)), block(32, 32);
    if (w_f32) k_columns_join<<<grid, block, 0, s>>>(a.partial, blocks, 1, a.cols, static_cast<float*>(a.dweight), static_cast<float*>(nullptr));
    else k_columns_join<<<grid, block, 0, s>>>(a.partial, blocks, 1, a.cols, static_cast<T*>(a.dweight), static_cast<T*>(nullptr));
  }
  return cudaGetLastError();
}

// a warp's share of a row's columns: whole steps of its unrolled loop (1024 columns), fewer rows' cut until the SMs are full
dim3 block_grid(int64_t rows, int64_t cols, int64_t* share) {
  const int64_t groups = (rows + 7) / 8, steps = (cols + 255) / 256;
  const int64_t cuts = std::clamp<int64_t>(kSms * 8 / groups, 1, std::min<int64_t>(steps, 65535));
  *share = (steps + cuts - 1) / cuts * 256;
  return dim3((unsigned)groups, (unsigned)((cols + *share - 1) / *share));
}

template <typename T>
cudaError_t quantize(const RmsArgs& a, cudaStream_t s) {
  if (a.rows == 0) return cudaSuccess;
  int64_t share;
  const dim3 grid = block_grid((a.rows + 127) / 128 * 128, a.cols, &share);
  const int width = load_width<T>(a.rows, a.cols, 0, {}, {{a.x, a.x_stride}});
  constexpr int V = 16 / sizeof(T);
  if (width == V) k_quantize<T, V><<<grid, 256, 0, s>>>(a, share);
  else if (width == 2) k_quantize<T, 2><<<grid, 256, 0, s>>>(a, share);
  else k_quantize<T, 1><<<grid, 256, 0, s>>>(a, share);
  return cudaGetLastError();
}
template <typename T>
cudaError_t dequantize(const RmsArgs& a, cudaStream_t s) {
  if (a.rows == 0) return cudaSuccess;
  int64_t share;
  const dim3 grid = block_grid(a.rows, a.cols, &share);
  if (starts_on(a.y, 16) && (a.rows <= 1 || a.y_stride * sizeof(T) % 16 == 0)) k_dequantize<T, true><<<grid, 256, 0, s>>>(a, share);
  else k_dequantize<T, false><<<grid, 256, 0, s>>>(a, share);
  return cudaGetLastError();
}

}  // namespace

#define BY_TYPE(call, t) ((t) == NDVM_F32 ? call<float> : (t) == NDVM_F16 ? call<__half> : call<__nv_bfloat16>)

cudaError_t launch_rms_forward(const RmsArgs& a, ndvm_dtype t, ndvm_dtype wt, cudaStream_t s) {
  const int f = wt == NDVM_F32;
  if (a.values) return t == NDVM_F32 ? rms_forward<float, true>(a, f, s) : t == NDVM_F16 ? rms_forward<__half, true>(a, f, s) : rms_forward<__nv_bfloat16, true>(a, f, s);
  return t == NDVM_F32 ? rms_forward<float, false>(a, f, s) : t == NDVM_F16 ? rms_forward<__half, false>(a, f, s) : rms_forward<__nv_bfloat16, false>(a, f, s);
}
cudaError_t launch_rms_backward(const RmsArgs& a, ndvm_dtype t, ndvm_dtype wt, cudaStream_t s) { return BY_TYPE(rms_backward, t)(a, wt == NDVM_F32, s); }
size_t rms_workspace(int64_t rows, int64_t cols) {
  return (size_t)std::clamp<int64_t>(rows, 1, cols > kHeld ? kLongBlocks : kMostBlocks) * (size_t)cols * sizeof(float);
}
cudaError_t launch_quantize(const RmsArgs& a, ndvm_dtype t, cudaStream_t s) { return BY_TYPE(quantize, t)(a, s); }
cudaError_t launch_dequantize(const RmsArgs& a, ndvm_dtype t, cudaStream_t s) { return BY_TYPE(dequantize, t)(a, s); }

}  // namespace ndvm
