// Root-mean-square norm over a row of C elements with the residual stream's sum, and its backward pass:
//   s = round(x + residual) (s = x without one), r = 1 / sqrt(mean(s^2) + eps), y = s r w
//   g = dy w, sh = s r: dx = dresidual = dsum + r (g - sh mean(g sh)), dw = sum over rows of dy sh
// and 8-bit blocks (blocks.cuh): of y instead of y, or of any rows.
//
// All of it is bound by memory: forward reads x and the residual and writes s and y, backward reads s, dy and dsum and
// writes dx.  A row is read once and held in the registers of the threads that share it, as in the layer norm; the stream
// is rounded to its type before it is normalised, so that the backward pass sees from s alone what the forward pass saw.
#include <atomic>

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

// Rows longer than the registers of a block hold: two passes over the row, the later one from L2, one element a load.  (The sum's
// rounded values are made again where they are not stored.)  With a residual, 2048 rows: 20000 columns of bf16 148 us (2.2 TB/s; 16384, which
// are held, 43), 12288 of f32 108.
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

// Backward: a group of kRow threads takes every so-manieth row.  Each thread asks for its part of the rows to come by asynchronous
// copies, kDepth - 1 rows ahead, to shared memory that it alone reads: registers would hold one row ahead, which left the latency of
// memory in the open (16384 x 1024 bf16 with a residual 37 us; 25 so, and 65536 x 2048 154 us, 7.0 TB/s).  Rows off 16 bytes do take
// registers, one row ahead.
// partial[block][c] = the block's sum of dy sh.
template <int V, int N, int kRow, int kResident, int kBytes>
constexpr int kDepth = V * kBytes != 16 ? 0 : std::min(4, 221184 / kResident / (3 * N * kBackBlock<kRow> * 16));

__device__ __forceinline__ void copy16(uint32_t to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
template <int kLeft>
__device__ __forceinline__ void copies_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
}

template <typename T, int V, int N, int kRow, int kResident>
__global__ void __launch_bounds__(kBackBlock<kRow>, kResident) k_rms_backward(RmsArgs a, int w_f32) {
  using P = Pairs<V>;
  constexpr int H = kPairs<V>, kBlockRows = kBackBlock<kRow> / kRow, D = kDepth<V, N, kRow, kResident, sizeof(T)>;
  extern __shared__ __align__(16) char ring[];  // [row ahead][array][pack][thread]
  __shared__ float2 part[2][kBlockRows][kRow > 32 ? kRow / 32 : 1];
  const int t = threadIdx.x % kRow, group = threadIdx.x / kRow, cols = (int)a.cols, arrays = a.dsum ? 3 : 2;
  const float inv = 1.0f / (float)cols;
  P dw[N][H];
#pragma unroll
  for (int j = 0; j < N; j++)
#pragma unroll
    for (int e = 0; e < H; e++) dw[j][e] = both(0.0f, P());
  Pack<T, V> nx[N], nd[N], ns[N];
  float nrstd = 0.0f;
  const int64_t step = (int64_t)gridDim.x * kBlockRows;
  const auto pack_at = [&](int slot, int array, int j) { return ((slot * arrays + array) * N + j) * kBackBlock<kRow> * 16 + (int)threadIdx.x * 16; };
  // asks for a row; `slot` of the ring receives it
  const auto fetch = [&](int64_t row, int slot) {
    if (row < a.rows) {
      const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
      const T* d = static_cast<const T*>(a.dy) + row * a.dy_stride;
      const T* s = static_cast<const T*>(a.dsum) + row * a.dsum_stride;
#pragma unroll
      for (int j = 0; j < N; j++) {
        const int c = (j * kRow + t) * V;
        if (c >= cols) continue;
        if constexpr (D > 0) {
          const uint32_t to = (uint32_t)__cvta_generic_to_shared(ring);
          copy16(to + pack_at(slot, 0, j), x + c);
          copy16(to + pack_at(slot, 1, j), d + c);
          if (a.dsum) copy16(to + pack_at(slot, 2, j), s + c);
        } else {
          nx[j] = load_pack<T, V>(x + c);
          nd[j] = load_pack<T, V>(d + c);
          if (a.dsum) ns[j] = load_pack<T, V>(s + c);
        }
      }
    }
    if constexpr (D > 0) asm volatile("cp.async.commit_group;" ::: "memory");
  };
  const auto ask_rstd = [&](int64_t row) {
    if (row < a.rows) nrstd = a.rstd[row];
  };
  // weights stay in registers where the ring has left room for them
  P w[N][H];
  const auto ask_weight = [&](int j) {
    const int c = (j * kRow + t) * V;
    if (c < cols) load_weight<T, V>(w[j], a.weight, w_f32, c, 1.0f);
  };
  int64_t row = (int64_t)blockIdx.x * kBlockRows + group;
  ask_rstd(row);
  if constexpr (D > 0) {
#pragma unroll
    for (int q = 0; q < D - 1; q++) fetch(row + q * step, q);
#pragma unroll
    for (int j = 0; j < N; j++) ask_weight(j);
  } else {
    fetch(row, 0);
  }
  int slot = 0;
  for (int turn = 0; row < a.rows; row += step, turn ^= 1) {
    const float rstd = nrstd;
    const P scale = both(rstd, P());
    ask_rstd(row + step);
    if constexpr (D > 0) {
      fetch(row + (D - 1) * step, slot == 0 ? D - 1 : slot - 1);
      copies_wait<D - 1>();
    }
    P sh[N][H], g[N][H], sgs = both(0.0f, P());
    Pack<T, V> ds[N];
#pragma unroll
    for (int j = 0; j < N; j++) {
      const int c = (j * kRow + t) * V;
      if (c >= cols) continue;
      if constexpr (D == 0) ask_weight(j);
      if constexpr (D > 0) {
        nx[j] = load_pack<T, V>(reinterpret_cast<const T*>(ring + pack_at(slot, 0, j)));
        nd[j] = load_pack<T, V>(reinterpret_cast<const T*>(ring + pack_at(slot, 1, j)));
        if (a.dsum) ns[j] = load_pack<T, V>(reinterpret_cast<const T*>(ring + pack_at(slot, 2, j)));
      }
      widen<T, V>(nx[j], sh[j]);
      widen<T, V>(nd[j], g[j]);
      ds[j] = ns[j];
#pragma unroll
      for (int e = 0; e < H; e++) {
        sh[j][e] = mul(sh[j][e], scale);
        dw[j][e] = fma(g[j][e], sh[j][e], dw[j][e]);
        g[j][e] = mul(g[j][e], w[j][e]);
        sgs = fma(g[j][e], sh[j][e], sgs);
      }
    }
    if constexpr (D > 0) slot = slot + 1 == D ? 0 : slot + 1;
    else fetch(row + step, 0);
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
  if constexpr (D > 0) copies_wait<0>();
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

// (one element a load, and dw by a kernel of its own: 2048 rows with a residual, 12288 columns of bf16 129 us, 1.6 TB/s, against 29 for 8192, which
// k_rms_backward holds; of f32 149)
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
// A warp a row (gridDim.y warps, each its share of whole 128s of the columns), 16 bytes a lane wherever the rows start.
template <typename T, bool kVectors>
__global__ void __launch_bounds__(256) k_quantize(RmsArgs a, int64_t share) {
  constexpr int V = 16 / sizeof(T), H = kPairs<V>, kUnroll = 4;
  using P = Pairs<V>;
  const int lane = threadIdx.x % 32;
  const int64_t row = (int64_t)blockIdx.x * 8 + threadIdx.x / 32, chunks = (a.cols + 127) / 128;
  const int64_t from = blockIdx.y * share, to = min(from + share, chunks * 128);
  if (row >= whole(a.rows)) return;
  const bool real = row < a.rows;
  const T* x = static_cast<const T*>(a.x) + (real ? row : 0) * a.x_stride;
  uint8_t *values = a.values + row * a.v_stride, *scales = a.scales + scale_at(row, 0, chunks);  // (a row's: 4 of every 512 bytes)
  const char *begin = reinterpret_cast<const char*>(x), *end = reinterpret_cast<const char*>(x + a.cols);
  const int off = (int)(reinterpret_cast<uintptr_t>(x) % 16);
  const uint32_t lanes = (0xffffffffu >> (32 - 32 / V)) << (lane / (32 / V) * (32 / V));
  for (int64_t c0 = from + lane * V; c0 < to; c0 += kUnroll * 32 * V) {
    Pack<T, V> p[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; u++) {
      const int64_t c = c0 + u * 32 * V;
      if (!real || c >= to || c >= a.cols) continue;
      if constexpr (kVectors) {
        p[u] = load_pack<T, V>(x + c);
      } else {
        union { uint4 u; Pack<T, V> p; } b;
        b.u = row_bytes(begin + c * sizeof(T), begin, end, off);
        p[u] = b.p;
      }
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
      store_block<V>(v, lanes, values + c, real && c < a.v_cols, scales + c / 128 * 512 + (c / 32 & 3));
    }
  }
}

template <typename T, bool kVectors>
__global__ void __launch_bounds__(256) k_dequantize(RmsArgs a, int64_t share) {
  constexpr int kUnroll = 4;
  __shared__ T staging[kVectors ? 1 : 8][256];
  const int lane = threadIdx.x % 32;
  const int64_t row = (int64_t)blockIdx.x * 8 + threadIdx.x / 32, chunks = (a.cols + 127) / 128;
  const int64_t from = blockIdx.y * share, to = min(from + share, a.cols);
  if (row >= a.rows) return;
  T* y = static_cast<T*>(a.y) + row * a.y_stride;
  const uint8_t *values = a.values + row * a.v_stride, *scales = a.scales + scale_at(row, 0, chunks);
  for (int64_t first = from; first < to; first += kUnroll * 256) {
    uint2 words[kUnroll];
    uint32_t codes[kUnroll];
#pragma unroll
    for (int u = 0; u < kUnroll; u++) {
      const int64_t c = first + u * 256 + lane * 8;
      if (c >= to) continue;
      words[u] = *reinterpret_cast<const uint2*>(values + c);
      codes[u] = scales[c / 128 * 512 + (c / 32 & 3)];
    }
#pragma unroll
    for (int u = 0; u < kUnroll; u++) {
      const int64_t c0 = first + u * 256, c = c0 + lane * 8;
      if (c0 >= to) break;
      Pack<T, 8> out;
      if (c < to) {
        const float scale = block_scale(codes[u]);
#pragma unroll
        for (int e = 0; e < 4; e++)
          narrow(out.v + 2 * e, held<T>(from_e4m3((uint16_t)((e < 2 ? words[u].x : words[u].y) >> (e % 2 * 16))), scale, codes[u]));
      }
      if (kVectors && c + 8 <= a.cols) {
        if constexpr (sizeof(T) == 2) {
          store_pack(y + c, out);
        } else {
          *reinterpret_cast<float4*>(y + c) = make_float4(out.v[0], out.v[1], out.v[2], out.v[3]);
          *reinterpret_cast<float4*>(y + c + 4) = make_float4(out.v[4], out.v[5], out.v[6], out.v[7]);
        }
      } else if (kVectors) {
#pragma unroll
        for (int e = 0; e < 8; e++)
          if (c + e < a.cols) y[c + e] = out.v[e];
      } else {  // by way of shared memory, so that a warp stores neighbours
        T* mine = staging[threadIdx.x / 32];
        if (c < to) {
#pragma unroll
          for (int e = 0; e < 8; e++) mine[lane * 8 + e] = out.v[e];
        }
        __syncwarp();
#pragma unroll
        for (int e = 0; e < 8; e++)
          if (c0 + e * 32 + lane < a.cols) y[c0 + e * 32 + lane] = mine[e * 32 + lane];
        __syncwarp();
      }
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
    constexpr int V = decltype(v)::value, R = decltype(r)::value, N = decltype(n)::value;
    // 8-bit blocks want 32 consecutive elements in one turn of a row's threads, and two warps rather than one for a row of eight
    // loads a thread: the blocks' instructions are what a row waits for (one warp and two, with a residual, us: bf16 16384 x 2048 45
    // and 39, x 1536 37 and 31, x 1280 33 and 28, x 1032 31 and 28; 64 rows 4.8 to 6.3 and 3.1 to 3.8; f32 16384 x 1024 45 and
    // 36, x 516 29 and 23)
    constexpr bool kTwo = kBlocks && R == 32 && N == 8 && V > 1;
    constexpr int kRow = kTwo ? 64 : kBlocks && R * V < 32 ? 32 : R, kRows = kBlock<kRow> / kRow;
    k_rms_forward<T, V, kTwo ? 4 : N, kRow, kTwo ? 8 : decltype(b)::value, kBlocks>
        <<<(unsigned)((rows + kRows - 1) / kRows), kBlock<kRow>, 0, s>>>(a, w_f32);
  });
  if (!held) k_rms_forward_long<T, kBlocks><<<(unsigned)rows, kLong, 0, s>>>(a, w_f32);
  return cudaGetLastError();
}

template <typename T>
cudaError_t rms_backward(RmsArgs a, int w_f32, cudaStream_t s) {
  if (!a.dweight) a.partial = nullptr;
  int blocks = 0;
  cudaError_t failed = cudaSuccess;
  if (a.rows > 0 && (a.dx || a.dweight)) {
    const int width = load_width<T>(a.rows, a.cols, w_f32, {a.weight},
                                    {{a.x, a.x_stride}, {a.dy, a.dy_stride}, {a.dsum, a.dsum ? a.dsum_stride : 0}, {a.dx, a.dx ? a.dx_stride : 0}});
    // (rows: not the layer norm's rule for many of them, whose one load a thread leaves more barriers a row: with the rows ahead in
    // shared memory two loads are the faster, 65536 x 2048 154 us against 190)
    const bool held = backward_variant<T>(width, 0, a.cols, [&](auto v, auto n, auto r, auto b) {
      constexpr int kRow = decltype(r)::value, kThreads = kBackBlock<kRow>, kRows = kThreads / kRow;
      constexpr auto kernel = k_rms_backward<T, decltype(v)::value, decltype(n)::value, kRow, decltype(b)::value>;
      constexpr int kRing = kDepth<decltype(v)::value, decltype(n)::value, kRow, decltype(b)::value, sizeof(T)> * decltype(n)::value * kThreads * 16;
      // as many blocks as stay resident, or a block a group of rows where there are fewer
      static std::atomic<uint64_t> allowed{0};  // devices on which the kernel may take its shared memory
      static std::atomic<int> resident{0};
      int device = 0;
      if (failed == cudaSuccess) failed = cudaGetDevice(&device);
      if (failed == cudaSuccess && (device >= 64 || !(allowed.load(std::memory_order_acquire) >> device & 1))) {
        if (kRing) failed = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 3 * kRing);
        int fit = 0;
        if (failed == cudaSuccess) failed = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&fit, kernel, kThreads, 3 * kRing);
        resident.store(std::clamp(fit * kSms, kSms, kMostBlocks), std::memory_order_relaxed);
        if (failed == cudaSuccess && device < 64) allowed.fetch_or((uint64_t)1 << device, std::memory_order_release);
      }
      if (failed != cudaSuccess) return;
      blocks = (int)std::min<int64_t>(resident.load(std::memory_order_relaxed), (a.rows + kRows - 1) / kRows);
      kernel<<<blocks, kThreads, (a.dsum ? 3 : 2) * kRing, s>>>(a, w_f32);
    });
    if (failed != cudaSuccess) return failed;
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
  if (width == 16 / (int)sizeof(T)) k_quantize<T, true><<<grid, 256, 0, s>>>(a, share);
  else k_quantize<T, false><<<grid, 256, 0, s>>>(a, share);
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
