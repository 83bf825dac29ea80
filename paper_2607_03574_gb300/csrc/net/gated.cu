// Gated projection h = act(G) U with G = x Wg^T, U = x Wu^T, and its backward pass:
//   dU = dh act(G), dG = dh U act'(G), dx = dG Wg + dU Wu, dWg = dG^T x, dWu = dU^T x.
// The backward pass computes G and U again, or takes those that the forward pass kept: in binary32 (8 bytes an
// element of h), so that dG and dU are rounded once, to the operands' type, which the next products need (and
// where there are few of them, not even that: in_halves).
//
// All products run in one kernel frame (product.cu).
#include "activation.cuh"
#include "net.h"
#include "product.h"
#include "types.cuh"

namespace ndvm {
namespace {

// dG and dU of G and U that the forward pass kept: 8 columns a thread.  halves: and what their rounding left, `rows`
// rows further on.
template <typename T, bool kVectors>
__global__ void __launch_bounds__(256) k_gradient(const float* kept, int64_t kept_stride, const T* dh, int64_t dh_stride, int64_t rows,
                                                  int64_t n, int act, T* dg, T* du, int64_t pitch, bool halves) {
  const int64_t eights = pitch / 8, total = rows * eights;
  const float* up = kept + rows * kept_stride;
  by_activation(act, [&](auto k) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
      const int64_t row = i / eights, c = (i - row * eights) * 8;
      Pack<T, 8> d;
      float4 g[2], u[2];
      const bool all = c + 8 <= n;
#pragma unroll
      for (int q = 0; q < 2; q++) {
        if (all || c + 4 * q < n) {  // (rows of G and U hold whole fours)
          g[q] = *reinterpret_cast<const float4*>(kept + row * kept_stride + c + 4 * q);
          u[q] = *reinterpret_cast<const float4*>(up + row * kept_stride + c + 4 * q);
        } else {
          g[q] = u[q] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        }
      }
      if (kVectors && all) {
        d = load_pack<T, 8>(dh + row * dh_stride + c);
      } else {
#pragma unroll
        for (int e = 0; e < 8; e++) d.v[e] = c + e < n ? dh[row * dh_stride + c + e] : from_f32<T>(0.0f);
      }
      Pack<T, 8> og, ou, lg, lu;
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float4 gq = g[e / 4], uq = u[e / 4];
        const float2 ge = e % 4 ? make_float2(gq.z, gq.w) : make_float2(gq.x, gq.y);
        const float2 ue = e % 4 ? make_float2(uq.z, uq.w) : make_float2(uq.x, uq.y);
        float2 a, da;
        activate<decltype(k)::value>(ge, &a, &da);
        const float2 f = widen(d.v + e);
        const float2 vg = mul(mul(f, ue), da), vu = mul(f, a);
        narrow(og.v + e, vg);
        narrow(ou.v + e, vu);
        if (halves) {
          lg.v[e] = rest_of(vg.x, og.v[e]), lg.v[e + 1] = rest_of(vg.y, og.v[e + 1]);
          lu.v[e] = rest_of(vu.x, ou.v[e]), lu.v[e + 1] = rest_of(vu.y, ou.v[e + 1]);
        }
      }
      if (halves) {
        store_pack(dg + (rows + row) * pitch + c, lg);
        store_pack(du + (rows + row) * pitch + c, lu);
      }
      store_pack(dg + row * pitch + c, og);
      store_pack(du + row * pitch + c, ou);
    }
  });
}

// ------------------------------------------------------------------------------------ one row: vectors
// Forward alone.  The weights are read once and are nearly all the traffic: a warp takes kPer rows of each weight, 16 bytes a
// lane and load, against x (from L1), sums in binary32.  (From two rows on the tensor cores are the faster: 8
// rows, 2048 -> 8192, took 53 us this way and 17 us that way.)
template <typename T, int V, int kPer>
__global__ void __launch_bounds__(128) k_one(GatedArgs a) {
  using P = Pairs<V>;
  constexpr int H = kPairs<V>, kUnroll = 16 / (2 * kPer);
  const int lane = threadIdx.x % 32;
  const int64_t j0 = ((int64_t)blockIdx.x * 4 + threadIdx.x / 32) * kPer;
  if (j0 >= a.n) return;
  const T *wg[kPer], *wu[kPer];
  P g[kPer], u[kPer];
#pragma unroll
  for (int q = 0; q < kPer; q++) {
    const int64_t j = j0 + q < a.n ? j0 + q : j0;
    wg[q] = static_cast<const T*>(a.w_gate) + j * a.g_stride;
    wu[q] = static_cast<const T*>(a.w_up) + j * a.u_stride;
    g[q] = u[q] = both(0.0f, P());
  }
  const T* x = static_cast<const T*>(a.x);
#pragma unroll kUnroll
  for (int64_t c = lane * V; c < a.k; c += 32 * V) {
    P vx[H], vg[kPer][H], vu[kPer][H];
    Pack<T, V> pg[kPer], pu[kPer];
#pragma unroll
    for (int q = 0; q < kPer; q++) pg[q] = load_pack<T, V>(wg[q] + c), pu[q] = load_pack<T, V>(wu[q] + c);
    widen<T, V>(load_pack<T, V>(x + c), vx);
#pragma unroll
    for (int q = 0; q < kPer; q++) {
      widen<T, V>(pg[q], vg[q]);
      widen<T, V>(pu[q], vu[q]);
#pragma unroll
      for (int e = 0; e < H; e++) {
        g[q] = fma(vx[e], vg[q][e], g[q]);
        u[q] = fma(vx[e], vu[q][e], u[q]);
      }
    }
  }
#pragma unroll
  for (int q = 0; q < kPer; q++) {
    float sg = total(g[q]), su = total(u[q]);
#pragma unroll
    for (int o = 16; o; o >>= 1) {
      sg += __shfl_xor_sync(~0u, sg, o);
      su += __shfl_xor_sync(~0u, su, o);
    }
    const int64_t j = j0 + q;
    if (lane != q || j >= a.n) continue;
    if (a.kept) {
      a.kept[j] = sg;
      a.kept[a.kept_stride + j] = su;
    }
    by_activation(a.act, [&](auto k) {
      float2 act, da;
      activate<decltype(k)::value>(make_float2(sg, sg), &act, &da);
      static_cast<T*>(a.h)[j] = from_f32<T>(act.x * su);
    });
  }
}

template <typename T>
void one(const GatedArgs& a, bool vectors, cudaStream_t s) {
  // two rows of each weight a warp halve the loads of x; fewer outputs than would fill the SMs go one a warp
  const bool two = a.n >= 4096;
  const unsigned grid = (unsigned)((a.n + (two ? 7 : 3)) / (two ? 8 : 4));
  if (vectors && two) k_one<T, 8, 2><<<grid, 128, 0, s>>>(a);
  else if (vectors) k_one<T, 8, 1><<<grid, 128, 0, s>>>(a);
  else if (two) k_one<T, 1, 2><<<grid, 128, 0, s>>>(a);
  else k_one<T, 1, 1><<<grid, 128, 0, s>>>(a);
}

// ------------------------------------------------------------------------------------ launches
// The workspace: aligned copies of what TMA cannot read, dG and dU, and split sums (dx's and the weights'
// take turns).
struct Layout {
  int64_t k_pitch, n_pitch;
  int parts;
  size_t x, gate, up, dh, grad, partial, kept, h, total;
  Layout(int64_t rows, int64_t k, int64_t n, bool backward, bool copies) {
    k_pitch = ndvm::up(k, 8);
    n_pitch = ndvm::up(n, 8);
    parts = in_halves(rows, k, n) ? 2 : 1;
    total = 0;
    const auto take = [&](int64_t bytes) {
      const size_t at = total;
      total += (size_t)ndvm::up(bytes, 256);
      return at;
    };
    x = take(copies ? rows * k_pitch * 2 : 0);
    gate = take(copies ? n * k_pitch * 2 : 0);
    up = take(copies ? n * k_pitch * 2 : 0);
    dh = take(copies && backward ? rows * n_pitch * 2 : 0);
    grad = take(backward ? 2 * parts * rows * n_pitch * 2 : 0);
    int64_t sums = 0;
    if (backward && rows > 0) {
      const Cut i = cut(kInput, rows * parts, k, n, 2, 1), w = cut(kWeight, n, k, rows, parts, 2);
      if (i.splits > 1 || parts > 1) sums = i.splits * parts * rows * ndvm::up(k, 4);
      if (w.splits > 1) sums = std::max(sums, 2 * w.splits * n * ndvm::up(k, 4));
    }
    partial = take(sums * 4);
    // halves are made from G and U in binary32: where the forward pass has not kept them, it runs again
    kept = take(backward && parts > 1 ? 2 * rows * ndvm::up(n, 4) * 4 : 0);
    h = take(backward && parts > 1 ? rows * n_pitch * 2 : 0);
  }
};

bool all_ready(const GatedArgs& a) {
  return (!a.dh || tma_ready(a.dh, a.dh_stride, a.rows, a.n)) && tma_ready(a.x, a.x_stride, a.rows, a.k) && tma_ready(a.w_gate, a.g_stride, a.n, a.k) &&
         tma_ready(a.w_up, a.u_stride, a.n, a.k);
}

void make_ready(GatedArgs& a, const Layout& l, bool x, bool weights, cudaStream_t s) {
  char* ws = static_cast<char*>(a.workspace);
  PackArgs p{};
  int count = 0;
  int64_t most = 0;
  const auto add = [&](const void*& from, int64_t& stride, int64_t rows, size_t at) {
    if (tma_ready(from, stride, rows, a.k)) return;
    p.from[count] = from; p.stride[count] = stride; p.rows[count] = rows; p.to[count] = ws + at;
    most = std::max(most, rows);
    from = ws + at;
    stride = l.k_pitch;
    count++;
  };
  if (x) add(a.x, a.x_stride, a.rows, l.x);
  if (weights) add(a.w_gate, a.g_stride, a.n, l.gate), add(a.w_up, a.u_stride, a.n, l.up);
  p.cols = a.k;
  p.pitch = l.k_pitch;
  if (count) launch_pack(p, count, most, s);
}

// G and U, and h or dG and dU of them
template <typename T, Mode kMode>
cudaError_t products(const GatedArgs& a, void* out0, void* out1, int64_t stride, cudaStream_t s) {
  const Cut k = cut(kMode, a.rows, a.n, a.k, 1, 1);
  ProductArgs p{};
  if (!map_matrix(&p.a[0], kType<T>, a.x, a.rows, a.k, a.x_stride, a_box(a.rows)) || !map_matrix(&p.b[0], kType<T>, a.w_gate, a.n, a.k, a.g_stride, k.width / 2) ||
      !map_matrix(&p.b[1], kType<T>, a.w_up, a.n, a.k, a.u_stride, k.width / 2))
    return cudaErrorInvalidValue;
  p.m = (int)a.rows; p.n = (int)a.n; p.c = (int)a.k;
  if (kMode == kForward && a.kept) {
    p.keep = 1;
    if (!map_partial(&p.kept, a.kept, 2, a.rows, a.n, a.kept_stride)) return cudaErrorInvalidValue;
  }
  p.matrices = 1;
  if (kMode == kGradient && !map_matrix(&p.dh, kType<T>, a.dh, a.rows, a.n, a.dh_stride, 32, true)) return cudaErrorInvalidValue;
  p.act = a.act; p.out[0] = out0; p.out[1] = out1; p.stride = stride;
  return launch_product(kMode, kType<T>, p, k, s);
}

template <typename T>
cudaError_t forward(GatedArgs a, cudaStream_t s) {
  if (a.rows == 0) return cudaSuccess;
  if (a.rows == 1) {
    one<T>(a, all_ready(a) && a.k % 8 == 0, s);
    return cudaGetLastError();
  }
  const Layout l(a.rows, a.k, a.n, false, !all_ready(a));
  make_ready(a, l, true, true, s);
  return products<T, kForward>(a, a.h, nullptr, a.h_stride, s);
}

template <typename T>
cudaError_t backward(GatedArgs a, cudaStream_t s) {
  if (a.rows == 0) {
    cudaError_t e = cudaSuccess;
    if (a.dw_gate) e = cudaMemsetAsync(a.dw_gate, 0, (size_t)(a.n * a.k) * 2, s);
    if (a.dw_up && e == cudaSuccess) e = cudaMemsetAsync(a.dw_up, 0, (size_t)(a.n * a.k) * 2, s);
    return e;
  }
  const bool weights = a.dw_gate || a.dw_up;
  if (!a.dx && !weights) return cudaSuccess;
  const Layout l(a.rows, a.k, a.n, true, !all_ready(a));
  char* ws = static_cast<char*>(a.workspace);
  T* dg = reinterpret_cast<T*>(ws + l.grad);
  T* du = dg + l.parts * a.rows * l.n_pitch;
  cudaError_t e;
  if (l.parts > 1 && !a.kept) {
    GatedArgs f = a;
    f.dh = nullptr;
    f.kept = reinterpret_cast<float*>(ws + l.kept);
    f.kept_stride = up(a.n, 4);
    f.h = ws + l.h;
    f.h_stride = l.n_pitch;
    if ((e = forward<T>(f, s)) != cudaSuccess) return e;
    a.kept = f.kept;
    a.kept_stride = f.kept_stride;
  }
  if (a.kept) {
    make_ready(a, l, weights, a.dx != nullptr, s);
    const int64_t blocks = std::min<int64_t>(ceil_div(a.rows * (l.n_pitch / 8), 256), kSms * 32);
    const T* dh = static_cast<const T*>(a.dh);
    const bool vectors = reinterpret_cast<uintptr_t>(dh) % 16 == 0 && (a.rows == 1 || a.dh_stride % 8 == 0);
    const auto kernel = vectors ? k_gradient<T, true> : k_gradient<T, false>;
    kernel<<<(unsigned)blocks, 256, 0, s>>>(a.kept, a.kept_stride, dh, a.dh_stride, a.rows, a.n, a.act, dg, du, l.n_pitch, l.parts > 1);
  } else {
    make_ready(a, l, true, true, s);
    if (!tma_ready(a.dh, a.dh_stride, a.rows, a.n)) {
      PackArgs p{};
      p.from[0] = a.dh; p.stride[0] = a.dh_stride; p.rows[0] = a.rows; p.to[0] = ws + l.dh;
      p.cols = a.n;
      p.pitch = l.n_pitch;
      launch_pack(p, 1, a.rows, s);
      a.dh = ws + l.dh;
      a.dh_stride = l.n_pitch;
    }
    if ((e = products<T, kGradient>(a, dg, du, l.n_pitch, s)) != cudaSuccess) return e;
  }
  ProductArgs p{};
  p.partial = reinterpret_cast<float*>(ws + l.partial);
  if (a.dx) {
    p.parts = 2;
    const int64_t m = a.rows * l.parts;
    const Cut k = cut(kInput, m, a.k, a.n, 2, 1);
    const int box = a_box(m);
    if (!map_matrix(&p.a[0], kType<T>, dg, m, a.n, l.n_pitch, box) || !map_matrix(&p.a[1], kType<T>, du, m, a.n, l.n_pitch, box) ||
        !map_matrix(&p.b[0], kType<T>, a.w_gate, a.n, a.k, a.g_stride, 64) || !map_matrix(&p.b[1], kType<T>, a.w_up, a.n, a.k, a.u_stride, 64))
      return cudaErrorInvalidValue;
    p.m = (int)m; p.n = (int)a.k; p.c = (int)a.n; p.matrices = 1;
    p.out[0] = a.dx; p.out[1] = nullptr; p.stride = a.dx_stride;
    if ((e = launch_product(kInput, kType<T>, p, k, s, l.parts > 1)) != cudaSuccess) return e;
  }
  if (weights) {
    const Cut k = cut(kWeight, a.n, a.k, a.rows, l.parts, 2);
    p.matrices = 0;
    p.parts = l.parts;
    for (int w = 0; w < 2; w++) {
      void* out = w ? a.dw_up : a.dw_gate;
      if (!out) continue;
      for (int half = 0; half < l.parts; half++)
        if (!map_matrix(&p.a[p.matrices * l.parts + half], kType<T>, (w ? du : dg) + half * a.rows * l.n_pitch, a.rows, a.n, l.n_pitch, 64))
          return cudaErrorInvalidValue;
      p.out[p.matrices++] = out;
    }
    if (!map_matrix(&p.b[0], kType<T>, a.x, a.rows, a.k, a.x_stride, 64)) return cudaErrorInvalidValue;
    p.m = (int)a.n; p.n = (int)a.k; p.c = (int)a.rows; p.stride = a.k;
    if (p.matrices == 1) p.out[1] = nullptr;
    if ((e = launch_product(kWeight, kType<T>, p, k, s)) != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace

cudaError_t launch_gated_forward(const GatedArgs& a, ndvm_dtype t, cudaStream_t s) {
  return t == NDVM_F16 ? forward<__half>(a, s) : forward<__nv_bfloat16>(a, s);
}
cudaError_t launch_gated_backward(const GatedArgs& a, ndvm_dtype t, cudaStream_t s) {
  return t == NDVM_F16 ? backward<__half>(a, s) : backward<__nv_bfloat16>(a, s);
}
size_t gated_workspace(int64_t rows, int64_t k, int64_t n, bool backward, bool copies) {
  if (rows == 0 || (!backward && rows == 1)) return 0;
  return Layout(rows, k, n, backward, copies).total;
}
size_t gated_workspace(const GatedArgs& a, bool backward) { return gated_workspace(a.rows, a.k, a.n, backward, !all_ready(a)); }

}  // namespace ndvm
