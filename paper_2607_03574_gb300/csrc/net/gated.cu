// Gated projection h = act(G) U with G = x Wg^T, U = x Wu^T, and its backward pass:
//   dU = dh act(G), dG = dh U act'(G), dx = dG Wg + dU Wu, dWg = dG^T x, dWu = dU^T x.
// The backward pass computes G and U again, or takes those that the forward pass kept: in binary32 (8 bytes an
// element of h), so that dG and dU are rounded once, to the operands' type, which the next products need (and
// where there are few of them, not even that: in_halves).
//
// All products run in one kernel frame (k_product): D[m, n] = sum over c of A[m, c] B[n, c], 128 rows a tile,
// operands by TMA, sums in tensor memory.
//   forward   A = x, B = a tile's rows of Wg and then of Wu: G and U land in the two halves of a tile's columns
//   gradient  the same products; the epilogue reads dh and writes dG and dU to the workspace
//   dx        A = dG, B = Wg^T, then A = dU, B = Wu^T into the same sums
//   dW        A = dG^T (or dU^T), B = x^T
// Transposes are read as they lie: the operand's rows are contiguous instead of its contraction.
#include <atomic>

#include "net.h"
#include "tc.cuh"
#include "types.cuh"

namespace ndvm {
namespace {

__device__ int g_stopped;  // a wait in k_product ran out (ndvm_check_operators)

// act(g) and act'(g), two at a time: off by a few units of binary32's last place, and by a share of |g| (gelu: g^2) of
// them where the value itself vanishes.  Powers of two and reciprocals are the hardware's.
__device__ __forceinline__ float power2(float x) {  // (down to binary32's smallest)
  float y;
  asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float reciprocal(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <int kAct>
__device__ __forceinline__ void activate(float2 g, float2* a, float2* da) {
  const float2 one = make_float2(1.0f, 1.0f);
  if constexpr (kAct == NDVM_ACT_RELU) {
    *a = make_float2(g.x > 0.0f ? g.x : (g.x != g.x ? g.x : 0.0f), g.y > 0.0f ? g.y : (g.y != g.y ? g.y : 0.0f));
    *da = make_float2(g.x > 0.0f ? 1.0f : 0.0f, g.y > 0.0f ? 1.0f : 0.0f);
  } else if constexpr (kAct == NDVM_ACT_GELU) {
    // The normal distribution function by its tail, cdf(-|g|) = e^(-g^2 / 2) t Q(t) with t = 1 / (1 + 0.35 |g|): relative
    // accuracy on both sides (1 + erf cancels below zero, to 4 % at -5 and to nothing from -5.5 on).  Q is the polynomial
    // of degree 8 with the least largest relative error on 0 <= |g| <= 15 (3.2e-8), by reweighted least squares.
    const float2 q = mul(mul(g, g), make_float2(-0.72134752f, -0.72134752f));  // -g^2 / 2 in powers of two
    const float2 e = make_float2(power2(q.x), power2(q.y));
    const float2 d = make_float2(fmaf(fabsf(g.x), 0.35f, 1.0f), fmaf(fabsf(g.y), 0.35f, 1.0f));
    const float2 t = make_float2(reciprocal(d.x), reciprocal(d.y));
    constexpr float kQ[9] = {0.139621258f, 0.139864326f,  0.119815566f, 0.105574533f,   -0.0232631564f,
                             0.15939188f,  -0.255900919f, 0.144060329f, -0.0291638281f};
    float2 tail = make_float2(kQ[8], kQ[8]);
#pragma unroll
    for (int i = 7; i >= 0; i--) tail = fma(tail, t, make_float2(kQ[i], kQ[i]));
    tail = mul(mul(e, t), tail);
    const float2 cdf = make_float2(g.x < 0.0f ? tail.x : 1.0f - tail.x, g.y < 0.0f ? tail.y : 1.0f - tail.y);
    *a = mul(g, cdf);
    *da = fma(mul(g, e), make_float2(0.39894228f, 0.39894228f), cdf);
  } else {
    // s = 1 / (1 + e^-g) and 1 - s are r and e r, with e = e^-|g| and r = 1 / (1 + e), the one or the other way round: nothing
    // cancels, overflows or is flushed in either tail
    const float2 e = make_float2(power2(fabsf(g.x) * -1.44269504f), power2(fabsf(g.y) * -1.44269504f));
    const float2 d = add(e, one), r = make_float2(reciprocal(d.x), reciprocal(d.y)), er = mul(e, r);
    const float2 s = make_float2(g.x < 0.0f ? er.x : r.x, g.y < 0.0f ? er.y : r.y);
    const float2 rest = make_float2(g.x < 0.0f ? r.x : er.x, g.y < 0.0f ? r.y : er.y);
    *a = kAct == NDVM_ACT_SILU ? mul(g, s) : s;
    *da = kAct == NDVM_ACT_SILU ? fma(*a, rest, s) : mul(s, rest);
  }
}
// f(activation as a constant): one branch around a loop over many elements, not one in each
template <typename F>
__device__ __forceinline__ void by_activation(int act, F&& f) {
  if (act == NDVM_ACT_SILU) f(std::integral_constant<int, NDVM_ACT_SILU>());
  else if (act == NDVM_ACT_GELU) f(std::integral_constant<int, NDVM_ACT_GELU>());
  else if (act == NDVM_ACT_RELU) f(std::integral_constant<int, NDVM_ACT_RELU>());
  else f(std::integral_constant<int, NDVM_ACT_SIGMOID>());
}

// ------------------------------------------------------------------ products on the tensor cores
enum Mode { kForward, kGradient, kInput, kWeight };

constexpr int kM = 128, kC = 64;  // rows of a tile, contraction of a step (128 bytes)
constexpr int kReaders = 8;       // warps that read the sums: two for each quarter of a tile's rows
constexpr int kThreads = 64 + 32 * kReaders;  // and one that loads, one that multiplies

__host__ __device__ constexpr bool a_rows(Mode m) { return m == kWeight; }
__host__ __device__ constexpr bool b_rows(Mode m) { return m == kInput || m == kWeight; }
__host__ __device__ constexpr bool dual(Mode m) { return m == kForward || m == kGradient; }

// A block's share: kN columns of sums for its 128 rows, of whose operand B a pair's blocks hold half each.
template <int kN, int kCtas> constexpr int kStageBytes = (kM + kN / kCtas) * kC * 2;
// Of each warp that reads sums: what its stores are made from (twice as much for a block alone would cost it a stage:
// 16384 x 512 -> 2048 forward 54 -> 58 us), and two pieces of dh that it has asked for.
template <Mode kMode, int kCtas> constexpr int kStaging = kMode == kGradient ? 4096 : 4096 * kCtas;
template <Mode kMode> constexpr int kAsked = kMode == kGradient ? 4096 : 0;
template <Mode kMode, int kN, int kCtas>
constexpr int kStages = std::min(8, (229376 - kReaders * (kStaging<kMode, kCtas> + kAsked<kMode>)) / kStageBytes<kN, kCtas>);
template <Mode kMode, int kN, int kCtas>
constexpr int kSmem = kStages<kMode, kN, kCtas> * kStageBytes<kN, kCtas> + kReaders * (kStaging<kMode, kCtas> + kAsked<kMode>) +
                      1024 /* alignment */ + 384 /* barriers */;

struct ProductArgs {
  CUtensorMap a[4], b[2];        // kWeight: a's are gate's parts, then up's
  CUtensorMap o[2];              // the results (kGradient: dG and dU), or o[0] the split sums
  CUtensorMap dh;                // kGradient
  CUtensorMap kept;              // kForward: where G and U go in binary32, if keep
  int keep;
  int m, n, c;                   // rows and columns of the result, contraction of one segment
  int tiles_m, tiles_n, matrices;  // matrices: results of one shape, by the a's (kWeight: 1 or 2), else 1
  int parts;                     // kWeight: segments of a matrix (dG, or its two halves)
  int steps, splits;             // contraction steps of a result, and how many parts they are cut into
  int act;
  int a_box;                     // rows of A that a tile loads (fewer than 128 where the result has fewer)
  int sums;                      // results are binary32 sums, which k_join finishes
  int copies;                    // results are stored by copies (their rows start on 16 bytes)
  void* out[2]; int64_t stride;  // kWeight: both matrices'; kGradient: dG and dU; else out[0]
  float* partial; int64_t partial_pitch;  // splits > 1: [split][matrix][m][pitch]
};

// 32 values of a row to the staging buffer, in the 64-byte swizzle (a line of 64 bytes a row: the 16-byte
// pieces of two lines that share banks are spread over all of them)
template <typename T>
__device__ __forceinline__ void stage_row(uint32_t buffer, int lane, const float (&v)[32]) {
#pragma unroll
  for (int q = 0; q < 4; q++) {
    union { uint4 u; T t[8]; } o;
#pragma unroll
    for (int e = 0; e < 8; e += 2) narrow(o.t + e, make_float2(v[q * 8 + e], v[q * 8 + e + 1]));
    tc::store16(buffer + lane * 64 + ((q ^ (lane >> 1 & 3)) << 4), o.u);
  }
}
// and as they are, a line of 128 bytes a row, in the 128-byte swizzle
__device__ __forceinline__ void stage_row(uint32_t buffer, int lane, const float (&v)[32]) {
#pragma unroll
  for (int q = 0; q < 8; q++)
    tc::store16(buffer + lane * 128 + ((q ^ (lane & 7)) << 4),
                make_uint4(__float_as_uint(v[q * 4]), __float_as_uint(v[q * 4 + 1]), __float_as_uint(v[q * 4 + 2]),
                           __float_as_uint(v[q * 4 + 3])));
}
// the buffer's rows to rows that start anywhere, a row at a time
template <typename T>
__device__ __forceinline__ void unstage(const char* buffer, int lane, T* out, int64_t stride, int rows, int cols) {
  for (int r = 0; r < rows; r++)
    if (lane < cols) out[r * stride + lane] = *reinterpret_cast<const T*>(buffer + r * 64 + ((lane / 8 ^ (r >> 1 & 3)) << 4) + lane % 8 * 2);
}

template <typename T, Mode kMode, int kN, int kCtas>
__global__ void __launch_bounds__(kThreads, 1) k_product(const __grid_constant__ ProductArgs p) {
  extern __shared__ char raw[];
  constexpr int S = kStages<kMode, kN, kCtas>, kStage = kStageBytes<kN, kCtas>;
  constexpr uint32_t kABytes = kM * kC * 2;
  constexpr int kColumns = 2 * kN;  // of tensor memory: two tiles' sums
  constexpr int kOutN = dual(kMode) ? kN / 2 : kN;
  __shared__ uint32_t s_tmem;
  __shared__ int s_stop;
  const uint32_t base = (tc::smem(raw) + 1023) & ~1023u;
  const uint32_t staging = base + S * kStage, asked_at = staging + kReaders * kStaging<kMode, kCtas>;
  const uint32_t bars = asked_at + kReaders * kAsked<kMode>;
  const auto full = [&](int i) { return bars + i * 8; };
  const auto empty = [&](int i) { return bars + (S + i) * 8; };
  const auto done = [&](int i) { return bars + (2 * S + i) * 8; };       // a tile's sums are complete
  const auto taken = [&](int i) { return bars + (2 * S + 2 + i) * 8; };  // and have been read
  const uint32_t drain = bars + (2 * S + 4) * 8;
  const auto dh_in = [&](int reader, int b) { return bars + (2 * S + 5 + 2 * reader + b) * 8; };  // a piece of dh has come
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  const int rank = kCtas == 1 ? 0 : (int)tc::cluster_rank(), unit = blockIdx.x / kCtas, units = gridDim.x / kCtas;
  volatile int* stop = &s_stop;

  if (threadIdx.x == 0) {
    s_stop = 0;
    for (int i = 0; i < S; i++) tc::barrier_init(full(i), 1), tc::barrier_init(empty(i), 1);
    for (int i = 0; i < 2; i++) tc::barrier_init(done(i), 1), tc::barrier_init(taken(i), kReaders * kCtas);
    tc::barrier_init(drain, 1);
    if (kMode == kGradient)
      for (int i = 0; i < 2 * kReaders; i++) tc::barrier_init(dh_in(i / 2, i % 2), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tc::tmem_alloc<kCtas, kColumns>(tc::smem(&s_tmem));
  tc::fence_before();
  __syncthreads();
  if (kCtas == 2) tc::cluster_sync();
  tc::fence_after();
  const uint32_t tmem = s_tmem;

  const int tiles = p.tiles_m * p.tiles_n, items = tiles * p.matrices * p.splits;
  const int segment = (p.c + kC - 1) / kC;  // steps of one segment
  struct Item { int m0, n0, matrix, split, from, to; };
  constexpr int kBand = 16 / kCtas;
  // tiles in bands of 2048 rows, down a band first: blocks that run together share operands in L2
  const auto item = [&](int i) {
    Item it;
    it.split = i / (tiles * p.matrices);
    i -= it.split * (tiles * p.matrices);
    it.matrix = i / tiles;
    i -= it.matrix * tiles;
    const int band = i / (kBand * p.tiles_n), first = band * kBand, height = min(kBand, p.tiles_m - first);
    i -= band * kBand * p.tiles_n;
    it.m0 = ((first + i % height) * kCtas + rank) * kM;
    it.n0 = i / height * kOutN;
    it.from = (int)((int64_t)p.steps * it.split / p.splits);
    it.to = (int)((int64_t)p.steps * (it.split + 1) / p.splits);
    return it;
  };

  if (warp == 0 && lane == 0) {
    // ---- loads
    int stage = 0;
    uint32_t phase = 0;
    int issued = 0;
    bool ok = true;
    for (int i = unit; ok && i < items; i += units) {
      const Item it = item(i);
      for (int s = it.from; s < it.to; s++) {
        if (!(ok = tc::barrier_wait(empty(stage), phase ^ 1, stop))) break;
        const uint32_t a = base + stage * kStage, b = a + kABytes, bar = kCtas == 1 ? full(stage) : tc::in_first(full(stage));
        const int bytes = a_rows(kMode) ? kStage : kStage - (int)kABytes + p.a_box * kC * 2;
        if (rank == 0) tc::barrier_expect(full(stage), kCtas * bytes);
        const int part = kMode == kInput || kMode == kWeight ? s / segment : 0, seg = kMode == kWeight ? it.matrix * p.parts + part : part;
        const int c = (s - part * segment) * kC;
        if (a_rows(kMode)) {
          for (int q = 0; q < kM / 64; q++) tc::load_box<kCtas>(a + q * 8192, &p.a[seg], it.m0 + q * 64, c, bar);
        } else {
          tc::load_box<kCtas>(a, &p.a[seg], c, it.m0, bar);
        }
        if (dual(kMode) && kCtas == 2) {
          tc::load_box<kCtas>(b, &p.b[rank], c, it.n0, bar);
        } else if (dual(kMode)) {
          tc::load_box<kCtas>(b, &p.b[0], c, it.n0, bar);
          tc::load_box<kCtas>(b + kN / 2 * kC * 2, &p.b[1], c, it.n0, bar);
        } else {
          for (int q = 0; q < kN / kCtas / 64; q++)
            tc::load_box<kCtas>(b + q * 8192, &p.b[kMode == kInput ? seg : 0], it.n0 + rank * (kN / kCtas) + q * 64, c, bar);
        }
        issued++;
        if (++stage == S) stage = 0, phase ^= 1;
      }
    }
    // The block stays until the products have let go of its stages (their arrivals come from outside, a pair's from
    // the other block too); if the launch gives up, until its copies have landed (a pair's second waits for its first).
    for (int k = min(issued, S); k >= 1; k--) {
      const int at = (issued - k) % S, turn = (issued - k) / S;
      if (ok) ok = tc::barrier_wait(empty(at), turn & 1, stop);
      if (!ok && rank == 0) tc::barrier_drain(full(at), turn & 1);
    }
  } else if (warp == 1 && lane == 0 && rank == 0) {
    // ---- products
    constexpr uint32_t desc = tc::instruction(std::is_same<T, __nv_bfloat16>::value, a_rows(kMode), b_rows(kMode), kM * kCtas, kN);
    int stage = 0, slot = 0;
    uint32_t phase = 0, slot_phase = 0;
    bool ok = true;
    for (int i = unit; ok && i < items; i += units) {
      const Item it = item(i);
      if (!(ok = tc::barrier_wait(taken(slot), slot_phase ^ 1, stop))) break;
      tc::fence_after();
      for (int s = it.from; s < it.to; s++) {
        if (!(ok = tc::barrier_wait(full(stage), phase, stop))) break;
        tc::fence_after();
        const uint32_t at = base + stage * kStage;
        const uint64_t a = tc::operand(at, a_rows(kMode)), b = tc::operand(at + kABytes, b_rows(kMode));
#pragma unroll
        for (int q = 0; q < kC / 16; q++)  // 16 of the contraction: 32 bytes along a line, or 16 lines
          tc::mma<kCtas>(tmem + slot * kN, a + q * (a_rows(kMode) ? 2048 >> 4 : 32 >> 4), b + q * (b_rows(kMode) ? 2048 >> 4 : 32 >> 4),
                  desc, s > it.from || q > 0);
        tc::commit<kCtas>(empty(stage));
        if (++stage == S) stage = 0, phase ^= 1;
      }
      tc::commit<kCtas>(done(slot));
      if (++slot == 2) slot = 0, slot_phase ^= 1;
    }
    if (!ok) {  // the products in flight end before tensor memory is freed
      tc::commit<kCtas>(drain);
      tc::barrier_drain(drain, 0);
    }
  } else if (warp >= 2) {
    // ---- sums to memory: a warp reads the 32 lanes (rows of the tile) that are its own, every other 32
    // columns, by way of staging that asynchronous copies empty.  (Two warps a scheduler: one alone left the
    // latencies of the reads, the copies and dh in the open: backward of 4096 x 1024 -> 4096 174 and 159 us.)
    const int lanes = (warp % 4) * 32;
    const uint32_t mine = staging + (warp - 2) * kStaging<kMode, kCtas>;
    const char* const mine_ptr = raw + (mine - tc::smem(raw));
    const int first = (warp - 2) / 4 * 32;
    int slot = 0, buffer = 0;
    uint32_t slot_phase = 0;
    // kGradient: the pieces of dh that this warp needs, in the order it needs them, two of them asked for ahead
    const int reader = warp - 2;
    struct Place { int i, j; Item it; } ask{unit, first, {}};
    const auto settle = [&] {  // past the tiles that have no columns of this warp's
      while (ask.i < items && ask.it.n0 + first >= p.n) {
        ask.i += units;
        if (ask.i < items) ask.it = item(ask.i);
      }
    };
    int asked = 0, had = 0;
    const auto ask_next = [&] {
      if (ask.i >= items) return;
      if (lane == 0) {
        const uint32_t bar = dh_in(reader, asked & 1);
        tc::barrier_expect(bar, 2048);
        tc::load_box<1>(asked_at + reader * kAsked<kMode> + (asked & 1) * 2048, &p.dh, ask.it.n0 + ask.j, ask.it.m0 + lanes, bar);
      }
      asked++;
      ask.j += 64;
      if (ask.j >= kOutN || ask.it.n0 + ask.j >= p.n) {
        ask.j = first;
        ask.i += units;
        if (ask.i < items) ask.it = item(ask.i);
        settle();
      }
    };
    if (kMode == kGradient) {
      if (first >= kOutN) ask.i = items;
      if (ask.i < items) ask.it = item(ask.i);
      settle();
      ask_next();
      ask_next();
    }
    bool ok = true;
    for (int i = unit; ok && i < items; i += units) {
      const Item it = item(i);
      const int row0 = it.m0 + lanes;
      // (the whole warp goes on or gives up: reading tensor memory is a warp's instruction)
      if (!__all_sync(~0u, tc::barrier_wait(done(slot), slot_phase, stop))) break;
      tc::fence_after();
      const uint32_t at = tmem + slot * kN + ((uint32_t)lanes << 16);
#pragma unroll 1
      for (int j = first; ok && j < kOutN; j += 64) {
        const int col = it.n0 + j, count = min(32, p.n - col);
        if (count <= 0) break;
        float v[32], u[32];
        Pack<T, 8> dh[4];
        tc::tmem_load32(v, at + j);
        if (dual(kMode)) tc::tmem_load32(u, at + kN / 2 + j);
        if (kMode == kGradient) {
          const int b = had & 1;
          ok = __all_sync(~0u, tc::barrier_wait(dh_in(reader, b), had >> 1 & 1, stop));
          const char* from = raw + (asked_at - tc::smem(raw)) + reader * kAsked<kMode> + b * 2048 + lane * 64;
#pragma unroll
          for (int q = 0; q < 4; q++) dh[q] = load_pack<T, 8>(reinterpret_cast<const T*>(from + ((q ^ (lane >> 1 & 3)) << 4)));
          __syncwarp();
          if (ok) had++, ask_next();
        }
        tc::tmem_loaded(v);
        if (dual(kMode)) tc::tmem_loaded(u);
        if (kMode == kForward && p.keep) {  // G and then U to memory, as binary32
          if (lane == 0) tc::stores_read<0>();
          __syncwarp();
          stage_row(mine, lane, v);
          if (kCtas == 2) stage_row(mine + 4096, lane, u);
          tc::fence_async();
          __syncwarp();
          if (lane == 0) {
            if (row0 < p.m) tc::store_box(&p.kept, col, row0, 0, mine);
            if (row0 < p.m && kCtas == 2) tc::store_box(&p.kept, col, row0, 1, mine + 4096);
            tc::stores_commit();
            if (kCtas == 1) tc::stores_read<0>();
          }
          if (kCtas == 1) {
            __syncwarp();
            stage_row(mine, lane, u);
            tc::fence_async();
            __syncwarp();
            if (lane == 0) {
              if (row0 < p.m) tc::store_box(&p.kept, col, row0, 1, mine);
              tc::stores_commit();
            }
          }
        }
        if (dual(kMode))
          by_activation(p.act, [&](auto act) {
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
              const float2 up = make_float2(u[e], u[e + 1]);
              float2 a, da, out;
              activate<decltype(act)::value>(make_float2(v[e], v[e + 1]), &a, &da);
              if (kMode == kForward) {
                out = mul(a, up);
              } else {
                const float2 d = widen(dh[e / 8].v + e % 8), other = mul(d, a);
                out = mul(mul(d, up), da);
                u[e] = other.x, u[e + 1] = other.y;
              }
              v[e] = out.x, v[e + 1] = out.y;
            }
          });
        // A piece takes 2048 bytes of 16-bit results, or 4096 for both of dG and dU or for binary32; while it is
        // made, the copies of as many others as the staging holds may be under way (none where it held G and U).
        constexpr int kSmall = kStaging<kMode, kCtas> / 2048, kLarge = kStaging<kMode, kCtas> / 4096;
        const bool large = kMode == kGradient || (!dual(kMode) && p.sums), alone = kMode == kForward && p.keep;
        const uint32_t to = mine + (alone ? 0 : large ? buffer % kLarge * 4096 : buffer * 2048);
        if (lane == 0) {
          if (alone) tc::stores_read<0>();
          else if (large) tc::stores_read<kLarge - 1>();
          else tc::stores_read<kSmall - 1>();
        }
        __syncwarp();
        if (!dual(kMode) && p.sums) {
          stage_row(to, lane, v);
          tc::fence_async();
          __syncwarp();
          if (lane == 0 && row0 < p.m) tc::store_box(&p.o[0], col, row0, it.split * p.matrices + it.matrix, to);
        } else {
          stage_row<T>(to, lane, v);
          if (kMode == kGradient) stage_row<T>(to + 2048, lane, u);
          if (p.copies) {
            tc::fence_async();
            __syncwarp();
            if (lane == 0 && row0 < p.m) {
              tc::store_box(&p.o[kMode == kWeight ? it.matrix : 0], col, row0, to);
              if (kMode == kGradient) tc::store_box(&p.o[1], col, row0, to + 2048);
            }
          } else {
            __syncwarp();
            T* out = static_cast<T*>(p.out[kMode == kWeight ? it.matrix : 0]) + row0 * p.stride + col;
            unstage<T>(mine_ptr + (to - mine), lane, out, p.stride, min(32, p.m - row0), count);
          }
        }
        if (lane == 0) tc::stores_commit();
        buffer = (buffer + 1) % kSmall;
      }
      tc::fence_before();
      __syncwarp();
      if (lane == 0) {
        if (kCtas == 1) tc::barrier_arrive(taken(slot));
        else tc::barrier_arrive_cluster(tc::in_first(taken(slot)));
      }
      if (++slot == 2) slot = 0, slot_phase ^= 1;
    }
    if (lane == 0) {
      tc::stores_read<0>();  // (what they write is there when the kernel ends)
      if (kMode == kGradient)  // (pieces that a launch that gave up has left)
        for (; had < asked; had++) tc::barrier_drain(dh_in(reader, had & 1), had >> 1 & 1);
    }
  }
  __syncwarp();
  __syncthreads();
  if (threadIdx.x == 0 && s_stop) g_stopped = 1;
  __syncwarp();
  tc::fence_before();
  if (kCtas == 2) tc::cluster_sync();  // neither block's memory is in the other's use any more
  tc::fence_after();
  if (warp == 1) tc::tmem_free<kCtas, kColumns>(tmem);
}

// the parts of split sums added up in order, and rounded: 4 columns a thread.  fold: each matrix's rows come
// twice, and are added up too.
template <typename T>
__global__ void __launch_bounds__(256) k_join(const float* partial, int64_t pitch, int splits, int matrices, int fold, int64_t m,
                                              int64_t n, T* out0, T* out1, int64_t stride) {
  const int64_t quads = pitch / 4, total = matrices * m * quads, part = total << fold;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / quads, c = (i - row * quads) * 4;
    const float* p = partial + (i + (fold && row >= m ? m * quads : 0)) * 4;
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (int k = 0; k < splits; k++) {
      const float4 v = *reinterpret_cast<const float4*>(p + k * part * 4);
      s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
      if (fold) {
        const float4 l = *reinterpret_cast<const float4*>(p + (k * part + m * quads) * 4);
        s.x += l.x, s.y += l.y, s.z += l.z, s.w += l.w;
      }
    }
    T* out = row >= m ? out1 + (row - m) * stride + c : out0 + row * stride + c;
    const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int e = 0; e < 4; e++)
      if (c + e < n) out[e] = from_f32<T>(v[e]);
  }
}

// what rounding v to the operands' type leaves, rounded too (0 beside what is not finite)
template <typename T>
__device__ __forceinline__ T rest_of(float v, T rounded) {
  const float r = to_f32(rounded);
  return from_f32<T>(fabsf(r) <= 3.0e38f ? v - r : 0.0f);
}
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

// Up to three matrices of `cols` columns to rows that start on 16 bytes (TMA reads no others): a warp a row, 16 bytes
// a lane, out of the one or two aligned 16-byte blocks that hold them.  What lies before and behind a row is not read
// (it need not be the caller's): the blocks at its two ends are read element by element.
struct PackArgs {
  const void* from[3];
  void* to[3];
  int64_t stride[3], rows[3];
  int64_t cols, pitch;
};
// the aligned 16 bytes at `block`, 0 where they are not of the row
__device__ __forceinline__ uint4 row_block(const char* block, const char* row, const char* end) {
  if (block >= row && block + 16 <= end) return *reinterpret_cast<const uint4*>(block);
  uint32_t e[8];
#pragma unroll
  for (int i = 0; i < 8; i++)
    e[i] = block + 2 * i >= row && block + 2 * i < end ? *reinterpret_cast<const uint16_t*>(block + 2 * i) : 0;
  return make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
}
__global__ void __launch_bounds__(256) k_pack(const __grid_constant__ PackArgs a) {
  const int w = blockIdx.y, lane = threadIdx.x % 32;
  for (int64_t row = (int64_t)blockIdx.x * 8 + threadIdx.x / 32; row < a.rows[w]; row += (int64_t)gridDim.x * 8) {
    const char* from = static_cast<const char*>(a.from[w]) + row * a.stride[w] * 2;
    char* to = static_cast<char*>(a.to[w]) + row * a.pitch * 2;
    const int off = (int)(reinterpret_cast<uintptr_t>(from) % 16);  // even, the same for all of the row's pieces
    const char* end = from + a.cols * 2;
    for (int64_t c = lane * 16; c < a.pitch * 2; c += 32 * 16) {
      const char* block = from + c - off;
      uint32_t v[9] = {};
      const uint4 p = row_block(block, from, end), q = off ? row_block(block + 16, from, end) : make_uint4(0, 0, 0, 0);
      v[0] = p.x, v[1] = p.y, v[2] = p.z, v[3] = p.w;
      v[4] = q.x, v[5] = q.y, v[6] = q.z, v[7] = q.w;
#pragma unroll
      for (int i = 0; i < 7; i++) v[i] = off & 8 ? v[i + 2] : v[i];
#pragma unroll
      for (int i = 0; i < 5; i++) v[i] = off & 4 ? v[i + 1] : v[i];
      const int bits = off % 4 * 8;
      *reinterpret_cast<uint4*>(to + c) = make_uint4(__funnelshift_r(v[0], v[1], bits), __funnelshift_r(v[1], v[2], bits),
                                                     __funnelshift_r(v[2], v[3], bits), __funnelshift_r(v[3], v[4], bits));
    }
  }
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
constexpr int kSms = 152;

int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

bool tma_ready(const void* p, int64_t stride, int64_t rows, int64_t cols) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows == 1 || (stride % 8 == 0 && stride >= cols));
}

using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                            const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                            CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
Encode encoder() {
  static const Encode e = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      f = nullptr;
    return reinterpret_cast<Encode>(f);
  }();
  return e;
}

// A matrix of `rows` rows of `cols` contiguous elements, read in boxes of 64 columns and `box` rows in the
// 128-byte swizzle; or in boxes of 32 by 32 (results, and dh: 64 bytes a row, the 64-byte swizzle).
template <typename T>
bool map_matrix(CUtensorMap* map, const void* p, int64_t rows, int64_t cols, int64_t stride, int box, bool piece = false) {
  if (!encoder()) return false;
  if (rows == 1) stride = up(cols, 8);  // (never taken)
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride * 2};
  const cuuint32_t boxes[2] = {piece ? 32u : 64u, (cuuint32_t)box}, ones[2] = {1, 1};
  const CUtensorMapDataType type = std::is_same<T, __half>::value ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  return encoder()(map, type, 2, const_cast<void*>(p), dims, strides, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   piece ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// split sums: `parts` matrices of m rows, written in boxes of 32 by 32
bool map_partial(CUtensorMap* map, float* p, int64_t parts, int64_t m, int64_t n, int64_t pitch) {
  if (!encoder()) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)n, (cuuint64_t)m, (cuuint64_t)parts};
  const cuuint64_t strides[2] = {(cuuint64_t)pitch * 4, (cuuint64_t)(pitch * m) * 4};
  const cuuint32_t boxes[3] = {32, 32, 1}, ones[3] = {1, 1, 1};
  return encoder()(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, p, dims, strides, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, Mode kMode, int kN, int kCtas>
cudaError_t launch_width(const ProductArgs& p, cudaStream_t s) {
  static std::atomic<uint64_t> allowed{0};  // devices on which the kernel may take its shared memory
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  if (device >= 64 || !(allowed.load(std::memory_order_relaxed) >> device & 1)) {
    e = cudaFuncSetAttribute(k_product<T, kMode, kN, kCtas>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem<kMode, kN, kCtas>);
    if (e != cudaSuccess) return e;
    if (device < 64) allowed.fetch_or((uint64_t)1 << device, std::memory_order_relaxed);
  }
  const int items = p.tiles_m * p.tiles_n * p.matrices * p.splits;
  cudaLaunchConfig_t c{};
  c.gridDim = dim3((unsigned)std::min(items, kSms / kCtas) * kCtas);
  c.blockDim = dim3(kThreads);
  c.dynamicSmemBytes = kSmem<kMode, kN, kCtas>;
  c.stream = s;
  cudaLaunchAttribute cluster{};
  cluster.id = cudaLaunchAttributeClusterDimension;
  cluster.val.clusterDim.x = kCtas;
  cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
  c.attrs = &cluster;
  c.numAttrs = kCtas == 1 ? 0 : 1;
  return cudaLaunchKernelEx(&c, k_product<T, kMode, kN, kCtas>, p);
}

// how a product of the given size is cut up: columns and rows of a tile's sums (256 rows are a pair's), parts
struct Cut { int width, ctas, splits; };

int a_box(int64_t m) { return (int)std::min<int64_t>(up(m, 8), kM); }

// The shape with the least estimated time, in steps of a tile 256 wide (0.27 us): a round of tiles takes its
// steps and about 8 more to fill and empty; narrower tiles' steps are shorter, but not in proportion (more bytes an
// operation), a pair's a little shorter (16384 x 2048 -> 8192 forward: 630 us alone, 576 in pairs) if there are 12 or
// more (pairs start and end together: 4096 x 256 -> 1024 takes 9.2 us alone, 10.6 in pairs).  Where tiles are fewer than
// SMs, a contraction is cut into parts of 8 steps or more, which costs the launch that joins them.  The weights'
// gradients are cut as if both were wanted: one of them alone has the same bits.
Cut cut(Mode mode, int64_t m, int64_t n, int64_t c, int parts = 1) {
  struct Shape { int width, ctas; double step; };
  static constexpr Shape shapes[] = {{256, 2, 0.9}, {256, 1, 1.0}, {128, 1, 0.6}, {64, 1, 0.4}};
  const int matrices = mode == kWeight ? 2 : 1;
  const int64_t steps = ceil_div(c, kC) * (mode == kInput ? 2 : mode == kWeight ? parts : 1);
  Cut best{};
  double least = 1e300;
  for (const Shape& s : shapes) {
    if (s.ctas == 2 && steps < 12) continue;
    const int64_t units = kSms / s.ctas, tiles = matrices * ceil_div(m, kM * s.ctas) * ceil_div(n, dual(mode) ? s.width / 2 : s.width);
    const int64_t splits = dual(mode) || tiles >= units ? 1 : std::clamp<int64_t>(units / tiles, 1, std::max<int64_t>(steps / 8, 1));
    const double time = (double)ceil_div(tiles * splits, units) * ((double)ceil_div(steps, splits) * s.step + 8) + (splits > 1 ? 13 : 0);
    if (time < least) least = time, best = Cut{s.width, s.ctas, (int)splits};
  }
  return best;
}

template <typename T, Mode kMode>
cudaError_t launch_product(ProductArgs& p, const Cut& k, cudaStream_t s, bool fold = false) {
  const int out = dual(kMode) ? k.width / 2 : k.width;
  p.tiles_m = (int)ceil_div(p.m, kM * k.ctas);
  p.tiles_n = (int)ceil_div(p.n, out);
  p.steps = (int)ceil_div(p.c, kC) * (kMode == kInput ? 2 : kMode == kWeight ? p.parts : 1);
  p.splits = k.splits;
  p.a_box = a_rows(kMode) ? kM : a_box(p.m);
  p.copies = 1;
  p.sums = p.splits > 1 || fold;
  if (p.sums) {
    p.partial_pitch = up(p.n, 4);
    if (!map_partial(&p.o[0], p.partial, (int64_t)p.splits * p.matrices, p.m, p.n, p.partial_pitch)) return cudaErrorInvalidValue;
  } else {
    for (int w = 0; w < 2; w++) {
      if (!p.out[w]) continue;
      p.copies &= tma_ready(p.out[w], p.stride, p.m, p.n);
      if (p.copies && !map_matrix<T>(&p.o[w], p.out[w], p.m, p.n, p.stride, 32, true)) return cudaErrorInvalidValue;
    }
  }
  if ((int64_t)p.tiles_m * p.tiles_n * p.matrices * p.splits > 0x40000000) return cudaErrorInvalidConfiguration;
  const cudaError_t e = k.ctas == 2      ? launch_width<T, kMode, 256, 2>(p, s)
                        : k.width == 256 ? launch_width<T, kMode, 256, 1>(p, s)
                        : k.width == 128 ? launch_width<T, kMode, 128, 1>(p, s)
                                         : launch_width<T, kMode, 64, 1>(p, s);
  if (e != cudaSuccess || !p.sums) return e;
  const int64_t m = fold ? p.m / 2 : p.m, total = (int64_t)p.matrices * m * p.partial_pitch / 4;
  k_join<T><<<(unsigned)std::min<int64_t>(ceil_div(total, 256), kSms * 8), 256, 0, s>>>(
      p.partial, p.partial_pitch, p.splits, p.matrices, fold, m, p.n, static_cast<T*>(p.out[0]), static_cast<T*>(p.out[1]), p.stride);
  return cudaGetLastError();
}

// Few elements: dG and dU are handed on in two halves of 16 bits, so that next to nothing is lost before the last
// rounding.  (Over many elements the rounding of dG and dU adds to the results' own as squares add, 1.41 times in
// all; over few it scatters, to more than twice: 4096 elements leave 1.2 to 1.55, 16384 1.37 to 1.49.)  dx has the halves' rows
// one after the other in its tiles, the weights' gradients twice the steps, and G and U are made in binary32 first.  A step with
// the products kept, bf16, with and without halves: 8 x 2048 -> 8192 63 / 56 us, 16 x 1024 -> 4096 32 / 30, 64 x 256 -> 512 20.3 /
// 19.5, 4096 x 32 -> 64 23 / 20; the cost grows with the rows where n k is small (65536 x 32 -> 64 67 / 52, and 77 / 50 with
// nothing kept) and with n where k is (1000 x 16 -> 8192 76 / 62).
bool in_halves(int64_t rows, int64_t k, int64_t n) { return rows * std::min(n, k) <= 16384 || n * k <= 2048; }

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
      const Cut i = cut(kInput, rows * parts, k, n), w = cut(kWeight, n, k, rows, parts);
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

void launch_pack(const PackArgs& p, int count, int64_t most_rows, cudaStream_t s) {
  const int64_t blocks = std::min<int64_t>(ceil_div(most_rows, 8), kSms * 32);
  k_pack<<<dim3((unsigned)blocks, (unsigned)count), 256, 0, s>>>(p);
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
  const Cut k = cut(kMode, a.rows, a.n, a.k);
  ProductArgs p{};
  if (!map_matrix<T>(&p.a[0], a.x, a.rows, a.k, a.x_stride, a_box(a.rows)) || !map_matrix<T>(&p.b[0], a.w_gate, a.n, a.k, a.g_stride, k.width / 2) ||
      !map_matrix<T>(&p.b[1], a.w_up, a.n, a.k, a.u_stride, k.width / 2))
    return cudaErrorInvalidValue;
  p.m = (int)a.rows; p.n = (int)a.n; p.c = (int)a.k;
  if (kMode == kForward && a.kept) {
    p.keep = 1;
    if (!map_partial(&p.kept, a.kept, 2, a.rows, a.n, a.kept_stride)) return cudaErrorInvalidValue;
  }
  p.matrices = 1;
  if (kMode == kGradient && !map_matrix<T>(&p.dh, a.dh, a.rows, a.n, a.dh_stride, 32, true)) return cudaErrorInvalidValue;
  p.act = a.act; p.out[0] = out0; p.out[1] = out1; p.stride = stride;
  return launch_product<T, kMode>(p, k, s);
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
  p.parts = l.parts;
  if (a.dx) {
    const int64_t m = a.rows * l.parts;
    const Cut k = cut(kInput, m, a.k, a.n);
    const int box = a_box(m);
    if (!map_matrix<T>(&p.a[0], dg, m, a.n, l.n_pitch, box) || !map_matrix<T>(&p.a[1], du, m, a.n, l.n_pitch, box) ||
        !map_matrix<T>(&p.b[0], a.w_gate, a.n, a.k, a.g_stride, 64) || !map_matrix<T>(&p.b[1], a.w_up, a.n, a.k, a.u_stride, 64))
      return cudaErrorInvalidValue;
    p.m = (int)m; p.n = (int)a.k; p.c = (int)a.n; p.matrices = 1;
    p.out[0] = a.dx; p.out[1] = nullptr; p.stride = a.dx_stride;
    if ((e = launch_product<T, kInput>(p, k, s, l.parts > 1)) != cudaSuccess) return e;
  }
  if (weights) {
    const Cut k = cut(kWeight, a.n, a.k, a.rows, l.parts);
    p.matrices = 0;
    for (int w = 0; w < 2; w++) {
      void* out = w ? a.dw_up : a.dw_gate;
      if (!out) continue;
      for (int half = 0; half < l.parts; half++)
        if (!map_matrix<T>(&p.a[p.matrices * l.parts + half], (w ? du : dg) + half * a.rows * l.n_pitch, a.rows, a.n, l.n_pitch, 64))
          return cudaErrorInvalidValue;
      p.out[p.matrices++] = out;
    }
    if (!map_matrix<T>(&p.b[0], a.x, a.rows, a.k, a.x_stride, 64)) return cudaErrorInvalidValue;
    p.m = (int)a.n; p.n = (int)a.k; p.c = (int)a.rows; p.stride = a.k;
    if (p.matrices == 1) p.out[1] = nullptr;
    if ((e = launch_product<T, kWeight>(p, k, s)) != cudaSuccess) return e;
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
cudaError_t gated_stopped(int* flag) {
  cudaError_t e = cudaMemcpyFromSymbol(flag, g_stopped, sizeof *flag);
  const int none = 0;
  if (e == cudaSuccess && *flag) e = cudaMemcpyToSymbol(g_stopped, &none, sizeof none);
  return e;
}

}  // namespace ndvm
