// The products of the gated projection and of the dense layers' backward passes, in one kernel frame: 128 rows a tile,
// operands by TMA, sums in tensor memory.
//   forward   A = x, B = a tile's rows of Wg and then of Wu: G and U land in the two halves of a tile's columns
//   gradient  the same products; the epilogue reads dh and writes dG and dU to the workspace
//   input     dx: A = dG, B = Wg^T, then A = dU, B = Wu^T into the same sums (a dense layer's: A = dz, B = w^T alone)
//   weight    dW: A = dG^T (or dU^T, dz^T), B = x^T
//   both      a dense layer's dw and dx in one launch
// Transposes are read as they lie: the operand's rows are contiguous instead of its contraction.
#include <atomic>
#include <cmath>
#include <cstdint>
#include <initializer_list>

#include "activation.cuh"
#include "product.h"
#include "tc.cuh"
#include "types.cuh"

namespace ndvm {
namespace {

__device__ int g_stopped;  // a wait in k_product ran out (ndvm_check_operators)

// Warps that read the sums: two for each quarter of a tile's rows, or four where each needs little staging.
template <Mode kMode> constexpr int kReaders = kMode == kForward || kMode == kGradient ? 8 : 16;
template <Mode kMode> constexpr int kThreads = 64 + 32 * kReaders<kMode>;  // and one that loads, one that multiplies

__host__ __device__ constexpr bool a_rows(Mode m) { return m == kWeight; }
__host__ __device__ constexpr bool b_rows(Mode m) { return m == kInput || m == kWeight || m == kBoth; }
__host__ __device__ constexpr bool dual(Mode m) { return m == kForward || m == kGradient; }

// A block's share: kN columns of sums for its 128 rows, of whose operand B a pair's blocks hold half each.
template <int kN, int kCtas> constexpr int kStageBytes = (kM + kN / kCtas) * kC * 2;
// Of each warp that reads sums: what its stores are made from (twice as much for a block alone would cost it a stage:
// 16384 x 512 -> 2048 forward 54 -> 58 us), and two pieces of dh that it has asked for.
template <Mode kMode, int kCtas> constexpr int kStaging = kMode == kForward ? 4096 * kCtas : 4096;
template <Mode kMode> constexpr int kAsked = kMode == kGradient ? 4096 : 0;
template <Mode kMode, int kN, int kCtas>
constexpr int kStages = std::min(8, (229376 - kReaders<kMode> * (kStaging<kMode, kCtas> + kAsked<kMode>)) / kStageBytes<kN, kCtas>);
template <Mode kMode, int kN, int kCtas>
constexpr int kSmem = kStages<kMode, kN, kCtas> * kStageBytes<kN, kCtas> + kReaders<kMode> * (kStaging<kMode, kCtas> + kAsked<kMode>) +
                      1024 /* alignment */ + 384 /* barriers */;

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
// What a launch computes: one product, or (kBoth) two, the one with the longer items first.  Of two, each unit takes every
// so-manieth of the first's items (full of them, the first `rest` units one more) and then of the second's: all units for `rounds`
// rounds, from there on those that did not have one more of the first's.
struct Single { ProductArgs of[1]; };
struct Double { ProductArgs of[2]; int full, rest, rounds; };
template <Mode kMode> using Launch = std::conditional_t<kMode == kBoth, Double, Single>;

template <typename T, Mode kMode, int kN, int kCtas>
__global__ void __launch_bounds__(kThreads<kMode>, 1) k_product(const __grid_constant__ Launch<kMode> launch) {
  extern __shared__ char raw[];
  constexpr int S = kStages<kMode, kN, kCtas>, kStage = kStageBytes<kN, kCtas>, R = kReaders<kMode>, kNext = R / 4 * 32;
  constexpr uint32_t kABytes = kM * kC * 2;
  constexpr int kColumns = 2 * kN;  // of tensor memory: two tiles' sums
  constexpr int kOutN = dual(kMode) ? kN / 2 : kN;
  __shared__ uint32_t s_tmem;
  __shared__ int s_stop;
  const uint32_t base = (tc::smem(raw) + 1023) & ~1023u;
  const uint32_t staging = base + S * kStage, asked_at = staging + R * kStaging<kMode, kCtas>;
  const uint32_t bars = asked_at + R * kAsked<kMode>;
  const auto full = [&](int i) { return bars + i * 8; };
  const auto empty = [&](int i) { return bars + (S + i) * 8; };
  const auto done = [&](int i) { return bars + (2 * S + i) * 8; };       // a tile's sums are complete
  const auto taken = [&](int i) { return bars + (2 * S + 2 + i) * 8; };  // and have been read
  const uint32_t drain = bars + (2 * S + 4) * 8;
  const auto dh_in = [&](int reader, int b) { return bars + (2 * S + 5 + 2 * reader + b) * 8; };  // a piece of dh has come
  const int warp = __shfl_sync(~0u, threadIdx.x / 32, 0), lane = threadIdx.x % 32;  // (the same for all of a warp, as the compiler sees)
  const int rank = kCtas == 1 ? 0 : (int)tc::cluster_rank(), unit = blockIdx.x / kCtas, units = gridDim.x / kCtas;
  volatile int* stop = &s_stop;

  if (threadIdx.x == 0) {
    s_stop = 0;
    for (int i = 0; i < S; i++) tc::barrier_init(full(i), 1), tc::barrier_init(empty(i), 1);
    for (int i = 0; i < 2; i++) tc::barrier_init(done(i), 1), tc::barrier_init(taken(i), R * kCtas);
    tc::barrier_init(drain, 1);
    if (kMode == kGradient)
      for (int i = 0; i < 2 * R; i++) tc::barrier_init(dh_in(i / 2, i % 2), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tc::tmem_alloc<kCtas, kColumns>(tc::smem(&s_tmem));
  tc::fence_before();
  __syncthreads();
  if (kCtas == 2) tc::cluster_sync();
  tc::fence_after();
  const uint32_t tmem = s_tmem;

  const auto count = [&](const ProductArgs& p) { return p.tiles_m * p.tiles_n * p.matrices * p.splits; };
  const int items0 = count(launch.of[0]), items = items0 + (kMode == kBoth ? count(launch.of[kMode == kBoth]) : 0);
  struct Item { int which, m0, n0, matrix, split, from, to; };
  constexpr int kBand = 16 / kCtas;
  // tiles in bands of 2048 rows, down a band first: blocks that run together share operands in L2
  const auto item = [&](int i) {
    Item it;
    it.which = kMode == kBoth && i >= items0;
    i -= it.which * items0;
    const ProductArgs& p = launch.of[it.which];
    const int tiles = p.tiles_m * p.tiles_n;
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
  const auto nth = [&](int r) {  // a unit's items; `items` and more: no more of them
    if constexpr (kMode != kBoth) {
      return r * units + unit;
    } else {
      const bool more = unit < launch.rest;
      if (r < launch.full + more) return r * units + unit;
      r -= launch.full + more;
      if (r < launch.rounds) return items0 + r * units + unit;
      return more ? items : items0 + launch.rounds * units + (r - launch.rounds) * (units - launch.rest) + unit - launch.rest;
    }
  };
  // whether an item's A has its rows contiguous, and not its contraction
  const auto rows_of = [&](const Item& it) { return kMode == kBoth ? launch.of[it.which].rows != 0 : a_rows(kMode); };

  // (the whole warp waits, and goes on or gives up)
  const auto wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(~0u, tc::barrier_wait(bar, parity, stop)) != 0; };
  if (warp == 0) {
    // ---- loads
    int stage = 0;
    uint32_t phase = 0;
    int issued = 0;
    bool ok = true;
    for (int r = 0, i = nth(0); ok && i < items; i = nth(++r)) {
      const Item it = item(i);
      const ProductArgs& p = launch.of[it.which];
      const bool a_r = rows_of(it);
      const int segment = (p.c + kC - 1) / kC;  // steps of one segment
      for (int s = it.from; s < it.to; s++) {
        if (!(ok = wait(empty(stage), phase ^ 1))) break;
        const int bytes = a_r ? kStage : kStage - (int)kABytes + p.a_box * kC * 2;
        const int part = dual(kMode) ? 0 : s / segment, seg = a_r ? it.matrix * p.parts + part : part;
        const int c = (s - part * segment) * kC;
        if (tc::elect()) {
          const uint32_t a = base + stage * kStage, b = a + kABytes, bar = kCtas == 1 ? full(stage) : tc::in_first(full(stage));
          if (rank == 0) tc::barrier_expect(full(stage), kCtas * bytes);
          if (a_r) {
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
              tc::load_box<kCtas>(b + q * 8192, &p.b[a_r ? 0 : seg], it.n0 + rank * (kN / kCtas) + q * 64, c, bar);
          }
        }
        __syncwarp();
        issued++;
        if (++stage == S) stage = 0, phase ^= 1;
      }
    }
    // The block stays until the products have let go of its stages (their arrivals come from outside, a pair's from
    // the other block too); if the launch gives up, until its copies have landed (a pair's second waits for its first).
    for (int k = min(issued, S); k >= 1; k--) {
      const int at = (issued - k) % S, turn = (issued - k) / S;
      if (ok) ok = wait(empty(at), turn & 1);
      if (!ok && rank == 0) tc::barrier_drain(full(at), turn & 1);
    }
  } else if (warp == 1 && rank == 0) {
    // ---- products
    int stage = 0, slot = 0;
    uint32_t phase = 0, slot_phase = 0;
    bool ok = true;
    for (int r = 0, i = nth(0); ok && i < items; i = nth(++r)) {
      const Item it = item(i);
      const bool a_r = rows_of(it);
      const uint32_t desc = tc::instruction(std::is_same<T, __nv_bfloat16>::value, a_r, b_rows(kMode), kM * kCtas, kN);
      if (!(ok = wait(taken(slot), slot_phase ^ 1))) break;
      tc::fence_after();
      for (int s = it.from; s < it.to; s++) {
        if (!(ok = wait(full(stage), phase))) break;
        tc::fence_after();
        if (tc::elect()) {
          const uint32_t at = base + stage * kStage;
          const uint64_t a = tc::operand(at, a_r), b = tc::operand(at + kABytes, b_rows(kMode));
#pragma unroll
          for (int q = 0; q < kC / 16; q++)  // 16 of the contraction: 32 bytes along a line, or 16 lines
            tc::mma<kCtas>(tmem + slot * kN, a + q * (a_r ? 2048 >> 4 : 32 >> 4), b + q * (b_rows(kMode) ? 2048 >> 4 : 32 >> 4),
                           desc, s > it.from || q > 0);
          tc::commit<kCtas>(empty(stage));
          if (s + 1 == it.to) tc::commit<kCtas>(done(slot));
        }
        __syncwarp();
        if (++stage == S) stage = 0, phase ^= 1;
      }
      if (++slot == 2) slot = 0, slot_phase ^= 1;
    }
    if (!ok) {  // the products in flight end before tensor memory is freed
      if (tc::elect()) tc::commit<kCtas>(drain);
      __syncwarp();
      tc::barrier_drain(drain, 0);
    }
  } else if (warp >= 2) {
    // ---- sums to memory: a warp reads the 32 lanes (rows of the tile) that are its own, 32 columns at a time, by way of
    // staging that asynchronous copies empty.  (Two warps a scheduler or four: one alone left the latencies of the reads, the
    // copies and dh in the open.)
    const int lanes = (warp % 4) * 32;
    const uint32_t mine = staging + (warp - 2) * kStaging<kMode, kCtas>;
    const char* const mine_ptr = raw + (mine - tc::smem(raw));
    const int first = (warp - 2) / 4 * 32;
    int slot = 0, buffer = 0;
    uint32_t slot_phase = 0;
    bool was_large = false;  // (kBoth: of one product binary32 sums are staged, of the other results)
    // kGradient: the pieces of dh that this warp needs, in the order it needs them, two of them asked for ahead
    const int reader = warp - 2;
    const ProductArgs& p = launch.of[0];
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
      ask.j += kNext;
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
    for (int r = 0, i = nth(0); ok && i < items; i = nth(++r)) {
      const Item it = item(i);
      const ProductArgs& p = launch.of[it.which];
      const int row0 = it.m0 + lanes;
      if (!wait(done(slot), slot_phase)) break;
      tc::fence_after();
      const uint32_t at = tmem + slot * kN + ((uint32_t)lanes << 16);
#pragma unroll 1
      for (int j = first; ok && j < kOutN; j += kNext) {
        const int col = it.n0 + j, count = min(32, p.n - col);
        if (count <= 0) break;
        float v[32], u[32];
        Pack<T, 8> dh[4];
        tc::tmem_load32(v, at + j);
        if (dual(kMode)) tc::tmem_load32(u, at + kN / 2 + j);
        if (kMode == kGradient) {
          const int b = had & 1;
          ok = wait(dh_in(reader, b), had >> 1 & 1);
          const char* from = raw + (asked_at - tc::smem(raw)) + reader * kAsked<kMode> + b * 2048 + lane * 64;
#pragma unroll
          for (int q = 0; q < 4; q++) dh[q] = load_pack<T, 8>(reinterpret_cast<const T*>(from + ((q ^ (lane >> 1 & 3)) << 4)));
          if (ok) had++;
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
        // made, the copies of as many others as the staging holds may be under way (none where it held G and U, or where the
        // last piece, of the launch's other product, took all of it).
        constexpr int kSmall = kStaging<kMode, kCtas> / 2048, kLarge = kStaging<kMode, kCtas> / 4096;
        const bool large = kMode == kGradient || (!dual(kMode) && p.sums), alone = kMode == kForward && p.keep;
        const uint32_t to = mine + (alone ? 0 : large ? buffer % kLarge * 4096 : buffer * 2048);
        if (lane == 0) {
          if (alone || (kMode == kBoth && was_large)) tc::stores_read<0>();
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
              tc::store_box(&p.o[it.matrix], col, row0, to);
              if (kMode == kGradient) tc::store_box(&p.o[1], col, row0, to + 2048);
            }
          } else {
            __syncwarp();
            T* out = static_cast<T*>(p.out[it.matrix]) + row0 * p.stride + col;
            tc::unstage<T>(mine_ptr + (to - mine), lane, out, p.stride, min(32, p.m - row0), count);
          }
        }
        if (lane == 0) tc::stores_commit();
        buffer = (buffer + 1) % kSmall;
        was_large = large;
        // The next but one piece of dh takes this one's place: asked for behind the stores of what was made of it, which cannot be
        // issued before its reads have come back.  (A read alone that is issued can still wait when a copy asked for behind it lands.)
        if (kMode == kGradient && ok) {
          __syncwarp();
          ask_next();
        }
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

// The parts of split sums added up in order, and rounded: 4 columns a thread; blockIdx.y says of which product.  fold: each
// matrix's rows come twice, and are added up too.
struct JoinArgs {
  const float* partial; int64_t pitch;
  int splits, matrices, fold;
  int64_t m, n;
  void* out[2]; int64_t stride;
};
struct Joins { JoinArgs of[2]; };
template <typename T>
__global__ void __launch_bounds__(256) k_join(const __grid_constant__ Joins joins) {
  const JoinArgs& a = joins.of[blockIdx.y];
  const int64_t quads = a.pitch / 4, total = a.matrices * a.m * quads, part = total << a.fold;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / quads, c = (i - row * quads) * 4;
    const float* p = a.partial + (i + (a.fold && row >= a.m ? a.m * quads : 0)) * 4;
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (int k = 0; k < a.splits; k++) {
      const float4 v = *reinterpret_cast<const float4*>(p + k * part * 4);
      s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
      if (a.fold) {
        const float4 l = *reinterpret_cast<const float4*>(p + (k * part + a.m * quads) * 4);
        s.x += l.x, s.y += l.y, s.z += l.z, s.w += l.w;
      }
    }
    T* out = row >= a.m ? static_cast<T*>(a.out[1]) + (row - a.m) * a.stride + c : static_cast<T*>(a.out[0]) + row * a.stride + c;
    const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int e = 0; e < 4; e++)
      if (c + e < a.n) out[e] = from_f32<T>(v[e]);
  }
}

__global__ void __launch_bounds__(256) k_pack(const __grid_constant__ PackArgs a) {
  const int w = blockIdx.y, lane = threadIdx.x % 32;
  for (int64_t row = (int64_t)blockIdx.x * 8 + threadIdx.x / 32; row < a.rows[w]; row += (int64_t)gridDim.x * 8) {
    const char* from = static_cast<const char*>(a.from[w]) + row * a.stride[w] * 2;
    char* to = static_cast<char*>(a.to[w]) + row * a.pitch * 2;
    const int off = (int)(reinterpret_cast<uintptr_t>(from) % 16);  // even, the same for all of the row's pieces
    const char* end = from + a.cols * 2;
    for (int64_t c = lane * 16; c < a.pitch * 2; c += 32 * 16) {
      *reinterpret_cast<uint4*>(to + c) = row_bytes(from + c, from, end, off);
    }
  }
}

int items_of(const ProductArgs& p) { return p.tiles_m * p.tiles_n * p.matrices * p.splits; }

template <typename T, Mode kMode, int kN, int kCtas>
cudaError_t launch_width(const Launch<kMode>& l, cudaStream_t s) {
  static std::atomic<uint64_t> allowed{0};  // devices on which the kernel may take its shared memory
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  if (device >= 64 || !(allowed.load(std::memory_order_relaxed) >> device & 1)) {
    e = cudaFuncSetAttribute(k_product<T, kMode, kN, kCtas>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem<kMode, kN, kCtas>);
    if (e != cudaSuccess) return e;
    if (device < 64) allowed.fetch_or((uint64_t)1 << device, std::memory_order_relaxed);
  }
  int items = 0;
  for (const ProductArgs& p : l.of) items += items_of(p);
  cudaLaunchConfig_t c{};
  c.gridDim = dim3((unsigned)std::min(items, kSms / kCtas) * kCtas);
  c.blockDim = dim3(kThreads<kMode>);
  c.dynamicSmemBytes = kSmem<kMode, kN, kCtas>;
  c.stream = s;
  cudaLaunchAttribute cluster{};
  cluster.id = cudaLaunchAttributeClusterDimension;
  cluster.val.clusterDim.x = kCtas;
  cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
  c.attrs = &cluster;
  c.numAttrs = kCtas == 1 ? 0 : 1;
  return cudaLaunchKernelEx(&c, k_product<T, kMode, kN, kCtas>, l);
}

// what a product's size and cut say of its arguments
template <typename T, Mode kMode>
bool settle(ProductArgs& p, const Cut& k, bool fold) {
  const int out = dual(kMode) ? k.width / 2 : k.width;
  p.tiles_m = (int)ceil_div(p.m, kM * k.ctas);
  p.tiles_n = (int)ceil_div(p.n, out);
  p.steps = (int)ceil_div(p.c, kC) * (dual(kMode) ? 1 : p.parts);
  p.splits = k.splits;
  p.rows = a_rows(kMode);
  p.a_box = a_rows(kMode) ? kM : a_box(p.m);
  p.copies = 1;
  p.sums = p.splits > 1 || fold;
  if (p.sums) {
    p.partial_pitch = up(p.n, 4);
    if (!map_partial(&p.o[0], p.partial, (int64_t)p.splits * p.matrices, p.m, p.n, p.partial_pitch)) return false;
  } else {
    for (int w = 0; w < 2; w++) {
      if (!p.out[w]) continue;
      p.copies &= tma_ready(p.out[w], p.stride, p.m, p.n);
      if (p.copies && !map_matrix(&p.o[w], kType<T>, p.out[w], p.m, p.n, p.stride, 32, true)) return false;
    }
  }
  return (int64_t)p.tiles_m * p.tiles_n * p.matrices * p.splits <= 0x20000000;
}

template <typename T, Mode kMode>
cudaError_t run(const Launch<kMode>& l, const Cut& k, cudaStream_t s, std::initializer_list<int> folds) {
  const cudaError_t e = k.ctas == 2      ? launch_width<T, kMode, 256, 2>(l, s)
                        : k.width == 256 ? launch_width<T, kMode, 256, 1>(l, s)
                        : k.width == 128 ? launch_width<T, kMode, 128, 1>(l, s)
                                         : launch_width<T, kMode, 64, 1>(l, s);
  if (e != cudaSuccess) return e;
  Joins joins{};
  int count = 0;
  int64_t most = 0;
  const int* fold = folds.begin();
  for (const ProductArgs& p : l.of) {
    const int f = *fold++;
    if (!p.sums) continue;
    JoinArgs& a = joins.of[count++];
    a = JoinArgs{p.partial, p.partial_pitch, p.splits, p.matrices, f, f ? p.m / 2 : p.m, p.n, {p.out[0], p.out[1]}, p.stride};
    most = std::max(most, a.matrices * a.m * a.pitch / 4);
  }
  if (!count) return e;
  k_join<T><<<dim3((unsigned)std::min<int64_t>(ceil_div(most, 256), kSms * 8), (unsigned)count), 256, 0, s>>>(joins);
  return cudaGetLastError();
}

template <typename T, Mode kMode>
cudaError_t launch_mode(ProductArgs& p, const Cut& k, cudaStream_t s, bool fold) {
  if (!settle<T, kMode>(p, k, fold)) return cudaErrorInvalidValue;
  return run<T, kMode>(Launch<kMode>{{p}}, k, s, {fold});
}
// the estimated time of an item (see cut)
double item_time(const Cut& k, int steps) {
  return (double)ceil_div(steps, k.splits) * (k.ctas == 2 ? 0.9 : k.width == 256 ? 1.0 : k.width == 128 ? 0.6 : 0.4) + 8;
}
template <typename T>
cudaError_t launch_both(ProductArgs& weight, ProductArgs& input, const Cuts& k, cudaStream_t s, bool fold) {
  if (!settle<T, kWeight>(weight, k.weight, false) || !settle<T, kInput>(input, k.input, fold)) return cudaErrorInvalidValue;
  // in units of the shorter items' time: how many of each a unit has
  const double item_w = item_time(k.weight, weight.steps), item_i = item_time(k.input, input.steps);
  const bool first = item_w >= item_i;
  Double l{first ? Double{{weight, input}} : Double{{input, weight}}};
  const int units = kSms / k.weight.ctas, a = items_of(l.of[0]), b = items_of(l.of[1]);
  const int longer = (int)std::lround(first ? item_w / item_i : item_i / item_w);
  l.full = a / units;
  l.rest = a % units;
  if (a + b > units) {  // the least time `slots` in which all of the second's items find room
    const auto room = [&](int64_t slots) {
      const int64_t less = std::max<int64_t>(slots - (int64_t)longer * (l.full + 1), 0), most = std::max<int64_t>(slots - (int64_t)longer * l.full, 0);
      return less * l.rest + most * (units - l.rest);
    };
    int64_t slots = ((int64_t)longer * a + b) / units;
    while (room(slots) < b) slots++;
    l.rounds = (int)std::max<int64_t>(slots - (int64_t)longer * (l.full + (l.rest > 0)), 0);
  }
  return run<T, kBoth>(l, k.weight, s, first ? std::initializer_list<int>{0, fold} : std::initializer_list<int>{fold, 0});
}

}  // namespace

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

bool map_matrix(CUtensorMap* map, ndvm_dtype t, const void* p, int64_t rows, int64_t cols, int64_t stride, int box, bool piece) {
  if (!encoder()) return false;
  if (rows == 1) stride = up(cols, 8);  // (never taken)
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride * 2};
  const cuuint32_t boxes[2] = {piece ? 32u : 64u, (cuuint32_t)box}, ones[2] = {1, 1};
  const CUtensorMapDataType type = t == NDVM_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
  return encoder()(map, type, 2, const_cast<void*>(p), dims, strides, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   piece ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool map_partial(CUtensorMap* map, float* p, int64_t parts, int64_t m, int64_t n, int64_t pitch) {
  if (!encoder()) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)n, (cuuint64_t)m, (cuuint64_t)parts};
  const cuuint64_t strides[2] = {(cuuint64_t)pitch * 4, (cuuint64_t)(pitch * m) * 4};
  const cuuint32_t boxes[3] = {32, 32, 1}, ones[3] = {1, 1, 1};
  return encoder()(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, p, dims, strides, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The shape with the least estimated time, in steps of a tile 256 wide (0.27 us): a round of tiles takes its
// steps and about 8 more to fill and empty; narrower tiles' steps are shorter, but not in proportion (more bytes an
// operation), a pair's a little shorter (16384 x 2048 -> 8192 forward: 612 us alone, 560 in pairs) if there are 12 or
// more (pairs start and end together: 4096 x 256 -> 1024 takes 9.2 us alone, 10.6 in pairs).  Where tiles are fewer than
// SMs, a contraction is cut into parts of 8 steps or more, which costs the launch that joins them.  (The gated
// projection's weight gradients are cut as if both were wanted: one of them alone has the same bits.)
Cut cut(Mode mode, int64_t m, int64_t n, int64_t c, int parts, int matrices) {
  struct Shape { int width, ctas; double step; };
  static constexpr Shape shapes[] = {{256, 2, 0.9}, {256, 1, 1.0}, {128, 1, 0.6}, {64, 1, 0.4}};
  const int64_t steps = ceil_div(c, kC) * parts;
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

// The same for a dense layer's two gradients, which share a launch: as the items are dealt out, the longer ones first, a unit
// has its share of the work and up to one item more (half of a shorter one, on average).  A part more of a sum costs 1.1 to 1.6 ps an
// element of the result (16384 x 1024 -> 1024, dw in 2, 4, 8, 16, 32 parts: 51.1, 53.5, 60.1, 73.6, 98.4 us; whole 78.7).  Against the
// best of all widths and parts the rule takes 51.2 / 51.1 us there, 4096 x 4096 -> 1024 45.9 / 45.8, 16384 x 256 -> 2048 33.4 / 33.4,
// 65536 x 256 -> 256 41.6 / 41.8, 1501 x 776 -> 336 10.5 / 10.5, 16384 x 1024 -> 256 35.8 / 33.9; farther off with few steps on one side:
// 16384 x 1024 -> 64 28.8 / 25.9, 64 x 2048 -> 8192 27.6 / 25.1, 150 x 1000 -> 4096 17.4 / 14.8.
Cuts cut_both(int64_t rows, int64_t k, int64_t n, int parts) {
  // (a call asks three times: for its workspace, whether it fits, and for the launch)
  thread_local struct { int64_t rows = -1, k, n; int parts; Cuts cuts; } last;
  if (last.rows == rows && last.k == k && last.n == n && last.parts == parts) return last.cuts;
  struct Shape { int width, ctas; double step; };
  static constexpr Shape shapes[] = {{256, 2, 0.9}, {256, 1, 1.0}, {128, 1, 0.6}, {64, 1, 0.4}};
  const int64_t steps_w = ceil_div(rows, kC) * parts, steps_i = ceil_div(n, kC);
  const double sum_w = (double)(n * k) * 4e-6, sum_i = (double)(rows * parts * k) * 4e-6;  // steps (of 0.27 us) to write and read one part
  Cuts best{};
  double least = 1e300;
  for (const Shape& s : shapes) {
    if (s.ctas == 2 && std::min(steps_w, steps_i) < 12) continue;
    const double units = kSms / s.ctas;
    const int64_t tiles_w = ceil_div(n, kM * s.ctas) * ceil_div(k, s.width), tiles_i = ceil_div(rows * parts, kM * s.ctas) * ceil_div(k, s.width);
    for (const int w : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
      if (w > 1 && w > steps_w / 8) break;
      for (const int i : {1, 2, 4, 8}) {
        if (i > 1 && i > steps_i / 8) break;
        const double item_w = (double)ceil_div(steps_w, w) * s.step + 8, item_i = (double)ceil_div(steps_i, i) * s.step + 8;
        const double count_w = (double)(tiles_w * w), count_i = (double)(tiles_i * i), work = (count_w * item_w + count_i * item_i) / units;
        const double rounds = count_w + count_i > units ? work + 0.5 * std::min(item_w, item_i) : 0;
        const double time = std::max({rounds, item_w, item_i}) + (w > 1 || i > 1 ? 13 : 0) + (w > 1 ? w * sum_w : 0) + (i > 1 ? i * sum_i : 0);
        if (time < least) least = time, best = Cuts{{s.width, s.ctas, w}, {s.width, s.ctas, i}};
      }
    }
  }
  last = {rows, k, n, parts, best};
  return best;
}

void launch_pack(const PackArgs& p, int count, int64_t most_rows, cudaStream_t s) {
  const int64_t blocks = std::min<int64_t>(ceil_div(most_rows, 8), kSms * 32);
  k_pack<<<dim3((unsigned)blocks, (unsigned)count), 256, 0, s>>>(p);
}

cudaError_t launch_product(Mode mode, ndvm_dtype t, ProductArgs& p, const Cut& k, cudaStream_t s, bool fold) {
  const bool half = t == NDVM_F16;
  if (mode == kForward) return half ? launch_mode<__half, kForward>(p, k, s, fold) : launch_mode<__nv_bfloat16, kForward>(p, k, s, fold);
  if (mode == kGradient) return half ? launch_mode<__half, kGradient>(p, k, s, fold) : launch_mode<__nv_bfloat16, kGradient>(p, k, s, fold);
  if (mode == kInput) return half ? launch_mode<__half, kInput>(p, k, s, fold) : launch_mode<__nv_bfloat16, kInput>(p, k, s, fold);
  return half ? launch_mode<__half, kWeight>(p, k, s, fold) : launch_mode<__nv_bfloat16, kWeight>(p, k, s, fold);
}

cudaError_t launch_products(ndvm_dtype t, ProductArgs& weight, ProductArgs& input, const Cuts& k, cudaStream_t s, bool fold) {
  return t == NDVM_F16 ? launch_both<__half>(weight, input, k, s, fold) : launch_both<__nv_bfloat16>(weight, input, k, s, fold);
}

cudaError_t product_stopped(int* flag) {
  cudaError_t e = cudaMemcpyFromSymbol(flag, g_stopped, sizeof *flag);
  const int none = 0;
  if (e == cudaSuccess && *flag) e = cudaMemcpyToSymbol(g_stopped, &none, sizeof none);
  return e;
}

}  // namespace ndvm
