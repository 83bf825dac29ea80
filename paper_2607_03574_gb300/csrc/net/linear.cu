// Dense layer z = x w^T + b, y = act(z) + residual, and its backward pass:
//   dz = dy act'(z), dx = dz w, dw = dz^T x, db = sum over rows of dz, dresidual = dy.
// The forward pass keeps z if there is an activation: in binary32 (so that dz is rounded once, to the operands' type, which
// its products need; where there are few elements not even that: in_halves), or as 8-bit blocks.  db sums dz in binary32.
//
// Operands are 16-bit, or e4m3 in 8-bit blocks (blocks.cuh) whose scales the tensor cores apply: twice the operations a second
// and half the bytes.  The backward pass's products are product.cu's.
#include <atomic>
#include <cstdint>

#include "activation.cuh"
#include "blocks.cuh"
#include "net.h"
#include "product.h"
#include "rows.cuh"
#include "tc.cuh"
#include "types.cuh"

namespace ndvm {
namespace {

__device__ int g_linear_stopped;  // a wait in k_linear ran out (ndvm_check_operators)

// ---------------------------------------------------------------------------------- the product
// Warps that read the sums: four (in 8 bits, whose tiles have at most 192 columns, three) for each quarter of a tile's rows, which
// share its columns; a tile of 64 columns has work for two.
template <bool kEight, int kN> constexpr int kReaders = kN == 64 ? 8 : kEight ? 12 : 16;
template <bool kEight, int kN> constexpr int kThreads = 64 + 32 * kReaders<kEight, kN>;  // and one that loads, one that multiplies
constexpr int kRoom = 4096;                   // bytes of each: what its stores are made from
constexpr int kLine = 128;                    // bytes of a row in a step: 64 elements of the contraction, or 128 in 8 bits

template <int kN, int kCtas> constexpr int kTileBytes = (kM + kN / kCtas) * kLine;
// scales of a step, in 8 bits: 128 rows' of A, and those of the one or two 128s of rows that B's lie in
template <int kN> constexpr int kScaleTiles = kN > 128 ? 2 : 1;
template <bool kEight, int kN> constexpr int kScaleBytes = kEight ? 512 * (1 + kScaleTiles<kN>) : 0;
template <bool kEight, int kN, int kCtas>
constexpr int kSteps = std::min(8, (229376 - kReaders<kEight, kN> * kRoom) / (kTileBytes<kN, kCtas> + kScaleBytes<kEight, kN>));
template <bool kEight, int kN, int kCtas>
constexpr int kShared = kSteps<kEight, kN, kCtas> * (kTileBytes<kN, kCtas> + kScaleBytes<kEight, kN>) + kReaders<kEight, kN> * kRoom +
                        1024 /* alignment */ + 256 /* barriers */;
// of tensor memory: two tiles' sums, and two steps' scales
template <bool kEight, int kN> constexpr int kColumns = !kEight ? 2 * kN : kN == 64 ? 256 : 512;

enum Keep { kNothing, kFloats, kBlocks };

struct ForwardArgs {
  CUtensorMap a, b;                 // operands
  CUtensorMap a_scales, b_scales;   // in 8 bits
  CUtensorMap o;                    // y, or the split sums
  CUtensorMap z;                    // z in binary32
  int m, n, c;                      // rows and columns of the result, contraction
  int tiles_m, tiles_n, steps, splits;
  int act, keep;
  int a_box;                        // rows of A that a tile loads (fewer than 128 where the result has fewer)
  int copies;                       // y is stored by copies (its rows start on 16 bytes)
  int wide, bias_wide;              // the residual's rows, and the bias, start on 16 bytes
  uint32_t band_magic, band_shift;  // i / (a band's tiles) = (i * magic) >> (32 + shift)
  const void* bias; int bias_f32;
  const void* residual; int64_t r_stride;
  void* out; int64_t stride;
  uint8_t* z_values; int64_t z_pitch; uint8_t* z_scales;
};

template <typename T>
__device__ __forceinline__ float bias_at(const void* bias, int f32, int64_t c) {
  return !bias ? 0.0f : f32 ? static_cast<const float*>(bias)[c] : to_f32(static_cast<const T*>(bias)[c]);
}

// 32 values of a row to a warp's staging, in the 64-byte swizzle (a line of 64 bytes a row), or as binary32 in the 128-byte one
template <typename T>
__device__ __forceinline__ void stage_narrow(uint32_t buffer, int lane, const float (&v)[32]) {
#pragma unroll
  for (int q = 0; q < 4; q++) {
    union { uint4 u; T t[8]; } o;
#pragma unroll
    for (int e = 0; e < 8; e += 2) narrow(o.t + e, make_float2(v[q * 8 + e], v[q * 8 + e + 1]));
    tc::store16(buffer + lane * 64 + ((q ^ (lane >> 1 & 3)) << 4), o.u);
  }
}
__device__ __forceinline__ void stage_floats(uint32_t buffer, int lane, const float (&v)[32]) {
#pragma unroll
  for (int q = 0; q < 8; q++)
    tc::store16(buffer + lane * 128 + ((q ^ (lane & 7)) << 4),
                make_uint4(__float_as_uint(v[q * 4]), __float_as_uint(v[q * 4 + 1]), __float_as_uint(v[q * 4 + 2]),
                           __float_as_uint(v[q * 4 + 3])));
}

// A block of a row (values beyond its end are 0) to e4m3, `room` (16 or 32) bytes of which are the row's
__device__ __forceinline__ void keep_block(const float (&v)[32], uint8_t* values, int room, uint8_t* scale) {
  float most[4] = {};
#pragma unroll
  for (int e = 0; e < 32; e++) most[e % 4] = larger(most[e % 4], v[e]);
  const uint32_t code = block_code(__float_as_uint(larger(larger(most[0], most[1]), larger(most[2], most[3]))));
  const float inverse = block_inverse(code);
  uint32_t q[8];
#pragma unroll
  for (int e = 0; e < 8; e++) q[e] = to_e4m3(v[4 * e] * inverse, v[4 * e + 1] * inverse, v[4 * e + 2] * inverse, v[4 * e + 3] * inverse);
  *reinterpret_cast<uint4*>(values) = make_uint4(q[0], q[1], q[2], q[3]);
  if (room > 16) *reinterpret_cast<uint4*>(values + 16) = make_uint4(q[4], q[5], q[6], q[7]);
  *scale = (uint8_t)code;
}

// 32 consecutive values of a row from memory, `count` of which there are; wide: they start on 16 bytes
template <typename T>
__device__ __forceinline__ void load32(Pack<T, 8> (&v)[4], const T* from, int count, bool wide) {
  if (wide && count >= 32) {
#pragma unroll
    for (int q = 0; q < 4; q++) v[q] = load_pack<T, 8>(from + 8 * q);
  } else {
#pragma unroll
    for (int e = 0; e < 32; e++)
      if (e < count) v[e / 8].v[e % 8] = from[e];
  }
}
template <typename T>
__device__ __forceinline__ void add32(float (&v)[32], const Pack<T, 8> (&a)[4]) {
#pragma unroll
  for (int e = 0; e < 32; e += 2) {
    const float2 s = add(make_float2(v[e], v[e + 1]), widen(a[e / 8].v + e % 8));
    v[e] = s.x, v[e + 1] = s.y;
  }
}
template <typename T>
__device__ __forceinline__ void prefetch_bias(const void* bias, int f32, int64_t c) {
  const void* p = f32 ? static_cast<const void*>(static_cast<const float*>(bias) + c) : static_cast<const T*>(bias) + c;
  asm volatile("prefetch.global.L1 [%0];" ::"l"(p));
}
// the same 32 values for every lane (a broadcast from L1)
template <typename T>
__device__ __forceinline__ void add_bias(float (&v)[32], const void* bias, int f32, int col, int count, bool wide) {
  if (f32 && wide && count >= 32) {
#pragma unroll
    for (int q = 0; q < 8; q++) {
      const float4 b = *reinterpret_cast<const float4*>(static_cast<const float*>(bias) + col + 4 * q);
      const float2 s = add(make_float2(v[4 * q], v[4 * q + 1]), make_float2(b.x, b.y)), t = add(make_float2(v[4 * q + 2], v[4 * q + 3]), make_float2(b.z, b.w));
      v[4 * q] = s.x, v[4 * q + 1] = s.y, v[4 * q + 2] = t.x, v[4 * q + 3] = t.y;
    }
  } else if (f32) {
#pragma unroll
    for (int e = 0; e < 32; e++)
      if (e < count) v[e] += static_cast<const float*>(bias)[col + e];
  } else {
    Pack<T, 8> b[4] = {};
    load32<T>(b, static_cast<const T*>(bias) + col, count, wide);
    add32<T>(v, b);
  }
}

// One warp loads, one issues the products, the others read the sums of a tile while the next one's are made.  A block has
// kN columns of sums for its 128 rows; a pair's blocks (kCtas = 2) hold half of those rows of B each.  Bound by the tensor
// cores where the contraction is long, by the epilogue's instructions where it is short: 16384 x 2048 -> 8192 bf16 295 us (1.86 PFLOP/s), 302
// with gelu, 347 with z kept in binary32 too; in 8 bits 177 us (3.1 PFLOP/s) and 204, which no counter explains (it is not the scales'
// copies: 177 without them);
// 16384 x 256 -> 8192 74 us and 127 with gelu.  In 8 bits two tiles' sums of 256 columns would leave no room for scales, and
// 128 columns read more bytes an operation (360 us).
template <typename T, bool kEight, int kN, int kCtas>
__global__ void __launch_bounds__(kThreads<kEight, kN>, 1) k_linear(const __grid_constant__ ForwardArgs p) {
  extern __shared__ char raw[];
  constexpr int S = kSteps<kEight, kN, kCtas>, kTile = kTileBytes<kN, kCtas>, kScales = kScaleBytes<kEight, kN>;
  constexpr int kABytes = kM * kLine, kElements = kEight ? 128 : 64, R = kReaders<kEight, kN>;  // (of the contraction a step)
  __shared__ uint32_t s_tmem;
  __shared__ int s_stop;
  const uint32_t base = (tc::smem(raw) + 1023) & ~1023u;
  const uint32_t staging = base + S * kTile, scales = staging + R * kRoom, bars = scales + S * kScales;
  const auto full = [&](int i) { return bars + i * 8; };
  const auto empty = [&](int i) { return bars + (S + i) * 8; };
  const auto done = [&](int i) { return bars + (2 * S + i) * 8; };       // a tile's sums are complete
  const auto taken = [&](int i) { return bars + (2 * S + 2 + i) * 8; };  // and have been read
  const uint32_t drain = bars + (2 * S + 4) * 8;
  const int warp = __shfl_sync(~0u, threadIdx.x / 32, 0), lane = threadIdx.x % 32;  // (the same for all of a warp, as the compiler sees)
  const int rank = kCtas == 1 ? 0 : (int)tc::cluster_rank(), unit = blockIdx.x / kCtas, units = gridDim.x / kCtas;
  volatile int* stop = &s_stop;

  if (threadIdx.x == 32) {
    tc::prefetch_map(&p.a), tc::prefetch_map(&p.b);
    if (kEight) tc::prefetch_map(&p.a_scales), tc::prefetch_map(&p.b_scales);
  }
  if (threadIdx.x == 0) {
    s_stop = 0;
    for (int i = 0; i < S; i++) tc::barrier_init(full(i), 1), tc::barrier_init(empty(i), 1);
    for (int i = 0; i < 2; i++) tc::barrier_init(done(i), 1), tc::barrier_init(taken(i), R * kCtas);
    tc::barrier_init(drain, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tc::tmem_alloc<kCtas, kColumns<kEight, kN>>(tc::smem(&s_tmem));
  tc::fence_before();
  __syncthreads();
  if (kCtas == 2) tc::cluster_sync();
  tc::fence_after();
  const uint32_t tmem = s_tmem;

  const int tiles = p.tiles_m * p.tiles_n, items = tiles * p.splits;
  struct Item { int m0, n0, split, from, to; };
  constexpr int kBand = 16 / kCtas;
  // tiles in bands of 2048 rows, down a band first: blocks that run together share operands in L2
  const auto item = [&](int i) {
    Item it;
    it.split = p.splits > 1 ? i / tiles : 0;
    i -= it.split * tiles;
    const int band = (int)((uint64_t)i * p.band_magic >> 32 >> p.band_shift), first = band * kBand, height = min(kBand, p.tiles_m - first);
    i -= band * kBand * p.tiles_n;
    const int across = height == kBand ? i / kBand : i / height;
    it.m0 = ((first + i - across * height) * kCtas + rank) * kM;
    it.n0 = across * kN;
    if (p.splits == 1) {
      it.from = 0, it.to = p.steps;
      return it;
    }
    it.from = (int)((int64_t)p.steps * it.split / p.splits);
    it.to = (int)((int64_t)p.steps * (it.split + 1) / p.splits);
    return it;
  };

  // (the whole warp waits, and goes on or gives up)
  const auto wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(~0u, tc::barrier_wait(bar, parity, stop)) != 0; };
  if (warp == 0) {
    // ---- loads
    int stage = 0;
    uint32_t phase = 0;
    int issued = 0;
    bool ok = true;
    const int bytes = kTile - kABytes + p.a_box * kLine + kScales;
    for (int i = unit; ok && i < items; i += units) {
      const Item it = item(i);
      for (int s = it.from; s < it.to; s++) {
        if (!(ok = wait(empty(stage), phase ^ 1))) break;
        if (tc::elect()) {
          const uint32_t at = base + stage * kTile, bar = kCtas == 1 ? full(stage) : tc::in_first(full(stage));
          if (rank == 0) tc::barrier_expect(full(stage), kCtas * bytes);
          tc::load_box<kCtas>(at, &p.a, s * kElements, it.m0, bar);
          tc::load_box<kCtas>(at + kABytes, &p.b, s * kElements, it.n0 + rank * (kN / kCtas), bar);
          if constexpr (kEight) {  // (scales behind the last row of either are filled with 0; a pair's blocks both hold all of B's)
            const uint32_t to = scales + stage * kScales;
            tc::load_box<kCtas>(to, &p.a_scales, 0, s, it.m0 / 128, bar);
            tc::load_box<kCtas>(to + 512, &p.b_scales, 0, s, it.n0 / 128, bar);
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
    constexpr uint32_t desc = tc::instruction(std::is_same<T, __nv_bfloat16>::value, false, false, kM * kCtas, kN);
    int stage = 0, slot = 0, turn = 0;
    uint32_t phase = 0, slot_phase = 0;
    bool ok = true;
    for (int i = unit; ok && i < items; i += units) {
      const Item it = item(i);
      if (!(ok = wait(taken(slot), slot_phase ^ 1))) break;
      tc::fence_after();
      for (int s = it.from; s < it.to; s++) {
        if (!(ok = wait(full(stage), phase))) break;
        tc::fence_after();
        if (tc::elect()) {
          const uint32_t at = base + stage * kTile;
          const uint64_t a = tc::operand(at, false), b = tc::operand(at + kABytes, false);
          if constexpr (kEight) {
            // scales to tensor memory, two steps' by turns; B's columns begin in the middle of a 128 where its tile does
            const uint32_t from = scales + stage * kScales, to = tmem + 2 * kN + turn * 16, to_b = to + 4 + it.n0 % 128 / 32;
            tc::copy_scales<kCtas>(to, from);
#pragma unroll
            for (int q = 0; q < kScaleTiles<kN>; q++) tc::copy_scales<kCtas>(to + 4 + 4 * q, from + 512 + 512 * q);
            const int blocks = (p.c - s * kElements + 31) / 32;  // (none behind the row's last: its scale need not be one)
#pragma unroll
            for (int q = 0; q < 4; q++)
              if (q < blocks)
                tc::mma_blocks<kCtas>(tmem + slot * kN, a + q * (32 >> 4), b + q * (32 >> 4), tc::instruction_blocks(kM * kCtas, kN, q), to, to_b,
                                      s > it.from || q > 0);
          } else {
#pragma unroll
            for (int q = 0; q < 4; q++)  // 16 of the contraction: 32 bytes along a line
              tc::mma<kCtas>(tmem + slot * kN, a + q * (32 >> 4), b + q * (32 >> 4), desc, s > it.from || q > 0);
          }
          tc::commit<kCtas>(empty(stage));
          if (s + 1 == it.to) tc::commit<kCtas>(done(slot));
        }
        __syncwarp();
        turn ^= 1;
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
    // ---- sums to memory: a warp reads the 32 lanes (rows of the tile) that are its own, and 32 columns at a time: a block
    // of one row a thread.  The residual is asked for a piece ahead: by copies of neighbours to half of the staging, where z does not
    // take that whole, or a thread its own row (16384 x 256 -> 8192 with a residual 116 us so, 134 by its own row).  (What these warps do for each other is hide the waits between
    // their instructions: 16384 x 256 -> 8192 takes 74 us, with eight of them, and the bias by way of shared memory, it took 147.)
    const int lanes = (warp % 4) * 32, reader = warp - 2, first = reader / 4 * 32;
    constexpr int kNext = R / 4 * 32;
    const uint32_t mine = staging + reader * kRoom;
    const char* const mine_ptr = raw + (mine - tc::smem(raw));
    const bool sums = p.splits > 1, floats = !sums && p.keep == kFloats;
    int slot = 0, buffer = 0;
    uint32_t slot_phase = 0;
    Pack<T, 8> next[4];
    const bool by_copies = p.residual && p.wide && !sums && !floats;
    const uint32_t residual_at = mine + 2048;
    const auto ask = [&](int row, int col) {
      if (!p.residual || sums || col >= p.n) return;
      if (by_copies) {  // four lanes a row of 64 bytes, in the 64-byte swizzle; nothing behind a row's end is read
        const int c = col + lane % 4 * 8, bytes = min(16, max(0, p.n - c) * 2);
#pragma unroll
        for (int q = 0; q < 4; q++) {
          const int r = q * 8 + lane / 4, from = row - lane + r;
          if (from < p.m && bytes > 0)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(residual_at + r * 64 + ((lane % 4 ^ (r >> 1 & 3)) << 4)),
                         "l"(static_cast<const T*>(p.residual) + from * p.r_stride + c), "r"(bytes) : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
      } else if (row < p.m) {
        load32<T>(next, static_cast<const T*>(p.residual) + row * p.r_stride + col, p.n - col, p.wide);
      }
    };
    for (int i = unit; i < items; i += units) {
      const Item it = item(i);
      const int row0 = it.m0 + lanes, row = row0 + lane;
      ask(row, it.n0 + first);
      if (p.bias && !sums)  // (so that L1 has it when the sums come)
        for (int j = first; j < kN; j += kNext)
          if (it.n0 + j + lane < p.n) prefetch_bias<T>(p.bias, p.bias_f32, it.n0 + j + lane);
      if (!wait(done(slot), slot_phase)) break;
      tc::fence_after();
      const uint32_t at = tmem + slot * kN + ((uint32_t)lanes << 16);
#pragma unroll 1
      for (int j = first; j < kN && row0 < p.m; j += kNext) {
        const int col = it.n0 + j, count = min(32, p.n - col);
        if (count <= 0) break;
        float v[32];
        tc::tmem_load32(v, at + j);
        // binary32 takes the staging whole, y half of it by turns, or one half beside the residual
        const uint32_t to = mine + (sums || floats || by_copies ? 0 : (buffer++ & 1) * 2048);
        if (lane == 0) {
          if (sums || floats || by_copies) tc::stores_read<0>();
          else tc::stores_read<1>();
        }
        __syncwarp();
        tc::tmem_loaded(v);
        if (sums) {
          stage_floats(to, lane, v);
          tc::fence_async();
          __syncwarp();
          if (lane == 0 && row0 < p.m) tc::store_box(&p.o, col, row0, it.split, to);
          if (lane == 0) tc::stores_commit();
          continue;
        }
        if (p.bias) add_bias<T>(v, p.bias, p.bias_f32, col, count, p.bias_wide);
        if (floats) {
          stage_floats(mine, lane, v);
          tc::fence_async();
          __syncwarp();
          if (lane == 0) {
            if (row0 < p.m) tc::store_box(&p.z, col, row0, 0, mine);
            tc::stores_commit();
          }
        } else if (p.keep == kBlocks) {
          if (count < 32) {
#pragma unroll
            for (int e = 0; e < 32; e++) v[e] = e < count ? v[e] : 0.0f;
          }
          if (row < p.m) keep_block(v, p.z_values + row * p.z_pitch + col, count > 16 ? 32 : 16, p.z_scales + scale_at(row, col / 32, (p.n + 127) / 128));
        }
        by_activation_or_none(p.act, [&](auto act) {
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const float2 a = activation<decltype(act)::value>(make_float2(v[e], v[e + 1]));
            v[e] = a.x, v[e + 1] = a.y;
          }
        });
        if (by_copies) {
          asm volatile("cp.async.wait_group 0;" ::: "memory");
          __syncwarp();
          const char* from = mine_ptr + 2048 + lane * 64;
#pragma unroll
          for (int q = 0; q < 4; q++) next[q] = load_pack<T, 8>(reinterpret_cast<const T*>(from + ((q ^ (lane >> 1 & 3)) << 4)));
        }
        if (p.residual) add32<T>(v, next);
        if (floats) {
          if (lane == 0) tc::stores_read<0>();
          __syncwarp();
        }
        stage_narrow<T>(to, lane, v);
        if (p.copies) {
          tc::fence_async();
          __syncwarp();
          if (lane == 0 && row0 < p.m) tc::store_box(&p.o, col, row0, to);
        } else {
          __syncwarp();
          tc::unstage<T>(mine_ptr + (to - mine), lane, static_cast<T*>(p.out) + row0 * p.stride + col, p.stride, min(32, p.m - row0), count);
        }
        if (lane == 0) tc::stores_commit();
        // (behind the stores of what the residual went into: its reads have come back, and copies may take its place)
        if (p.residual && j + kNext < kN) {
          __syncwarp();
          ask(row, col + kNext);
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
    if (lane == 0) tc::stores_read<0>();  // (what they write is there when the kernel ends)
    asm volatile("cp.async.wait_all;" ::: "memory");  // (what a launch that gave up had asked for)
  }
  __syncwarp();
  __syncthreads();
  if (threadIdx.x == 0 && s_stop) g_linear_stopped = 1;
  __syncwarp();
  tc::fence_before();
  if (kCtas == 2) tc::cluster_sync();  // neither block's memory is in the other's use any more
  tc::fence_after();
  if (warp == 1) tc::tmem_free<kCtas, kColumns<kEight, kN>>(tmem);
}

// What k_linear does with its sums, for those that were split: added up in order, 4 columns a thread (8 threads a block of z).
template <typename T>
__global__ void __launch_bounds__(256) k_finish(const float* partial, int64_t pitch, int splits, LinearArgs a, int64_t chunks) {
  const int64_t quads = (a.n + 31) / 32 * 8, total = a.rows * quads, part = a.rows * pitch;
  const uint32_t lanes = 0xffu << (threadIdx.x % 32 / 8 * 8);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / quads, c = (i - row * quads) * 4;
    float v[4] = {};
    if (c < a.n) {
      const float* p = partial + row * pitch + c;
#pragma unroll 4
      for (int k = 0; k < splits; k++) {
        const float4 f = *reinterpret_cast<const float4*>(p + k * part);
        v[0] += f.x, v[1] += f.y, v[2] += f.z, v[3] += f.w;
      }
    }
#pragma unroll
    for (int e = 0; e < 4; e++) v[e] = c + e < a.n ? v[e] + bias_at<T>(a.bias, a.bias_f32, c + e) : 0.0f;
    if (a.z && c < a.z_stride) *reinterpret_cast<float4*>(a.z + row * a.z_stride + c) = make_float4(v[0], v[1], v[2], v[3]);
    if (a.z_values) {
      const float2 pairs[2] = {make_float2(v[0], v[1]), make_float2(v[2], v[3])};
      store_block<4>(pairs, lanes, a.z_values + row * a.z_pitch + c, c < a.z_pitch, a.z_scales + scale_at(row, c / 32, chunks));
    }
    if (c >= a.n) continue;
    by_activation_or_none(a.act, [&](auto act) {
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        const float2 o = activation<decltype(act)::value>(make_float2(v[e], v[e + 1]));
        v[e] = o.x, v[e + 1] = o.y;
      }
    });
#pragma unroll
    for (int e = 0; e < 4; e++) {
      if (c + e >= a.n) continue;
      if (a.residual) v[e] += to_f32(static_cast<const T*>(a.residual)[row * a.r_stride + c + e]);
      static_cast<T*>(a.y)[row * a.y_stride + c + e] = from_f32<T>(v[e]);
    }
  }
}

// ------------------------------------------------------------------------------------ one row: vectors
// w is read once and is nearly all the traffic, so what counts is how much of it is under way: kSplits warps share a row of w, 16
// bytes a lane and two loads at once past L1, against x (from L1); a block's sums are joined in shared memory.  Many warps of few
// loads beat few of many (8192 -> 8192: 22.6 us at 64 warps an SM, 32.8 at 32 with four loads), and keeping w out of L1 helps
// both (25.6 with it).
template <typename T, int V, int kSplits>
__global__ void __launch_bounds__(256, 8) k_linear_one(LinearArgs a) {
  using P = Pairs<V>;
  constexpr int H = kPairs<V>, kUnroll = 2, kPer = 8 / kSplits;  // rows of w a block
  __shared__ float part[8];
  const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, split = warp % kSplits;
  const int64_t j = (int64_t)blockIdx.x * kPer + warp / kSplits;
  P s = both(0.0f, P());
  float bias = 0.0f, residual = 0.0f;
  if (j < a.n) {
    if (lane == 0) {  // (asked for first: what the end waits for)
      bias = bias_at<T>(a.bias, a.bias_f32, j);
      if (a.residual) residual = to_f32(static_cast<const T*>(a.residual)[j]);
    }
    const T *w = static_cast<const T*>(a.w) + j * a.w_stride, *x = static_cast<const T*>(a.x);
    constexpr int kStep = kSplits * 32 * V;
    for (int64_t c0 = (split * 32 + lane) * V; c0 < a.k; c0 += kUnroll * kStep) {
      Pack<T, V> pw[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; u++)
        if (c0 + u * kStep < a.k) pw[u] = load_once<T, V>(w + c0 + u * kStep);
#pragma unroll
      for (int u = 0; u < kUnroll; u++) {
        if (c0 + u * kStep >= a.k) break;
        P vx[H], vw[H];
        widen<T, V>(load_pack<T, V>(x + c0 + u * kStep), vx);
        widen<T, V>(pw[u], vw);
#pragma unroll
        for (int e = 0; e < H; e++) s = fma(vx[e], vw[e], s);
      }
    }
  }
  float z = total(s);
#pragma unroll
  for (int o = 16; o; o >>= 1) z += __shfl_xor_sync(~0u, z, o);
  if constexpr (kSplits > 1) {
    if (lane == 0) part[warp] = z;
    __syncthreads();
    if (split) return;
    z = part[warp];
#pragma unroll
    for (int q = 1; q < kSplits; q++) z += part[warp + q];
  }
  if (lane || j >= a.n) return;
  z += bias;
  if (a.z) a.z[j] = z;
  by_activation_or_none(a.act, [&](auto k) {
    const float2 act = activation<decltype(k)::value>(make_float2(z, z));
    static_cast<T*>(a.y)[j] = from_f32<T>(act.x + residual);
  });
}

template <typename T, int V>
void one_of(const LinearArgs& a, cudaStream_t s) {
  // as many warps a row as 64 on each SM have room for, each with two batches of loads at least (4096 -> 4096 7.4 us; 8.4 with 40 and four)
  const int64_t room = kSms * 64 / a.n, most = a.k / (4 * 32 * V);
  if (std::min(room, most) >= 8) k_linear_one<T, V, 8><<<(unsigned)a.n, 256, 0, s>>>(a);
  else if (std::min(room, most) >= 4) k_linear_one<T, V, 4><<<(unsigned)ceil_div(a.n, 2), 256, 0, s>>>(a);
  else if (std::min(room, most) >= 2) k_linear_one<T, V, 2><<<(unsigned)ceil_div(a.n, 4), 256, 0, s>>>(a);
  else k_linear_one<T, V, 1><<<(unsigned)ceil_div(a.n, 8), 256, 0, s>>>(a);
}
template <typename T>
void one(const LinearArgs& a, bool vectors, cudaStream_t s) {
  if (vectors) one_of<T, 8>(a, s);
  else one_of<T, 1>(a, s);
}

// ----------------------------------------------------------------------------------------- dz and db
struct SlopeArgs {
  int64_t rows, n;
  const void* dy; int64_t dy_stride;
  int act;
  const float* z; int64_t z_stride;
  const uint8_t* z_values; int64_t z_pitch; const uint8_t* z_scales;
  void* dz; int64_t pitch;  // null: not wanted
  int halves;               // and what dz's rounding leaves, `rows` rows further on
  float* sums;              // [gridDim.y][n], or null
};
// z of 8 columns of a row: two words of a block and its scale, or binary32
struct HeldZ { uint2 q; uint32_t code; };
// 8 columns a thread, 256 a block, every so-manieth 8 rows, kRows of them asked for at once; a block's 8 row sums are joined in
// shared memory.  Bound by memory where z is binary32 (16384 x 8192, db alone: 805 MB in 136 us), by the activation's instructions where it
// is 8-bit blocks (402 MB, 136 us); two rows at once and three blocks an SM beat four and two (139 and 155 us).
template <typename T, bool kVectors, int kZ>
__global__ void __launch_bounds__(256, 3) k_slope(SlopeArgs a) {
  constexpr int kRows = kZ == kNothing ? 8 : 2;
  using Z = std::conditional_t<kZ == kFloats, Pack<float, 8>, HeldZ>;
  const int t = threadIdx.x % 32, r = threadIdx.x / 32;
  const int64_t c = (int64_t)blockIdx.x * 256 + t * 8, chunks = (a.n + 127) / 128, step = (int64_t)gridDim.y * 8;
  const bool all = c + 8 <= a.n, some = c < a.n;
  float2 sum[4] = {};
  for (int64_t row0 = (int64_t)blockIdx.y * 8 + r; some && row0 < a.rows; row0 += kRows * step) {
    Pack<T, 8> d[kRows];
    Z held_z[kZ == kNothing ? 1 : kRows];
#pragma unroll
    for (int u = 0; u < kRows; u++) {
      const int64_t row = row0 + u * step;
      if (row >= a.rows) continue;
      const T* dy = static_cast<const T*>(a.dy) + row * a.dy_stride + c;
      if (kVectors && all) {
        d[u] = load_once<T, 8>(dy);
      } else {
#pragma unroll
        for (int e = 0; e < 8; e++) d[u].v[e] = c + e < a.n ? dy[e] : from_f32<T>(0.0f);
      }
      if constexpr (kZ == kFloats) {  // (its rows hold whole fours)
#pragma unroll
        for (int q = 0; q < 2; q++) {
          const float4 f = all || c + 4 * q < a.n ? *reinterpret_cast<const float4*>(a.z + row * a.z_stride + c + 4 * q) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          held_z[u].v[4 * q] = f.x, held_z[u].v[4 * q + 1] = f.y, held_z[u].v[4 * q + 2] = f.z, held_z[u].v[4 * q + 3] = f.w;
        }
      } else if constexpr (kZ == kBlocks) {
        held_z[u].q = *reinterpret_cast<const uint2*>(a.z_values + row * a.z_pitch + c);
        held_z[u].code = a.z_scales[scale_at(row, c / 32, chunks)];
      }
    }
    by_activation_or_none(kZ == kNothing ? NDVM_ACT_NONE : a.act, [&](auto k) {
#pragma unroll
      for (int u = 0; u < kRows; u++) {
        const int64_t row = row0 + u * step;
        if (row >= a.rows) break;
        if constexpr (kZ == kNothing) {
#pragma unroll
          for (int e = 0; e < 4; e++) sum[e] = add(sum[e], widen(d[u].v + 2 * e));
        } else {
          Pack<T, 8> o, l;
#pragma unroll
          for (int e = 0; e < 4; e++) {
            float2 z;
            if constexpr (kZ == kFloats) {
              z = make_float2(held_z[u].v[2 * e], held_z[u].v[2 * e + 1]);
            } else {
              const float scale = block_scale(held_z[u].code);
              z = from_e4m3((uint16_t)((e < 2 ? held_z[u].q.x : held_z[u].q.y) >> (e % 2 * 16)));
              z = held<float>(z, scale, held_z[u].code);
            }
            const float2 v = mul(widen(d[u].v + 2 * e), derivative<decltype(k)::value>(z));
            sum[e] = add(sum[e], v);
            narrow(o.v + 2 * e, v);
            if (a.halves) l.v[2 * e] = rest_of(v.x, o.v[2 * e]), l.v[2 * e + 1] = rest_of(v.y, o.v[2 * e + 1]);
          }
          if (!a.dz) continue;
          if (!all) {  // (the pitch's last columns are 0)
#pragma unroll
            for (int e = 0; e < 8; e++)
              if (c + e >= a.n) o.v[e] = l.v[e] = from_f32<T>(0.0f);
          }
          T* dz = static_cast<T*>(a.dz) + row * a.pitch + c;
          store_pack(dz, o);
          if (a.halves) store_pack(dz + a.rows * a.pitch, l);
        }
      }
    });
  }
  if (!a.sums) return;
  __shared__ __align__(16) float2 all_sums[8][4][32];
#pragma unroll
  for (int e = 0; e < 4; e++) all_sums[r][e][t] = sum[e];
  __syncthreads();
  if (r >= 4) return;
  float2 s = all_sums[0][r][t];
#pragma unroll
  for (int q = 1; q < 8; q++) s = add(s, all_sums[q][r][t]);
  float* out = a.sums + (int64_t)blockIdx.y * a.n + c + 2 * r;
  if (c + 2 * r < a.n) out[0] = s.x;
  if (c + 2 * r + 1 < a.n) out[1] = s.y;
}

// ------------------------------------------------------------------------------------------- launches
// 8-bit operands in boxes of 128 columns and `box` rows in the 128-byte swizzle
bool map_values(CUtensorMap* map, const uint8_t* p, int64_t rows, int64_t cols, int64_t stride, int box) {
  if (!encoder()) return false;
  if (rows == 1) stride = up(cols, 16);  // (never taken)
  const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride};
  const cuuint32_t boxes[2] = {128, (cuuint32_t)box}, ones[2] = {1, 1};
  return encoder()(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(p), dims, strides, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// their scales, in boxes of `tiles` 512s
bool map_scales(CUtensorMap* map, const uint8_t* p, int64_t rows, int64_t cols, int tiles) {
  if (!encoder()) return false;
  const int64_t chunks = ceil_div(cols, 128);
  const cuuint64_t dims[3] = {128, (cuuint64_t)chunks, (cuuint64_t)ceil_div(rows, 128)};
  const cuuint64_t strides[2] = {512, (cuuint64_t)chunks * 512};
  const cuuint32_t boxes[3] = {128, 1, (cuuint32_t)tiles}, ones[3] = {1, 1, 1};
  return encoder()(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 3, const_cast<uint8_t*>(p), dims, strides, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// How a product of 8-bit operands is cut up, as cut() for 16-bit ones (in the same units: 0.27 us).  Pairs of 192 columns, 192 alone, 128
// and 64, us: 16384 x 2048 -> 8192 178, 236, 239, 401; 16384 x 256 -> 8192 (2 steps: no pairs) 88, 62, 83, 92; 4096 x 4096 -> 1024 22,
// 25, 21, 32; 64 x 1024 -> 4096 8.1, 7.3, 6.7, 6.0; 64 x 8192 -> 1024 whole 21, 24, 19, 18 and in 8 parts 12.0, 11.3, 10.5, 10.1.
// What the rule takes is the best of them, but for 1000 x 2000 -> 500 (10.0 in two parts, 8.7 whole) and 16384 x 1024 -> 1024 (22.7 in
// pairs, 21.5 alone).
Cut cut_blocks(int64_t m, int64_t n, int64_t c) {
  struct Shape { int width, ctas; double step; };
  static constexpr Shape shapes[] = {{192, 2, 0.68}, {192, 1, 0.75}, {128, 1, 0.55}, {64, 1, 0.4}};
  const int64_t steps = ceil_div(c, 128);
  Cut best{};
  double least = 1e300;
  for (const Shape& s : shapes) {
    if (s.ctas == 2 && steps < 8) continue;
    const int64_t units = kSms / s.ctas, tiles = ceil_div(m, kM * s.ctas) * ceil_div(n, s.width);
    const int64_t splits = tiles >= units ? 1 : std::clamp<int64_t>(units / tiles, 1, std::max<int64_t>(steps / 8, 1));
    const double time = (double)ceil_div(tiles * splits, units) * ((double)ceil_div(steps, splits) * s.step + 8) + (splits > 1 ? 13 : 0);
    if (time < least) least = time, best = Cut{s.width, s.ctas, (int)splits};
  }
  return best;
}

template <typename T, bool kEight, int kN, int kCtas>
cudaError_t launch_shape(const ForwardArgs& p, cudaStream_t s) {
  static std::atomic<uint64_t> allowed{0};  // devices on which the kernel may take its shared memory
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  if (device >= 64 || !(allowed.load(std::memory_order_relaxed) >> device & 1)) {
    e = cudaFuncSetAttribute(k_linear<T, kEight, kN, kCtas>, cudaFuncAttributeMaxDynamicSharedMemorySize, kShared<kEight, kN, kCtas>);
    if (e != cudaSuccess) return e;
    if (device < 64) allowed.fetch_or((uint64_t)1 << device, std::memory_order_relaxed);
  }
  cudaLaunchConfig_t c{};
  c.gridDim = dim3((unsigned)std::min(p.tiles_m * p.tiles_n * p.splits, kSms / kCtas) * kCtas);
  c.blockDim = dim3(kThreads<kEight, kN>);
  c.dynamicSmemBytes = kShared<kEight, kN, kCtas>;
  c.stream = s;
  cudaLaunchAttribute cluster{};
  cluster.id = cudaLaunchAttributeClusterDimension;
  cluster.val.clusterDim.x = kCtas;
  cluster.val.clusterDim.y = cluster.val.clusterDim.z = 1;
  c.attrs = &cluster;
  c.numAttrs = kCtas == 1 ? 0 : 1;
  return cudaLaunchKernelEx(&c, k_linear<T, kEight, kN, kCtas>, p);
}

// the product and what follows it, of operands that TMA can read; `partial`: room for the split sums
template <typename T, bool kEight>
cudaError_t product(const LinearArgs& a, const Cut& k, float* partial, cudaStream_t s) {
  ForwardArgs p{};
  p.m = (int)a.rows; p.n = (int)a.n; p.c = (int)a.k;
  p.tiles_m = (int)ceil_div(a.rows, kM * k.ctas);
  p.tiles_n = (int)ceil_div(a.n, k.width);
  p.steps = (int)ceil_div(a.k, kEight ? 128 : kC);
  p.splits = k.splits;
  if ((int64_t)p.tiles_m * p.tiles_n * p.splits > 0x40000000) return cudaErrorInvalidConfiguration;
  p.act = a.act;
  p.keep = a.z ? kFloats : a.z_values ? kBlocks : kNothing;
  p.a_box = a_box(a.rows);
  p.bias = a.bias; p.bias_f32 = a.bias_f32;
  p.residual = a.residual; p.r_stride = a.r_stride;
  p.wide = a.residual && tma_ready(a.residual, a.r_stride, a.rows, 0);
  p.bias_wide = reinterpret_cast<uintptr_t>(a.bias) % 16 == 0;
  // floor(2^(32 + shift) / d) + 1 with 2^shift < d <= 2^(shift + 1): over by less than i / 2^(32 + shift), below 1 / d for i below 2^31
  const uint32_t band = (uint32_t)(16 / k.ctas * p.tiles_n);
  while (((uint64_t)2 << p.band_shift) < band) p.band_shift++;
  p.band_magic = (uint32_t)(((uint64_t)1 << (32 + p.band_shift)) / band + 1);
  p.out = a.y; p.stride = a.y_stride;
  p.z_values = a.z_values; p.z_pitch = a.z_pitch; p.z_scales = a.z_scales;
  bool ok = true;
  if (kEight) {
    ok = map_values(&p.a, a.x_values, a.rows, a.k, a.xv_stride, p.a_box) && map_values(&p.b, a.w_values, a.n, a.k, a.wv_stride, k.width / k.ctas) &&
         map_scales(&p.a_scales, a.x_scales, a.rows, a.k, 1) && map_scales(&p.b_scales, a.w_scales, a.n, a.k, k.width > 128 ? 2 : 1);
  } else {
    ok = map_matrix(&p.a, kType<T>, a.x, a.rows, a.k, a.x_stride, p.a_box) && map_matrix(&p.b, kType<T>, a.w, a.n, a.k, a.w_stride, k.width / k.ctas);
  }
  const int64_t pitch = up(a.n, 4);
  if (k.splits > 1) {
    ok = ok && map_partial(&p.o, partial, k.splits, a.rows, a.n, pitch);
  } else {
    p.copies = tma_ready(a.y, a.y_stride, a.rows, a.n);
    if (p.copies) ok = ok && map_matrix(&p.o, kType<T>, a.y, a.rows, a.n, a.y_stride, 32, true);
    if (p.keep == kFloats) ok = ok && map_partial(&p.z, a.z, 1, a.rows, a.n, a.z_stride);
  }
  if (!ok) return cudaErrorInvalidValue;
  cudaError_t e;
  if constexpr (kEight)
    e = k.ctas == 2      ? launch_shape<T, true, 192, 2>(p, s)
        : k.width == 192 ? launch_shape<T, true, 192, 1>(p, s)
        : k.width == 128 ? launch_shape<T, true, 128, 1>(p, s)
                         : launch_shape<T, true, 64, 1>(p, s);
  else
    e = k.ctas == 2      ? launch_shape<T, false, 256, 2>(p, s)
        : k.width == 256 ? launch_shape<T, false, 256, 1>(p, s)
        : k.width == 128 ? launch_shape<T, false, 128, 1>(p, s)
                         : launch_shape<T, false, 64, 1>(p, s);
  if (e != cudaSuccess || k.splits == 1) return e;
  const int64_t blocks = std::min<int64_t>(ceil_div(a.rows * up(a.n, 32) / 4, 256), kSms * 8);
  k_finish<T><<<(unsigned)blocks, 256, 0, s>>>(partial, pitch, k.splits, a, ceil_div(a.n, 128));
  return cudaGetLastError();
}

// The workspace: aligned copies of what TMA cannot read (or x out of its blocks), dz, split sums (the forward product's or dx's,
// and dw's) and db's.
bool x_ready(const LinearArgs& a) { return a.x && tma_ready(a.x, a.x_stride, a.rows, a.k); }
bool w_ready(const LinearArgs& a) { return tma_ready(a.w, a.w_stride, a.n, a.k); }
bool dy_ready(const LinearArgs& a) { return tma_ready(a.dy, a.dy_stride, a.rows, a.n); }

// row ranges of k_slope: as many blocks as stay resident
int64_t slope_splits(int64_t rows, int64_t n) { return std::clamp<int64_t>(kSms * 3 / ceil_div(n, 256), 1, ceil_div(rows, 8)); }

struct Layout {
  int64_t k_pitch, n_pitch;
  int parts;
  size_t x, w, dz, partial, partial_w, sums, total;
  Cuts cuts;  // of the backward pass's products
  Layout(int64_t rows, int64_t k, int64_t n, bool activated, bool backward, bool x_copy, bool w_copy, bool dy_copy) {
    k_pitch = up(k, 8);
    n_pitch = up(n, 8);
    parts = activated && in_halves(rows, k, n) ? 2 : 1;
    total = 0;
    const auto take = [&](int64_t bytes) {
      const size_t at = total;
      total += (size_t)up(bytes, 256);
      return at;
    };
    x = take(x_copy ? rows * k_pitch * 2 : 0);
    w = take(w_copy ? n * k_pitch * 2 : 0);
    dz = take(backward && (activated || dy_copy) ? parts * rows * n_pitch * 2 : 0);
    int64_t most = 0, most_w = 0;
    if (rows > 0 && backward) {
      cuts = cut_both(rows, k, n, parts);
      if (cuts.input.splits > 1 || parts > 1) most = cuts.input.splits * parts * rows * up(k, 4);
      if (cuts.weight.splits > 1) most_w = cuts.weight.splits * n * up(k, 4);
    } else if (rows > 0) {
      const Cut f = cut(kInput, rows, n, k, 1, 1);
      if (f.splits > 1) most = f.splits * rows * up(n, 4);
    }
    partial = take(most * 4);
    partial_w = take(most_w * 4);
    sums = take(backward && rows > 0 ? slope_splits(rows, n) * n * 4 : 0);
  }
  static Layout of(const LinearArgs& a, bool backward) {
    return Layout(a.rows, a.k, a.n, a.act != NDVM_ACT_NONE, backward, (!backward || a.dw) && !x_ready(a), (!backward || a.dx) && !w_ready(a),
                  backward && (a.dx || a.dw) && !dy_ready(a));
  }
};

bool vectors_alone(const LinearArgs& a) { return a.rows == 1 && !a.z_values; }

// aligned copies of x and w where they are wanted and not aligned
void make_ready(LinearArgs& a, const Layout& l, bool x, bool w, cudaStream_t s) {
  char* ws = static_cast<char*>(a.workspace);
  PackArgs p{};
  int count = 0;
  int64_t most = 0;
  const auto add = [&](const void*& from, int64_t& stride, int64_t rows, size_t at) {
    p.from[count] = from; p.stride[count] = stride; p.rows[count] = rows; p.to[count] = ws + at;
    most = std::max(most, rows);
    from = ws + at;
    stride = l.k_pitch;
    count++;
  };
  if (x && !x_ready(a)) add(a.x, a.x_stride, a.rows, l.x);
  if (w && !w_ready(a)) add(a.w, a.w_stride, a.n, l.w);
  p.cols = a.k;
  p.pitch = l.k_pitch;
  if (count) launch_pack(p, count, most, s);
}

template <typename T>
cudaError_t forward(LinearArgs a, cudaStream_t s) {
  if (a.rows == 0) return cudaSuccess;
  if (vectors_alone(a)) {
    one<T>(a, x_ready(a) && w_ready(a) && a.k % 8 == 0, s);
    return cudaGetLastError();
  }
  const Layout l = Layout::of(a, false);
  make_ready(a, l, true, true, s);
  return product<T, false>(a, cut(kInput, a.rows, a.n, a.k, 1, 1), reinterpret_cast<float*>(static_cast<char*>(a.workspace) + l.partial), s);
}

template <typename T>
cudaError_t backward(LinearArgs a, cudaStream_t s) {
  cudaError_t e = cudaSuccess;
  if (a.rows == 0) {
    if (a.dw) e = cudaMemsetAsync(a.dw, 0, (size_t)(a.n * a.k) * 2, s);
    if (a.dbias && e == cudaSuccess) e = cudaMemsetAsync(a.dbias, 0, (size_t)a.n * (a.bias_f32 ? 4 : 2), s);
    return e;
  }
  const Layout l = Layout::of(a, true);
  char* ws = static_cast<char*>(a.workspace);
  const bool activated = a.act != NDVM_ACT_NONE, products = a.dx || a.dw;
  const void* dz = a.dy;
  int64_t dz_stride = a.dy_stride;
  if (products && (activated || !dy_ready(a))) dz = ws + l.dz, dz_stride = l.n_pitch;
  if ((products && activated) || a.dbias) {
    SlopeArgs d{};
    d.rows = a.rows; d.n = a.n; d.dy = a.dy; d.dy_stride = a.dy_stride; d.act = a.act;
    d.z = a.z; d.z_stride = a.z_stride; d.z_values = a.z_values; d.z_pitch = a.z_pitch; d.z_scales = a.z_scales;
    if (products && activated) d.dz = ws + l.dz;
    d.pitch = l.n_pitch;
    d.halves = l.parts > 1;
    d.sums = a.dbias ? reinterpret_cast<float*>(ws + l.sums) : nullptr;
    const int64_t splits = slope_splits(a.rows, a.n);
    const dim3 grid((unsigned)ceil_div(a.n, 256), (unsigned)splits);
    const auto launch = [&](auto vectors) {
      constexpr bool kVectors = decltype(vectors)::value;
      if (!activated) k_slope<T, kVectors, kNothing><<<grid, 256, 0, s>>>(d);
      else if (a.z) k_slope<T, kVectors, kFloats><<<grid, 256, 0, s>>>(d);
      else k_slope<T, kVectors, kBlocks><<<grid, 256, 0, s>>>(d);
    };
    if (tma_ready(a.dy, a.dy_stride, a.rows, 0)) launch(std::true_type());
    else launch(std::false_type());
    if (a.dbias) {
      const dim3 join((unsigned)ceil_div(a.n, 32)), block(32, 32);
      if (a.bias_f32) k_columns_join<<<join, block, 0, s>>>(d.sums, (int)splits, 1, a.n, static_cast<float*>(a.dbias), static_cast<float*>(nullptr));
      else k_columns_join<<<join, block, 0, s>>>(d.sums, (int)splits, 1, a.n, static_cast<T*>(a.dbias), static_cast<T*>(nullptr));
    }
  }
  if (products && !activated && !dy_ready(a)) {
    PackArgs p{};
    p.from[0] = a.dy; p.stride[0] = a.dy_stride; p.rows[0] = a.rows; p.to[0] = ws + l.dz;
    p.cols = a.n;
    p.pitch = l.n_pitch;
    launch_pack(p, 1, a.rows, s);
  }
  if (!products) return cudaGetLastError();
  if (a.dw && !a.x) {
    RmsArgs d{};
    d.rows = a.rows; d.cols = a.k; d.values = const_cast<uint8_t*>(a.x_values); d.v_stride = a.xv_stride; d.scales = const_cast<uint8_t*>(a.x_scales);
    d.y = ws + l.x; d.y_stride = l.k_pitch;
    if ((e = launch_dequantize(d, kType<T>, s)) != cudaSuccess) return e;
    a.x = d.y;
    a.x_stride = l.k_pitch;
  }
  make_ready(a, l, a.dw != nullptr, a.dx != nullptr, s);
  // (one of the two alone is cut as if both were wanted: the same bits)
  ProductArgs input{}, weight{};
  if (a.dx) {
    const int64_t m = a.rows * l.parts;
    if (!map_matrix(&input.a[0], kType<T>, dz, m, a.n, dz_stride, a_box(m)) || !map_matrix(&input.b[0], kType<T>, a.w, a.n, a.k, a.w_stride, 64))
      return cudaErrorInvalidValue;
    input.partial = reinterpret_cast<float*>(ws + l.partial);
    input.matrices = input.parts = 1;
    input.m = (int)m; input.n = (int)a.k; input.c = (int)a.n; input.out[0] = a.dx; input.stride = a.dx_stride;
  }
  if (a.dw) {
    for (int half = 0; half < l.parts; half++)
      if (!map_matrix(&weight.a[half], kType<T>, static_cast<const T*>(dz) + half * a.rows * dz_stride, a.rows, a.n, dz_stride, 64)) return cudaErrorInvalidValue;
    if (!map_matrix(&weight.b[0], kType<T>, a.x, a.rows, a.k, a.x_stride, 64)) return cudaErrorInvalidValue;
    weight.partial = reinterpret_cast<float*>(ws + l.partial_w);
    weight.matrices = 1;
    weight.parts = l.parts;
    weight.m = (int)a.n; weight.n = (int)a.k; weight.c = (int)a.rows; weight.out[0] = a.dw; weight.stride = a.k;
  }
  if (a.dx && a.dw) return launch_products(kType<T>, weight, input, l.cuts, s, l.parts > 1);
  if (a.dx) return launch_product(kInput, kType<T>, input, l.cuts.input, s, l.parts > 1);
  return launch_product(kWeight, kType<T>, weight, l.cuts.weight, s);
}

}  // namespace

cudaError_t launch_linear_forward(const LinearArgs& a, ndvm_dtype t, cudaStream_t s) {
  return t == NDVM_F16 ? forward<__half>(a, s) : forward<__nv_bfloat16>(a, s);
}
cudaError_t launch_linear_blocks(const LinearArgs& a, ndvm_dtype t, cudaStream_t s) {
  if (a.rows == 0) return cudaSuccess;
  const Cut k = cut_blocks(a.rows, a.n, a.k);
  float* partial = static_cast<float*>(a.workspace);
  return t == NDVM_F16 ? product<__half, true>(a, k, partial, s) : product<__nv_bfloat16, true>(a, k, partial, s);
}
cudaError_t launch_linear_backward(const LinearArgs& a, ndvm_dtype t, cudaStream_t s) {
  return t == NDVM_F16 ? backward<__half>(a, s) : backward<__nv_bfloat16>(a, s);
}
size_t linear_workspace(int64_t rows, int64_t k, int64_t n, ndvm_activation act, bool backward, bool copies, bool blocks) {
  if (rows == 0) return 0;
  return Layout(rows, k, n, act != NDVM_ACT_NONE, backward, copies || blocks, copies, backward && copies).total;
}
size_t linear_workspace(const LinearArgs& a, bool backward) {
  if (a.rows == 0 || (!backward && vectors_alone(a))) return 0;
  return Layout::of(a, backward).total;
}
size_t linear_blocks_workspace(int64_t rows, int64_t k, int64_t n) {
  if (rows == 0) return 0;
  const Cut c = cut_blocks(rows, n, k);
  return c.splits > 1 ? (size_t)(c.splits * rows * up(n, 4)) * 4 : 0;
}
cudaError_t linear_stopped(int* flag) {
  cudaError_t e = cudaMemcpyFromSymbol(flag, g_linear_stopped, sizeof *flag);
  const int none = 0;
  if (e == cudaSuccess && *flag) e = cudaMemcpyToSymbol(g_linear_stopped, &none, sizeof none);
  return e;
}

}  // namespace ndvm
