// Products on the tensor cores that the gated projection and the dense layers share: D[m, n] = sum over c of
// A[m, c] B[n, c] (product.cu), what cuts them up, the tensor maps of their operands, and aligned copies of operands
// that TMA cannot read.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>

#include <algorithm>

#include "net.h"

namespace ndvm {

enum Mode { kForward, kGradient, kInput, kWeight, kBoth };

constexpr int kM = 128, kC = 64;  // rows of a tile, contraction of a step (128 bytes)

struct ProductArgs {
  CUtensorMap a[4], b[2];        // kWeight: a's are the first matrix's parts, then the second's
  CUtensorMap o[2];              // the results (kGradient: dG and dU), or o[0] the split sums
  CUtensorMap dh;                // kGradient
  CUtensorMap kept;              // kForward: where G and U go in binary32, if keep
  int keep;
  int m, n, c;                   // rows and columns of the result, contraction of one segment
  int tiles_m, tiles_n, matrices;  // matrices: results of one shape, by the a's (kWeight: 1 or 2), else 1
  int parts;                     // segments of the contraction, by the a's: kInput (dG and dU), kWeight (a matrix, or its two halves)
  int steps, splits;             // contraction steps of a result, and how many parts they are cut into
  int act;
  int a_box;                     // rows of A that a tile loads (fewer than 128 where the result has fewer)
  int rows;                      // A's rows are contiguous, and not its contraction
  int sums;                      // results are binary32 sums, which k_join finishes
  int copies;                    // results are stored by copies (their rows start on 16 bytes)
  void* out[2]; int64_t stride;  // kWeight: both matrices'; kGradient: dG and dU; else out[0]
  float* partial; int64_t partial_pitch;  // splits > 1: [split][matrix][m][pitch]
};

// how a product of the given size is cut up: columns and rows of a tile's sums (256 rows are a pair's), parts
struct Cut { int width, ctas, splits; };
Cut cut(Mode mode, int64_t m, int64_t n, int64_t c, int parts, int matrices);
struct Cuts { Cut weight, input; };  // (of one width)
Cuts cut_both(int64_t rows, int64_t k, int64_t n, int parts);
// t: half or bfloat16.  fold: the result's rows come twice (two halves of A), and are added up.
cudaError_t launch_product(Mode mode, ndvm_dtype t, ProductArgs& p, const Cut& k, cudaStream_t s, bool fold = false);
// a dense layer's two gradients in one launch (fold: of the input's)
cudaError_t launch_products(ndvm_dtype t, ProductArgs& weight, ProductArgs& input, const Cuts& k, cudaStream_t s, bool fold);

inline int64_t up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int a_box(int64_t m) { return (int)std::min<int64_t>(up(m, 8), kM); }
inline bool tma_ready(const void* p, int64_t stride, int64_t rows, int64_t cols) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (rows == 1 || (stride % 8 == 0 && stride >= cols));
}

using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                            const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                            CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
Encode encoder();  // null: the driver has no such function
// A matrix of `rows` rows of `cols` contiguous elements, read in boxes of 64 columns and `box` rows in the
// 128-byte swizzle; or in boxes of 32 by 32 (results, and dh: 64 bytes a row, the 64-byte swizzle).
bool map_matrix(CUtensorMap* map, ndvm_dtype t, const void* p, int64_t rows, int64_t cols, int64_t stride, int box, bool piece = false);
// split sums: `parts` matrices of m rows, written in boxes of 32 by 32
bool map_partial(CUtensorMap* map, float* p, int64_t parts, int64_t m, int64_t n, int64_t pitch);

// Up to three matrices of `cols` columns to rows that start on 16 bytes (TMA reads no others): a warp a row, 16 bytes
// a lane, out of the one or two aligned 16-byte blocks that hold them.  What lies before and behind a row is not read
// (it need not be the caller's): the blocks at its two ends are read element by element.
struct PackArgs {
  const void* from[3];
  void* to[3];
  int64_t stride[3], rows[3];
  int64_t cols, pitch;
};
void launch_pack(const PackArgs& p, int count, int64_t most_rows, cudaStream_t s);

// Few elements: dG and dU are handed on in two halves of 16 bits, so that next to nothing is lost before the last
// rounding.  (Over many elements the rounding of dG and dU adds to the results' own as squares add, 1.41 times in
// all; over few it scatters, to more than twice: 4096 elements leave 1.2 to 1.55, 16384 1.37 to 1.49.)  dx has the halves' rows
// one after the other in its tiles, the weights' gradients twice the steps, and G and U are made in binary32 first.  A gated step with
// the products kept, bf16, with and without halves: 8 x 2048 -> 8192 66 / 55 us, 16 x 1024 -> 4096 32 / 27, 64 x 256 -> 512 20.0 /
// 18.8, 4096 x 32 -> 64 25 / 21; the cost grows with the rows where n k is small (65536 x 32 -> 64 72 / 61, and 82 / 60 with
// nothing kept) and with n where k is (1000 x 16 -> 8192 76 / 64).
inline bool in_halves(int64_t rows, int64_t k, int64_t n) { return rows * std::min(n, k) <= 16384 || n * k <= 2048; }

}  // namespace ndvm
