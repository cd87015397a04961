// Internal declarations of the dense layers in 8-bit floating point.  Not part of
// the public ABI; see include/shiftquant.h.
#pragma once

#include "sq_mx.h"

namespace sq {

// ---------------------------------------------------------------------------
// Matrix [rows, K] in E4M3 with one E8M0 scale for 128 consecutive elements of a
// row (or for 128 x 128, repeated for each row), laid out for the matrix cores
// (v_mfma_scale_f32_*_f8f6f4, 32 elements a lane): a tile of 16 rows x 128 elements
// is 2 KB, [16 elements][row][16 bytes], its halves of 64 elements 1 KB each, so a
// wave loads either and reads its operands in whole contiguous lines.  Which inner
// elements meet in a lane does not matter to a sum as long as both operands agree,
// and one scale covers the tile.  Tiles of a 16-row group follow each other along
// K; K is padded to units of 512, whose scales are 64 bytes, [row][tile].
// ---------------------------------------------------------------------------
constexpr int kF8TileBytes = 2048, kF8HalfBytes = 1024, kF8UnitBytes = 8192, kF8UnitScales = 64;

inline int64_t f8_code_bytes(int64_t rows, int64_t k) { return mx_groups(rows) * mx_units(k) * kF8UnitBytes; }
inline int64_t f8_scale_bytes(int64_t rows, int64_t k) { return mx_groups(rows) * mx_units(k) * kF8UnitScales; }

struct F8QuantArgs {
    const void* x;
    int type;                           // SQ_TYPE_*
    int64_t rows, cols, ld;
    int square;                         // one scale for 128 x 128
    uint8_t *codes, *scales;            // blocks along the columns (may be null)
    uint8_t *codes_t, *scales_t;        // the transpose, blocks along the rows (may be null)
};
hipError_t launch_f8_quantize(const F8QuantArgs& a, hipStream_t s);
hipError_t launch_f8_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* out, int type,
                                int64_t ld, hipStream_t s);

// C[i, j] = sum_k A(i, k) B(j, k)
struct F8GemmArgs {
    int64_t M, N, K;
    const uint8_t *A, *As, *B, *Bs;
    void* C;
    int type;
    int64_t ldc;
    float* part;                        // split-K partials [splits, M, N]
};
int64_t f8_gemm_splits(int64_t M, int64_t N, int64_t K, int type);      // type of the result
hipError_t launch_f8_gemm(const F8GemmArgs& a, hipStream_t s);
// Both products, in one launch where they take the same tiles; their partials must not overlap.
hipError_t launch_f8_gemm_pair(const F8GemmArgs& a, const F8GemmArgs& b, hipStream_t s);

// Few rows: Y = X W^T with the rows of X quantized on the way.
struct F8RowsArgs {
    const void* x;
    int type;
    int64_t M, K, ld;
    const uint8_t *W, *Ws;
    int64_t N;
    void* Y;
    int out_type;
    int64_t ldy;
};
bool f8_rows_ok(int64_t M, int64_t K, int64_t N, int type);
hipError_t launch_f8_rows(const F8RowsArgs& a, hipStream_t s);

#if defined(__HIPCC__)
// Scale byte of a block whose largest |x| has the bits `b`: the smallest power of
// two 2^(s - 127) with max |x| / 2^(s - 127) <= 464 = 1.8125 2^8 (rounds to 448,
// half a step).  Inf and NaN: 255.
__device__ __forceinline__ uint32_t f8_scale(uint32_t b) {
    return b >= 0x7F800000u ? 255u : (uint32_t)max((int)((b + 0x17FFFFu) >> 23) - 8, 0);
}
#endif

}  // namespace sq
