// Internal declarations of the microscaled 4-bit path and of the activations
// with 8-bit checkpoints.  Not part of the public ABI; see include/shiftquant.h.
#pragma once

#include <algorithm>
#include <string>

#include "sq_internal.h"

namespace sq {

// Error reporting of the entry points (sq_abi.hip): the message behind
// sq_last_error, and the status returned.
sq_status fail(sq_status s, const std::string& msg);
sq_status hip_status(hipError_t e, const char* what);

// ---------------------------------------------------------------------------
// Microscaled 4-bit matrix [rows, K]: E2M1 codes with one E8M0 scale for 32
// consecutive elements of a row, laid out as the matrix cores take them
// (v_mfma_scale_f32_16x16x128_f8f6f4: lane l of a wave holds the 32 elements
// of row l % 16 and block l / 16 of a 16 x 128 operand, 16 bytes, and their
// scale).  So a 16 x 128 tile is 1 KB in lane order, [block][row][16 bytes],
// and the scales of 16 x 512 elements are 256 bytes, [block of a tile][row]
// [tile]: one word per lane holds its scales of four consecutive tiles.  The
// tiles of a 16-row group follow each other along K; K is padded to whole
// 512-element units, rows to whole groups.
// ---------------------------------------------------------------------------
constexpr int kMxBlock = 32, kMxTile = 128, kMxUnit = 512, kMxRows = 16;
constexpr int kMxTileBytes = 1024, kMxUnitBytes = 4096, kMxUnitScales = 256;

__host__ __device__ inline int64_t mx_units(int64_t k) { return (k + kMxUnit - 1) / kMxUnit; }
__host__ __device__ inline int64_t mx_groups(int64_t rows) { return (rows + kMxRows - 1) / kMxRows; }
inline int64_t mx_code_bytes(int64_t rows, int64_t k) { return mx_groups(rows) * mx_units(k) * kMxUnitBytes; }
inline int64_t mx_scale_bytes(int64_t rows, int64_t k) { return mx_groups(rows) * mx_units(k) * kMxUnitScales; }
// Inner elements of a matrix whose inner axis holds the rows of `experts`
// segments, each from a multiple of kMxUnit: enough for any split of `rows`.
inline int64_t mx_segment_cols(int64_t rows, int64_t experts) {
    return (rows + (kMxUnit - 1) * std::min(experts, rows)) / kMxUnit * kMxUnit;
}

struct MxQuantArgs {
    const void* x;
    int type;                                  // SQ_TYPE_*
    int64_t batch, rows, cols, ld, stride;     // elements; stride: from matrix to matrix
    const int32_t* offsets;                    // rows of expert e: [offsets[e], offsets[e + 1]); null: one segment
    int experts;
    uint8_t *codes, *scales;                   // blocks along the columns (may be null)
    uint8_t *codes_t, *scales_t;               // the transpose, blocks along the rows (may be null)
    int64_t cap_t;                             // inner elements of the transpose
    int32_t* keep;                             // a copy of the offsets (may be null)
};
hipError_t launch_mx_quantize(const MxQuantArgs& a, hipStream_t s);
hipError_t launch_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* out,
                                int type, int64_t ld, hipStream_t s);

// C[i, j] = sum_k A(i, k) B(j, k).
//   kDense         one product
//   kExpertRows    rows [offsets[e], offsets[e + 1]) of A and C with matrix e of B
//   kExpertInner   C[e] from the inner elements of segment e of A and B (launch_mx_quantize's segments)
enum MxMode { kDense = 0, kExpertRows = 1, kExpertInner = 2 };
struct MxGemmArgs {
    MxMode mode;
    int64_t M, N, K;                       // kExpertInner: K = inner elements of A and B (mx_segment_cols)
    const uint8_t *A, *As, *B, *Bs;
    const int32_t* offsets;
    int experts;
    int64_t rows;                          // kExpertInner: rows that the offsets split
    void* C;
    int type;
    int64_t ldc;                           // kExpertInner: matrix e at e * M * ldc
    float* part;                           // split-K partials [splits, M, N] (kDense)
};
int64_t mx_gemm_splits(const MxGemmArgs& a);      // K splits of the product (1 unless kDense)
hipError_t launch_mx_gemm(const MxGemmArgs& a, hipStream_t s);
// Both products, one launch where they take the same tiles: two of kDense, or
// kExpertRows and kExpertInner.  Their K splits' partials must not overlap.
hipError_t launch_mx_gemm_pair(const MxGemmArgs& a, const MxGemmArgs& b, hipStream_t s);

// Few rows: Y = X W^T with the rows of X quantized on the way.
struct MxRowsArgs {
    const void* x;
    int type;
    int64_t M, K, ld;
    const uint8_t *W, *Ws;
    int64_t N;
    const int32_t* offsets;
    int experts;
    void* Y;
    int out_type;
    int64_t ldy;
};
bool mx_rows_ok(int64_t M, int64_t K, int64_t N, int64_t experts, int type);
hipError_t launch_mx_rows(const MxRowsArgs& a, hipStream_t s);

// ---- activations (sq_act.hip) ----
struct ActArgs {
    int kind, gated, type;
    int64_t M, F, ld_x, ld_h;      // x [M, F or 2 F] (gate first), h [M, F]
    const void* x;                 // forward: input; backward: unused
    void* h;                       // forward: output; backward: dh (read)
    void* dx;                      // backward: [M, F or 2 F], leading dimension ld_x
    int8_t* codes;                 // [M, ld_codes], gate columns [0, Fp), then up columns [Fp, 2 Fp), Fp = roundup(F, 32)
    uint8_t* scales;               // [M, ld_codes / 32]
};
hipError_t launch_act_forward(const ActArgs& a, hipStream_t s);
hipError_t launch_act_backward(const ActArgs& a, hipStream_t s);

// ---- device helpers ----
#if defined(__HIPCC__)
// Scale byte of a block whose largest |x| has the bits `b` (an fp32 without its
// sign): the smallest power of two 2^(s - 127) with max |x| / 2^(s - 127)
// rounding into the format.  4-bit: at most 7 (rounds to 6, half a step), so
// a significand above 1.75 carries into the exponent; 8-bit: below 127.5.
// Inf and NaN: 255.
__device__ __forceinline__ uint32_t mx_scale4(uint32_t b) {
    return b >= 0x7F800000u ? 255u : (uint32_t)max((int)((b + 0x1FFFFFu) >> 23) - 2, 0);
}
__device__ __forceinline__ uint32_t mx_scale8(uint32_t b) {
    return b >= 0x7F800000u ? 255u : (uint32_t)max((int)((b + 0x10000u) >> 23) - 6, 0);
}
// 2^(127 - s), the factor from values to codes; 0 for s = 255 (every code 0)
__device__ __forceinline__ float mx_inverse(uint32_t s) {
    return s == 255u ? 0.0f : __uint_as_float((254u - s) << 23);
}
// 2^(s - 127); NaN for s = 255
__device__ __forceinline__ float mx_value(uint32_t s) {
    return __uint_as_float(s == 255u ? 0x7FC00000u : s == 0u ? 0x00400000u : s << 23);
}

// The expert whose tiles of `unit` rows hold tile `index`, counted over all
// experts; offsets out of order or out of range cut the expert short, never
// past `rows`.  Called by whole waves.
struct Segment {
    int expert = -1;      // -1: past the last tile
    int lo = 0, hi = 0;   // rows of the expert
    int tile = 0;         // index of the tile within it
    int64_t inner = 0;    // first inner element of the expert in a segmented transpose
};
__device__ __forceinline__ void segment_of(const int32_t* offsets, int experts, int rows, int e, int& lo, int& hi) {
    lo = hi = 0;
    if (e < experts) {
        lo = min(max(offsets[e], 0), rows);
        hi = min(max(offsets[e + 1], lo), rows);
    }
}
// Inclusive sum over the lanes of a wave: within rows of 16 lanes by shifts,
// then the row totals broadcast onward.  Every lane must be active.
__device__ __forceinline__ int wave_scan(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);   // row_shr:1
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);   // row_shr:2
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);   // row_shr:4
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);   // row_shr:8
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);   // row_bcast:15 into rows 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);   // row_bcast:31 into rows 2 and 3
    return v;
}
__device__ __forceinline__ Segment find_segment(const int32_t* offsets, int experts, int rows, int unit, int index) {
    const int lane = threadIdx.x & 63;
    Segment r;
    int tiles = 0;
    int64_t inner = 0;
    for (int base = 0; base < experts; base += 64) {
        int lo, hi;
        segment_of(offsets, experts, rows, base + lane, lo, hi);
        const int t = (hi - lo + unit - 1) / unit, k = (hi - lo + kMxUnit - 1) / kMxUnit;
        const int ti = wave_scan(t), ki = wave_scan(k);
        const uint64_t hit = __ballot(index >= tiles + ti - t && index < tiles + ti);
        if (hit) {
            const int src = __ffsll((unsigned long long)hit) - 1;
            r.expert = base + src;
            r.lo = __builtin_amdgcn_readlane(lo, src);
            r.hi = __builtin_amdgcn_readlane(hi, src);
            r.tile = index - tiles - __builtin_amdgcn_readlane(ti - t, src);
            r.inner = inner + (int64_t)__builtin_amdgcn_readlane(ki - k, src) * kMxUnit;
            return r;
        }
        tiles += __builtin_amdgcn_readlane(ti, 63);
        inner += (int64_t)__builtin_amdgcn_readlane(ki, 63) * kMxUnit;
    }
    return r;
}
// find_segment(index_of(tiles of all experts)); none for a negative index.  Up to
// 64 experts take one look at the offsets.
template <class F>
__device__ __forceinline__ Segment find_segment_of(const int32_t* offsets, int experts, int rows, int unit, F index_of) {
    const int lane = threadIdx.x & 63;
    int lo, hi;
    segment_of(offsets, experts, rows, lane, lo, hi);
    const int t = (hi - lo + unit - 1) / unit, ti = wave_scan(t), first = __builtin_amdgcn_readlane(ti, 63);
    int total = first;
    for (int base = 64; base < experts; base += 64) {
        int l, h;
        segment_of(offsets, experts, rows, base + lane, l, h);
        total += __builtin_amdgcn_readlane(wave_scan((h - l + unit - 1) / unit), 63);
    }
    const int index = index_of(total);
    Segment r;
    if (index < 0) return r;
    if (index >= first) return find_segment(offsets, experts, rows, unit, index);
    const uint64_t hit = __ballot(index >= ti - t && index < ti);
    if (!hit) return r;
    const int src = __ffsll((unsigned long long)hit) - 1;
    r.expert = src;
    r.lo = __builtin_amdgcn_readlane(lo, src);
    r.hi = __builtin_amdgcn_readlane(hi, src);
    r.tile = index - __builtin_amdgcn_readlane(ti - t, src);
    return r;
}
// Inner elements before expert e in a segmented transpose, and its rows.
__device__ __forceinline__ void segment_inner(const int32_t* offsets, int experts, int rows, int e, int64_t& inner,
                                              int& len) {
    const int lane = threadIdx.x & 63;
    inner = 0;
    len = 0;
    for (int base = 0; base < experts; base += 64) {
        int lo, hi;
        segment_of(offsets, experts, rows, base + lane, lo, hi);
        const int k = (hi - lo + kMxUnit - 1) / kMxUnit, ki = wave_scan(k);
        if (e < base + 64) {
            inner += (int64_t)__builtin_amdgcn_readlane(ki - k, e - base) * kMxUnit;
            len = __builtin_amdgcn_readlane(hi - lo, e - base);
            return;
        }
        inner += (int64_t)__builtin_amdgcn_readlane(ki, 63) * kMxUnit;
    }
}

// 16 bytes at any element's address: gfx950 loads and stores them unaligned, so
// odd row strides and views need no path of their own.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

__device__ __forceinline__ float bf16_value(uint32_t b) { return __uint_as_float(b << 16); }
// round to nearest even; NaN stays NaN
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
    typedef float v2f __attribute__((ext_vector_type(2)));
    typedef __bf16 v2b __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v2f{a, b}, v2b));
}
__device__ __forceinline__ uint32_t bf16_bits(float v) { return bf16_pair(v, 0.0f) & 0xFFFFu; }
#endif

}  // namespace sq
