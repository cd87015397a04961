// Quantizer of the microscaled 4-bit format (layout: sq_mx.h) and its inverse.
//
// For each block of 32 consecutive elements: s from max |x| (mx_scale4), codes
// x 2^(127 - s) rounded to E2M1.  Every step is exact but the rounding itself:
// the scale is a power of two taken from the exponent of the maximum.
#include <algorithm>

#include "sq_mx.h"

namespace sq {

namespace {

typedef float v4f __attribute__((ext_vector_type(4)));

// codes of 8 values already divided by their scale, element 0 in the low bits
__device__ __forceinline__ uint32_t codes8(const float* v) {
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[0], v[1], 1.0f, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2], v[3], 1.0f, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4], v[5], 1.0f, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6], v[7], 1.0f, 3);
    return r;
}

// Tile of a quantizer block: 128 rows x TC columns, in LDS as they came, for
// both directions.  128 rows are one tile of the transpose's inner axis.
template <typename T>
struct QuantTile;
template <>
struct QuantTile<float> {
    static constexpr int TC = 64;
};
template <>
struct QuantTile<uint16_t> {   // bf16 bits
    static constexpr int TC = 128;
};

template <typename T>
__device__ __forceinline__ float value_of(T v);
template <>
__device__ __forceinline__ float value_of<float>(float v) { return v; }
template <>
__device__ __forceinline__ float value_of<uint16_t>(uint16_t v) { return bf16_value(v); }

// Eight lanes (fp32) or sixteen (bf16) hold a row of the tile, 8 elements
// each, so a block of 32 is four lanes' and its maximum two exchanges away.
// The transposed direction reads the tile's columns from LDS, one word (one
// or two columns) a lane.
template <typename T>
__global__ __launch_bounds__(256) void k_mx_quantize(MxQuantArgs p, int64_t tiles_c, bool vec) {
    constexpr int TC = QuantTile<T>::TC, kLanes = TC / 8, kPass = 256 / kLanes, kPasses = 128 / kPass;
    constexpr int kCols = 4 / sizeof(T);                 // columns a lane takes of the transpose
    __shared__ __attribute__((aligned(16))) T tile[128][TC];

    const int tid = threadIdx.x;
    const int64_t tr = blockIdx.x / tiles_c, tc = blockIdx.x - tr * tiles_c, mat = blockIdx.y;
    int64_t row0 = tr * 128, row_end = p.rows, inner = row0;
    if (p.offsets) {
        const Segment g = find_segment(p.offsets, p.experts, (int)p.rows, 128, (int)tr);
        if (g.expert < 0) return;
        row0 = (int64_t)g.lo + (int64_t)g.tile * 128;
        row_end = g.hi;
        inner = g.inner + (int64_t)g.tile * 128;
    }
    const int64_t col0 = tc * TC;
    const T* x = static_cast<const T*>(p.x) + mat * p.stride;

    const int q = tid % kLanes, r0 = tid / kLanes;
    const int64_t c = col0 + 8 * q;
    T v[kPasses][8];
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        const int64_t r = row0 + r0 + i * kPass;
        const T* src = x + r * p.ld + c;
        if (r < row_end && vec && c + 8 <= p.cols) {
#pragma unroll
            for (int w = 0; w < (int)(8 * sizeof(T) / 16); ++w)
                reinterpret_cast<uint4*>(v[i])[w] = reinterpret_cast<const uint4*>(src)[w];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[i][e] = r < row_end && c + e < p.cols ? src[e] : (T)0;
        }
    }
    if (p.codes) {
        const int64_t units = mx_units(p.cols);
        uint8_t* codes = p.codes + mat * mx_groups(p.rows) * units * kMxUnitBytes;
        uint8_t* scales = p.scales + mat * mx_groups(p.rows) * units * kMxUnitScales;
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const int64_t r = row0 + r0 + i * kPass;
            float f[8];
            uint32_t b = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                f[e] = value_of<T>(v[i][e]);
                b = max(b, __float_as_uint(f[e]) & 0x7FFFFFFFu);
            }
            b = max(b, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b, 0xB1, 0xF, 0xF, false));   // lane ^ 1
            b = max(b, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b, 0x4E, 0xF, 0xF, false));   // lane ^ 2
            const uint32_t s = mx_scale4(b);
            const float inv = mx_inverse(s);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = s == 255u ? 0.0f : f[e] * inv;
            if (r < row_end) {
                const int64_t group = r >> 4;
                const int slot = (int)(r & 15), blk = (int)(c >> 5) & 3;
                *reinterpret_cast<uint32_t*>(codes + (group * units * 4 + (c >> 7)) * kMxTileBytes + blk * 256 + slot * 16 +
                                             (q & 3) * 4) = codes8(f);
                if ((q & 3) == 0)
                    scales[(group * units + (c >> 9)) * kMxUnitScales + blk * 64 + slot * 4 + ((c >> 7) & 3)] = (uint8_t)s;
            }
        }
    }
    if (!p.codes_t) return;
#pragma unroll
    for (int i = 0; i < kPasses; ++i)
#pragma unroll
        for (int w = 0; w < (int)(8 * sizeof(T) / 16); ++w)
            reinterpret_cast<uint4*>(&tile[r0 + i * kPass][8 * q])[w] = reinterpret_cast<uint4*>(v[i])[w];
    __syncthreads();
    if (inner + 128 > p.cap_t) return;   // offsets out of order
    const int64_t units = mx_units(p.cap_t);
    uint8_t* codes = p.codes_t + mat * mx_groups(p.cols) * units * kMxUnitBytes;
    uint8_t* scales = p.scales_t + mat * mx_groups(p.cols) * units * kMxUnitScales;
    const int word = tid & 63, blk = tid >> 6;
    uint32_t w[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) w[i] = reinterpret_cast<const uint32_t*>(&tile[32 * blk + i][0])[word];
#pragma unroll
    for (int h = 0; h < kCols; ++h) {
        const int64_t col = col0 + word * kCols + h;
        float f[32];
        uint32_t b = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            f[i] = kCols == 1 ? __uint_as_float(w[i]) : __uint_as_float(h ? w[i] & 0xFFFF0000u : w[i] << 16);
            b = max(b, __float_as_uint(f[i]) & 0x7FFFFFFFu);
        }
        const uint32_t s = mx_scale4(b);
        const float inv = mx_inverse(s);
#pragma unroll
        for (int i = 0; i < 32; ++i) f[i] = s == 255u ? 0.0f : f[i] * inv;
        if (col < p.cols) {
            const int64_t group = col >> 4;
            const int slot = (int)(col & 15);
            *reinterpret_cast<uint4*>(codes + (group * units * 4 + (inner >> 7)) * kMxTileBytes + blk * 256 + slot * 16) =
                make_uint4(codes8(f), codes8(f + 8), codes8(f + 16), codes8(f + 24));
            scales[(group * units + (inner >> 9)) * kMxUnitScales + blk * 64 + slot * 4 + ((inner >> 7) & 3)] = (uint8_t)s;
        }
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows,
                                                       int64_t cols, T* out, int64_t ld) {
    // a thread per block of 32
    const int64_t blocks = (cols + kMxBlock - 1) / kMxBlock, units = mx_units(cols);
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= rows * blocks) return;
    const int64_t r = i / blocks, c = (i - r * blocks) * kMxBlock, group = r >> 4;
    const int slot = (int)(r & 15), blk = (int)(c >> 5) & 3;
    const uint8_t* src = codes + (group * units * 4 + (c >> 7)) * kMxTileBytes + blk * 256 + slot * 16;
    const float scale =
        mx_value(scales[(group * units + (c >> 9)) * kMxUnitScales + blk * 64 + slot * 4 + ((c >> 7) & 3)]);
    for (int e = 0; e < kMxBlock && c + e < cols; ++e) {
        const uint32_t k = (src[e >> 1] >> (4 * (e & 1))) & 15u, m = k & 7u;
        // 0, 0.5, then 2^(m / 2 - 1) (1 + (m % 2) / 2)
        const float a = m < 2 ? 0.5f * (float)m : __uint_as_float((m / 2 + 126u) << 23 | (m & 1u) << 22);
        const float v = (k & 8u ? -a : a) * scale;
        if constexpr (sizeof(T) == 4) out[r * ld + c + e] = v;
        else out[r * ld + c + e] = (T)bf16_bits(v);
    }
}

template <typename T>
hipError_t quantize(const MxQuantArgs& a, hipStream_t s) {
    constexpr int TC = QuantTile<T>::TC;
    // whole 128-element tiles of the columns, so that the row codes' padding is written too
    const int64_t tiles_c = round_up(a.cols, kMxTile) / TC;
    const int64_t tiles_r = a.offsets ? a.rows / 128 + std::min<int64_t>(a.experts, a.rows) : (a.rows + 127) / 128;
    const bool vec = (reinterpret_cast<uintptr_t>(a.x) & 15) == 0 && (a.ld * sizeof(T)) % 16 == 0 &&
                     (a.batch == 1 || (a.stride * sizeof(T)) % 16 == 0);
    k_mx_quantize<T><<<dim3((uint32_t)(tiles_r * tiles_c), (uint32_t)a.batch), 256, 0, s>>>(a, tiles_c, vec);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_quantize(const MxQuantArgs& a, hipStream_t s) {
    if (a.batch == 0 || a.rows == 0 || a.cols == 0) return hipSuccess;
    return a.type == SQ_TYPE_F32 ? quantize<float>(a, s) : quantize<uint16_t>(a, s);
}

hipError_t launch_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* out,
                                int type, int64_t ld, hipStream_t s) {
    const int64_t n = rows * ((cols + kMxBlock - 1) / kMxBlock);
    if (n == 0) return hipSuccess;
    const dim3 grid((uint32_t)((n + 255) / 256));
    if (type == SQ_TYPE_F32) k_mx_dequantize<float><<<grid, 256, 0, s>>>(codes, scales, rows, cols, (float*)out, ld);
    else k_mx_dequantize<uint16_t><<<grid, 256, 0, s>>>(codes, scales, rows, cols, (uint16_t*)out, ld);
    return hipGetLastError();
}

}  // namespace sq
