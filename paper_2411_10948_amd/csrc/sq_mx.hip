// Quantizer of the microscaled 4-bit format (layout: sq_mx.h) and its inverse.
//
// For each block of 32 consecutive elements: s from max |x| (mx_scale4), codes
// x 2^(127 - s) rounded to E2M1.  Every step is exact but the rounding itself:
// the scale is a power of two taken from the exponent of the maximum.
#include <algorithm>

#include "sq_mx.h"

namespace sq {

namespace {

typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef uint16_t v2u16 __attribute__((ext_vector_type(2)));

// Codes of 8 values, element 0 in the low bits.  The conversion divides by the
// scale and rounds once (to the nearest even, saturating), for every scale
// 2^-127 .. 2^126 and subnormal inputs too.
__device__ __forceinline__ uint32_t codes8(const float* v, float scale) {
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[0], v[1], scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[2], v[3], scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[4], v[5], scale, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, v[6], v[7], scale, 3);
    return r;
}
__device__ __forceinline__ v2bf as_bf16(uint32_t w) {
    v2bf b;
    __builtin_memcpy(&b, &w, 4);
    return b;
}
__device__ __forceinline__ uint32_t codes8(uint32_t a, uint32_t b, uint32_t c, uint32_t d, float scale) {   // bf16 pairs
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, as_bf16(a), scale, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, as_bf16(b), scale, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, as_bf16(c), scale, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, as_bf16(d), scale, 3);
    return r;
}
// running maximum of the magnitudes of two bf16 at once
__device__ __forceinline__ uint32_t pair_max(uint32_t m, uint32_t w) {
    v2u16 a, b;
    w &= 0x7FFF7FFFu;
    __builtin_memcpy(&a, &m, 4);
    __builtin_memcpy(&b, &w, 4);
    a = __builtin_elementwise_max(a, b);
    __builtin_memcpy(&m, &a, 4);
    return m;
}

template <int CTRL>
__device__ __forceinline__ uint32_t quad(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false);
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E;   // quad_perm [1,0,3,2], [2,3,0,1]

// c[i] of lane j of a quad to c[j] of lane i.
__device__ __forceinline__ void transpose4(uint32_t* c, int lane) {
    const bool odd = lane & 1, high = lane & 2;
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
        const uint32_t got = quad<kXor1>(odd ? c[i] : c[i + 1]);
        c[odd ? i : i + 1] = got;
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t got = quad<kXor2>(high ? c[i] : c[i + 2]);
        c[high ? i : i + 2] = got;
    }
}

// Tile of a quantizer block: 128 rows x TC columns, in LDS as they came, for
// the transpose; 128 rows are one tile of the transpose's inner axis.
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

// A wave takes 32 rows of the tile; a row is 8 lanes' (fp32) or 16 lanes'
// (bf16), 8 elements each, so a block of 32 is a quad's and its maximum two
// exchanges away.  After four passes over the rows the quad's codes are
// transposed among its lanes: a lane then holds a whole block, and the wave's
// 16-byte stores cover whole 1 KB tiles.  The other direction reads the tile's
// columns from LDS, one word (one or two columns) a lane.  bf16 stays packed
// from load to code (maximum, conversion): vector instructions, some 20 an
// element, bound the kernel when each one was unpacked and multiplied by the
// scale's inverse.  Bound by HBM now: 8192 x 11008 in bf16 both ways 84 -> 55 us
// (276 MB, 5.0 TB/s, the rate of a large copy), along the columns only 8192 x
// 4096 in 16 us (5.3 TB/s); small inputs by their chain of one load, one
// barrier and one store, 768 x 768 in fp32 both ways 3.5 us.
template <typename T, bool NT>
__global__ __launch_bounds__(256) void k_mx_quantize(MxQuantArgs p, uint32_t tiles_c) {
    constexpr int TC = QuantTile<T>::TC, kLanes = TC / 8, kPass = 64 / kLanes, kPasses = 32 / kPass;
    constexpr int kWords = 8 * sizeof(T) / 4;            // words a lane loads of a row
    constexpr int kCols = 4 / sizeof(T);                 // columns a lane takes of the transpose
    __shared__ __attribute__((aligned(16))) uint32_t tile[128][TC * sizeof(T) / 4];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t tr = blockIdx.x / tiles_c, tc = blockIdx.x - tr * tiles_c;
    const int64_t mat = blockIdx.y;
    int64_t row0 = (int64_t)tr * 128, row_first = row0, row_end = p.rows, inner = row0;
    if (p.offsets) {
        if (p.keep && blockIdx.x == 0)
            for (int i = tid; i <= p.experts; i += 256) p.keep[i] = p.offsets[i];
        if (p.codes_t) {
            const Segment g = find_segment(p.offsets, p.experts, (int)p.rows, 128, (int)tr);
            if (g.expert < 0) return;
            row0 = row_first = (int64_t)g.lo + (int64_t)g.tile * 128;
            row_end = g.hi;
            inner = g.inner + (int64_t)g.tile * 128;
        } else {    // blocks along the columns alone: no tile has to start at an expert's first row, rows of none stay out
            row_first = min(max((int64_t)p.offsets[0], (int64_t)0), p.rows);
            row_end = min(max((int64_t)p.offsets[p.experts], row_first), p.rows);
            if (row0 + 128 <= row_first || row0 >= row_end) return;
        }
    }
    const int64_t col0 = (int64_t)tc * TC;
    const T* x = static_cast<const T*>(p.x) + mat * p.stride;

    const int q = lane % kLanes, r0 = wave * 32 + lane / kLanes;
    const int64_t c = col0 + 8 * q;
    const int left = (int)(p.cols - c);
    uint32_t v[kPasses][kWords];
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        const int64_t r = row0 + r0 + i * kPass;
        const T* src = x + r * p.ld + c;
#pragma unroll
        for (int w = 0; w < kWords; ++w) v[i][w] = 0;
        if (r < row_first || r >= row_end || left <= 0) continue;
        if (left >= 8) {
#pragma unroll
            for (int w = 0; w < kWords; w += 4) {
                const u32x4_any* at = reinterpret_cast<const u32x4_any*>(src + w * 4 / sizeof(T));
                u32x4_any l;
                if constexpr (NT) l = __builtin_nontemporal_load(at);
                else l = *at;
                v[i][w] = l.x;
                v[i][w + 1] = l.y;
                v[i][w + 2] = l.z;
                v[i][w + 3] = l.w;
            }
        } else {    // the last columns: loads without branches, those past the end cleared
            T t[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) t[e] = src[min(e, left - 1)];
#pragma unroll
            for (int e = 0; e < 8; ++e) t[e] = e < left ? t[e] : (T)0;
            __builtin_memcpy(v[i], t, sizeof(t));
        }
    }
    if (p.codes_t) {
#pragma unroll
        for (int i = 0; i < kPasses; ++i)
#pragma unroll
            for (int w = 0; w < kWords; w += 4)
                *reinterpret_cast<uint4*>(&tile[r0 + i * kPass][q * kWords + w]) =
                    make_uint4(v[i][w], v[i][w + 1], v[i][w + 2], v[i][w + 3]);
    }
    if (p.codes) {
        const int64_t units = mx_units(p.cols);
        uint8_t* codes = p.codes + mat * mx_groups(p.rows) * units * kMxUnitBytes;
        uint8_t* scales = p.scales + mat * mx_groups(p.rows) * units * kMxUnitScales;
        const int blk = (int)(c >> 5) & 3;
        codes += (c >> 7) * kMxTileBytes + blk * 256;
        scales += (c >> 9) * kMxUnitScales + blk * 64 + ((c >> 7) & 3);
#pragma unroll
        for (int i = 0; i < kPasses; i += 4) {
            uint32_t k[4], s[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t* w = v[i + j];
                uint32_t b = 0;
                if constexpr (sizeof(T) == 4) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) b = max(b, w[e] & 0x7FFFFFFFu);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) b = pair_max(b, w[e]);
                    b = max(b << 16, b & 0xFFFF0000u);
                }
                b = max(b, quad<kXor1>(b));
                b = max(b, quad<kXor2>(b));
                s[j] = mx_scale4(b);
                const float scale = mx_value(s[j]);
                if constexpr (sizeof(T) == 4) {
                    float f[8];
                    __builtin_memcpy(f, w, sizeof(f));
                    k[j] = codes8(f, scale);
                } else {
                    k[j] = codes8(w[0], w[1], w[2], w[3], scale);
                }
                k[j] = s[j] == 255u ? 0u : k[j];
            }
            transpose4(k, lane);
            const int j = lane & 3;
            const int64_t r = row0 + r0 + (i + j) * kPass, group = (r >> 4) * units;
            const int slot = (int)(r & 15);
            if (r >= row_first && r < row_end) {
                *reinterpret_cast<uint4*>(codes + group * kMxUnitBytes + slot * 16) = make_uint4(k[0], k[1], k[2], k[3]);
                scales[group * kMxUnitScales + slot * 4] = (uint8_t)(j & 2 ? (j & 1 ? s[3] : s[2]) : (j & 1 ? s[1] : s[0]));
            }
        }
    }
    if (!p.codes_t) return;
    __syncthreads();
    if (inner + 128 > p.cap_t) return;   // offsets out of order
    const int64_t units = mx_units(p.cap_t);
    uint8_t* codes = p.codes_t + mat * mx_groups(p.cols) * units * kMxUnitBytes + (inner >> 7) * kMxTileBytes + wave * 256;
    uint8_t* scales = p.scales_t + mat * mx_groups(p.cols) * units * kMxUnitScales + (inner >> 9) * kMxUnitScales + wave * 64 +
                      ((inner >> 7) & 3);
    uint32_t w[32], m = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        w[i] = tile[32 * wave + i][lane];
        if constexpr (sizeof(T) == 4) m = max(m, w[i] & 0x7FFFFFFFu);
        else m = pair_max(m, w[i]);
    }
#pragma unroll
    for (int h = 0; h < kCols; ++h) {
        const int64_t col = col0 + lane * kCols + h;
        const uint32_t s = mx_scale4(kCols == 1 ? m : (h ? m & 0xFFFF0000u : m << 16));
        const float scale = mx_value(s);
        uint32_t k[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (kCols == 1) {
                float f[8];
                __builtin_memcpy(f, w + 8 * i, sizeof(f));
                k[i] = codes8(f, scale);
            } else {
                uint32_t t[4];   // two rows' elements of this column
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    t[e] = __builtin_amdgcn_perm(w[8 * i + 2 * e + 1], w[8 * i + 2 * e], h ? 0x07060302u : 0x05040100u);
                k[i] = codes8(t[0], t[1], t[2], t[3], scale);
            }
            k[i] = s == 255u ? 0u : k[i];
        }
        if (col < p.cols) {
            const int64_t group = (col >> 4) * units;
            const int slot = (int)(col & 15);
            *reinterpret_cast<uint4*>(codes + group * kMxUnitBytes + slot * 16) = make_uint4(k[0], k[1], k[2], k[3]);
            scales[group * kMxUnitScales + slot * 4] = (uint8_t)s;
        }
    }
}

// A thread per block of 32; for looking at codes, not for a hot path.
template <typename T>
__global__ __launch_bounds__(256) void k_mx_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows,
                                                       int64_t cols, T* out, int64_t ld) {
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
    const int64_t tiles_r = a.offsets && a.codes_t ? a.rows / 128 + std::min<int64_t>(a.experts, a.rows) : (a.rows + 127) / 128;
    // Inputs that the last-level cache would not keep anyway are read past it, so
    // that the codes stay there for the product: 8192 x 4096 in bf16 and its product
    // with 11008 columns 208 -> 195 us; a step of 3152 x 768 x 768 in fp32 29.0 ->
    // 31.9 with such loads.  Not where blocks share the lines of a row: 4617 x 7614
    // in fp32 38 us, 52 with them.
    const dim3 grid((uint32_t)(tiles_r * tiles_c), (uint32_t)a.batch);
    if ((double)a.batch * (double)a.rows * (double)a.cols * sizeof(T) >= 32e6 && a.ld * sizeof(T) % 128 == 0)
        k_mx_quantize<T, true><<<grid, 256, 0, s>>>(a, (uint32_t)tiles_c);
    else
        k_mx_quantize<T, false><<<grid, 256, 0, s>>>(a, (uint32_t)tiles_c);
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
