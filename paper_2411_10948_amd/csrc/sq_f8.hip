// Quantizer of the 8-bit floating-point format (layout: sq_f8.h) and its inverse.
//
// For each block of 128 consecutive elements, or of 128 x 128: s from max |x|
// (f8_scale), codes x 2^(127 - s) rounded to E4M3.  Every step is exact but the
// rounding itself: the scale is a power of two taken from the exponent of the
// maximum.  One read for both axes, bound by HBM: 8192 x 11008 in bf16 to codes along
// both 62 us, 5.8 TB/s; 3152 x 768 in fp32 6.1 us, where the launch and the two
// dependent passes count.
#include <algorithm>
#include <type_traits>

#include "sq_f8.h"

namespace sq {

namespace {

typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef uint16_t v2u16 __attribute__((ext_vector_type(2)));
typedef short v2i16 __attribute__((ext_vector_type(2)));

// Codes of 4 values, element 0 in the low byte.  The conversion divides by the scale
// and rounds once, to the nearest even, for every scale 2^-127 .. 2^126 and
// subnormal inputs too; nothing is past 464, so nothing overflows.
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, float scale) {
    v2i16 r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, a, b, scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, c, d, scale, true);
    return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ uint32_t codes4(uint32_t ab, uint32_t cd, float scale) {     // bf16 pairs
    v2i16 r = {0, 0};
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(v2bf, ab), scale, false);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(v2bf, cd), scale, true);
    return __builtin_bit_cast(uint32_t, r);
}
// running maximum of the magnitudes of two bf16 at once
__device__ __forceinline__ uint32_t pair_max(uint32_t m, uint32_t w) {
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(v2u16, m), __builtin_bit_cast(v2u16, w & 0x7FFF7FFFu)));
}
template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false);
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kMirror8 = 0x141, kMirror16 = 0x140;
// maximum over the 16 lanes of a row
__device__ __forceinline__ uint32_t max16(uint32_t b) {
    b = max(b, moved<kXor1>(b));
    b = max(b, moved<kXor2>(b));
    b = max(b, moved<kMirror8>(b));
    return max(b, moved<kMirror16>(b));
}

// A block takes 128 x 128 elements.  A row is 16 lanes', 8 elements each, and its
// maximum four exchanges away; after two passes over the rows neighbouring lanes
// trade halves, so that each holds 16 elements of one row and stores 16 bytes, 128
// contiguous ones for 8 rows.  The other direction reads the tile's columns from
// LDS, one word (one or two columns) and 32 rows a lane, and takes the waves' maxima
// together there.  APART: two blocks take a tile, the first `tiles` of them one axis each,
// the others the other one.
template <typename T, bool SQUARE, bool APART>
__global__ __launch_bounds__(sizeof(T) == 4 ? 512 : 256) void k_f8_quantize(F8QuantArgs p, uint32_t tiles_c, uint32_t tiles) {
    constexpr int kWaves = sizeof(T) == 4 ? 8 : 4, kPasses = 32 / kWaves;     // 4 rows a pass
    constexpr int kWords = 8 * sizeof(T) / 4, kCols = 4 / sizeof(T);
    constexpr int kRowWords = 128 * sizeof(T) / 4;
    __shared__ __attribute__((aligned(16))) uint32_t tile[128][kRowWords];
    __shared__ uint32_t most[4][128];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint32_t block = blockIdx.x;
    if constexpr (APART) {
        if (block < tiles) {
            p.codes_t = nullptr;
        } else {
            p.codes = nullptr;
            block -= tiles;
        }
    }
    const uint32_t tr = block / tiles_c, tc = block - tr * tiles_c;
    const int64_t row0 = (int64_t)tr * 128, col0 = (int64_t)tc * 128;
    const T* x = static_cast<const T*>(p.x);
    const int q = lane & 15, r0 = wave * (4 * kPasses) + (lane >> 4);
    const int64_t c = col0 + 8 * q;
    const int left = (int)min(p.cols - c, (int64_t)8);
    uint32_t v[kPasses][kWords], peak[kPasses];
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        const int64_t r = row0 + r0 + 4 * i;
        const T* src = x + r * p.ld + c;
#pragma unroll
        for (int w = 0; w < kWords; ++w) v[i][w] = 0;
        if (r >= p.rows || left <= 0) continue;
        if (left == 8) {
#pragma unroll
            for (int w = 0; w < kWords; w += 4) {
                const u32x4_any l = *reinterpret_cast<const u32x4_any*>(src + w * 4 / sizeof(T));
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
                *reinterpret_cast<uint4*>(&tile[r0 + 4 * i][q * kWords + w]) = make_uint4(v[i][w], v[i][w + 1], v[i][w + 2], v[i][w + 3]);
    }
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        uint32_t b = 0;
        if (APART && !SQUARE && !p.codes) break;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int e = 0; e < 8; ++e) b = max(b, v[i][e] & 0x7FFFFFFFu);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) b = pair_max(b, v[i][e]);
            b = max(b << 16, b & 0xFFFF0000u);
        }
        peak[i] = max16(b);
    }
    uint32_t whole = 0;
    if constexpr (SQUARE) {
        uint32_t b = peak[0];
#pragma unroll
        for (int i = 1; i < kPasses; ++i) b = max(b, peak[i]);
        if (q == 0) most[0][tid >> 4] = b;      // of 16 lanes
        __syncthreads();
        for (int i = 0; i < 4 * kWaves; ++i) whole = max(whole, most[0][i]);
        whole = f8_scale(whole);
    }
    if (p.codes) {
        const int64_t units = mx_units(p.cols);
        uint8_t* codes = p.codes + (col0 >> 7) * kF8TileBytes + (q >> 1) * 256;
        uint8_t* scales = p.scales + (col0 >> 9) * kF8UnitScales + ((col0 >> 7) & 3);
#pragma unroll
        for (int i = 0; i < kPasses; i += 2) {
            uint32_t k[2][2], s[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t* w = v[i + j];
                s[j] = SQUARE ? whole : f8_scale(peak[i + j]);
                const float scale = mx_value(s[j]);
                if constexpr (sizeof(T) == 4) {
                    float f[8];
                    __builtin_memcpy(f, w, sizeof(f));
                    k[j][0] = codes4(f[0], f[1], f[2], f[3], scale);
                    k[j][1] = codes4(f[4], f[5], f[6], f[7], scale);
                } else {
                    k[j][0] = codes4(w[0], w[1], scale);
                    k[j][1] = codes4(w[2], w[3], scale);
                }
                if (s[j] == 255u) k[j][0] = k[j][1] = 0;
            }
            // an even lane keeps the first row's elements and gets its neighbour's, an odd one the second's
            const bool odd = lane & 1;
            const uint32_t g0 = moved<kXor1>(odd ? k[0][0] : k[1][0]), g1 = moved<kXor1>(odd ? k[0][1] : k[1][1]);
            const uint4 out = odd ? make_uint4(g0, g1, k[1][0], k[1][1]) : make_uint4(k[0][0], k[0][1], g0, g1);
            const int64_t r = row0 + r0 + 4 * (i + (odd ? 1 : 0)), group = (r >> 4) * units;
            const int slot = (int)(r & 15);
            if (r < p.rows) {
                *reinterpret_cast<uint4*>(codes + group * kF8UnitBytes + slot * 16) = out;
                if (q < 2) scales[group * kF8UnitScales + slot * 4] = (uint8_t)(odd ? s[1] : s[0]);
            }
        }
    }
    if (!p.codes_t) return;
    __syncthreads();
    const int64_t units = mx_units(p.rows);
    const int part = sizeof(T) == 4 ? wave >> 1 : wave;                             // which 32 rows
    const int word = sizeof(T) == 4 ? (wave & 1) * 64 + lane : lane;                // which column or two
    uint8_t* codes = p.codes_t + (row0 >> 7) * kF8TileBytes + part * 512;
    uint8_t* scales = p.scales_t + (row0 >> 9) * kF8UnitScales + ((row0 >> 7) & 3);
    uint32_t w[32], m = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        w[i] = tile[32 * part + i][word];
        if constexpr (!SQUARE) {
            if constexpr (sizeof(T) == 4) m = max(m, w[i] & 0x7FFFFFFFu);
            else m = pair_max(m, w[i]);
        }
    }
    if constexpr (!SQUARE) {
        most[part][word] = m;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (sizeof(T) == 4) m = max(m, most[i][word]);
            else m = pair_max(m, most[i][word]);
        }
    }
#pragma unroll
    for (int h = 0; h < kCols; ++h) {
        const int64_t col = col0 + word * kCols + h;
        const uint32_t s = SQUARE ? whole : f8_scale(kCols == 1 ? m : (h ? m & 0xFFFF0000u : m << 16));
        const float scale = mx_value(s);
        uint32_t k[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (kCols == 1) {
                float f[4];
                __builtin_memcpy(f, w + 4 * i, sizeof(f));
                k[i] = codes4(f[0], f[1], f[2], f[3], scale);
            } else {
                // two rows' elements of this column
                const uint32_t sel = h ? 0x07060302u : 0x05040100u;
                k[i] = codes4(__builtin_amdgcn_perm(w[4 * i + 1], w[4 * i], sel), __builtin_amdgcn_perm(w[4 * i + 3], w[4 * i + 2], sel), scale);
            }
            k[i] = s == 255u ? 0u : k[i];
        }
        if (col < p.cols) {
            const int64_t group = (col >> 4) * units;
            const int slot = (int)(col & 15);
            uint8_t* to = codes + group * kF8UnitBytes + slot * 16;
            *reinterpret_cast<uint4*>(to) = make_uint4(k[0], k[1], k[2], k[3]);
            *reinterpret_cast<uint4*>(to + 256) = make_uint4(k[4], k[5], k[6], k[7]);
            if (part == 0) scales[group * kF8UnitScales + slot * 4] = (uint8_t)s;
        }
    }
}

// A thread per 16 elements; for looking at codes, not for a hot path.
template <typename T>
__global__ __launch_bounds__(256) void k_f8_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, T* out,
                                                       int64_t ld) {
    const int64_t pieces = (cols + 15) / 16, units = mx_units(cols);
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= rows * pieces) return;
    const int64_t r = i / pieces, c = (i - r * pieces) * 16, group = (r >> 4) * units;
    const int slot = (int)(r & 15);
    const uint8_t* src = codes + group * kF8UnitBytes + (c >> 7) * kF8TileBytes + ((c >> 4) & 7) * 256 + slot * 16;
    const float scale = mx_value(scales[(group + (c >> 9)) * kF8UnitScales + slot * 4 + ((c >> 7) & 3)]);
    for (int e = 0; e < 16 && c + e < cols; ++e) {
        const uint32_t k = src[e], x = (k >> 3) & 15u, m = k & 7u;
        const float a = x ? __uint_as_float((x + 120u) << 23 | m << 20) : (float)m * 0.001953125f;
        const float v = (k & 128u ? -a : a) * scale;
        if constexpr (sizeof(T) == 4) out[r * ld + c + e] = v;
        else out[r * ld + c + e] = (T)bf16_bits(v);
    }
}

template <typename T>
hipError_t quantize(const F8QuantArgs& a, hipStream_t s) {
    const int64_t tiles_c = (a.cols + 127) / 128, tiles = tiles_c * ((a.rows + 127) / 128);
    constexpr int threads = sizeof(T) == 4 ? 512 : 256;
    const auto launch = [&](auto APART) {
        constexpr bool apart = decltype(APART)::value;
        const uint32_t blocks = (uint32_t)(apart ? 2 * tiles : tiles);
        if (a.square) k_f8_quantize<T, true, apart><<<blocks, threads, 0, s>>>(a, (uint32_t)tiles_c, (uint32_t)tiles);
        else k_f8_quantize<T, false, apart><<<blocks, threads, 0, s>>>(a, (uint32_t)tiles_c, (uint32_t)tiles);
        return hipGetLastError();
    };
    // Few tiles: the chip has room for a block an axis, which takes half of the steps, where the second read does not count.
    // Inputs from HBM, in fp32 768 x 768 (36 tiles) 5.1 us together and 4.3 apart, 2048 x 1024 (128) 6.0 and 5.4, 3152 x 768
    // (150) 6.1 and 6.7; in bf16 5.1 and 4.0, 5.7 and 4.7, 5.9 and 5.6, 2048 x 2048 (256) 6.8 and 6.2.
    return a.codes && a.codes_t && tiles <= (sizeof(T) == 4 ? 128 : 256) ? launch(std::true_type()) : launch(std::false_type());
}

}  // namespace

hipError_t launch_f8_quantize(const F8QuantArgs& a, hipStream_t s) {
    if (a.rows == 0 || a.cols == 0) return hipSuccess;
    return a.type == SQ_TYPE_F32 ? quantize<float>(a, s) : quantize<uint16_t>(a, s);
}

hipError_t launch_f8_dequantize(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, void* out, int type,
                                int64_t ld, hipStream_t s) {
    const int64_t n = rows * ((cols + 15) / 16);
    if (n == 0) return hipSuccess;
    const dim3 grid((uint32_t)((n + 255) / 256));
    if (type == SQ_TYPE_F32) k_f8_dequantize<float><<<grid, 256, 0, s>>>(codes, scales, rows, cols, (float*)out, ld);
    else k_f8_dequantize<uint16_t><<<grid, 256, 0, s>>>(codes, scales, rows, cols, (uint16_t*)out, ld);
    return hipGetLastError();
}

}  // namespace sq
