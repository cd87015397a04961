// Activations between two layers, and their backward pass from a copy of the
// input in 8 bits:
//   h = act(x), or gated h = act(g) u;   act(x) = x sigma(t(x)),
//   t(x) = x (SiLU) or 2 sqrt(2 / pi) (x + 0.044715 x^3) (GELU, tanh form).
//   dg = dh u act'(g), du = dh act(g),  act'(x) = sg + x sg (1 - sg) t'(x),
// the backward at the values that the copy holds: code 2^(s - 127) with one
// scale byte for 32 consecutive elements of g or of u (mx_scale8).  A training
// step keeps 33/32 bytes per input element instead of 2 or 4.  One pass over the
// data, eight elements a thread, bound by HBM: gated SiLU of 8192 x 11008 in bf16
// (727 MB a direction), each repeated, 125 us forward and 119 backward (5.8 and 6.1
// TB/s); in turn, as in a training step, 114 and 135, together 249.  With ordinary
// instead of nontemporal stores and twice the vector instructions (a 64-bit
// division a thread, maxima and codes element by element) 132 and 130.
#include <algorithm>

#include "sq_mx.h"

namespace sq {

namespace {

// 8 consecutive elements as they came, 4 words of bf16 pairs or 8 of fp32;
// columns at and past `cols` read as zero.
template <typename T>
__device__ __forceinline__ void load8(const T* row, int64_t c, int64_t cols, uint32_t* w) {
    if (c + 8 <= cols) {
#pragma unroll
        for (int i = 0; i < (int)(8 * sizeof(T) / 4); i += 4) {
            const u32x4_any v = *reinterpret_cast<const u32x4_any*>(row + c + i * 4 / sizeof(T));
            w[i] = v.x;
            w[i + 1] = v.y;
            w[i + 2] = v.z;
            w[i + 3] = v.w;
        }
    } else {
        T v[8];     // loads without branches, those past the end cleared
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = row[min(c + e, cols - 1)];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = c + e < cols ? v[e] : (T)0;
        __builtin_memcpy(w, v, sizeof(v));
    }
}
template <typename T>
__device__ __forceinline__ void values8(const uint32_t* w, float* f) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if constexpr (sizeof(T) == 4) f[e] = __uint_as_float(w[e]);
        else f[e] = __uint_as_float(e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
    }
}

template <typename T>
__device__ __forceinline__ void store8(T* row, int64_t c, int64_t cols, const float* f) {
    if (c + 8 <= cols) {
        u32x4_any* to = reinterpret_cast<u32x4_any*>(row + c);
        if constexpr (sizeof(T) == 4) {
            __builtin_nontemporal_store(u32x4_any{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])}, to);
            __builtin_nontemporal_store(u32x4_any{__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7])}, to + 1);
        } else {
            __builtin_nontemporal_store(u32x4_any{bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7])}, to);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e < cols) {
                if constexpr (sizeof(T) == 4) row[c + e] = f[e];
                else row[c + e] = (T)bf16_bits(f[e]);
            }
    }
}

constexpr float kGeluA = 1.5957691216057308f, kGeluB = 0.044715f;   // 2 sqrt(2 / pi)

// sigma(t), 1 - sigma(t), and t' for the slope.  sigma is 1 or t's exponential to
// fp32 well before |x| = 60, so GELU's cube is taken there, where nothing overflows.
// fp32: e = exp(-|t|) to 1 ulp and sigma = e / (1 + e) or 1 / (1 + e), so that
// neither end loses digits; with __expf, which rounds the argument's product with
// log2 e, SiLU at -80 is off by 4e-6 of its value.  bf16 rounds both to the same.
template <int KIND, bool F32>
__device__ __forceinline__ float gate(float x, float& rest, float& slope) {
    float t = x;
    slope = 1.0f;
    if constexpr (KIND == SQ_ACT_GELU) {
        const float y = __builtin_isnan(x) ? x : fminf(fmaxf(x, -60.0f), 60.0f), y2 = y * y;
        t = kGeluA * (y + kGeluB * y2 * y);
        slope = kGeluA * (1.0f + 3.0f * kGeluB * y2);
    }
    if constexpr (F32) {
        const float e = expf(-fabsf(t)), r = __builtin_amdgcn_rcpf(1.0f + e), er = e * r;
        rest = t < 0.0f ? r : er;
        return t < 0.0f ? er : r;
    } else {
        const float sg = __builtin_amdgcn_rcpf(1.0f + __expf(-t));
        rest = 1.0f - sg;
        return sg;
    }
}

// The 8-bit copy of 8 elements; four lanes hold a block of 32.
template <typename T>
__device__ __forceinline__ void copy8(const uint32_t* raw, const float* f, int8_t* codes, uint8_t* scale, bool first) {
    uint32_t b = 0;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < 8; ++e) b = max(b, raw[e] & 0x7FFFFFFFu);
    } else {
        typedef uint16_t v2u16 __attribute__((ext_vector_type(2)));
        v2u16 m = {0, 0};
#pragma unroll
        for (int e = 0; e < 4; ++e) m = __builtin_elementwise_max(m, __builtin_bit_cast(v2u16, raw[e] & 0x7FFF7FFFu));
        b = (uint32_t)max(m.x, m.y) << 16;
    }
    b = max(b, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b, 0xB1, 0xF, 0xF, false));   // lane ^ 1
    b = max(b, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b, 0x4E, 0xF, 0xF, false));   // lane ^ 2
    const uint32_t s = mx_scale8(b);
    const float inv = mx_inverse(s);
    // x inv is exact (a power of two), so 1.5 2^23 + x inv rounds once, to the
    // nearest even integer, which its low byte holds in two's complement
    uint32_t k[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) k[e] = __float_as_uint(__builtin_fmaf(f[e], inv, 12582912.0f));
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t lo = __builtin_amdgcn_perm(k[4 * h + 1], k[4 * h], 0x0C0C0400u);
        const uint32_t hi = __builtin_amdgcn_perm(k[4 * h + 3], k[4 * h + 2], 0x04000C0Cu);
        w[h] = s == 255u ? 0u : lo | hi;
    }
    *reinterpret_cast<uint2*>(codes) = make_uint2(w[0], w[1]);
    if (first) *scale = (uint8_t)s;
}
__device__ __forceinline__ void from_copy8(const int8_t* codes, const uint8_t* scale, float* f) {
    const uint2 w = *reinterpret_cast<const uint2*>(codes);
    const float s = mx_value(*scale);
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = (float)(int8_t)((e < 4 ? w.x : w.y) >> (8 * (e & 3))) * s;
}

// Row and column of a thread: item / chunks by a multiplication, exact for
// items below 2^31 (mul = ceil(2^(31 + shift) / chunks), 2^shift >= chunks).
struct ActGrid {
    uint32_t items, chunks, mul;
    int shift;
};
__device__ __forceinline__ uint32_t row_of(const ActGrid& g, uint32_t i) {
    return (uint32_t)(((uint64_t)i * g.mul) >> (31 + g.shift));
}

// A thread takes 8 columns of a row of the padded width Fp = roundup(F, 32).
template <typename T, int KIND, bool GATED>
__global__ __launch_bounds__(256) void k_act_forward(ActArgs p, ActGrid q) {
    const uint32_t i = blockIdx.x * 256u + threadIdx.x;
    if (i >= q.items) return;
    const uint32_t row = row_of(q, i);
    const int64_t r = row, c = (int64_t)(i - row * q.chunks) * 8, fp = (int64_t)q.chunks * 8;
    const int64_t ldc = GATED ? 2 * fp : fp;
    const T* x = static_cast<const T*>(p.x) + r * p.ld_x;
    int8_t* codes = p.codes + r * ldc;
    uint8_t* scales = p.scales + r * (ldc / 32);
    constexpr int kWords = 8 * sizeof(T) / 4;
    uint32_t gw[kWords], uw[kWords];
    float g[8], u[8], h[8];
    load8<T>(x, c, p.F, gw);
    if constexpr (GATED) load8<T>(x + p.F, c, p.F, uw);
    const bool first = (threadIdx.x & 3) == 0;
    values8<T>(gw, g);
    copy8<T>(gw, g, codes + c, scales + (c >> 5), first);
    if constexpr (GATED) {
        values8<T>(uw, u);
        copy8<T>(uw, u, codes + fp + c, scales + ((fp + c) >> 5), first);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float rest, slope;
        h[e] = g[e] * gate<KIND, sizeof(T) == 4>(g[e], rest, slope);
        if constexpr (GATED) h[e] *= u[e];
    }
    store8<T>(static_cast<T*>(p.h) + r * p.ld_h, c, p.F, h);
}

template <typename T, int KIND, bool GATED>
__global__ __launch_bounds__(256) void k_act_backward(ActArgs p, ActGrid q) {
    const uint32_t i = blockIdx.x * 256u + threadIdx.x;
    if (i >= q.items) return;
    const uint32_t row = row_of(q, i);
    const int64_t r = row, c = (int64_t)(i - row * q.chunks) * 8, fp = (int64_t)q.chunks * 8;
    const int64_t ldc = GATED ? 2 * fp : fp;
    const int8_t* codes = p.codes + r * ldc;
    const uint8_t* scales = p.scales + r * (ldc / 32);
    uint32_t dw[8 * sizeof(T) / 4];
    float g[8], u[8], d[8];
    load8<T>(static_cast<const T*>(p.h) + r * p.ld_h, c, p.F, dw);
    from_copy8(codes + c, scales + (c >> 5), g);
    if constexpr (GATED) from_copy8(codes + fp + c, scales + ((fp + c) >> 5), u);
    values8<T>(dw, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float rest, slope;
        const float sg = gate<KIND, sizeof(T) == 4>(g[e], rest, slope), a = g[e] * sg;
        const float da = sg + a * rest * slope;
        if constexpr (GATED) {
            g[e] = d[e] * u[e] * da;
            u[e] = d[e] * a;
        } else {
            g[e] = d[e] * da;
        }
    }
    T* dx = static_cast<T*>(p.dx) + r * p.ld_x;
    store8<T>(dx, c, p.F, g);
    if constexpr (GATED) store8<T>(dx + p.F, c, p.F, u);
}

template <typename T, int KIND, bool GATED>
hipError_t act(const ActArgs& args, bool forward, hipStream_t s) {
    ActArgs a = args;
    const int64_t chunks = round_up(a.F, 32) / 8, fp = chunks * 8, codes_ld = GATED ? 2 * fp : fp;
    ActGrid q{};
    q.chunks = (uint32_t)chunks;
    while (((int64_t)1 << q.shift) < chunks) ++q.shift;
    q.mul = (uint32_t)((((uint64_t)1 << (31 + q.shift)) + (uint64_t)chunks - 1) / (uint64_t)chunks);
    // as many rows a launch as keep its items below 2^31
    const int64_t most = (((int64_t)1 << 31) - 256) / chunks;
    for (int64_t left = args.M; left > 0; left -= most) {
        q.items = (uint32_t)(std::min(left, most) * chunks);
        const uint32_t blocks = (q.items + 255) / 256;
        if (forward) k_act_forward<T, KIND, GATED><<<blocks, 256, 0, s>>>(a, q);
        else k_act_backward<T, KIND, GATED><<<blocks, 256, 0, s>>>(a, q);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        a.x = a.x ? static_cast<const T*>(a.x) + most * a.ld_x : nullptr;
        a.dx = a.dx ? static_cast<T*>(a.dx) + most * a.ld_x : nullptr;
        a.h = static_cast<T*>(a.h) + most * a.ld_h;
        a.codes += most * codes_ld;
        a.scales += most * (codes_ld / 32);
    }
    return hipSuccess;
}

template <typename T>
hipError_t act_of(const ActArgs& a, bool forward, hipStream_t s) {
    if (a.M == 0 || a.F == 0) return hipSuccess;
    if (a.kind == SQ_ACT_SILU) return a.gated ? act<T, SQ_ACT_SILU, true>(a, forward, s) : act<T, SQ_ACT_SILU, false>(a, forward, s);
    return a.gated ? act<T, SQ_ACT_GELU, true>(a, forward, s) : act<T, SQ_ACT_GELU, false>(a, forward, s);
}

}  // namespace

hipError_t launch_act_forward(const ActArgs& a, hipStream_t s) {
    return a.type == SQ_TYPE_F32 ? act_of<float>(a, true, s) : act_of<uint16_t>(a, true, s);
}
hipError_t launch_act_backward(const ActArgs& a, hipStream_t s) {
    return a.type == SQ_TYPE_F32 ? act_of<float>(a, false, s) : act_of<uint16_t>(a, false, s);
}

}  // namespace sq
