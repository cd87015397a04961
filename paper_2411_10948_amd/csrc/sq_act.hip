// Activations between two layers, and their backward pass from a copy of the
// input in 8 bits:
//   h = act(x), or gated h = act(g) u;   act(x) = x sigma(t(x)),
//   t(x) = x (SiLU) or 2 sqrt(2 / pi) (x + 0.044715 x^3) (GELU, tanh form).
//   dg = dh u act'(g), du = dh act(g),  act'(x) = sg + x sg (1 - sg) t'(x),
// the backward at the values that the copy holds: code 2^(s - 127) with one
// scale byte for 32 consecutive elements of g or of u (mx_scale8).  Bound by
// HBM: a training step keeps 33/32 bytes per input element instead of 2 or 4.
#include <algorithm>

#include "sq_mx.h"

namespace sq {

namespace {

template <typename T>
__device__ __forceinline__ float value_of(T v) {
    if constexpr (sizeof(T) == 4) return v;
    else return bf16_value(v);
}

// 8 consecutive elements; columns at and past `cols` read as zero.
template <typename T>
__device__ __forceinline__ void load8(const T* row, int64_t c, int64_t cols, bool vec, float* f) {
    if (vec && c + 8 <= cols) {
        T v[8];
#pragma unroll
        for (int w = 0; w < (int)(8 * sizeof(T) / 16); ++w)
            reinterpret_cast<uint4*>(v)[w] = reinterpret_cast<const uint4*>(row + c)[w];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = value_of<T>(v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = c + e < cols ? value_of<T>(row[c + e]) : 0.0f;
    }
}

template <typename T>
__device__ __forceinline__ void store8(T* row, int64_t c, int64_t cols, bool vec, const float* f) {
    if (vec && c + 8 <= cols) {
        if constexpr (sizeof(T) == 4) {
            reinterpret_cast<float4*>(row + c)[0] = make_float4(f[0], f[1], f[2], f[3]);
            reinterpret_cast<float4*>(row + c)[1] = make_float4(f[4], f[5], f[6], f[7]);
        } else {
            *reinterpret_cast<uint4*>(row + c) =
                make_uint4(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7]));
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

// sigma(t), and t' for the slope.  sigma is 1 or t's exponential to fp32 well
// before |x| = 60, so GELU's cube is taken there, where nothing overflows.
template <int KIND>
__device__ __forceinline__ float gate(float x, float& slope) {
    float t = x;
    slope = 1.0f;
    if constexpr (KIND == SQ_ACT_GELU) {
        const float y = __builtin_isnan(x) ? x : fminf(fmaxf(x, -60.0f), 60.0f), y2 = y * y;
        t = kGeluA * (y + kGeluB * y2 * y);
        slope = kGeluA * (1.0f + 3.0f * kGeluB * y2);
    }
    return __builtin_amdgcn_rcpf(1.0f + __expf(-t));
}

// The 8-bit copy of 8 elements; four lanes hold a block of 32.
__device__ __forceinline__ void copy8(const float* f, int8_t* codes, uint8_t* scale, bool first) {
    uint32_t b = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) b = max(b, __float_as_uint(f[e]) & 0x7FFFFFFFu);
    b = max(b, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b, 0xB1, 0xF, 0xF, false));   // lane ^ 1
    b = max(b, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)b, 0x4E, 0xF, 0xF, false));   // lane ^ 2
    const uint32_t s = mx_scale8(b);
    const float inv = mx_inverse(s);
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int k = s == 255u ? 0 : (int)__builtin_rintf(f[e] * inv);
        w[e >> 2] |= ((uint32_t)k & 255u) << (8 * (e & 3));
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

// A thread takes 8 columns of a row of the padded width Fp = roundup(F, 32).
template <typename T, int KIND, bool GATED>
__global__ __launch_bounds__(256) void k_act_forward(ActArgs p, int64_t n, uint32_t chunks, bool vec) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const int64_t r = i / chunks, c = (i - r * chunks) * 8, fp = (int64_t)chunks * 8;
    const int64_t ldc = GATED ? 2 * fp : fp;
    const T* x = static_cast<const T*>(p.x) + r * p.ld_x;
    int8_t* codes = p.codes + r * ldc;
    uint8_t* scales = p.scales + r * (ldc / 32);
    float g[8], u[8], h[8];
    load8<T>(x, c, p.F, vec, g);
    if constexpr (GATED) load8<T>(x + p.F, c, p.F, vec, u);
    const bool first = (threadIdx.x & 3) == 0;
    copy8(g, codes + c, scales + (c >> 5), first);
    if constexpr (GATED) copy8(u, codes + fp + c, scales + ((fp + c) >> 5), first);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float slope;
        h[e] = g[e] * gate<KIND>(g[e], slope);
        if constexpr (GATED) h[e] *= u[e];
    }
    store8<T>(static_cast<T*>(p.h) + r * p.ld_h, c, p.F, vec, h);
}

template <typename T, int KIND, bool GATED>
__global__ __launch_bounds__(256) void k_act_backward(ActArgs p, int64_t n, uint32_t chunks, bool vec) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const int64_t r = i / chunks, c = (i - r * chunks) * 8, fp = (int64_t)chunks * 8;
    const int64_t ldc = GATED ? 2 * fp : fp;
    const int8_t* codes = p.codes + r * ldc;
    const uint8_t* scales = p.scales + r * (ldc / 32);
    float g[8], u[8], d[8];
    load8<T>(static_cast<const T*>(p.h) + r * p.ld_h, c, p.F, vec, d);
    from_copy8(codes + c, scales + (c >> 5), g);
    if constexpr (GATED) from_copy8(codes + fp + c, scales + ((fp + c) >> 5), u);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float slope;
        const float sg = gate<KIND>(g[e], slope), a = g[e] * sg;
        const float da = sg + a * (1.0f - sg) * slope;
        if constexpr (GATED) {
            g[e] = d[e] * u[e] * da;
            u[e] = d[e] * a;
        } else {
            g[e] = d[e] * da;
        }
    }
    T* dx = static_cast<T*>(p.dx) + r * p.ld_x;
    store8<T>(dx, c, p.F, vec, g);
    if constexpr (GATED) store8<T>(dx + p.F, c, p.F, vec, u);
}

template <typename T, int KIND, bool GATED>
hipError_t act(const ActArgs& a, bool forward, hipStream_t s) {
    const int64_t chunks = round_up(a.F, 32) / 8, n = a.M * chunks;
    auto ok = [](const void* p, int64_t ld) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (ld * sizeof(T)) % 16 == 0; };
    const bool vec = ok(forward ? a.x : a.dx, a.ld_x) && ok(a.h, a.ld_h) && (!GATED || (a.F * sizeof(T)) % 16 == 0);
    const uint32_t blocks = (uint32_t)((n + 255) / 256);
    if (forward) k_act_forward<T, KIND, GATED><<<blocks, 256, 0, s>>>(a, n, (uint32_t)chunks, vec);
    else k_act_backward<T, KIND, GATED><<<blocks, 256, 0, s>>>(a, n, (uint32_t)chunks, vec);
    return hipGetLastError();
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
