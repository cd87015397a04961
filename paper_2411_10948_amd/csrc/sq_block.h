// Internal declarations of what stands around an expert layer's products: layer
// norm, router, exchange of rows.  Not part of the public ABI; see
// include/shiftquant.h.
#pragma once

#include "sq_mx.h"

namespace sq {

// ---- layer norm (sq_norm.hip) ----
struct NormArgs {
    int type, param_type;               // SQ_TYPE_* of the rows; of gamma and beta
    int64_t M, C;
    float eps;
    const void *x, *residual;           // forward: input, addend (may be null)
    void *h, *y;                        // forward: x + residual (null without one), output
    const void *gamma, *beta;
    float* stats;                       // [M, 4]: mean, its remainder, 1 / sqrt(var + eps), 0 (forward: may be null)
    const void *dy, *dh;                // backward: gradients of y and of h (may be null)
    void* dx;
    float *dgamma, *dbeta;
    float* part;                        // backward: the blocks' sums of dgamma and dbeta, [parts, 2, C]
    int64_t ld_x, ld_r, ld_h, ld_y, ld_dy, ld_dh, ld_dx;
};
int64_t norm_parts(int64_t M, int64_t C, int type);     // rows of `part`
hipError_t launch_norm_forward(const NormArgs& a, hipStream_t s);
hipError_t launch_norm_backward(const NormArgs& a, hipStream_t s);   // x is the forward's h, or its x without a residual

// ---- router (sq_route.hip) ----
constexpr int kRouteMaxExperts = 1024, kRouteMaxTopK = 64, kRouteMaxGroups = 64;
constexpr int64_t kRouteMaxTokens = ((int64_t)1 << 26) - 4;     // at most: four a block of 256 threads, below 2^32 threads
constexpr int kRouteTokens = 64;        // of a block: a bit each in a word by expert
struct RouteArgs {
    int type, score, renorm;            // SQ_TYPE_*, SQ_SCORE_*
    int64_t T, ld;
    int E, k, groups, top_groups;
    float scale;
    const void* logits;
    const float* bias;                  // may be null
    float* share;                       // [T, k]
    int32_t *chosen, *place;            // [T, k]
    int32_t* offsets;                   // [E + 1]
    uint8_t* counts;                    // [blocks, route_stride(E)] rows of a block by expert
    int32_t* base;                      // [blocks + 1, E]: rows before the block's by expert; last row: all
    const float* dshare;                // backward
    void* dlogits;
    int64_t ld_d;
};
__host__ __device__ inline int64_t route_stride(int64_t E) { return (E + 3) / 4 * 4; }     // whole words
inline int64_t route_blocks(int64_t T) { return (T + kRouteTokens - 1) / kRouteTokens; }
hipError_t launch_route_forward(const RouteArgs& a, hipStream_t s);
hipError_t launch_route_backward(const RouteArgs& a, hipStream_t s);

// ---- exchange of rows (sq_exchange.hip) ----
constexpr int kExchangeMaxTopK = 64;
struct ExchangeArgs {
    int type;
    int64_t T, rows, D;                 // tokens; sorted rows
    int k;
    const int32_t* place;               // [T, k]; outside [0, rows): no row
    const float* share;                 // [T, k]; combine: null for 1
    const void* x;                      // [T, D]: dispatch's input, combine_backward's dout
    const void* rows_in;                // [rows, D]: combine's y (or gradients of dispatched rows), combine_backward's y
    const void* add;                    // [T, D] combine's addend (may be null)
    void* out;                          // combine's output [T, D]
    void* rows_out;                     // dispatch's output [rows, D], combine_backward's dy
    float* dshare;                      // combine_backward [T, k]
    int64_t ld_x, ld_in, ld_add, ld_out, ld_rows;
};
hipError_t launch_dispatch(const ExchangeArgs& a, hipStream_t s);
hipError_t launch_combine(const ExchangeArgs& a, hipStream_t s);
hipError_t launch_combine_backward(const ExchangeArgs& a, hipStream_t s);

// ---- device helpers ----
#if defined(__HIPCC__)
template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);       // elements of a 16-byte piece

// 16 bytes of a row from column c < cols as they came; columns at and past `cols`
// read as zero.  WHOLE: there are none, rows are whole pieces.  NT: past the caches.
template <bool WHOLE = false, bool NT = false, typename T>
__device__ __forceinline__ void load16(const T* row, int c, int cols, uint32_t* w) {
    if (WHOLE || c + kVec<T> <= cols) {
        const u32x4_any* at = reinterpret_cast<const u32x4_any*>(row + (uint32_t)c);
        u32x4_any v;
        if constexpr (NT) v = __builtin_nontemporal_load(at);
        else v = *at;
        w[0] = v.x;
        w[1] = v.y;
        w[2] = v.z;
        w[3] = v.w;
    } else {
        T t[kVec<T>];       // loads without branches, those past the end cleared
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) t[e] = row[(uint32_t)min(c + e, cols - 1)];
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e) t[e] = c + e < cols ? t[e] : (T)0;
        __builtin_memcpy(w, t, 16);
    }
}
template <bool WHOLE = false, bool NT = false, typename T>
__device__ __forceinline__ void store16(T* row, int c, int cols, const uint32_t* w) {
    if (WHOLE || c + kVec<T> <= cols) {
        u32x4_any* to = reinterpret_cast<u32x4_any*>(row + (uint32_t)c);
        if constexpr (NT) __builtin_nontemporal_store(u32x4_any{w[0], w[1], w[2], w[3]}, to);
        else *to = u32x4_any{w[0], w[1], w[2], w[3]};
    } else {
        T t[kVec<T>];
        __builtin_memcpy(t, w, 16);
#pragma unroll
        for (int e = 0; e < kVec<T>; ++e)
            if (c + e < cols) row[(uint32_t)(c + e)] = t[e];
    }
}
// fp32 values of a piece, and back (rounded once to bf16)
template <typename T>
__device__ __forceinline__ void values16(const uint32_t* w, float* f) {
#pragma unroll
    for (int e = 0; e < kVec<T>; ++e) {
        if constexpr (sizeof(T) == 4) f[e] = __uint_as_float(w[e]);
        else f[e] = __uint_as_float(e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
    }
}
template <typename T>
__device__ __forceinline__ void pack16(const float* f, uint32_t* w) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if constexpr (sizeof(T) == 4) w[e] = __float_as_uint(f[e]);
        else w[e] = bf16_pair(f[2 * e], f[2 * e + 1]);
    }
}

// A lane's value moved along the wave: row_shr 1, 2, 4, 8 (0x111, 2, 4, 8), then
// row_bcast 15 and 31; lanes that get none keep their own.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t wave_move(uint32_t own, uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp((int)own, (int)v, CTRL, ROWS, 0xF, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ float wave_move(float own, float v) {
    return __uint_as_float(wave_move<CTRL, ROWS>(__float_as_uint(own), __float_as_uint(v)));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ double wave_move(double own, double v) {
    const uint64_t o = __builtin_bit_cast(uint64_t, own), b = __builtin_bit_cast(uint64_t, v);
    const uint64_t lo = wave_move<CTRL, ROWS>((uint32_t)o, (uint32_t)b);
    const uint64_t hi = wave_move<CTRL, ROWS>((uint32_t)(o >> 32), (uint32_t)(b >> 32));
    return __builtin_bit_cast(double, hi << 32 | lo);
}
__device__ __forceinline__ float wave_lane(float v, int lane) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), lane));
}
__device__ __forceinline__ double wave_lane(double v, int lane) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint64_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, lane);
    const uint64_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
    return __builtin_bit_cast(double, hi << 32 | lo);
}
// Sum and maximum over the wave in a fixed order, the same in every lane; every
// lane must be active.  The maximum of values that hold no NaN.
template <typename F>
__device__ __forceinline__ F wave_sum(F v) {
    v += wave_move<0x111, 0xF>((F)0, v);
    v += wave_move<0x112, 0xF>((F)0, v);
    v += wave_move<0x114, 0xF>((F)0, v);
    v += wave_move<0x118, 0xF>((F)0, v);
    v += wave_move<0x142, 0xA>((F)0, v);
    v += wave_move<0x143, 0xC>((F)0, v);
    return wave_lane(v, 63);
}
template <typename F>
__device__ __forceinline__ F larger(F a, F b) { return a < b ? b : a; }
template <typename F>
__device__ __forceinline__ F wave_max(F v) {
    v = larger(v, wave_move<0x111, 0xF>(v, v));
    v = larger(v, wave_move<0x112, 0xF>(v, v));
    v = larger(v, wave_move<0x114, 0xF>(v, v));
    v = larger(v, wave_move<0x118, 0xF>(v, v));
    v = larger(v, wave_move<0x142, 0xA>(v, v));
    v = larger(v, wave_move<0x143, 0xC>(v, v));
    return wave_lane(v, 63);
}
template <int CTRL, typename F>
__device__ __forceinline__ F row_move(F v) {
    return wave_move<CTRL, 0xF>(v, v);
}
constexpr int kLane1 = 0xB1, kLane2 = 0x4E, kMirror8 = 0x141, kMirror16 = 0x140;     // partners in a sum over 2, 4, 8, 16 lanes
// f over the `lanes` lanes (1, 2, 4, 8 or 16) that start at a multiple of it
template <typename F, class Op>
__device__ __forceinline__ F over_lanes(F v, int lanes, Op op) {
    if (lanes > 1) v = op(v, row_move<kLane1>(v));
    if (lanes > 2) v = op(v, row_move<kLane2>(v));
    if (lanes > 4) v = op(v, row_move<kMirror8>(v));
    if (lanes > 8) v = op(v, row_move<kMirror16>(v));
    return v;
}
#endif

}  // namespace sq
