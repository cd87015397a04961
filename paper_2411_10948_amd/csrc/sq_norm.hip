// Layer norm over the rows of a matrix, with the residual sum before it, and
// its backward pass.
//   h = x + residual (rounded to the type); mean, var over a row of h
//   y = (h - mean) r gamma + beta,  r = 1 / sqrt(var + eps)
//   q = dy gamma, xh = (h - mean) r:
//   dx = r (q - mean(q) - xh mean(q xh)) [+ dh],  dgamma = sum dy xh,  dbeta = sum dy
// A row stays in registers between its two reductions: h read once a direction.
// The mean is a sum of two fp32 numbers: the rounded mean, and the mean of what
// is left once that is taken off, so that a row far from zero loses no digits
// (var = mean (h - mean)^2 - rest^2).
#include <algorithm>

#include "sq_block.h"

namespace sq {

namespace {

// Sum of N values over the TPR threads of a row, the same in all of them; `slot`:
// a row's LDS words for one of the reductions between two barriers.
template <int TPR, int N>
__device__ __forceinline__ void row_sum(float* v, float (*slot)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
    if constexpr (TPR > 64) {
        const int wave = (threadIdx.x % TPR) >> 6;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) slot[wave][i] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = 0.0f;
        for (int w = 0; w < TPR / 64; ++w)
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += slot[w][i];
    }
}

// V pieces of gamma or beta that a thread's columns take, in fp32.
template <typename T, int TPR, int V>
__device__ __forceinline__ void load_param(const void* p, int type, int64_t C, float* f) {
    constexpr int N = kVec<T>;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int64_t c = ((int64_t)v * TPR + threadIdx.x % TPR) * N;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const int64_t at = min(c + e, C - 1);
            const float w = type == SQ_TYPE_F32 ? static_cast<const float*>(p)[at] : bf16_value(static_cast<const uint16_t*>(p)[at]);
            f[v * N + e] = c + e < C ? w : 0.0f;
        }
    }
}

// TPR threads a row, V pieces of 16 bytes a thread; THREADS / TPR rows at a time.
template <typename T, int TPR, int V, int THREADS>
__global__ __launch_bounds__(THREADS) void k_norm_forward(NormArgs p) {
    constexpr int N = kVec<T>, ROWS = THREADS / TPR;
    __shared__ float red1[ROWS][TPR / 64][1], red2[ROWS][TPR / 64][2];
    const int grp = threadIdx.x / TPR, tid = threadIdx.x % TPR;
    float g[V * N], b[V * N];
    load_param<T, TPR, V>(p.gamma, p.param_type, p.C, g);
    load_param<T, TPR, V>(p.beta, p.param_type, p.C, b);
    const float inv = 1.0f / (float)p.C;
    for (int64_t row0 = (int64_t)blockIdx.x * ROWS; row0 < p.M; row0 += (int64_t)gridDim.x * ROWS) {
        const int64_t row = row0 + grp;
        const bool live = row < p.M;
        const T* x = static_cast<const T*>(p.x) + row * p.ld_x;
        const T* res = static_cast<const T*>(p.residual) + row * p.ld_r;
        uint32_t w[V][4], r[V][4];
        float f[V * N];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int64_t c = ((int64_t)v * TPR + tid) * N;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[v][i] = r[v][i] = 0;
            if (!live || c >= p.C) continue;
            load16(x, c, p.C, w[v]);
            if (p.residual) load16(res, c, p.C, r[v]);
        }
        float s[1] = {0.0f};
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int64_t c = ((int64_t)v * TPR + tid) * N;
            values16<T>(w[v], f + v * N);
            if (p.residual) {
                float a[N];
                values16<T>(r[v], a);
#pragma unroll
                for (int e = 0; e < N; ++e) a[e] += f[v * N + e];
                pack16<T>(a, w[v]);
                values16<T>(w[v], f + v * N);
                if (live && c < p.C) store16(static_cast<T*>(p.h) + row * p.ld_h, c, p.C, w[v]);
            }
#pragma unroll
            for (int e = 0; e < N; ++e) s[0] += f[v * N + e];
        }
        row_sum<TPR, 1>(s, red1[grp]);
        const float mean = s[0] * inv;
        float t[2] = {0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int64_t c = ((int64_t)v * TPR + tid) * N;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float d = c + e < p.C ? f[v * N + e] - mean : 0.0f;
                f[v * N + e] = d;
                t[0] += d;
                t[1] = __builtin_fmaf(d, d, t[1]);
            }
        }
        row_sum<TPR, 2>(t, red2[grp]);
        const float rest = t[0] * inv, var = fmaxf(__builtin_fmaf(-rest, rest, t[1] * inv), 0.0f);
        // a NaN in the row is one in var, which fmaxf would drop
        const float rstd = t[1] != t[1] ? t[1] : 1.0f / sqrtf(var + p.eps);
        if (!live) continue;
        if (p.stats && tid == 0) *reinterpret_cast<float4*>(p.stats + row * 4) = make_float4(mean, rest, rstd, 0.0f);
        T* y = static_cast<T*>(p.y) + row * p.ld_y;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int64_t c = ((int64_t)v * TPR + tid) * N;
            if (c >= p.C) continue;
            float o[N];
#pragma unroll
            for (int e = 0; e < N; ++e) o[e] = __builtin_fmaf((f[v * N + e] - rest) * rstd, g[v * N + e], b[v * N + e]);
            pack16<T>(o, w[v]);
            store16(y, c, p.C, w[v]);
        }
    }
}

// The same rows of dy, h and dh; the block keeps its rows' sums of dgamma and
// dbeta, a thread those of its columns, and writes them to `part`.
template <typename T, int TPR, int V, int THREADS>
__global__ __launch_bounds__(THREADS) void k_norm_backward(NormArgs p) {
    constexpr int N = kVec<T>, ROWS = THREADS / TPR;
    __shared__ float red[2][ROWS][TPR / 64][2];
    __shared__ float cols[ROWS > 1 ? TPR * V * N : 1];
    const int grp = threadIdx.x / TPR, tid = threadIdx.x % TPR;
    float g[V * N], dg[V * N], db[V * N];
    load_param<T, TPR, V>(p.gamma, p.param_type, p.C, g);
#pragma unroll
    for (int i = 0; i < V * N; ++i) dg[i] = db[i] = 0.0f;
    const float inv = 1.0f / (float)p.C;
    int turn = 0;
    for (int64_t row0 = (int64_t)blockIdx.x * ROWS; row0 < p.M; row0 += (int64_t)gridDim.x * ROWS, turn ^= 1) {
        const int64_t row = row0 + grp;
        const bool live = row < p.M;
        uint32_t wd[V][4], wx[V][4], wh[V][4];
        float4 st = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (live) st = *reinterpret_cast<const float4*>(p.stats + row * 4);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int64_t c = ((int64_t)v * TPR + tid) * N;
#pragma unroll
            for (int i = 0; i < 4; ++i) wd[v][i] = wx[v][i] = wh[v][i] = 0;
            if (!live || c >= p.C) continue;
            load16(static_cast<const T*>(p.dy) + row * p.ld_dy, c, p.C, wd[v]);
            load16(static_cast<const T*>(p.x) + row * p.ld_x, c, p.C, wx[v]);
            if (p.dh) load16(static_cast<const T*>(p.dh) + row * p.ld_dh, c, p.C, wh[v]);
        }
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float d[N], x[N];
            values16<T>(wd[v], d);
            values16<T>(wx[v], x);
            const bool in = live && ((int64_t)v * TPR + tid) * N < p.C;     // columns past the end have dy = gamma = 0
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int i = v * N + e;
                const float xh = in ? ((x[e] - st.x) - st.y) * st.z : 0.0f, q = d[e] * g[i];
                s[0] += q;
                s[1] = __builtin_fmaf(q, xh, s[1]);
                dg[i] = __builtin_fmaf(d[e], xh, dg[i]);
                db[i] += d[e];
            }
        }
        row_sum<TPR, 2>(s, red[turn][grp]);     // the next row's words are others: one barrier a row
        const float a = s[0] * inv, b = s[1] * inv;
        if (!live) continue;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int64_t c = ((int64_t)v * TPR + tid) * N;
            if (c >= p.C) continue;
            float d[N], x[N], o[N], h[N];
            values16<T>(wd[v], d);
            values16<T>(wx[v], x);
            values16<T>(wh[v], h);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float xh = ((x[e] - st.x) - st.y) * st.z;
                o[e] = __builtin_fmaf(st.z, __builtin_fmaf(-xh, b, d[e] * g[v * N + e] - a), h[e]);
            }
            pack16<T>(o, wd[v]);
            store16(static_cast<T*>(p.dx) + row * p.ld_dx, c, p.C, wd[v]);
        }
    }
    // the rows' sums of the block, in the order of its row groups
    float* part = p.part + (int64_t)blockIdx.x * 2 * p.C;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float* mine = which ? db : dg;
#pragma unroll
        for (int k = 1; k < ROWS; ++k) {
            __syncthreads();
            if (grp == k)
#pragma unroll
                for (int i = 0; i < V * N; ++i) cols[i * TPR + tid] = mine[i];
            __syncthreads();
            if (grp == 0)
#pragma unroll
                for (int i = 0; i < V * N; ++i) mine[i] += cols[i * TPR + tid];
        }
        if (grp == 0)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int64_t c = ((int64_t)v * TPR + tid) * N;
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (c + e < p.C) part[which * p.C + c + e] = mine[v * N + e];
            }
    }
}

// dgamma and dbeta: sums over the rows of `part`, 64 columns a block, in the order
// of the rows within each of 16 waves, then of the waves.
__global__ __launch_bounds__(1024) void k_norm_reduce(const float* part, int64_t parts, int64_t C, float* dgamma, float* dbeta) {
    __shared__ float sums[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    float s = 0.0f;
    if (c < 2 * C)
        for (int64_t r = wave; r < parts; r += 16) s += part[r * 2 * C + c];
    sums[wave][lane] = s;
    __syncthreads();
    if (wave || c >= 2 * C) return;
#pragma unroll
    for (int w = 1; w < 16; ++w) s += sums[w][lane];
    if (c < C) dgamma[c] = s;
    else dbeta[c - C] = s;
}

// ---------------------------------------------------------------------------
// Rows too long for registers: a block of 1024 threads a row, which reads it
// again for each step (from the caches), and the columns' sums in a kernel of
// their own.
// ---------------------------------------------------------------------------
constexpr int kLong = 1024;

template <typename T, class F>
__device__ __forceinline__ void pieces(int64_t C, F f) {
    for (int64_t c = (int64_t)threadIdx.x * kVec<T>; c < C; c += kLong * kVec<T>) f(c);
}

template <typename T>
__global__ __launch_bounds__(kLong) void k_norm_forward_long(NormArgs p) {
    constexpr int N = kVec<T>;
    __shared__ float red1[kLong / 64][1], red2[kLong / 64][2];
    const float inv = 1.0f / (float)p.C;
    for (int64_t row = blockIdx.x; row < p.M; row += gridDim.x) {
        const T* x = static_cast<const T*>(p.x) + row * p.ld_x;
        float s[1] = {0.0f}, t[2] = {0.0f, 0.0f};
        pieces<T>(p.C, [&](int64_t c) {
            uint32_t w[4], r[4];
            float f[N], a[N];
            load16(x, c, p.C, w);
            values16<T>(w, f);
            if (p.residual) {
                load16(static_cast<const T*>(p.residual) + row * p.ld_r, c, p.C, r);
                values16<T>(r, a);
#pragma unroll
                for (int e = 0; e < N; ++e) a[e] += f[e];
                pack16<T>(a, w);
                values16<T>(w, f);
                store16(static_cast<T*>(p.h) + row * p.ld_h, c, p.C, w);
            }
#pragma unroll
            for (int e = 0; e < N; ++e) s[0] += f[e];
        });
        if (p.residual) x = static_cast<const T*>(p.h) + row * p.ld_h;      // a thread's own stores
        row_sum<kLong, 1>(s, red1);
        const float mean = s[0] * inv;
        pieces<T>(p.C, [&](int64_t c) {
            uint32_t w[4];
            float f[N];
            load16(x, c, p.C, w);
            values16<T>(w, f);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float d = c + e < p.C ? f[e] - mean : 0.0f;
                t[0] += d;
                t[1] = __builtin_fmaf(d, d, t[1]);
            }
        });
        row_sum<kLong, 2>(t, red2);
        const float rest = t[0] * inv, var = fmaxf(__builtin_fmaf(-rest, rest, t[1] * inv), 0.0f);
        const float rstd = t[1] != t[1] ? t[1] : 1.0f / sqrtf(var + p.eps);
        if (p.stats && threadIdx.x == 0) *reinterpret_cast<float4*>(p.stats + row * 4) = make_float4(mean, rest, rstd, 0.0f);
        pieces<T>(p.C, [&](int64_t c) {
            uint32_t w[4];
            float f[N];
            load16(x, c, p.C, w);
            values16<T>(w, f);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int64_t at = min(c + e, p.C - 1);
                const float g = p.param_type == SQ_TYPE_F32 ? static_cast<const float*>(p.gamma)[at]
                                                            : bf16_value(static_cast<const uint16_t*>(p.gamma)[at]);
                const float b = p.param_type == SQ_TYPE_F32 ? static_cast<const float*>(p.beta)[at]
                                                            : bf16_value(static_cast<const uint16_t*>(p.beta)[at]);
                f[e] = __builtin_fmaf(((f[e] - mean) - rest) * rstd, g, b);
            }
            pack16<T>(f, w);
            store16(static_cast<T*>(p.y) + row * p.ld_y, c, p.C, w);
        });
        __syncthreads();    // the reductions' words are free again
    }
}

template <typename T>
__global__ __launch_bounds__(kLong) void k_norm_backward_long(NormArgs p) {
    constexpr int N = kVec<T>;
    __shared__ float red[kLong / 64][2];
    const float inv = 1.0f / (float)p.C;
    for (int64_t row = blockIdx.x; row < p.M; row += gridDim.x) {
        const float4 st = *reinterpret_cast<const float4*>(p.stats + row * 4);
        auto terms = [&](int64_t c, float* q, float* xh) {
            uint32_t wd[4], wx[4];
            load16(static_cast<const T*>(p.dy) + row * p.ld_dy, c, p.C, wd);
            load16(static_cast<const T*>(p.x) + row * p.ld_x, c, p.C, wx);
            values16<T>(wd, q);
            values16<T>(wx, xh);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int64_t at = min(c + e, p.C - 1);
                q[e] *= p.param_type == SQ_TYPE_F32 ? static_cast<const float*>(p.gamma)[at]
                                                    : bf16_value(static_cast<const uint16_t*>(p.gamma)[at]);
                xh[e] = c + e < p.C ? ((xh[e] - st.x) - st.y) * st.z : 0.0f;
                q[e] = c + e < p.C ? q[e] : 0.0f;
            }
        };
        float s[2] = {0.0f, 0.0f};
        pieces<T>(p.C, [&](int64_t c) {
            float q[N], xh[N];
            terms(c, q, xh);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                s[0] += q[e];
                s[1] = __builtin_fmaf(q[e], xh[e], s[1]);
            }
        });
        row_sum<kLong, 2>(s, red);
        const float a = s[0] * inv, b = s[1] * inv;
        pieces<T>(p.C, [&](int64_t c) {
            float q[N], xh[N], h[N];
            uint32_t w[4] = {0, 0, 0, 0};
            terms(c, q, xh);
            if (p.dh) load16(static_cast<const T*>(p.dh) + row * p.ld_dh, c, p.C, w);
            values16<T>(w, h);
#pragma unroll
            for (int e = 0; e < N; ++e) h[e] = __builtin_fmaf(st.z, __builtin_fmaf(-xh[e], b, q[e] - a), h[e]);
            pack16<T>(h, w);
            store16(static_cast<T*>(p.dx) + row * p.ld_dx, c, p.C, w);
        });
        __syncthreads();    // the reductions' words are free again
    }
}

// A thread per column, blockIdx.y of gridDim.y of the rows.
template <typename T>
__global__ __launch_bounds__(256) void k_norm_columns(NormArgs p) {
    const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (c >= p.C) return;
    float dg = 0.0f, db = 0.0f;
    for (int64_t row = blockIdx.y; row < p.M; row += gridDim.y) {
        const float4 st = *reinterpret_cast<const float4*>(p.stats + row * 4);
        const T d = static_cast<const T*>(p.dy)[row * p.ld_dy + c], x = static_cast<const T*>(p.x)[row * p.ld_x + c];
        float df, xf;
        if constexpr (sizeof(T) == 4) df = d, xf = x;
        else df = bf16_value(d), xf = bf16_value(x);
        dg = __builtin_fmaf(df, ((xf - st.x) - st.y) * st.z, dg);
        db += df;
    }
    float* part = p.part + (int64_t)blockIdx.y * 2 * p.C;
    part[c] = dg;
    part[p.C + c] = db;
}

// How a row is held: threads and 16-byte pieces a thread.
struct RowPlan {
    int tpr, v;     // tpr 0: too long for registers
};
RowPlan row_plan(int64_t C, int type) {
    const int64_t n = (C + (type == SQ_TYPE_F32 ? 4 : 8) - 1) / (type == SQ_TYPE_F32 ? 4 : 8);
    if (n <= 256) return {64, (int)((n + 63) / 64)};
    if (n <= 512) return {256, 2};
    if (n <= 1024) return {256, 4};
    if (n <= 2048) return {512, 4};
    if (n <= 4096) return {1024, 4};
    return {0, 0};
}
// f(threads a row, pieces) as compile-time constants
template <class F>
hipError_t with_plan(RowPlan r, F f) {
#define SQ_ROW(t, v) return f(std::integral_constant<int, t>(), std::integral_constant<int, v>())
    if (r.tpr == 64) {
        switch (r.v) {
            case 1: SQ_ROW(64, 1);
            case 2: SQ_ROW(64, 2);
            case 3: SQ_ROW(64, 3);
            default: SQ_ROW(64, 4);
        }
    }
    if (r.tpr == 256) {
        if (r.v == 2) SQ_ROW(256, 2);
        SQ_ROW(256, 4);
    }
    if (r.tpr == 512) SQ_ROW(512, 4);
    SQ_ROW(1024, 4);
#undef SQ_ROW
}

constexpr int64_t kLongSlices = 64, kLongGrid = 1 << 20;

template <typename T>
hipError_t forward(const NormArgs& a, hipStream_t s) {
    const RowPlan r = row_plan(a.C, a.type);
    if (r.tpr == 0) {
        k_norm_forward_long<T><<<(uint32_t)std::min<int64_t>(a.M, kLongGrid), kLong, 0, s>>>(a);
        return hipGetLastError();
    }
    return with_plan(r, [&](auto TPR, auto V) {
        constexpr int tpr = decltype(TPR)::value, threads = tpr < 256 ? 256 : tpr, rows = threads / tpr;
        const int64_t blocks = std::min<int64_t>((a.M + rows - 1) / rows, 2048);
        k_norm_forward<T, tpr, decltype(V)::value, threads><<<(uint32_t)blocks, threads, 0, s>>>(a);
        return hipGetLastError();
    });
}

template <typename T>
hipError_t backward(const NormArgs& a, hipStream_t s) {
    const RowPlan r = row_plan(a.C, a.type);
    const int64_t parts = norm_parts(a.M, a.C, a.type);
    hipError_t e;
    if (r.tpr == 0) {
        if (a.M) k_norm_backward_long<T><<<(uint32_t)std::min<int64_t>(a.M, kLongGrid), kLong, 0, s>>>(a);
        e = hipGetLastError();
        if (e == hipSuccess) {
            k_norm_columns<T><<<dim3((uint32_t)((a.C + 255) / 256), (uint32_t)parts), 256, 0, s>>>(a);
            e = hipGetLastError();
        }
    } else {
        e = with_plan(r, [&](auto TPR, auto V) {
            constexpr int tpr = decltype(TPR)::value, threads = tpr < 512 ? 512 : tpr;
            k_norm_backward<T, tpr, decltype(V)::value, threads><<<(uint32_t)parts, threads, 0, s>>>(a);
            return hipGetLastError();
        });
    }
    if (e != hipSuccess) return e;
    k_norm_reduce<<<(uint32_t)((2 * a.C + 63) / 64), 1024, 0, s>>>(a.part, parts, a.C, a.dgamma, a.dbeta);
    return hipGetLastError();
}

}  // namespace

int64_t norm_parts(int64_t M, int64_t C, int type) {
    const RowPlan r = row_plan(C, type);
    if (r.tpr == 0) return std::max<int64_t>(1, std::min(M, kLongSlices));
    const int64_t rows = std::max(512, r.tpr) / r.tpr;
    return std::max<int64_t>(1, std::min<int64_t>((M + rows - 1) / rows, 256));
}

hipError_t launch_norm_forward(const NormArgs& a, hipStream_t s) {
    if (a.M == 0 || a.C == 0) return hipSuccess;
    return a.type == SQ_TYPE_F32 ? forward<float>(a, s) : forward<uint16_t>(a, s);
}

hipError_t launch_norm_backward(const NormArgs& a, hipStream_t s) {
    if (a.C == 0) return hipSuccess;      // without rows the weights' gradients are zero
    return a.type == SQ_TYPE_F32 ? backward<float>(a, s) : backward<uint16_t>(a, s);
}

}  // namespace sq
