// Layer norm over the rows of a matrix, with the residual sum before it, and
// its backward pass.
//   h = x + residual (rounded to the type); mean, var over a row of h
//   y = (h - mean) r gamma + beta,  r = 1 / sqrt(var + eps)
//   q = dy gamma, xh = (h - mean) r:
//   dx = r (q - mean(q) - xh mean(q xh)) [+ dh],  dgamma = sum dy xh,  dbeta = sum dy
// A row stays in registers between its two reductions: h read once a direction, bound
// by HBM: 16384 x 4096 in bf16 with a residual 102 us forward (four matrices, 5.3 TB/s),
// 97 backward (5.5) and 5 for the sums of dgamma's and dbeta's parts; 3152 x 768 in fp32
// 6.0, 8.3 and 4.0, one row of 4096 3.5, which are launches and chains of loads and sums.
// The mean is a sum of two fp32 numbers: the rounded mean, and the mean of what
// is left once that is taken off, so that a row far from zero loses no digits
// (var = mean (h - mean)^2 - rest^2).  Where the squares leave fp32's range they are
// summed up once more of deviations times a power of two (square_scale).
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
        constexpr int kWaves = TPR / 64;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = over_lanes(slot[threadIdx.x & (kWaves - 1)][i], kWaves, [](float a, float b) { return a + b; });
    }
}

// N values of gamma or beta from column c in fp32, 0 past the last
template <int N, bool WHOLE = false>
__device__ __forceinline__ void load_values(const void* p, int type, int c, int C, float* f) {
    if (WHOLE && c >= C) {
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = 0.0f;
        return;
    }
    if (WHOLE || c + N <= C) {
        if (type == SQ_TYPE_F32) {
#pragma unroll
            for (int i = 0; i < N; i += 4) {
                const f32x4_any v = *reinterpret_cast<const f32x4_any*>(static_cast<const float*>(p) + (uint32_t)(c + i));
                f[i] = v.x;
                f[i + 1] = v.y;
                f[i + 2] = v.z;
                f[i + 3] = v.w;
            }
        } else {
            typedef uint32_t words_any __attribute__((ext_vector_type(N / 2), aligned(2)));
            const words_any w = *reinterpret_cast<const words_any*>(static_cast<const uint16_t*>(p) + (uint32_t)c);
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = __uint_as_float(i & 1 ? w[i >> 1] & 0xFFFF0000u : w[i >> 1] << 16);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const uint32_t at = (uint32_t)min(c + e, C - 1);
        const float w = type == SQ_TYPE_F32 ? static_cast<const float*>(p)[at] : bf16_value(static_cast<const uint16_t*>(p)[at]);
        f[e] = c + e < C ? w : 0.0f;
    }
}
// Those of a thread's V pieces.
template <typename T, int TPR, int V, bool WHOLE>
__device__ __forceinline__ void load_param(const void* p, int type, int C, float* f) {
#pragma unroll
    for (int v = 0; v < V; ++v) load_values<kVec<T>, WHOLE>(p, type, (v * TPR + (int)threadIdx.x % TPR) * kVec<T>, C, f + v * kVec<T>);
}

// Power of two for the deviations of a row whose sum of squares is `sum`, 1 where they are
// fine as they are.  Inf: of up to 2^20 deviations below 2^128 one is past 2^53.  Tiny ones,
// which count where eps does not: all are below 2^-45.
__device__ __forceinline__ float square_scale(float sum, float eps) {
    return sum == __builtin_inff() ? 0x1p-96f : sum < 0x1p-90f && eps < 0x1p-100f ? 0x1p96f : 1.0f;
}
// 1 / sqrt(var + eps) of a row from its sums of deviations times `up`, their plain sum (then
// their mean, without `up`) and that of their squares.  A NaN in the row is one in the
// squares, which fmaxf would drop.
__device__ __forceinline__ float row_rstd(float* t, float inv, float eps, float up) {
    const float rest = t[0] * inv, var = fmaxf(__builtin_fmaf(-rest, rest, t[1] * inv), 0.0f);
    t[0] = up == 1.0f ? rest : up < 1.0f ? rest * 0x1p96f : rest * 0x1p-96f;
    return t[1] != t[1] ? t[1] : up / sqrtf(var + eps * up * up);
}

// TPR threads a row, V pieces of 16 bytes a thread; THREADS / TPR rows at a time.
template <typename T, int TPR, int V, int THREADS, bool WHOLE, bool NT>
__global__ __launch_bounds__(THREADS, WHOLE ? 4 : 2) void k_norm_forward(NormArgs p) {
    constexpr int N = kVec<T>, ROWS = THREADS / TPR;
    __shared__ float red1[ROWS][TPR / 64][1], red2[ROWS][TPR / 64][2];
    const int grp = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR), tid = threadIdx.x % TPR, C = (int)p.C;
    float g[V * N], b[V * N];
    load_param<T, TPR, V, WHOLE>(p.gamma, p.param_type, C, g);
    load_param<T, TPR, V, WHOLE>(p.beta, p.param_type, C, b);
    const float inv = 1.0f / (float)C;
    for (int64_t row0 = (int64_t)blockIdx.x * ROWS; row0 < p.M; row0 += (int64_t)gridDim.x * ROWS) {
        const int64_t row = row0 + grp;
        const bool live = row < p.M;
        const T* x = static_cast<const T*>(p.x) + row * p.ld_x;
        const T* res = static_cast<const T*>(p.residual) + row * p.ld_r;
        uint32_t w[V][4], r[V][4];      // h as it is stored, unpacked for each step: fewer registers than its values
        float f[N];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = (v * TPR + tid) * N;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[v][i] = r[v][i] = 0;
            if (!live || c >= C) continue;
            load16<WHOLE, NT>(x, c, C, w[v]);
            if (p.residual) load16<WHOLE, NT>(res, c, C, r[v]);
        }
        float s[1] = {0.0f};
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = (v * TPR + tid) * N;
            values16<T>(w[v], f);
            if (p.residual) {
                float a[N];
                values16<T>(r[v], a);
#pragma unroll
                for (int e = 0; e < N; ++e) a[e] += f[e];
                pack16<T>(a, w[v]);
                values16<T>(w[v], f);
                if (live && c < C) store16<WHOLE, NT>(static_cast<T*>(p.h) + row * p.ld_h, c, C, w[v]);
            }
#pragma unroll
            for (int e = 0; e < N; ++e) s[0] += f[e];
        }
        row_sum<TPR, 1>(s, red1[grp]);
        const float mean = s[0] * inv;
        float t[2];
        auto squares = [&](float up) {
            t[0] = t[1] = 0.0f;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int c = (v * TPR + tid) * N;
                values16<T>(w[v], f);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float d = (WHOLE ? c : c + e) < C ? (f[e] - mean) * up : 0.0f;
                    t[0] += d;
                    t[1] = __builtin_fmaf(d, d, t[1]);
                }
            }
        };
        squares(1.0f);
        row_sum<TPR, 2>(t, red2[grp]);
        const float up = square_scale(t[1], p.eps);
        if (up != 1.0f) {       // of the whole row, which is the block's only one where it takes more than a wave
            squares(up);
            if constexpr (TPR > 64) __syncthreads();
            row_sum<TPR, 2>(t, red2[grp]);
        }
        const float rstd = row_rstd(t, inv, p.eps, up), rest = t[0];
        if (!live) continue;
        if (p.stats && tid == 0) *reinterpret_cast<float4*>(p.stats + row * 4) = make_float4(mean, rest, rstd, 0.0f);
        T* y = static_cast<T*>(p.y) + row * p.ld_y;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = (v * TPR + tid) * N;
            if (c >= C) continue;
            values16<T>(w[v], f);
#pragma unroll
            for (int e = 0; e < N; ++e) f[e] = __builtin_fmaf(((f[e] - mean) - rest) * rstd, g[v * N + e], b[v * N + e]);
            pack16<T>(f, w[v]);
            store16<WHOLE, NT>(y, c, C, w[v]);
        }
    }
}

// The same rows of dy, h and dh; the block keeps its rows' sums of dgamma and
// dbeta, a thread those of its columns, and writes them to `part`.
template <typename T, int TPR, int V, int THREADS, bool WHOLE, bool NT>
__global__ __launch_bounds__(THREADS, V * kVec<T> <= 16 ? 4 : 2) void k_norm_backward(NormArgs p) {
    constexpr int N = kVec<T>, ROWS = THREADS / TPR;
    __shared__ float red[2][ROWS][TPR / 64][2];
    __shared__ __attribute__((aligned(16))) float cols[ROWS][TPR * V * N];      // first gamma, then the rows' sums
    const int grp = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR), tid = threadIdx.x % TPR, C = (int)p.C;
    float dg[V * N], db[V * N];
    if (grp == 0) {
        float g[V * N];
        load_param<T, TPR, V, WHOLE>(p.gamma, p.param_type, C, g);
#pragma unroll
        for (int i = 0; i < V * N; i += 4)
            *reinterpret_cast<float4*>(&cols[0][((i / N) * TPR + tid) * N + i % N]) = make_float4(g[i], g[i + 1], g[i + 2], g[i + 3]);
    }
    __syncthreads();
    auto gammas = [&](int v, float* g) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const float4 w = *reinterpret_cast<const float4*>(&cols[0][(v * TPR + tid) * N + i]);
            g[i] = w.x;
            g[i + 1] = w.y;
            g[i + 2] = w.z;
            g[i + 3] = w.w;
        }
    };
#pragma unroll
    for (int i = 0; i < V * N; ++i) dg[i] = db[i] = 0.0f;
    const float inv = 1.0f / (float)C;
    int turn = 0;
    for (int64_t row0 = (int64_t)blockIdx.x * ROWS; row0 < p.M; row0 += (int64_t)gridDim.x * ROWS, turn ^= 1) {
        const int64_t row = row0 + grp;
        const bool live = row < p.M;
        uint32_t wd[V][4], wx[V][4], wh[V][4];
        float4 st = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (live) st = *reinterpret_cast<const float4*>(p.stats + row * 4);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = (v * TPR + tid) * N;
#pragma unroll
            for (int i = 0; i < 4; ++i) wd[v][i] = wx[v][i] = wh[v][i] = 0;
            if (!live || c >= C) continue;
            load16<WHOLE, NT>(static_cast<const T*>(p.dy) + row * p.ld_dy, c, C, wd[v]);
            load16<WHOLE, NT>(static_cast<const T*>(p.x) + row * p.ld_x, c, C, wx[v]);
            if (p.dh) load16<WHOLE, NT>(static_cast<const T*>(p.dh) + row * p.ld_dh, c, C, wh[v]);
        }
        float s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int v = 0; v < V; ++v) {
            float d[N], x[N], g[N];
            gammas(v, g);
            values16<T>(wd[v], d);
            values16<T>(wx[v], x);
            const bool in = live && (v * TPR + tid) * N < C;     // columns past the end have dy = gamma = 0
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int i = v * N + e;
                const float xh = in ? ((x[e] - st.x) - st.y) * st.z : 0.0f, q = d[e] * g[e];
                s[0] += q;
                s[1] = __builtin_fmaf(q, xh, s[1]);
                dg[i] = __builtin_fmaf(d[e], xh, dg[i]);
                db[i] += d[e];
            }
        }
        row_sum<TPR, 2>(s, red[turn][grp]);     // the next row's words are others: one barrier a row
        const float a = s[0] * inv, b = s[1] * inv;
        if (!live) continue;
        // unpacked again below, for fewer registers than the values of the first pass would take (a row of more than 4096
        // elements spilled them)
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(wd[v][i]), "+v"(wx[v][i]));
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const int c = (v * TPR + tid) * N;
            if (c >= C) continue;
            float d[N], x[N], o[N], h[N], g[N];
            gammas(v, g);
            values16<T>(wd[v], d);
            values16<T>(wx[v], x);
            values16<T>(wh[v], h);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float xh = ((x[e] - st.x) - st.y) * st.z;
                o[e] = __builtin_fmaf(st.z, __builtin_fmaf(-xh, b, d[e] * g[e] - a), h[e]);
            }
            pack16<T>(o, wd[v]);
            store16<WHOLE, NT>(static_cast<T*>(p.dx) + row * p.ld_dx, c, C, wd[v]);
        }
    }
    // the rows' sums of the block, in the order of its row groups
    float* part = p.part + (int64_t)blockIdx.x * 2 * p.C;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const float* mine = which ? db : dg;
        if constexpr (ROWS > 1) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < V * N; i += 4)
                *reinterpret_cast<float4*>(&cols[grp][((i / N) * TPR + tid) * N + i % N]) = make_float4(mine[i], mine[i + 1], mine[i + 2], mine[i + 3]);
            __syncthreads();
            for (int c = threadIdx.x; c < C; c += THREADS) {
                float s = cols[0][c];
#pragma unroll
                for (int k = 1; k < ROWS; ++k) s += cols[k][c];
                part[(int64_t)which * C + c] = s;
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int c = (v * TPR + tid) * N;
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if ((WHOLE ? c : c + e) < C) part[(int64_t)which * C + c + e] = mine[v * N + e];
            }
        }
    }
}

// dgamma and dbeta: sums over the rows of `part`, 32 columns a block, 32 threads each
// in the order of their rows, then in the threads' order.
__global__ __launch_bounds__(1024) void k_norm_reduce(const float* part, int64_t parts, int64_t C, float* dgamma, float* dbeta) {
    __shared__ float sums[32][33];
    const int col = threadIdx.x & 31, slice = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + col;
    float s = 0.0f;
    if (c < 2 * C) {
#pragma unroll 8
        for (int64_t r = slice; r < parts; r += 32) s += part[r * 2 * C + c];
    }
    sums[slice][col] = s;
    __syncthreads();
    if (slice || c >= 2 * C) return;
#pragma unroll
    for (int w = 1; w < 32; ++w) s += sums[w][col];
    if (c < C) dgamma[c] = s;
    else dbeta[c - C] = s;
}

// ---------------------------------------------------------------------------
// Rows too long for registers (more than 8192 elements in fp32, 16384 in bf16): a block of
// 1024 threads a row, which reads it again for each step (from the caches), and the
// columns' sums in a kernel of their own, which reads dy and h once more.  4000 x 12000 in
// fp32 113 us forward (384 MB, 3.4 TB/s) and 212 backward (576 MB, 2.7), 2048 x 16384 70 and 156,
// 2048 x 20000 in bf16 53 and 98.
// ---------------------------------------------------------------------------
constexpr int kLong = 1024;

template <typename T, class F>
__device__ __forceinline__ void pieces(int C, F f) {
    for (int c = threadIdx.x * kVec<T>; c < C; c += kLong * kVec<T>) f(c);
}

template <typename T>
__global__ __launch_bounds__(kLong) void k_norm_forward_long(NormArgs p) {
    constexpr int N = kVec<T>;
    __shared__ float red1[kLong / 64][1], red2[kLong / 64][2];
    const float inv = 1.0f / (float)p.C;
    for (int64_t row = blockIdx.x; row < p.M; row += gridDim.x) {
        const T* x = static_cast<const T*>(p.x) + row * p.ld_x;
        float s[1] = {0.0f}, t[2];
        pieces<T>(p.C, [&](int c) {
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
        auto squares = [&](float up) {
            t[0] = t[1] = 0.0f;
            pieces<T>(p.C, [&](int c) {
                uint32_t w[4];
                float f[N];
                load16(x, c, p.C, w);
                values16<T>(w, f);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float d = c + e < p.C ? (f[e] - mean) * up : 0.0f;
                    t[0] += d;
                    t[1] = __builtin_fmaf(d, d, t[1]);
                }
            });
        };
        squares(1.0f);
        row_sum<kLong, 2>(t, red2);
        const float up = square_scale(t[1], p.eps);
        if (up != 1.0f) {
            __syncthreads();
            squares(up);
            row_sum<kLong, 2>(t, red2);
        }
        const float rstd = row_rstd(t, inv, p.eps, up), rest = t[0];
        if (p.stats && threadIdx.x == 0) *reinterpret_cast<float4*>(p.stats + row * 4) = make_float4(mean, rest, rstd, 0.0f);
        pieces<T>(p.C, [&](int c) {
            uint32_t w[4];
            float f[N];
            load16(x, c, p.C, w);
            values16<T>(w, f);
            float g[N], b[N];
            load_values<N>(p.gamma, p.param_type, c, p.C, g);
            load_values<N>(p.beta, p.param_type, c, p.C, b);
#pragma unroll
            for (int e = 0; e < N; ++e) f[e] = __builtin_fmaf(((f[e] - mean) - rest) * rstd, g[e], b[e]);
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
        auto terms = [&](int c, float* q, float* xh) {
            uint32_t wd[4], wx[4];
            load16(static_cast<const T*>(p.dy) + row * p.ld_dy, c, p.C, wd);
            load16(static_cast<const T*>(p.x) + row * p.ld_x, c, p.C, wx);
            values16<T>(wd, q);
            values16<T>(wx, xh);
            float g[N];
            load_values<N>(p.gamma, p.param_type, c, p.C, g);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                q[e] *= g[e];       // 0 past the last column
                xh[e] = c + e < p.C ? ((xh[e] - st.x) - st.y) * st.z : 0.0f;
            }
        };
        float s[2] = {0.0f, 0.0f};
        pieces<T>(p.C, [&](int c) {
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
        pieces<T>(p.C, [&](int c) {
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

// How a row is held: threads and 16-byte pieces a thread.  A wave a row as long as its
// registers last, for want of barriers; a block of 256 threads a row instead, launches back to
// back, the backward with the sums of its parts: 3152 x 768 in fp32 (192 pieces) 5.4 -> 6.7 us
// forward, 11.1 -> 11.0 backward, in bf16 (96) 4.9 -> 6.6 and 10.6 -> 11.6; 16384 x 1024 in bf16
// (128) 14.6 -> 24.5 and 23.2 -> 35.2, 16384 x 1536 (192) 18.9 -> 25.0 and 36.0 -> 38.0,
// 16384 x 2048 (256) 25.1 -> 27.7 forward.
struct RowPlan {
    int tpr, v;     // tpr 0: too long for registers
};
int64_t row_pieces(int64_t C, int type) { return (C + (type == SQ_TYPE_F32 ? 4 : 8) - 1) / (type == SQ_TYPE_F32 ? 4 : 8); }
RowPlan forward_plan(int64_t C, int type) {
    const int64_t n = row_pieces(C, type);
    if (n <= 256) return {64, (int)((n + 63) / 64)};
    if (n <= 512) return {256, 2};
    if (n <= 1024) return {256, 4};
    if (n <= 2048) return {512, 4};
    return {0, 0};
}
// The sums of dgamma and dbeta take two registers an element; gamma waits in LDS.
RowPlan backward_plan(int64_t C, int type) {
    const int64_t n = row_pieces(C, type);
    if (n <= 192) return {64, (int)((n + 63) / 64)};
    if (n <= 512) return {256, (int)((n + 255) / 256)};
    if (n <= 1024) return {512, 2};
    if (n <= 2048) return {512, 4};
    return {0, 0};
}
// f(threads a row, pieces) as compile-time constants
#define SQ_ROW(t, w) \
    if (r.tpr == t && r.v == w) return f(std::integral_constant<int, t>(), std::integral_constant<int, w>())
template <class F>
hipError_t with_forward(RowPlan r, F f) {
    SQ_ROW(64, 1);
    SQ_ROW(64, 2);
    SQ_ROW(64, 3);
    SQ_ROW(64, 4);
    SQ_ROW(256, 2);
    SQ_ROW(256, 4);
    SQ_ROW(512, 4);
    return hipErrorInvalidValue;
}
template <class F>
hipError_t with_backward(RowPlan r, F f) {
    SQ_ROW(64, 1);
    SQ_ROW(64, 2);
    SQ_ROW(64, 3);
    SQ_ROW(256, 1);
    SQ_ROW(256, 2);
    SQ_ROW(512, 2);
    SQ_ROW(512, 4);
    return hipErrorInvalidValue;
}
#undef SQ_ROW
constexpr int64_t kBackwardThreads = 512;

constexpr int64_t kLongSlices = 64, kLongGrid = 1 << 20;

// Rows that the last-level cache would not keep anyway go past it: 16384 x 4096 in bf16,
// forward and backward in turn, 98 and 121 us through the caches, 102 and 97 past
// them (5.3 and 5.5 TB/s); 3152 x 768 in fp32, the backward, 8.0 and 8.6.
template <typename T>
bool past_caches(const NormArgs& a) {
    return a.C % kVec<T> == 0 && (double)a.M * (double)a.C * sizeof(T) >= 32e6;
}

template <typename T>
hipError_t forward(const NormArgs& a, hipStream_t s) {
    const RowPlan r = forward_plan(a.C, a.type);
    if (r.tpr == 0) {
        k_norm_forward_long<T><<<(uint32_t)std::min<int64_t>(a.M, kLongGrid), kLong, 0, s>>>(a);
        return hipGetLastError();
    }
    return with_forward(r, [&](auto TPR, auto V) {
        constexpr int tpr = decltype(TPR)::value, threads = tpr < 256 ? 256 : tpr, rows = threads / tpr;
        const int64_t blocks = std::min<int64_t>((a.M + rows - 1) / rows, 2048);
        constexpr int v = decltype(V)::value;
        if (past_caches<T>(a)) k_norm_forward<T, tpr, v, threads, true, true><<<(uint32_t)blocks, threads, 0, s>>>(a);
        else if (a.C % kVec<T> == 0) k_norm_forward<T, tpr, v, threads, true, false><<<(uint32_t)blocks, threads, 0, s>>>(a);
        else k_norm_forward<T, tpr, v, threads, false, false><<<(uint32_t)blocks, threads, 0, s>>>(a);
        return hipGetLastError();
    });
}

template <typename T>
hipError_t backward(const NormArgs& a, hipStream_t s) {
    const RowPlan r = backward_plan(a.C, a.type);
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
        e = with_backward(r, [&](auto TPR, auto V) {
            constexpr int tpr = decltype(TPR)::value, threads = 512;
            constexpr int v = decltype(V)::value;
            if (past_caches<T>(a)) k_norm_backward<T, tpr, v, threads, true, true><<<(uint32_t)parts, threads, 0, s>>>(a);
            else if (a.C % kVec<T> == 0) k_norm_backward<T, tpr, v, threads, true, false><<<(uint32_t)parts, threads, 0, s>>>(a);
            else k_norm_backward<T, tpr, v, threads, false, false><<<(uint32_t)parts, threads, 0, s>>>(a);
            return hipGetLastError();
        });
    }
    if (e != hipSuccess) return e;
    k_norm_reduce<<<(uint32_t)((2 * a.C + 31) / 32), 1024, 0, s>>>(a.part, parts, a.C, a.dgamma, a.dbeta);
    return hipGetLastError();
}

}  // namespace

int64_t norm_parts(int64_t M, int64_t C, int type) {
    const RowPlan r = backward_plan(C, type);
    if (r.tpr == 0) return std::max<int64_t>(1, std::min(M, kLongSlices));
    const int64_t rows = kBackwardThreads / r.tpr;
    return std::max<int64_t>(1, std::min<int64_t>((M + rows - 1) / rows, 512));
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
