// Rows between tokens and experts: token t's slot j owns row place[t, j] of the rows
// sorted by expert.
//   dispatch           rows[place[t, j]] = x[t]
//   combine            out[t] = sum_j share[t, j] rows[place[t, j]] (+ add[t])
//   combine's gradient drows[place[t, j]] = share[t, j] dout[t],
//                      dshare[t, j] = <dout[t], rows[place[t, j]]>
//   dispatch's         dx[t] = sum_j drows[place[t, j]] (+ add[t]): combine without shares
// A place outside [0, rows) is no row: nothing is read or written for it, its
// product is 0.  Each row is read or written once, 16 bytes a thread, a thread's next
// slots' rows on their way while it adds up or multiplies; bound by HBM, small calls by
// their one launch.  4096 tokens, 8 rows of 2048 each in bf16 (134 MB of rows): dispatch
// 27 us, combine 29, its gradient 53, dispatch's 30: 738 MB at 5.3 TB/s in all.
#include <algorithm>
#include <type_traits>

#include "sq_block.h"

namespace sq {

namespace {

constexpr int kThreads = 256;
constexpr int kMostSlots = 8;   // rows in flight a thread

constexpr int64_t kMaxGrid = 1 << 20;   // blocks along the tokens; more of them take turns

// f(token, column): tpr threads a token, a piece of 16 bytes each; blockIdx.y: which
// tpr pieces of it.
template <typename T, class F>
__device__ __forceinline__ void my_pieces(const ExchangeArgs& p, int tpr, F f) {
    const int64_t c = ((int64_t)blockIdx.y * tpr + threadIdx.x % tpr) * kVec<T>, per = kThreads / tpr;
    if (c >= p.D) return;
    for (int64_t t = blockIdx.x * per + threadIdx.x / tpr; t < p.T; t += gridDim.x * per) f(t, c);
}

template <typename T, bool NT>
__global__ __launch_bounds__(kThreads) void k_dispatch(ExchangeArgs p, int tpr) {
    my_pieces<T>(p, tpr, [&](int64_t t, int64_t c) {
        uint32_t w[4];
        load16(static_cast<const T*>(p.x) + t * p.ld_x, c, p.D, w);
        for (int j = 0; j < p.k; ++j) {
            const uint32_t at = (uint32_t)p.place[t * p.k + j];
            if (at < (uint64_t)p.rows) store16<false, NT>(static_cast<T*>(p.rows_out) + at * p.ld_rows, c, p.D, w);
        }
    });
}

template <typename T, bool SHARES, int kSlots, bool NT>
__global__ __launch_bounds__(kThreads) void k_combine(ExchangeArgs p, int tpr) {
    constexpr int N = kVec<T>;
    my_pieces<T>(p, tpr, [&](int64_t t, int64_t c) {
        float sum[N];
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] = 0.0f;
        if (p.add) {
            uint32_t w[4];
            load16(static_cast<const T*>(p.add) + t * p.ld_add, c, p.D, w);
            values16<T>(w, sum);
        }
        for (int j0 = 0; j0 < p.k; j0 += kSlots) {
            uint32_t w[kSlots][4];
            float share[kSlots];
#pragma unroll
            for (int j = 0; j < kSlots; ++j) {
#pragma unroll
                for (int i = 0; i < 4; ++i) w[j][i] = 0;
                share[j] = 0.0f;
                if (j0 + j >= p.k) continue;
                const uint32_t at = (uint32_t)p.place[t * p.k + j0 + j];
                if (at >= (uint64_t)p.rows) continue;
                share[j] = SHARES ? p.share[t * p.k + j0 + j] : 1.0f;
                load16<false, NT>(static_cast<const T*>(p.rows_in) + at * p.ld_in, c, p.D, w[j]);
            }
#pragma unroll
            for (int j = 0; j < kSlots; ++j) {
                float f[N];
                values16<T>(w[j], f);
#pragma unroll
                for (int e = 0; e < N; ++e) sum[e] = __builtin_fmaf(share[j], f[e], sum[e]);
            }
        }
        uint32_t w[4];
        pack16<T>(sum, w);
        store16<false, NT>(static_cast<T*>(p.out) + t * p.ld_out, c, p.D, w);
    });
}

// WAVES waves a token; the products' sums over a wave's pieces, its lanes and the
// waves, in that order.
template <typename T, int WAVES, int kSlots, bool NT>
__global__ __launch_bounds__(kThreads) void k_combine_backward(ExchangeArgs p) {
    constexpr int N = kVec<T>, TPR = 64 * WAVES;
    __shared__ float sums[kThreads / 64][kSlots];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    constexpr int64_t per = kThreads / TPR;
    for (int64_t t0 = blockIdx.x * per; t0 < p.T; t0 += gridDim.x * per) {
        const int64_t t = t0 + threadIdx.x / TPR;
        const bool live = t < p.T;
        for (int j0 = 0; j0 < p.k; j0 += kSlots) {
            const int slots = min(p.k - j0, kSlots);
            uint32_t at[kSlots];
            float share[kSlots], dot[kSlots];
#pragma unroll
            for (int j = 0; j < kSlots; ++j) {
                at[j] = live && j < slots ? (uint32_t)p.place[t * p.k + j0 + j] : ~0u;
                share[j] = at[j] < (uint64_t)p.rows ? p.share[t * p.k + j0 + j] : 0.0f;
                dot[j] = 0.0f;
            }
            for (int64_t c = (int64_t)(threadIdx.x % TPR) * N; live && c < p.D; c += TPR * N) {
                uint32_t d[4], y[kSlots][4];
                load16(static_cast<const T*>(p.x) + t * p.ld_x, c, p.D, d);
#pragma unroll
                for (int j = 0; j < kSlots; ++j)
                    if (at[j] < (uint64_t)p.rows) load16<false, NT>(static_cast<const T*>(p.rows_in) + at[j] * p.ld_in, c, p.D, y[j]);
                float df[N];
                values16<T>(d, df);
#pragma unroll
                for (int j = 0; j < kSlots; ++j) {
                    if (at[j] >= (uint64_t)p.rows) continue;
                    float f[N], o[N];
                    values16<T>(y[j], f);
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        dot[j] = __builtin_fmaf(df[e], f[e], dot[j]);
                        o[e] = share[j] * df[e];
                    }
                    pack16<T>(o, y[j]);
                    store16<false, NT>(static_cast<T*>(p.rows_out) + at[j] * p.ld_rows, c, p.D, y[j]);
                }
            }
#pragma unroll
            for (int j = 0; j < kSlots; ++j) {
                dot[j] = wave_sum(dot[j]);
                if (lane == 0) sums[wave][j] = dot[j];
            }
            __syncthreads();
            const int j = threadIdx.x % TPR;
            if (live && j < slots) {
                float s = 0.0f;
                for (int w = 0; w < WAVES; ++w) s += sums[threadIdx.x / TPR * WAVES + w][j];
                p.dshare[t * p.k + j0 + j] = s;
            }
            __syncthreads();
        }
    }
}

// Threads a token, a power of two up to a block, and the grid.
template <typename T>
dim3 grid_of(int64_t T_, int64_t D, int& tpr) {
    const int64_t n = (D + kVec<T> - 1) / kVec<T>;
    tpr = 8;
    while (tpr < kThreads && tpr < n) tpr *= 2;
    return dim3((uint32_t)std::min<int64_t>((T_ + kThreads / tpr - 1) / (kThreads / tpr), kMaxGrid), (uint32_t)((n + tpr - 1) / tpr));
}

// f(slots in flight, whether the rows go past the caches) as compile-time constants.  No
// more slots than there are: combine's gradient of 1187 x 1000 in fp32 with two 5.3 us,
// with room for eight 8.1; with four 8.8 and 12.5.
template <typename T, class F>
hipError_t with_rows(const ExchangeArgs& a, F f) {
    // Rows that the last-level cache would not keep anyway go past it: 134 MB, combine and dispatch's gradient 29 and 30 us
    // instead of 37 and 47, the two that write rows the same either way.  Smaller ones stay for the kernel that reads them next.
    const bool nt = (double)a.T * a.k * (double)a.D * sizeof(T) >= 32e6;
    const auto slots = [&](auto NT) {
        if (a.k <= 2) return f(std::integral_constant<int, 2>(), NT);
        if (a.k <= 4) return f(std::integral_constant<int, 4>(), NT);
        return f(std::integral_constant<int, kMostSlots>(), NT);
    };
    return nt ? slots(std::true_type()) : slots(std::false_type());
}

template <typename T>
hipError_t dispatch(const ExchangeArgs& a, hipStream_t s) {
    int tpr;
    const dim3 grid = grid_of<T>(a.T, a.D, tpr);
    return with_rows<T>(a, [&](auto, auto NT) {
        k_dispatch<T, decltype(NT)::value><<<grid, kThreads, 0, s>>>(a, tpr);
        return hipGetLastError();
    });
}
template <typename T>
hipError_t combine(const ExchangeArgs& a, hipStream_t s) {
    int tpr;
    const dim3 grid = grid_of<T>(a.T, a.D, tpr);
    return with_rows<T>(a, [&](auto SLOTS, auto NT) {
        constexpr int slots = decltype(SLOTS)::value;
        if (a.share) k_combine<T, true, slots, decltype(NT)::value><<<grid, kThreads, 0, s>>>(a, tpr);
        else k_combine<T, false, slots, decltype(NT)::value><<<grid, kThreads, 0, s>>>(a, tpr);
        return hipGetLastError();
    });
}
template <typename T>
hipError_t combine_backward(const ExchangeArgs& a, hipStream_t s) {
    const int64_t n = (a.D + kVec<T> - 1) / kVec<T>;
    return with_rows<T>(a, [&](auto SLOTS, auto NT) {
        constexpr int slots = decltype(SLOTS)::value;
        constexpr bool nt = decltype(NT)::value;
        if (n <= 64) k_combine_backward<T, 1, slots, nt><<<(uint32_t)std::min<int64_t>((a.T + 3) / 4, kMaxGrid), kThreads, 0, s>>>(a);
        else k_combine_backward<T, 4, slots, nt><<<(uint32_t)std::min<int64_t>(a.T, kMaxGrid), kThreads, 0, s>>>(a);
        return hipGetLastError();
    });
}

}  // namespace

hipError_t launch_dispatch(const ExchangeArgs& a, hipStream_t s) {
    if (a.T == 0 || a.D == 0 || a.k == 0) return hipSuccess;
    return a.type == SQ_TYPE_F32 ? dispatch<float>(a, s) : dispatch<uint16_t>(a, s);
}
hipError_t launch_combine(const ExchangeArgs& a, hipStream_t s) {
    if (a.T == 0 || a.D == 0) return hipSuccess;
    return a.type == SQ_TYPE_F32 ? combine<float>(a, s) : combine<uint16_t>(a, s);
}
hipError_t launch_combine_backward(const ExchangeArgs& a, hipStream_t s) {
    if (a.T == 0 || a.k == 0) return hipSuccess;
    return a.type == SQ_TYPE_F32 ? combine_backward<float>(a, s) : combine_backward<uint16_t>(a, s);
}

}  // namespace sq
