// Routing of tokens to experts and its backward pass.
//   s = softmax(l) or sigma(l) over E experts; an expert with l = -inf is never chosen
//   order: by l, with a bias by s + bias; ties: the lowest index
//   groups: a group counts as the sum of its two highest s (+ bias); experts outside
//           the best top_groups are left out
//   share_j = scale s_j, renormalised scale s_j / sum of the chosen s
//   place: position of (token, slot) in a stable sort of all of them by expert
// Gradients of the logits, S the chosen experts, d_j of share_j:
//   softmax                 scale p_i (d_i [i in S] - sum_S d_j p_j)
//   softmax, renormalised   scale r_j (d_j - sum_S d_i r_i) for j in S, r_j = s_j / sum_S s
//   sigmoid                 scale d_j s_j (1 - s_j)
//   sigmoid, renormalised   scale r_j (1 - s_j) (d_j - sum_S d_i r_i)
// The shares and gradients of the chosen experts are computed in 64 bits, a lane
// each: next to no time, and no ratio of scores that underflow.
#include <algorithm>

#include "sq_block.h"

namespace sq {

namespace {

constexpr double kLeast = 1e-300;       // below it a sum of chosen scores counts as this

__device__ __forceinline__ void wave_fence() {      // LDS words of a wave's own: in order, but not for the compiler
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The logits of experts V lane .. V lane + V - 1 in fp32, -inf past the last.
template <typename T, int V>
__device__ __forceinline__ void load_logits(const T* row, int E, int lane, float* l) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = lane * V + i;
        const T v = row[min(e, E - 1)];
        float f;
        if constexpr (sizeof(T) == 4) f = v;
        else f = bf16_value(v);
        l[i] = e < E ? f : -__builtin_inff();
    }
}

// Value of a lane's register `i`, i the same in all lanes or not.
template <int V, typename F>
__device__ __forceinline__ F pick(const F* v, int i) {
    F r = v[0];
#pragma unroll
    for (int k = 1; k < V; ++k) r = i == k ? v[k] : r;
    return r;
}

// The scores of a wave's experts in 64 bits (0 for those that are never chosen).
template <int V>
__device__ __forceinline__ void scores(const float* l, bool softmax, double* s) {
    if (softmax) {
        float m = l[0];
#pragma unroll
        for (int i = 1; i < V; ++i) m = fmaxf(m, l[i]);
        m = wave_max(m);
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            s[i] = l[i] > -__builtin_inff() ? exp((double)l[i] - (double)m) : 0.0;
            sum += s[i];
        }
        sum = wave_sum(sum);
        const double inv = 1.0 / fmax(sum, kLeast);
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] *= inv;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = l[i] > -__builtin_inff() ? 1.0 / (1.0 + exp(-(double)l[i])) : 0.0;
    }
}

// A wave's token: its k best experts, lane j those of slot j (chosen -1: none), and
// their scores.  key: what orders the experts, -inf for those left out.
template <int V, typename F>
__device__ __forceinline__ int choose(F* key, const double* s, int k, int lane, int& chosen, double& score) {
    const F none = -(F)__builtin_inff();
    chosen = -1;
    score = 0.0;
    for (int j = 0; j < k; ++j) {
        F best = key[0];
#pragma unroll
        for (int i = 1; i < V; ++i) best = larger(best, key[i]);
        const F top = wave_max(best);
        if (!(top > none)) return j;
        const int src = __ffsll((unsigned long long)__ballot(best == top)) - 1;
        int at = V - 1;     // the lowest of the lane's that has it
#pragma unroll
        for (int i = V - 2; i >= 0; --i) at = key[i] == top ? i : at;
        at = __builtin_amdgcn_readlane(at, src);
        const double sj = wave_lane(pick<V>(s, at), src);
        if (lane == j) {
            chosen = src * V + at;
            score = sj;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) key[i] = lane == src && i == at ? none : key[i];
    }
    return k;
}

// Leaves the groups that are not among the best top_groups out of key.  s: -inf for
// experts that are never chosen; lds: 64 V values of the wave's own.  A group's sum is
// that of its two scores plus that of their biases, so that groups which hold the
// same of each are equal, however the biases fall on the scores.
template <int V>
__device__ __forceinline__ void keep_groups(const RouteArgs& p, const double* s, double* key, double* lds, int lane) {
    const double none = -__builtin_inf();
#pragma unroll
    for (int i = 0; i < V; ++i) lds[lane * V + i] = s[i];
    wave_fence();
    // L lanes a group, each the two highest of every L-th expert, then those of all of them
    const int per = p.E / p.groups, shift = __builtin_clz((unsigned)max(p.groups - 1, 1)) - 26;     // 64 / L >= groups
    const int L = p.groups == 1 ? 64 : 1 << shift, g = lane / L, first = lane % L;
    double a = none, b = none;
    int at_a = 0, at_b = 0;
    auto take = [&](double v, int at) {
        const bool over = a < v;
        const double low = over ? a : v;
        const int at_low = over ? at_a : at;
        if (over) a = v, at_a = at;
        if (b < low) b = low, at_b = at_low;
    };
    if (g < p.groups)
        for (int i = first; i < per; i += L) {
            const int e = g * per + i;
            const double v = lds[e];
            take(v > none && p.bias ? v + (double)p.bias[e] : v, e);
        }
    for (int step = 1; step < L; step <<= 1) {
        const double oa = __shfl_xor(a, step), ob = __shfl_xor(b, step);
        const int pa = __shfl_xor(at_a, step), pb = __shfl_xor(at_b, step);
        take(oa, pa);
        take(ob, pb);
    }
    double total = none;
    if (a > none) {
        total = lds[at_a] + (b > none ? lds[at_b] : 0.0);
        if (p.bias) total += (double)p.bias[at_a] + (b > none ? (double)p.bias[at_b] : 0.0);
    }
    wave_fence();
    if (first == 0 && g < p.groups) lds[g] = total;
    wave_fence();
    int rank = 0;
    for (int o = 0; o < p.groups; ++o) {
        const double t = lds[o];
        rank += t > total || (t == total && o < g) ? 1 : 0;
    }
    const uint64_t kept = __ballot(first == 0 && g < p.groups && rank < p.top_groups);      // of group g at bit g L
    wave_fence();
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int e = lane * V + i, at = min(e / per, p.groups - 1);
        key[i] = kept >> (at * L) & 1 ? key[i] : none;
    }
}

// The shares of a token's slots from their scores, a lane each.
__device__ __forceinline__ float share_of(const RouteArgs& p, double score) {
    double v = score;
    if (p.renorm) v = score / fmax(wave_sum(score), kLeast);
    return (float)((double)p.scale * v);
}

// Tokens 64 b .. 64 b + 63 of block b, a wave each at a time.  A token takes an
// expert once at most, so a word with a bit for each token holds a block's rows
// of an expert in order: their count, and a row's rank, are counts of its bits.
// ONLY: the only block, which writes the places themselves; otherwise ranks.
template <typename T, int V, bool EXACT, bool ONLY>
__global__ __launch_bounds__(1024) void k_route(RouteArgs p) {
    __shared__ uint64_t rows[64 * V];
    __shared__ double lds[EXACT ? 16 : 1][EXACT ? 64 * V : 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int waves = blockDim.x >> 6;
    const int64_t t0 = (int64_t)blockIdx.x * kRouteTokens;
    const int tokens = (int)min(p.T - t0, (int64_t)kRouteTokens);
    for (int e = tid; e < p.E; e += blockDim.x) rows[e] = 0;
    __syncthreads();
    for (int i = wave; i < tokens; i += waves) {
        const int64_t t = t0 + i;
        float l[V];
        load_logits<T, V>(static_cast<const T*>(p.logits) + t * p.ld, p.E, lane, l);
        const bool softmax = p.score == SQ_SCORE_SOFTMAX;
        bool bad = false;
#pragma unroll
        for (int k = 0; k < V; ++k) bad |= l[k] != l[k] || (softmax && l[k] == __builtin_inff());
        double s[V];
        int chosen = -1;
        double score = 0.0;
        bool nan = __ballot(bad) != 0;
        if (!nan) {
            scores<V>(l, softmax, s);
            if constexpr (EXACT) {
                double key[V], of[V];
                const double none = -__builtin_inf();
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    const int e = min(lane * V + k, p.E - 1);
                    const bool live = l[k] > -__builtin_inff();
                    of[k] = live ? s[k] : none;
                    key[k] = !live ? none : p.bias ? s[k] + (double)p.bias[e] : (double)l[k];
                    bad |= key[k] != key[k];
                }
                nan = __ballot(bad) != 0;
                if (!nan) {
                    if (p.groups > 1) keep_groups<V>(p, of, key, lds[wave], lane);
                    choose<V>(key, s, p.k, lane, chosen, score);
                }
            } else {
                choose<V>(l, s, p.k, lane, chosen, score);
            }
        }
        const float share = share_of(p, score);
        if (lane < p.k) {
            p.share[t * p.k + lane] = nan ? __builtin_nanf("") : share;
            p.chosen[t * p.k + lane] = chosen;
            if (chosen >= 0) atomicOr((unsigned long long*)&rows[chosen], 1ull << i);
        }
    }
    __syncthreads();
    if constexpr (ONLY) {
        if (wave == 0) {        // counts of the experts before, in place of none
            int before = 0;
            for (int e0 = 0; e0 < p.E; e0 += 64) {
                const int n = e0 + lane < p.E ? __popcll(rows[e0 + lane]) : 0, sum = wave_scan(n);
                if (e0 + lane < p.E) p.offsets[e0 + lane] = before + sum - n;
                before += __builtin_amdgcn_readlane(sum, 63);
            }
            if (lane == 0) p.offsets[p.E] = before;
        }
        __syncthreads();
    } else {
        for (int e = tid; e < p.E; e += blockDim.x) p.counts[(int64_t)blockIdx.x * p.E + e] = (uint8_t)__popcll(rows[e]);
    }
    // the wave and lane that wrote a slot reads it again
    for (int i = wave; i < tokens; i += waves) {
        if (lane >= p.k) continue;
        const int64_t at = (t0 + i) * p.k + lane;
        const int e = p.chosen[at];
        int rank = e < 0 ? -1 : __popcll(rows[e] & ((1ull << i) - 1));
        if (ONLY && e >= 0) rank += p.offsets[e];
        p.place[at] = rank;
    }
}

// base[b][e]: rows of expert e in the blocks before b, b = blocks: in all.  64
// experts a block of 16 waves, each a run of the blocks.
__global__ __launch_bounds__(1024) void k_route_base(const uint8_t* counts, int32_t* base, int64_t blocks, int E) {
    __shared__ int sums[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = blockIdx.x * 64 + lane;
    const int64_t per = (blocks + 15) / 16, lo = min(wave * per, blocks), hi = min(lo + per, blocks);
    int n = 0;
    if (e < E)
        for (int64_t b = lo; b < hi; ++b) n += counts[b * E + e];
    sums[wave][lane] = n;
    __syncthreads();
    if (e >= E) return;
    int at = 0;
    for (int w = 0; w < wave; ++w) at += sums[w][lane];
    for (int64_t b = lo; b < hi; ++b) {
        base[b * E + e] = at;
        at += counts[b * E + e];
    }
    if (wave == 15) base[blocks * E + e] = at;
}

// Ranks within a block's tokens to places: plus the expert's first row, plus its
// rows in the blocks before.
__global__ __launch_bounds__(256) void k_route_place(RouteArgs p, int64_t blocks) {
    __shared__ int first[kRouteMaxExperts];
    const int tid = threadIdx.x, lane = tid & 63;
    const int32_t *total = p.base + blocks * p.E, *mine = p.base + (int64_t)blockIdx.x * p.E;
    if (tid < 64) {
        int before = 0;
        for (int e0 = 0; e0 < p.E; e0 += 64) {
            const int e = e0 + lane, n = e < p.E ? total[e] : 0, sum = wave_scan(n);
            if (e < p.E) first[e] = before + sum - n;
            before += __builtin_amdgcn_readlane(sum, 63);
        }
        if (blockIdx.x == 0 && lane == 0) p.offsets[p.E] = before;
    }
    __syncthreads();
    if (blockIdx.x == 0)
        for (int e = tid; e < p.E; e += 256) p.offsets[e] = first[e];
    const int64_t t0 = (int64_t)blockIdx.x * kRouteTokens;
    const int n = (int)min(p.T - t0, (int64_t)kRouteTokens) * p.k;
    for (int i = tid; i < n; i += 256) {
        const int64_t at = t0 * p.k + i;
        const int e = p.chosen[at];
        if (e >= 0) p.place[at] += first[e] + mine[e];
    }
}

// A wave a token.  Only softmax that is not renormalised has a gradient outside the
// chosen experts, and reads all logits; the others read those of the chosen ones.
template <typename T, int V>
__global__ __launch_bounds__(256) void k_route_backward(RouteArgs p) {
    __shared__ float lds[4][64 * V];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t = (int64_t)blockIdx.x * 4 + wave;
    if (t >= p.T) return;
    const T* row = static_cast<const T*>(p.logits) + t * p.ld;
    int e = lane < p.k ? p.chosen[t * p.k + lane] : -1;
    const float w = lane < p.k ? p.share[t * p.k + lane] : 0.0f;
    const double d = e >= 0 && e < p.E ? (double)p.dshare[t * p.k + lane] : 0.0;
    e = e < p.E ? e : -1;
    const bool nan = __ballot(w != w) != 0, softmax = p.score == SQ_SCORE_SOFTMAX;
    float* mine = lds[wave];
#pragma unroll
    for (int i = 0; i < V; ++i) mine[lane * V + i] = 0.0f;
    wave_fence();
    float g[V];
    if (softmax && !p.renorm) {
        if (e >= 0) mine[e] = (float)d;
        wave_fence();
        float l[V];
        load_logits<T, V>(row, p.E, lane, l);
        double s[V], sum = 0.0;
        scores<V>(l, true, s);
#pragma unroll
        for (int i = 0; i < V; ++i) sum += (double)mine[lane * V + i] * s[i];
        sum = wave_sum(sum);
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = (float)((double)p.scale * s[i] * ((double)mine[lane * V + i] - sum));
    } else {
        float l = -__builtin_inff();
        if (e >= 0) {
            if constexpr (sizeof(T) == 4) l = row[e];
            else l = bf16_value(row[e]);
        }
        const double none = -__builtin_inf(), x = (double)l;
        double s, v;
        if (softmax) s = x > none ? exp(x - fmax(wave_max(x), -1e308)) : 0.0;
        else s = x > none ? 1.0 / (1.0 + exp(-x)) : 0.0;
        if (p.renorm) {
            const double r = s / fmax(wave_sum(s), kLeast);
            v = r * (d - wave_sum(d * r));
            if (!softmax) v *= 1.0 - s;
        } else {
            v = d * s * (1.0 - s);
        }
        if (e >= 0) mine[e] = (float)((double)p.scale * v);
        wave_fence();
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = mine[lane * V + i];
    }
    T* out = static_cast<T*>(p.dlogits) + t * p.ld_d;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int at = lane * V + i;
        const float v = nan ? __builtin_nanf("") : g[i];
        if (at >= p.E) continue;
        if constexpr (sizeof(T) == 4) out[at] = v;
        else out[at] = (T)bf16_bits(v);
    }
}

// f(V) for the power of two of experts a lane
template <class F>
hipError_t with_width(int E, F f) {
    if (E <= 64) return f(std::integral_constant<int, 1>());
    if (E <= 128) return f(std::integral_constant<int, 2>());
    if (E <= 256) return f(std::integral_constant<int, 4>());
    if (E <= 512) return f(std::integral_constant<int, 8>());
    return f(std::integral_constant<int, 16>());
}

template <typename T>
hipError_t forward(const RouteArgs& a, hipStream_t s) {
    const int64_t blocks = route_blocks(a.T);
    const bool exact = a.bias || a.groups > 1;
    hipError_t e = with_width(a.E, [&](auto W) {
        constexpr int V = decltype(W)::value;
        if (blocks == 1) {
            const int threads = 64 * (int)std::min<int64_t>(a.T, 16);
            if (exact) k_route<T, V, true, true><<<1, threads, 0, s>>>(a);
            else k_route<T, V, false, true><<<1, threads, 0, s>>>(a);
        } else {
            if (exact) k_route<T, V, true, false><<<(uint32_t)blocks, 1024, 0, s>>>(a);
            else k_route<T, V, false, false><<<(uint32_t)blocks, 1024, 0, s>>>(a);
        }
        return hipGetLastError();
    });
    if (e != hipSuccess || blocks == 1) return e;
    k_route_base<<<(uint32_t)((a.E + 63) / 64), 1024, 0, s>>>(a.counts, a.base, blocks, a.E);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    k_route_place<<<(uint32_t)blocks, 256, 0, s>>>(a, blocks);
    return hipGetLastError();
}

template <typename T>
hipError_t backward(const RouteArgs& a, hipStream_t s) {
    return with_width(a.E, [&](auto W) {
        k_route_backward<T, decltype(W)::value><<<(uint32_t)((a.T + 3) / 4), 256, 0, s>>>(a);
        return hipGetLastError();
    });
}

// Without tokens the experts have no rows.
__global__ void k_route_none(int32_t* offsets, int E) {
    for (int e = threadIdx.x; e <= E; e += 256) offsets[e] = 0;
}

}  // namespace

hipError_t launch_route_forward(const RouteArgs& a, hipStream_t s) {
    if (a.T == 0) {
        k_route_none<<<1, 256, 0, s>>>(a.offsets, a.E);
        return hipGetLastError();
    }
    return a.type == SQ_TYPE_F32 ? forward<float>(a, s) : forward<uint16_t>(a, s);
}

hipError_t launch_route_backward(const RouteArgs& a, hipStream_t s) {
    if (a.T == 0) return hipSuccess;
    return a.type == SQ_TYPE_F32 ? backward<float>(a, s) : backward<uint16_t>(a, s);
}

}  // namespace sq
