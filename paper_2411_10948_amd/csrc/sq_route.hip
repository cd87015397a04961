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
// each: next to no time, and no ratio of scores that underflow.  But for one sum: a
// softmax that is not renormalised is divided by an fp32 sum of fp32 exponentials
// where four tokens share a wave (up to 512 experts and 16 slots), which is off by at
// most 20 2^-24: in 64 bits it would take an exponential for every expert.  A sigmoid's
// 1 - s is what 64 bits leave of it, off by 2^-53 at most.
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

// How many lanes keep_groups has for a group.
__device__ __forceinline__ int group_lanes(const RouteArgs& p) {
    return p.groups == 1 ? 64 : 1 << (__builtin_clz((unsigned)(p.groups - 1)) - 26);      // 64 / lanes >= groups
}

// The best top_groups groups, group g at bit g group_lanes.  s: -inf for experts
// that are never chosen; lds: 64 V values of the wave's own.  A group's sum is
// that of its two scores plus that of their biases, so that groups which hold the
// same of each are equal, however the biases fall on the scores.
template <int V>
__device__ __forceinline__ uint64_t keep_groups(const RouteArgs& p, const double* s, double* lds, int lane) {
    const double none = -__builtin_inf();
#pragma unroll
    for (int i = 0; i < V; ++i) lds[lane * V + i] = s[i];
    wave_fence();
    // L lanes a group, each the two highest of every L-th expert, then those of all of them
    const int per = p.E / p.groups, L = group_lanes(p), g = lane / L, first = lane % L;
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
    const uint64_t kept = __ballot(first == 0 && g < p.groups && rank < p.top_groups);
    wave_fence();
    return kept;
}

// The shares of a token's slots from their scores, a lane each.
__device__ __forceinline__ float share_of(const RouteArgs& p, double score) {
    double v = score;
    if (p.renorm) v = score / fmax(wave_sum(score), kLeast);
    return (float)((double)p.scale * v);
}

// A token by a whole wave, E <= 64 V: its choice and shares, and a bit in `rows` for
// each of its experts.  EXACT: the experts are not ordered by their logits alone;
// lds as in keep_groups.
template <typename T, int V, bool EXACT>
__device__ __forceinline__ void wave_token(const RouteArgs& p, int64_t t, int bit, uint64_t* rows, double* lds, int lane) {
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
                if (p.groups > 1) {
                    const uint64_t kept = keep_groups<V>(p, of, lds, lane);
                    const int per = p.E / p.groups, L = group_lanes(p);
#pragma unroll
                    for (int k = 0; k < V; ++k)
                        key[k] = kept >> (min((lane * V + k) / per, p.groups - 1) * L) & 1 ? key[k] : none;
                }
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
        if (chosen >= 0) atomicOr((unsigned long long*)&rows[chosen], 1ull << bit);
    }
}

// What a block's tokens leave once their bits are in `rows`: a token takes an expert
// once at most, so a word with a bit for each token holds the block's rows of an
// expert in order: their count, and a row's rank, are counts of its bits.  ONLY: the
// only block, which writes the places themselves; otherwise ranks.
template <bool ONLY>
__device__ __forceinline__ void block_places(const RouteArgs& p, const uint64_t* rows, int64_t t0, int tokens) {
    const int tid = threadIdx.x, lane = tid & 63;
    __syncthreads();
    if constexpr (ONLY) {
        if (tid < 64) {         // counts of the experts before, in place of none
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
        for (int e = tid; e < p.E; e += blockDim.x)
            p.counts[(int64_t)blockIdx.x * route_stride(p.E) + e] = (uint8_t)__popcll(rows[e]);
    }
    for (int i = tid; i < tokens * p.k; i += blockDim.x) {
        const int64_t at = t0 * p.k + i;
        const int e = p.chosen[at];
        int rank = e < 0 ? -1 : __popcll(rows[e] & ((1ull << (i / p.k)) - 1));
        if (ONLY && e >= 0) rank += p.offsets[e];
        p.place[at] = rank;
    }
}

// Tokens 64 b .. 64 b + 63 of block b, a wave each at a time.
template <typename T, int V, bool EXACT, bool ONLY>
__global__ __launch_bounds__(1024) void k_route(RouteArgs p) {
    __shared__ uint64_t rows[64 * V];
    __shared__ double lds[EXACT ? 16 : 1][EXACT ? 64 * V : 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t t0 = (int64_t)blockIdx.x * kRouteTokens;
    const int tokens = (int)min(p.T - t0, (int64_t)kRouteTokens);
    for (int e = tid; e < p.E; e += blockDim.x) rows[e] = 0;
    __syncthreads();
    for (int i = wave; i < tokens; i += blockDim.x >> 6)
        wave_token<T, V, EXACT>(p, t0 + i, i, rows, lds[EXACT ? wave : 0], lane);
    block_places<ONLY>(p, rows, t0, tokens);
}

// ---------------------------------------------------------------------------
// Four tokens a wave, 16 lanes each, for up to 16 slots: a reduction over a token is
// four steps for four tokens at once.  A group of experts is a run of lanes, a lane
// up to R consecutive experts of it, so the lowest index is in the lowest lane.
// Scores and sums with biases are fp32 here; where these leave the order in doubt
// (EXACT) the token is done again by the whole wave in fp64.  Bound by the instructions
// of its k turns over the keys, and where there are few tokens by the launch: 16384
// tokens, 8 of 256 experts by sigmoids, a bias and 4 of 8 groups, 22 us forward and 6.8
// backward (52 MB: 10 at the copy rate), a wave a token throughout 67 and 10; 8 of 64 by
// a softmax 10.6 and 4.1, a wave a token 21.4 and 7.4; one token 4.6 and 4.2.
// ---------------------------------------------------------------------------
template <typename F>
__device__ __forceinline__ F max16(F v) {
    return over_lanes(v, 16, [](F a, F b) { return larger(a, b); });
}
template <typename F>
__device__ __forceinline__ F sum16(F v) {
    return over_lanes(v, 16, [](F a, F b) { return a + b; });
}
// whether any of a token's lanes says so
__device__ __forceinline__ bool any16(bool b, int lane) { return (__ballot(b) >> (lane & 48) & 0xFFFF) != 0; }

// fp32 as unsigned numbers of the same order (both zeros alike), -inf as 0
__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t b = __float_as_uint(v + 0.0f);
    return v == -__builtin_inff() ? 0u : b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7FFFFFFFu : ~u); }

// n <= R values from element e0 of a row of E, `fill` past them
template <typename T, int R>
__device__ __forceinline__ void load_run(const T* row, int e0, int n, int E, float fill, float* out) {
    constexpr int N = kVec<T>;
    if constexpr (R >= N) {
#pragma unroll
        for (int i = 0; i < R; i += N) {
            uint32_t w[4] = {0, 0, 0, 0};
            if (i < n) load16(row, e0 + i, E, w);
            values16<T>(w, out + i);
        }
    } else {
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const T v = row[min(e0 + i, E - 1)];
            if constexpr (sizeof(T) == 4) out[i] = v;
            else out[i] = bf16_value(v);
        }
    }
#pragma unroll
    for (int i = 0; i < R; ++i) out[i] = i < n ? out[i] : fill;
}

constexpr int kLaneExperts = 512, kLaneSlots = 16;

template <typename T, int R, bool EXACT, bool ONLY>
__global__ __launch_bounds__(1024) void k_route_lanes(RouteArgs p, int lanes, int run) {
    __shared__ uint64_t rows[kLaneExperts];
    __shared__ double lds[EXACT ? 16 : 1][EXACT ? kLaneExperts : 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t t0 = (int64_t)blockIdx.x * kRouteTokens;
    const int tokens = (int)min(p.T - t0, (int64_t)kRouteTokens);
    for (int e = tid; e < p.E; e += blockDim.x) rows[e] = 0;
    __syncthreads();

    const int sub = lane & 15, i = wave * 4 + (lane >> 4);
    const bool live = i < tokens;
    const int64_t t = t0 + min(i, tokens - 1);
    const T* row = static_cast<const T*>(p.logits) + t * p.ld;
    const int per = p.E / p.groups, g = sub / lanes, first = (sub - g * lanes) * run;
    const int e0 = g * per + first, n = g < p.groups ? max(0, min(run, per - first)) : 0;
    const float none = -__builtin_inff();
    const bool softmax = p.score == SQ_SCORE_SOFTMAX;
    float l[R];
    load_run<T, R>(row, min(e0, p.E - 1), n, p.E, none, l);
    bool bad = false;
    float m = none;
    if (softmax || !EXACT) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if constexpr (!EXACT) bad |= l[r] != l[r] || (softmax && l[r] == __builtin_inff());
            m = fmaxf(m, l[r]);
        }
        m = max16(m);
    }
    float sum = 1.0f;
    if (softmax && (EXACT || !p.renorm)) {
        float part[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int r = 0; r < R; ++r) part[r & 3] += l[r] > none ? __expf(l[r] - m) : 0.0f;
        sum = sum16((part[0] + part[1]) + (part[2] + part[3]));
    }

    uint32_t key[R];
    float doubt = 0.0f;     // how far fp32 may be off the difference of two sums s + bias, without its rounding
    if constexpr (EXACT) {
        float bias[R], inv = 1.0f / sum, a = none, b = none;
#pragma unroll
        for (int r = 0; r < R; ++r) bias[r] = 0.0f;
        if (p.bias) load_run<float, R>(p.bias, min(e0, p.E - 1), n, p.E, 0.0f, bias);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float s = softmax ? __expf(l[r] - m) * inv : __builtin_amdgcn_rcpf(1.0f + __expf(-l[r]));
            // NaN in the logit or the bias, and +inf under softmax (inf - inf), are NaN here
            const float v = l[r] == none ? none : s + bias[r];
            bad |= v != v;
            b = __builtin_amdgcn_fmed3f(a, b, v);       // the second of three, as b <= a
            a = fmaxf(a, v);
            if (p.bias) {
                // a sum with a bias is in doubt anyway: its last bits say which of the lane's it is
                const uint32_t u = __float_as_uint(v), o = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
                key[r] = v == none ? 0u : (o & ~(uint32_t)(R - 1)) | (uint32_t)(R - 1 - r);
            } else {
                key[r] = ordered(l[r]);
            }
        }
        // exp(x): the rounding of x log2(e) moves a score by at most s |x| 2^-24 or, a sigmoid, s (1 - s) |x| 2^-24, less
        // than half of 2^-24 of the largest; the exponential and the reciprocal are good to 1 ulp, sums are rounded once.
        // So two sigmoids' difference is right to 2^-21; a softmax's sum of at most 14 additions one after the other is a
        // factor of all scores, which moves differences by 20 2^-24 of the largest at most.
        doubt = softmax ? inv * 0x1p-18f : 0x1p-21f;     // the largest softmax is 1 / sum
        if (p.groups > 1) {
            for (int step = 1; step < lanes; step <<= 1) {
                const float oa = step == 1 ? row_move<kLane1>(a) : step == 2 ? row_move<kLane2>(a) : row_move<kMirror8>(a);
                const float ob = step == 1 ? row_move<kLane1>(b) : step == 2 ? row_move<kLane2>(b) : row_move<kMirror8>(b);
                b = larger(larger(b, ob), a < oa ? a : oa);
                a = larger(a, oa);
            }
            const float total = b > none ? a + b : a;
            int rank = 0;
            for (int o = 0; o < p.groups; ++o) {
                const float other = __shfl(total, (lane & 48) + o * lanes);
                rank += other > total || (other == total && o < g) ? 1 : 0;
            }
            const bool mine = g < p.groups;
            bool kept = mine && rank < p.top_groups;
            const float low = -max16(kept ? -total : none), high = max16(mine && !kept ? total : none);
            // Of equal totals the lowest group, but only fp64 knows which are equal: two sums with a bias and their total
            // are rounded, 3 2^-24 of the summands' size, on either side.
            const float size = max16(mine && a > none ? fabsf(a) + (b > none ? fabsf(b) : 0.0f) : 0.0f);
            const bool unclear = high > none && !(low - high > 2.0f * doubt + 0x1p-21f * size);
            // These tokens' groups by the whole wave in fp64: 16384 tokens, 4 of 8 groups of 256 experts, where one or two are
            // unclear 28.5 -> 23 us.  With 32 experts a lane that spills, and every launch pays (34 -> 39.5 us, 2 of 4 groups of
            // 512 experts): there the whole token is done again.
            if constexpr (R > 16) bad |= unclear;
            else for (uint64_t todo = __ballot(live && unclear && sub == 0); todo; todo &= todo - 1) {
                constexpr int V = kLaneExperts / 64;
                const int from = __ffsll((unsigned long long)todo) - 1;
                float v[V];
                double of[V];
                load_logits<T, V>(static_cast<const T*>(p.logits) + (t0 + wave * 4 + (from >> 4)) * p.ld, p.E, lane, v);
                scores<V>(v, softmax, of);
#pragma unroll
                for (int r = 0; r < V; ++r) of[r] = v[r] > none ? of[r] : -__builtin_inf();
                const uint64_t best = keep_groups<V>(p, of, lds[wave], lane);
                if ((lane ^ from) < 16) kept = mine && (best >> (g * group_lanes(p)) & 1);
            }
#pragma unroll
            for (int r = 0; r < R; ++r) key[r] = kept ? key[r] : 0u;
        }
    } else {
#pragma unroll
        for (int r = 0; r < R; ++r) key[r] = ordered(l[r]);
    }

    // Sigmoids + bias: two candidates more than slots, whose order fp64 decides; only where the last of them is as
    // near to the last slot's as fp32 may be off is an expert that is none of them in question.  A softmax's sum is known
    // in fp32 only: every two neighbours have to differ by more than that.
    const bool biased = EXACT && p.bias, refine = biased && !softmax && p.k < kLaneSlots;
    const int picks = refine ? min(p.k + 2, kLaneSlots) : biased ? p.k + 1 : p.k;
    int chosen = -1;
    bool unsure = false;
    float last = none;
    if (biased) {
        // No two keys of a lane are equal, so those that are left are the ones up to a limit: its distance to them,
        // which is smallest for the best and wraps around for those above.
        uint32_t limit = ~0u;
        for (int j = 0; j < picks; ++j) {
            uint32_t down = ~0u;
#pragma unroll
            for (int r = 0; r < R; ++r) down = min(down, limit - key[r]);
            const uint32_t best = down <= limit ? limit - down : 0u;
            const uint32_t top = over_lanes(best, 16, [](uint32_t x, uint32_t y) { return max(x, y); });
            if (__ballot(top != 0) == 0) {
                last = none;
                break;
            }
            const float v = top != 0 ? unordered(top) : none;
            unsure |= !refine && j > 0 && top != 0 && !(last - v > doubt + 0x1p-17f * (fabsf(last) + fabsf(v)));
            last = v;
            const int src = __builtin_ctz(((uint32_t)(__ballot(best == top) >> (lane & 48)) & 0xFFFFu) | 0x10000u);
            const int e = __shfl(e0, (lane & 48) + src) + R - 1 - (int)(top & (uint32_t)(R - 1));
            if (sub == j && top != 0) chosen = e;
            limit = top != 0 ? top - (sub <= src ? 1u : 0u) : 0u;
        }
    } else {
        for (int j = 0; j < picks; ++j) {
            uint32_t best = 0;
#pragma unroll
            for (int r = 0; r < R; ++r) best = max(best, key[r]);
            const uint32_t top = over_lanes(best, 16, [](uint32_t x, uint32_t y) { return max(x, y); });
            if (__ballot(top != 0) == 0) break;
            const int src = __builtin_ctz(((uint32_t)(__ballot(best == top) >> (lane & 48)) & 0xFFFFu) | 0x10000u);
            bool open = top != 0 && sub == src;
            int at = 0;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const bool hit = open && key[r] == top;
                open = open && !hit;
                key[r] = hit ? 0u : key[r];
                at = hit ? r : at;
            }
            const int e = __shfl(e0 + at, (lane & 48) + src);
            if (sub == j && top != 0) chosen = e;
        }
    }

    const bool nan = any16(bad, lane);      // or in doubt
    double s = 0.0;
    if (chosen >= 0) {
        float x;
        if constexpr (sizeof(T) == 4) x = row[chosen];
        else x = bf16_value(row[chosen]);
        s = softmax ? exp((double)x - (double)m) / (double)sum : 1.0 / (1.0 + exp(-(double)x));
    }
    if constexpr (EXACT) {
        if (refine) {
            double v = chosen >= 0 ? s + (double)p.bias[chosen] : -__builtin_inf();
            const double after = __shfl_down(v, 1);
            const int e_after = __shfl_down(chosen, 1);
            const bool fine = sub + 1 >= picks || e_after < 0 || v > after || (v == after && chosen < e_after);
            if (__ballot(live && !fine) != 0) {     // sort them, each to the lane of its rank
                int rank = 0;
                for (int o = 0; o < picks; ++o) {
                    const double other = __shfl(v, (lane & 48) + o);
                    const int e = __shfl(chosen, (lane & 48) + o);
                    rank += e >= 0 && (chosen < 0 || other > v || (other == v && e < chosen)) ? 1 : 0;
                }
                int from = lane;
                for (int o = 0; o < picks; ++o)
                    if (__shfl(rank, (lane & 48) + o) == sub && __shfl(chosen, (lane & 48) + o) >= 0) from = (lane & 48) + o;
                const int found = __popcll(__ballot(chosen >= 0) >> (lane & 48) & 0xFFFF);
                s = __shfl(s, from);
                v = __shfl(v, from);
                chosen = __shfl(chosen, from);
                if (sub >= found) chosen = -1, s = 0.0, v = -__builtin_inf();
            }
            const double edge = __shfl(v, (lane & 48) + p.k - 1);
            // a last candidate of +inf is NaN here, by the register in its last bits: in doubt too
            unsure = last != none && !(edge - (double)last > (double)(doubt + 0x1p-17f * fabsf(last)));
        }
        if (sub >= p.k) chosen = -1, s = 0.0;
    }
    if (p.renorm) s /= fmax(sum16(s), kLeast);
    const bool again = EXACT && (nan || any16(unsure, lane));
    if (live && sub < p.k && !again) {
        p.share[t * p.k + sub] = nan ? __builtin_nanf("") : (float)((double)p.scale * s);
        p.chosen[t * p.k + sub] = nan ? -1 : chosen;
        if (chosen >= 0 && !nan) atomicOr((unsigned long long*)&rows[chosen], 1ull << i);
    }
    if constexpr (EXACT) {
        for (uint64_t todo = __ballot(live && again && sub == 0); todo; todo &= todo - 1) {
            const int bit = wave * 4 + ((__ffsll((unsigned long long)todo) - 1) >> 4);
            wave_token<T, kLaneExperts / 64, true>(p, t0 + bit, bit, rows, lds[wave], lane);
        }
    }
    block_places<ONLY>(p, rows, t0, tokens);
}

// base[b][e]: rows of expert e in the blocks before b, b = blocks: in all.  64
// experts a block of 16 waves, each a run of the blocks.
__global__ __launch_bounds__(1024) void k_route_base(const uint8_t* counts, int32_t* base, int64_t blocks, int E) {
    __shared__ int sums[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, e = blockIdx.x * 64 + lane;
    const int64_t per = (blocks + 15) / 16, lo = min(wave * per, blocks), hi = min(lo + per, blocks);
    int n = 0;
    if (e < E)
        for (int64_t b = lo; b < hi; ++b) n += counts[b * route_stride(E) + e];
    sums[wave][lane] = n;
    __syncthreads();
    if (e >= E) return;
    int at = 0;
    for (int w = 0; w < wave; ++w) at += sums[w][lane];
    for (int64_t b = lo; b < hi; ++b) {
        base[b * E + e] = at;
        at += counts[b * route_stride(E) + e];
    }
    if (wave == 15) base[blocks * E + e] = at;
}

// Ranks within a block's tokens to places: plus the expert's first row, plus its
// rows in the blocks before.  COUNT: these are counted here, by every block over all
// blocks' counts (four experts a thread); otherwise `base` holds them.
template <bool COUNT>
__global__ __launch_bounds__(1024) void k_route_place(RouteArgs p, int blocks) {
    __shared__ int first[kRouteMaxExperts], mine[kRouteMaxExperts];
    const int tid = threadIdx.x, lane = tid & 63;
    if constexpr (COUNT) {
        __shared__ int all[1024][4], below[1024][4];
        const int words = (p.E + 3) / 4, slices = min(1024 / words, 16), w = tid % words, slice = tid / words;
        int n[4] = {0, 0, 0, 0}, b[4] = {0, 0, 0, 0};
        if (slice < slices) {
#pragma unroll 8
            for (int r = slice; r < blocks; r += slices) {
                const uint8_t* at = p.counts + (int64_t)r * words * 4 + 4 * w;
                const uint32_t c = *reinterpret_cast<const uint32_t*>(at);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int v = (int)(c >> (8 * i) & 255u);
                    n[i] += v;
                    b[i] += r < (int)blockIdx.x ? v : 0;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) all[tid][i] = n[i], below[tid][i] = b[i];
        __syncthreads();
        for (int e = tid; e < p.E; e += 1024) {
            int sum = 0, before = 0;
            for (int k = 0; k < slices; ++k) {
                sum += all[k * words + e / 4][e & 3];
                before += below[k * words + e / 4][e & 3];
            }
            first[e] = sum;
            mine[e] = before;
        }
    } else {
        for (int e = tid; e < p.E; e += 1024) {
            first[e] = p.base[(int64_t)blocks * p.E + e];
            mine[e] = p.base[(int64_t)blockIdx.x * p.E + e];
        }
    }
    __syncthreads();
    if (tid < 64) {
        int before = 0;
        for (int e0 = 0; e0 < p.E; e0 += 64) {
            const int e = e0 + lane, n = e < p.E ? first[e] : 0, sum = wave_scan(n);
            if (e < p.E) first[e] = before + sum - n;
            before += __builtin_amdgcn_readlane(sum, 63);
        }
        if (blockIdx.x == 0 && lane == 0) p.offsets[p.E] = before;
    }
    __syncthreads();
    if (blockIdx.x == 0)
        for (int e = tid; e < p.E; e += 1024) p.offsets[e] = first[e];
    const int64_t t0 = (int64_t)blockIdx.x * kRouteTokens;
    const int n = (int)min(p.T - t0, (int64_t)kRouteTokens) * p.k;
    for (int i = tid; i < n; i += 1024) {
        const int64_t at = t0 * p.k + i;
        const int e = p.chosen[at];
        if (e >= 0) p.place[at] += first[e] + mine[e];
    }
}

// A wave a token.  Only softmax that is not renormalised has a gradient outside the
// chosen experts, and reads all logits; the others read those of the chosen ones.
// Bound by the fp64 exponentials, one for every expert: 16384 x 64 in fp32 7.5 us, 16384 x 256
// 14.3 (34 MB, 6.5 at the copy rate), 32768 x 512 61; the renormalised ones 4.6, 7.2 and 16.4.
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
        const double peak = wave_max(x);    // of every lane, also those without a slot
        double s, v;
        if (softmax) s = x > none ? exp(x - peak) : 0.0;
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

// The same where only the chosen experts have a gradient, four tokens a wave, 16
// lanes each: rows are put together in LDS and leave in 16-byte pieces.
template <typename T>
__global__ __launch_bounds__(256) void k_route_backward_lanes(RouteArgs p) {
    extern __shared__ uint32_t row_words[];
    constexpr int N = kVec<T>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), sub = lane & 15;
    const int pieces = (p.E + N - 1) / N;
    uint4* mine = reinterpret_cast<uint4*>(row_words) + wave * 4 * pieces;
    const int64_t t0 = ((int64_t)blockIdx.x * 4 + wave) * 4, t = t0 + (lane >> 4);
    const bool live = t < p.T, slot = live && sub < p.k;
    int e = slot ? p.chosen[t * p.k + sub] : -1;
    const float w = slot ? p.share[t * p.k + sub] : 0.0f;
    e = e < p.E ? e : -1;
    const double d = e >= 0 ? (double)p.dshare[t * p.k + sub] : 0.0;
    double x = -__builtin_inf();
    if (e >= 0) {
        const T v = static_cast<const T*>(p.logits)[t * p.ld + e];
        if constexpr (sizeof(T) == 4) x = (double)v;
        else x = (double)bf16_value(v);
    }
    const bool nan = any16(w != w, lane), softmax = p.score == SQ_SCORE_SOFTMAX;
    const uint32_t fill = !nan ? 0u : sizeof(T) == 4 ? 0x7FC00000u : 0x7FC07FC0u;
    for (int i = sub; i < pieces; i += 16) mine[(lane >> 4) * pieces + i] = make_uint4(fill, fill, fill, fill);
    wave_fence();
    const double peak = max16(x);       // of every lane, also those without a slot
    double s, v;
    if (softmax) s = e >= 0 ? exp(x - peak) : 0.0;
    else s = e >= 0 ? 1.0 / (1.0 + exp(-x)) : 0.0;
    if (p.renorm) {
        const double r = s / fmax(sum16(s), kLeast);
        v = r * (d - sum16(d * r));
        if (!softmax) v *= 1.0 - s;
    } else {
        v = d * s * (1.0 - s);
    }
    const float g = (float)((double)p.scale * v);
    T* row = reinterpret_cast<T*>(mine + (lane >> 4) * pieces);
    if (e >= 0 && !nan) {
        if constexpr (sizeof(T) == 4) row[e] = g;
        else row[e] = (T)bf16_bits(g);
    }
    wave_fence();
    for (int i = lane; i < 4 * pieces; i += 64) {
        const int at = i / pieces;
        if (t0 + at >= p.T) break;
        const uint4 q = mine[i];
        const uint32_t words[4] = {q.x, q.y, q.z, q.w};
        store16(static_cast<T*>(p.dlogits) + (t0 + at) * p.ld_d, (int64_t)(i - at * pieces) * N, p.E, words);
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

template <typename T, bool EXACT>
hipError_t choices(const RouteArgs& a, int64_t blocks, hipStream_t s) {
    // lanes of a group, experts of a lane
    int lanes = 16;
    while (lanes > 1 && lanes * a.groups > 16) lanes /= 2;
    const int run = (a.E / a.groups + lanes - 1) / lanes;
    if (lanes * a.groups <= 16 && run <= 32 && a.E <= kLaneExperts && a.k <= kLaneSlots) {
        const auto launch = [&](auto W) {
            constexpr int R = decltype(W)::value;
            if (blocks == 1) k_route_lanes<T, R, EXACT, true><<<1, 64 * (int)((a.T + 3) / 4), 0, s>>>(a, lanes, run);
            else k_route_lanes<T, R, EXACT, false><<<(uint32_t)blocks, 1024, 0, s>>>(a, lanes, run);
            return hipGetLastError();
        };
        if (run <= 1) return launch(std::integral_constant<int, 1>());
        if (run <= 4) return launch(std::integral_constant<int, 4>());
        if (run <= 8) return launch(std::integral_constant<int, 8>());
        if (run <= 16) return launch(std::integral_constant<int, 16>());
        return launch(std::integral_constant<int, 32>());
    }
    return with_width(a.E, [&](auto W) {
        constexpr int V = decltype(W)::value;
        if (blocks == 1) k_route<T, V, EXACT, true><<<1, 64 * (int)std::min<int64_t>(a.T, 16), 0, s>>>(a);
        else k_route<T, V, EXACT, false><<<(uint32_t)blocks, 1024, 0, s>>>(a);
        return hipGetLastError();
    });
}

// All blocks' counts are read by every block, to place its rows without a launch that
// sums them up first, up to these bytes in all and these blocks (a 16th of them a
// thread, one after the other: few experts are few bytes and as long).  With and without that
// launch: 16384 tokens, 4 of 64 experts (4 MB) 15.8 and 9.9 us; 65536 (64 MB) 43 and 28; 4 of 256,
// 32768 tokens (64 MB) 34.7 and 27.8, 65536 (256 MB) 61.7 and 67.4.  One of 4 experts: 65536
// tokens (1024 blocks) 30 and 25, 131072 (2048) 52 and 57, 262144 102 and 168, 370000 154 and 311;
// two of 8: 131072 63 and 51, 262144 117 and 161.
constexpr int64_t kCounted = 128 << 20, kCountedBlocks = 2048;

template <typename T>
hipError_t forward(const RouteArgs& a, hipStream_t s) {
    const int64_t blocks = route_blocks(a.T);
    hipError_t e = a.bias || a.groups > 1 ? choices<T, true>(a, blocks, s) : choices<T, false>(a, blocks, s);
    if (e != hipSuccess || blocks == 1) return e;
    if (blocks <= kCountedBlocks && blocks * blocks * route_stride(a.E) <= kCounted) {
        k_route_place<true><<<(uint32_t)blocks, 1024, 0, s>>>(a, (int)blocks);
        return hipGetLastError();
    }
    k_route_base<<<(uint32_t)((a.E + 63) / 64), 1024, 0, s>>>(a.counts, a.base, blocks, a.E);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    k_route_place<false><<<(uint32_t)blocks, 1024, 0, s>>>(a, (int)blocks);
    return hipGetLastError();
}

template <typename T>
hipError_t backward(const RouteArgs& a, hipStream_t s) {
    if (!(a.score == SQ_SCORE_SOFTMAX && !a.renorm) && a.k <= kLaneSlots) {
        const size_t lds = (size_t)(16 * ((a.E + kVec<T> - 1) / kVec<T>) * 16);
        k_route_backward_lanes<T><<<(uint32_t)((a.T + 15) / 16), 256, lds, s>>>(a);
        return hipGetLastError();
    }
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
