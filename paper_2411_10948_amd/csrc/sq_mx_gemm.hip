// Products of microscaled 4-bit matrices for gfx950,
//     C[i, j] = sum_k A(i, k) B(j, k),
// dense, by expert over ragged rows (forward pass, input gradient) and by
// expert over ragged inner segments (weight gradient).
//
// v_mfma_scale_f32_16x16x128_f8f6f4 takes 16 x 128 codes of either operand
// (16 bytes a lane) and one scale a lane, multiplies in full and accumulates
// in fp32.  The operand layout (sq_mx.h) is the instruction's, so a tile goes
// from memory to LDS and from LDS to registers in lane order: contiguous
// 1 KB loads and conflict-free reads, no swizzle.
#include <algorithm>
#include <cstdlib>
#include <type_traits>

#include "sq_mx.h"

namespace sq {

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void_t;

constexpr int kFp4 = 4;   // the instruction's code of E2M1 operands

// c + a b^T over 128 inner elements; byte `S` of each lane's scale words.
template <int S>
__device__ __forceinline__ v4f mfma4(v4i a, v4i b, v4f c, int sa, int sb) {
    const v8i x = {a.x, a.y, a.z, a.w, 0, 0, 0, 0}, y = {b.x, b.y, b.z, b.w, 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, kFp4, kFp4, S, sa, S, sb);
}

// s_waitcnt vmcnt(n) lgkmcnt(0) (gfx9 encoding): at most n loads in flight, and
// every LDS read of this wave done, so that the stage it read may be refilled
// once all waves have passed the barrier that follows.
template <int N>
__device__ __forceinline__ void wait_loads() {
    __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | (0x7 << 4));
}

// Block tile BM x BN of WM x WN waves, a ring of STAGES stages of 128 inner
// elements in LDS.
template <int BM_, int BN_, int WM_, int WN_, int STAGES_>
struct MxCfg {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_;
    static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves;
    static constexpr int TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16;
    static constexpr int kGroups = (BM + BN) / 16;            // 16-row operand groups of a stage
    static constexpr int LPW = kGroups / kWaves;              // 1 KB loads per wave per stage
    static constexpr int kStage = kGroups * kMxTileBytes;
    static constexpr int kSmem = STAGES * kStage;
    static constexpr int kCycle = STAGES == 3 ? 24 : 8;       // steps after which stage, buffer and scale byte recur
    static_assert(LPW * kWaves == kGroups && TM % 16 == 0 && TN % 16 == 0, "even split");
    static_assert(BM / 16 % kWaves == 0 && BN / 16 % kWaves == 0, "a wave's i-th loads are all of A or all of B");
    static_assert(STAGES == 3 || STAGES == 4, "ring");
};
using MxLarge = MxCfg<256, 256, 4, 2, 3>;   // 8 waves of 64 x 128, 96 KB: one block per CU
using MxDuo = MxCfg<256, 128, 4, 1, 3>;     // 4 waves of 64 x 128, 72 KB: two
using MxMid = MxCfg<128, 128, 2, 2, 3>;     // 4 waves of 64 x 64, 48 KB: three
using MxSmall = MxCfg<64, 64, 2, 2, 4>;     // 4 waves of 32 x 32, 32 KB: five

[[maybe_unused]] constexpr int64_t kXcds = 8, kGroupM = 8;

// Work item b of n, the items of an XCD (blocks go to them round-robin) contiguous.
[[maybe_unused]] __device__ __forceinline__ int64_t xcd_item(int64_t b, int64_t n) {
    const int64_t x = b % kXcds, i = b / kXcds, q = n / kXcds, r = n % kXcds;
    return x * q + min(x, r) + i;
}

__device__ __forceinline__ void store_out(void* C, int type, int64_t at, float v) {
    if (type == SQ_TYPE_F32) static_cast<float*>(C)[at] = v;
    else static_cast<uint16_t*>(C)[at] = (uint16_t)bf16_bits(v);
}

// f(0), f(1), ... f(N - 1) as compile-time constants, until one returns false.
template <int N, int I = 0, class F>
__device__ __forceinline__ void unrolled_steps(F f) {
    if constexpr (I < N) {
        if (f(std::integral_constant<int, I>())) unrolled_steps<N, I + 1>(f);
    }
}

template <class T, int MODE>
__global__ __launch_bounds__(T::kThreads, 2) void k_mx_gemm(MxGemmArgs p, int64_t tiles_m, int64_t tiles_n, int splits,
                                                            int64_t per_split) {
#if defined(__HIP_DEVICE_COMPILE__)   // buffer resources exist in the device pass only
    __shared__ __attribute__((aligned(1024))) uint8_t smem[T::kSmem];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / T::WN, wn = wave % T::WN;

    // ---- which product, which tile, which tiles of the inner axis ----
    int64_t item = xcd_item(blockIdx.x, gridDim.x), split = 0, expert = 0;
    int64_t m0, n0, row_end = p.M, t0 = 0, n_tiles = (p.K + kMxTile - 1) / kMxTile;
    if constexpr (MODE == kExpertRows) {
        const int64_t tm = item / tiles_n;
        n0 = (item - tm * tiles_n) * T::BN;
        const Segment g = find_segment(p.offsets, p.experts, (int)p.M, T::BM, (int)tm);
        if (g.expert < 0) return;
        expert = g.expert;
        m0 = (int64_t)g.lo + (int64_t)g.tile * T::BM;
        row_end = g.hi;
    } else {
        const int64_t nt = tiles_m * tiles_n, outer = item / nt, w = item - outer * nt;
        if constexpr (MODE == kExpertInner) {
            expert = outer;
            int64_t inner;
            int len;
            segment_inner(p.offsets, p.experts, (int)p.rows, (int)expert, inner, len);
            t0 = inner / kMxTile;
            n_tiles = max((int64_t)0, min(((int64_t)len + kMxTile - 1) / kMxTile, p.K / kMxTile - t0));
        } else {
            split = outer;
            t0 = split * per_split;
            n_tiles = max((int64_t)0, min(per_split, n_tiles - t0));
        }
        const int64_t per_group = kGroupM * tiles_n, first = (w / per_group) * kGroupM;
        const int64_t gsz = min(tiles_m - first, kGroupM), u = w % per_group;
        m0 = (first + u % gsz) * T::BM;
        n0 = (u / gsz) * T::BN;
    }

    // ---- operand loads: a fixed offset per lane, the group and the inner axis in a scalar ----
    // Group g of a stage: rows 16 g.. of A (g < BM / 16), then of B; groups
    // past the last one read it again, their results are never stored.  A's
    // rows may start inside a 16-row group (kExpertRows): then the lanes of its
    // later rows read one group further.
    const int64_t units = mx_units(p.K), gbytes = units * kMxUnitBytes, sbytes = units * kMxUnitScales;
    const int64_t bm = MODE == kExpertRows ? expert * mx_groups(p.N) : 0;
    auto rsrc = [](const uint8_t* base, int64_t bytes) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), (short)0,
                                                 (int)min(bytes, (int64_t)0x7FFFFFFF), 0x00020000);
    };
    const int last_a = (int)(mx_groups(p.M) - 1 - (m0 >> 4)), last_b = (int)(mx_groups(p.N) - 1 - (n0 >> 4));
    const __amdgpu_buffer_rsrc_t rA = rsrc(p.A + (m0 >> 4) * gbytes, (last_a + 1) * gbytes),
                                 rB = rsrc(p.B + (bm + (n0 >> 4)) * gbytes, (last_b + 1) * gbytes),
                                 rAs = rsrc(p.As + (m0 >> 4) * sbytes, (last_a + 1) * sbytes),
                                 rBs = rsrc(p.Bs + (bm + (n0 >> 4)) * sbytes, (last_b + 1) * sbytes);
    const uint32_t gb = (uint32_t)gbytes, gs = (uint32_t)sbytes;
    const uint32_t slot = MODE == kExpertRows ? (uint32_t)(m0 + lane) & 15u : (uint32_t)lane & 15u;
    const bool next = MODE == kExpertRows && ((uint32_t)m0 & 15u) + ((uint32_t)lane & 15u) >= 16u;
    // Tiles past the last one read it again (never multiplied), so that every
    // step issues the same loads and the waits below are fixed counts.
    const int n = (int)n_tiles;
    auto issue = [&](int t, int stage) {
        const int k = ((int)t0 + min(t, n - 1)) * kMxTileBytes;
#pragma unroll
        for (int i = 0; i < T::LPW; ++i) {
            const int g = i * T::kWaves + wave;
            const bool isa = i * T::kWaves < T::BM / 16;
            const int last = isa ? last_a : last_b, grp = min(isa ? g : g - T::BM / 16, last);
            uint32_t off = 16u * (uint32_t)lane;
            if (MODE == kExpertRows && isa)
                off = ((uint32_t)lane >> 4) * 256u + slot * 16u + (next && grp < last ? gb : 0u);
            const int soff = (int)((uint32_t)grp * gb) + k;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(isa ? rA : rB, (lds_void_t*)(smem + stage * T::kStage + g * kMxTileBytes),
                                                     16, off, soff, 0, 0);
        }
    };

    v4f acc[T::FM][T::FN];
#pragma unroll
    for (int i = 0; i < T::FM; ++i)
#pragma unroll
        for (int j = 0; j < T::FN; ++j) acc[i][j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    // Operands of a stage in registers, two buffers: stage t + 1 is read while
    // stage t is multiplied.  The scales of four tiles, one word a fragment,
    // come straight from memory, two buffers too.
    v4i fa[2][T::FM], fb[2][T::FN];
    int sa[2][T::FM], sb[2][T::FN];
    auto load_scales = [&](int unit, auto BUF) {
        constexpr int buf = decltype(BUF)::value;
        const int k = ((int)(t0 >> 2) + min(unit, (n - 1) >> 2)) * kMxUnitScales;
#pragma unroll
        for (int i = 0; i < T::FM; ++i) {
            const int grp = min(wm * T::FM + i, last_a);
            uint32_t off = 4u * (uint32_t)lane;
            if (MODE == kExpertRows)
                off = ((uint32_t)lane >> 4) * 64u + slot * 4u + (next && grp < last_a ? gs : 0u);
            sa[buf][i] = (int)__builtin_amdgcn_raw_buffer_load_b32(rAs, off, (int)((uint32_t)grp * gs) + k, 0);
        }
#pragma unroll
        for (int j = 0; j < T::FN; ++j)
            sb[buf][j] = (int)__builtin_amdgcn_raw_buffer_load_b32(rBs, 4u * (uint32_t)lane,
                                                                   (int)((uint32_t)min(wn * T::FN + j, last_b) * gs) + k, 0);
    };
    auto read_frags = [&](auto STG, auto BUF) {
        constexpr int stg = decltype(STG)::value, buf = decltype(BUF)::value;
        const uint8_t* st = smem + stg * T::kStage + 16 * lane;
#pragma unroll
        for (int i = 0; i < T::FM; ++i) fa[buf][i] = *reinterpret_cast<const v4i*>(st + (wm * T::FM + i) * kMxTileBytes);
#pragma unroll
        for (int j = 0; j < T::FN; ++j)
            fb[buf][j] = *reinterpret_cast<const v4i*>(st + (T::BM / 16 + wn * T::FN + j) * kMxTileBytes);
    };
    // Step t, of index S in the cycle: publish stage t + 1, refill stage t's
    // place (its operands were read in the step before), read stage t + 1's
    // operands, multiply stage t's.
    auto step = [&](int t, auto S) {
        constexpr int s = decltype(S)::value, nxt = (s + 1) % T::STAGES, buf = s & 1, grp = (s >> 2) & 1;
        wait_loads<(T::STAGES - 2) * T::LPW>();
        __builtin_amdgcn_s_barrier();
        if constexpr ((s & 3) == 0) load_scales((t >> 2) + 1, std::integral_constant<int, grp ^ 1>());
        issue(t + T::STAGES, s % T::STAGES);
        read_frags(std::integral_constant<int, nxt>(), std::integral_constant<int, buf ^ 1>());
#pragma unroll
        for (int j = 0; j < T::FN; ++j)
#pragma unroll
            for (int i = 0; i < T::FM; ++i)
                acc[i][j] = mfma4<(s & 3)>(fb[buf][j], fa[buf][i], acc[i][j], sb[grp][j], sa[grp][i]);
        constexpr int kReads = T::FM + T::FN, kMfma = T::FM * T::FN, kPer = kMfma / kReads > 0 ? kMfma / kReads : 1;
#pragma unroll
        for (int g = 0; g < kReads; ++g) {
            __builtin_amdgcn_sched_group_barrier(0x008, kPer, 0);   // MFMAs
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);      // one LDS read
        }
    };
    if (n > 0) {
        load_scales(0, std::integral_constant<int, 0>());
#pragma unroll
        for (int i = 0; i < T::STAGES; ++i) issue(i, i);
        wait_loads<(T::STAGES - 1) * T::LPW>();
        __builtin_amdgcn_s_barrier();
        read_frags(std::integral_constant<int, 0>(), std::integral_constant<int, 0>());
        for (int t = 0; t < n; t += T::kCycle)
            unrolled_steps<T::kCycle>([&](auto S) {
                constexpr int s = decltype(S)::value;
                if (t + s >= n) return false;
                step(t + s, S);
                return true;
            });
    }

    // ---- epilogue: 16 rows of a wave at a time through LDS, out in whole lines ----
    __builtin_amdgcn_s_waitcnt(0);
    __builtin_amdgcn_s_barrier();
    constexpr int kLd = T::TN + 4;
    static_assert(T::kWaves * 16 * kLd * 4 <= T::kSmem && 16 * (T::TN / 8) >= 64, "a fragment row per wave fits");
    float* tr = reinterpret_cast<float*>(smem) + wave * 16 * kLd;
    const int er = lane & 15, eq = lane >> 4;
    void* C = p.C;
    int64_t ldc = p.ldc, base = MODE == kExpertInner ? expert * p.M * p.ldc : 0;
    int type = p.type;
    if (MODE == kDense && splits > 1) {
        C = p.part;
        type = SQ_TYPE_F32;
        ldc = p.N;
        base = split * p.M * p.N;
    }
    const int esz = type == SQ_TYPE_F32 ? 4 : 2;
    const bool vec = (ldc * esz) % 16 == 0 && (reinterpret_cast<uintptr_t>(C) & 15) == 0 && (base * esz) % 16 == 0;
    const int64_t n_w = n0 + wn * T::TN;
#pragma unroll
    for (int i = 0; i < T::FM; ++i) {
        const int64_t m = m0 + wm * T::TM + i * 16;
#pragma unroll
        for (int j = 0; j < T::FN; ++j) *reinterpret_cast<v4f*>(tr + er * kLd + j * 16 + eq * 4) = acc[i][j];
        // lanes take 8 consecutive columns each (16 bytes of bf16, 32 of fp32)
        constexpr int kPer = T::TN / 8, kRows = 64 / kPer;
        const int q = lane % kPer, r0 = lane / kPer;
#pragma unroll
        for (int rr = 0; rr < 16; rr += kRows) {
            const int r = r0 + rr;
            const float* src = tr + r * kLd + 8 * q;
            const v4f a = *reinterpret_cast<const v4f*>(src), b = *reinterpret_cast<const v4f*>(src + 4);
            const int64_t row = m + r, col = n_w + 8 * q, at = base + row * ldc + col;
            if (row >= row_end || col >= p.N) continue;
            if (vec && col + 8 <= p.N) {
                if (type == SQ_TYPE_F32) {
                    *reinterpret_cast<v4f*>(static_cast<float*>(C) + at) = a;
                    *reinterpret_cast<v4f*>(static_cast<float*>(C) + at + 4) = b;
                } else {
                    *reinterpret_cast<uint4*>(static_cast<uint16_t*>(C) + at) =
                        make_uint4(bf16_pair(a.x, a.y), bf16_pair(a.z, a.w), bf16_pair(b.x, b.y), bf16_pair(b.z, b.w));
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (col + e < p.N) store_out(C, type, at + e, e < 4 ? a[e & 3] : b[e & 3]);
            }
        }
    }
#endif
}

// Sum of the split-K partials, in the order of the splits.
__global__ __launch_bounds__(256) void k_mx_reduce(const float* part, int splits, int64_t M, int64_t N, void* C, int type,
                                                   int64_t ldc) {
    const int64_t n = M * N;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        float s = 0.0f;
        for (int k = 0; k < splits; ++k) s += part[k * n + i];
        const int64_t r = i / N;
        store_out(C, type, r * ldc + (i - r * N), s);
    }
}

// ---------------------------------------------------------------------------
// Few rows: Y = X W^T.  Bound by the one read of W.  A block owns 16 rows
// (those of one expert) and 16 columns; its waves share the inner axis, tile
// w, w + 8, ...: each lane reads the 32 elements of X of its row and block,
// quantizes them in registers (mx_scale4, as the quantizer does) and
// multiplies them with 1 KB of W read straight into registers.  The waves'
// sums meet in LDS.
// ---------------------------------------------------------------------------
constexpr int kRowsWaves = 8;

template <typename T>
__global__ __launch_bounds__(64 * kRowsWaves) void k_mx_rows(MxRowsArgs p, int64_t tiles_n, bool vec) {
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ float sums[kRowsWaves][16][17];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t tm = blockIdx.x / tiles_n, n0 = (blockIdx.x - tm * tiles_n) * 16;
    int64_t m0 = tm * 16, row_end = p.M, expert = 0;
    if (p.offsets) {
        const Segment g = find_segment(p.offsets, p.experts, (int)p.M, 16, (int)tm);
        if (g.expert < 0) return;
        expert = g.expert;
        m0 = (int64_t)g.lo + (int64_t)g.tile * 16;
        row_end = g.hi;
    }
    const int64_t units = mx_units(p.K), group = expert * mx_groups(p.N) + (n0 >> 4);
    const uint8_t* W = p.W + group * units * kMxUnitBytes + lane * 16;
    const uint8_t* Ws = p.Ws + group * units * kMxUnitScales + lane * 4;
    const int64_t row = m0 + (lane & 15);
    const bool live = row < row_end;
    const T* x = static_cast<const T*>(p.x) + row * p.ld + (lane >> 4) * 32;
    const int64_t left = p.K - (lane >> 4) * 32;
    const int tiles = (int)((p.K + kMxTile - 1) / kMxTile);
    v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int t = wave; t < tiles; t += kRowsWaves) {
        const v4i w = *reinterpret_cast<const v4i*>(W + (int64_t)t * kMxTileBytes);
        const int ws = (int)(*reinterpret_cast<const uint32_t*>(Ws + (int64_t)(t >> 2) * kMxUnitScales) >> (8 * (t & 3)));
        T v[32];
        const int64_t k = (int64_t)t * kMxTile;
        if (live && vec && k + 32 <= left) {
#pragma unroll
            for (int i = 0; i < (int)(32 * sizeof(T) / 16); ++i)
                reinterpret_cast<uint4*>(v)[i] = reinterpret_cast<const uint4*>(x + k)[i];
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = live && k + i < left ? x[k + i] : (T)0;
        }
        float f[32];
        uint32_t b = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            if constexpr (sizeof(T) == 4) f[i] = v[i];
            else f[i] = bf16_value(v[i]);
            b = max(b, __float_as_uint(f[i]) & 0x7FFFFFFFu);
        }
        const uint32_t s = mx_scale4(b);
        const float inv = mx_inverse(s);
        v4i a;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t r = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) f[8 * i + e] = s == 255u ? 0.0f : f[8 * i + e] * inv;
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[8 * i], f[8 * i + 1], 1.0f, 0);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[8 * i + 2], f[8 * i + 3], 1.0f, 1);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[8 * i + 4], f[8 * i + 5], 1.0f, 2);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, f[8 * i + 6], f[8 * i + 7], 1.0f, 3);
            a[i] = (int)r;
        }
        acc = mfma4<0>(w, a, acc, ws, (int)s);
    }
    // a lane holds columns 4 (lane / 16).. of row lane % 16
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[wave][lane & 15][4 * (lane >> 4) + e] = acc[e];
    __syncthreads();
    if (tid >= 256) return;
    const int r = tid >> 4, c = tid & 15;
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kRowsWaves; ++w) s += sums[w][r][c];
    if (m0 + r < row_end && n0 + c < p.N) store_out(p.Y, p.out_type, (m0 + r) * p.ldy + n0 + c, s);
#endif
}

template <class T, int MODE>
hipError_t gemm(const MxGemmArgs& a, int splits, hipStream_t s) {
    const int64_t tiles_n = (a.N + T::BN - 1) / T::BN;
    const int64_t tiles_m = MODE == kExpertRows ? a.M / T::BM + std::min<int64_t>(a.experts, a.M) : (a.M + T::BM - 1) / T::BM;
    const int64_t outer = MODE == kExpertInner ? a.experts : splits;
    const int64_t tiles = (a.K + kMxTile - 1) / kMxTile;
    const int64_t per = round_up((tiles + splits - 1) / splits, 4);
    k_mx_gemm<T, MODE><<<(uint32_t)(tiles_m * tiles_n * outer), T::kThreads, 0, s>>>(a, tiles_m, tiles_n, splits, per);
    if (splits > 1) {
        const int64_t n = a.M * a.N;
        k_mx_reduce<<<(uint32_t)std::min<int64_t>((n + 255) / 256, 4096), 256, 0, s>>>(a.part, splits, a.M, a.N, a.C, a.type,
                                                                                      a.ldc);
    }
    return hipGetLastError();
}

template <int MODE>
hipError_t gemm_mode(const MxGemmArgs& a, hipStream_t s) {
    const int splits = (int)mx_gemm_splits(a);
    const double rows = MODE == kExpertRows ? (double)a.M / a.experts : (double)a.M;
    const double tiles = rows / 256.0 * ((double)a.N / 256.0) * (MODE == kDense ? 1.0 : (double)a.experts);
    if (!getenv("SQ_DUO") && rows > 128 && a.N > 128 && tiles >= 192) return gemm<MxLarge, MODE>(a, splits, s);
    if (rows > 128 && a.N > 128 && tiles >= 192) return gemm<MxDuo, MODE>(a, splits, s);
    if (rows > 64 && a.N > 64 && tiles >= 24) return gemm<MxMid, MODE>(a, splits, s);
    return gemm<MxSmall, MODE>(a, splits, s);
}

}  // namespace

int64_t mx_gemm_splits(const MxGemmArgs& a) {
    if (a.mode != kDense) return 1;
    const int64_t tiles = ((a.M + 63) / 64) * ((a.N + 63) / 64), k = (a.K + kMxTile - 1) / kMxTile;
    if (tiles >= 512 || k < 16) return 1;
    return std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(1024 / tiles, k / 8), 64));
}

hipError_t launch_mx_gemm(const MxGemmArgs& a, hipStream_t s) {
    if (a.M == 0 || a.N == 0) return hipSuccess;
    switch (a.mode) {
        case kDense: return gemm_mode<kDense>(a, s);
        case kExpertRows: return gemm_mode<kExpertRows>(a, s);
        default: return gemm_mode<kExpertInner>(a, s);
    }
}

bool mx_rows_ok(int64_t M, int64_t, int64_t, int64_t experts) {
    return M <= 16 * std::max<int64_t>(1, experts);
}

hipError_t launch_mx_rows(const MxRowsArgs& a, hipStream_t s) {
    if (a.M == 0 || a.N == 0) return hipSuccess;
    const int64_t tiles_n = (a.N + 15) / 16;
    const int64_t tiles_m = a.offsets ? a.M / 16 + std::min<int64_t>(a.experts, a.M) : (a.M + 15) / 16;
    const int64_t sz = a.type == SQ_TYPE_F32 ? 4 : 2;
    const bool vec = (reinterpret_cast<uintptr_t>(a.x) & 15) == 0 && (a.ld * sz) % 16 == 0;
    const dim3 grid((uint32_t)(tiles_m * tiles_n));
    if (a.type == SQ_TYPE_F32) k_mx_rows<float><<<grid, 64 * kRowsWaves, 0, s>>>(a, tiles_n, vec);
    else k_mx_rows<uint16_t><<<grid, 64 * kRowsWaves, 0, s>>>(a, tiles_n, vec);
    return hipGetLastError();
}

}  // namespace sq
