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
//
// What bounds the large products is power: the register-only loop of the
// instruction runs at 9.8 PFLOP/s on zeros and at 7.1 on random codes and scales,
// 7.2 with one operand of each instruction that of the one before, as the shader
// clock falls; and the same launch of this kernel is 20 to 28 % shorter on zeros.
// Back to back, on quantized normal values and on zeros: 8192 x 4096 x 44032 609
// and 500 us (4.85 and 5.9 PFLOP/s), 8192 x 4096 x 11008 172 and 124 (4.3 and 5.9),
// 8192 x 11008 x 4096 191 and 141 (3.9 and 5.2; a bf16 library product of this size
// takes 3.2 times as long).  With the clock that a launch happens to get the
// normal values' times spread by 167 to 197 and 183 to 216 us.
#include <algorithm>
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
// elements in LDS.  AHEAD: a stage's operands are read into registers while
// the one before is multiplied, which a wave of 64 x 128 outputs needs (two
// waves a SIMD); the smaller ones read and multiply in turn, with the registers
// for more blocks a CU instead.
template <int BM_, int BN_, int STAGES_, bool AHEAD_, int BLOCKS>
struct MxCfg {
    static constexpr int BM = BM_, BN = BN_, WM = 2, WN = 2, STAGES = STAGES_;
    static constexpr bool AHEAD = AHEAD_, kScalesInLds = BN >= 128;
    static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves, kOccupancy = BLOCKS * kWaves / 4;
    static constexpr int TM = BM / WM, TN = BN / WN, FM = TM / 16, FN = TN / 16;
    static constexpr int kGroups = (BM + BN) / 16;            // 16-row operand groups of a stage
    static constexpr int LPW = kGroups / kWaves;              // 1 KB loads per wave per stage
    static constexpr int kStage = kGroups * kMxTileBytes;
    static constexpr int kScales = kScalesInLds ? BN / 16 * kMxUnitScales : 0;   // of B, four tiles
    static constexpr int kSmem = STAGES * kStage + 2 * kScales;
    static constexpr int kCycle = STAGES == 3 ? 24 : 8;       // steps after which stage, buffer and scale byte recur
    static_assert(BM / 16 % kWaves == 0 && BN / 16 % kWaves == 0, "a wave's i-th loads are all of A or all of B");
    static_assert(STAGES >= 2 && STAGES <= 4 && BLOCKS * kSmem <= 160 * 1024, "ring");
};
using MxWide = MxCfg<128, 256, 3, true, 2>;    // waves of 64 x 128
using MxMid = MxCfg<128, 128, 3, false, 3>;    // waves of 64 x 64
using MxShort = MxCfg<128, 128, 2, false, 4>;  // the same, a block more a CU for a step less in flight
using MxSmall = MxCfg<64, 64, 4, true, 5>;     // waves of 32 x 32

__device__ __forceinline__ void store_out(void* C, int type, int64_t at, float v) {
    if (type == SQ_TYPE_F32) static_cast<float*>(C)[at] = v;
    else static_cast<uint16_t*>(C)[at] = (uint16_t)bf16_bits(v);
}

#if defined(__HIP_DEVICE_COMPILE__)   // buffer resources exist in the device pass only
__device__ __forceinline__ __amdgpu_buffer_rsrc_t mx_rsrc(const uint8_t* base, int64_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(base), (short)0, (int)min(bytes, (int64_t)0x7FFFFFFF),
                                             0x00020000);
}
constexpr uint32_t kXcds = 8, kGroupM = 8;

// Work item b of n, the items of an XCD (blocks go to them round-robin) contiguous.
__device__ __forceinline__ uint32_t xcd_item(uint32_t b, uint32_t n) {
    const uint32_t x = b % kXcds, i = b / kXcds, q = n / kXcds, r = n % kXcds;
    return x * q + min(x, r) + i;
}
#endif

// f(0), f(1), ... f(N - 1) as compile-time constants, until one returns false.
template <int N, int I = 0, class F>
__device__ __forceinline__ void unrolled_steps(F f) {
    if constexpr (I < N) {
        if (f(std::integral_constant<int, I>())) unrolled_steps<N, I + 1>(f);
    }
}

// A product, its tiles and K splits, and how many blocks it takes.
struct MxProduct {
    MxGemmArgs a;
    uint32_t tiles_m, tiles_n, blocks;
    int splits;
};

#if defined(__HIP_DEVICE_COMPILE__)   // buffer resources exist in the device pass only
template <class T, int MODE>
__device__ __forceinline__ void product(const MxProduct& d, uint32_t block, uint8_t* smem) {
    const MxGemmArgs& p = d.a;
    const uint32_t tiles_m = d.tiles_m, tiles_n = d.tiles_n;
    const int splits = d.splits;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / T::WN, wn = wave % T::WN;

    // ---- which product, which tile, which tiles of the inner axis ----
    int64_t expert = 0, split = 0;
    int64_t row_end = p.M, t0 = 0, n_tiles = (p.K + kMxTile - 1) / kMxTile;
    uint32_t item = 0;
    if constexpr (MODE == kDense) item = xcd_item(block, d.blocks);
    if constexpr (MODE == kExpertInner) {
        // Every expert over all the XCDs: with whole experts on each, the one with
        // most rows sets the time (gradients of 20000 rows, 8 uneven experts, 1200 x
        // 3000, 173 -> 150 us; 32768 rows, 16 rather even ones, 2048 x 4096, 411 -> 418).
        const uint32_t e = block / (tiles_m * tiles_n);
        item = xcd_item(block - e * tiles_m * tiles_n, tiles_m * tiles_n);
        expert = e;
        int64_t inner;
        int len;
        segment_inner(p.offsets, p.experts, (int)p.rows, (int)expert, inner, len);
        t0 = inner / kMxTile;
        n_tiles = max((int64_t)0, min(((int64_t)len + kMxTile - 1) / kMxTile, p.K / kMxTile - t0));
    }
    if (MODE == kDense && splits > 1) {     // whole units, for the scales' words
        const uint32_t sp = item / (tiles_m * tiles_n);
        item -= sp * tiles_m * tiles_n;
        split = sp;
        const int64_t per = ((n_tiles + splits - 1) / splits + 3) & ~(int64_t)3;
        t0 = min(split * per, n_tiles);
        n_tiles = min(per, n_tiles - t0);
    }
    // kGroupM tile rows at a time, so that an XCD's blocks share panels of B in its L2
    uint32_t un = 0;
    auto tile_row = [&](uint32_t it, uint32_t rows) {
        const uint32_t per_group = kGroupM * tiles_n, grp0 = it / per_group, first = grp0 * kGroupM;
        const uint32_t gsz = min(rows - first, kGroupM), u = it - grp0 * per_group;
        un = u / gsz;
        return first + u - un * gsz;
    };
    int64_t m0 = 0;
    if constexpr (MODE != kExpertRows) m0 = (int64_t)tile_row(item, tiles_m) * T::BM;
    if constexpr (MODE == kExpertRows) {
        // The grid has room for any split of the rows; the tiles that there are go
        // evenly over the XCDs (16384 rows, 64 experts, 2048 -> 1408: 53 -> 47 us).
        const Segment g = find_segment_of(p.offsets, p.experts, (int)p.M, T::BM, [&](int rows) {
            const uint32_t n = (uint32_t)rows * tiles_n;
            return rows > 0 && block < n ? (int)tile_row(xcd_item(block, n), (uint32_t)rows) : -1;
        });
        if (g.expert < 0) return;
        expert = g.expert;
        m0 = (int64_t)g.lo + (int64_t)g.tile * T::BM;
        row_end = g.hi;
    }
    const int64_t n0 = (int64_t)un * T::BN;

    // ---- operand loads: a fixed offset per lane, the group and the inner axis in a scalar ----
    // Group g of a stage: rows 16 g.. of A (g < BM / 16), then of B; groups
    // past the last one read it again, their results are never stored.  A's
    // rows may start inside a 16-row group (kExpertRows): then the lanes of its
    // later rows read one group further.
    const int64_t units = mx_units(p.K), gbytes = units * kMxUnitBytes, sbytes = units * kMxUnitScales;
    const int64_t bm = MODE == kExpertRows ? expert * mx_groups(p.N) : 0;
    const int last_a = (int)(mx_groups(p.M) - 1 - (m0 >> 4)), last_b = (int)(mx_groups(p.N) - 1 - (n0 >> 4));
    const __amdgpu_buffer_rsrc_t rA = mx_rsrc(p.A + (m0 >> 4) * gbytes, (last_a + 1) * gbytes),
                                 rB = mx_rsrc(p.B + (bm + (n0 >> 4)) * gbytes, (last_b + 1) * gbytes),
                                 rAs = mx_rsrc(p.As + (m0 >> 4) * sbytes, (last_a + 1) * sbytes),
                                 rBs = mx_rsrc(p.Bs + (bm + (n0 >> 4)) * sbytes, (last_b + 1) * sbytes);
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
    // Operands of a stage in registers (AHEAD: two buffers).  The scales of
    // four tiles, one word a fragment: A's straight from memory, two buffers; B's
    // through LDS where the tile is wide, 1 KB a load (with a load a fragment the
    // 32768-row product by expert of 4096 -> 2048 took 156 us, now 147).
    constexpr int kBufs = T::AHEAD ? 2 : 1;
    v4i fa[kBufs][T::FM], fb[kBufs][T::FN];
    int sa[2][T::FM], sb[T::kScalesInLds ? 1 : 2][T::FN];
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
            if constexpr (!T::kScalesInLds)
                sb[buf][j] = (int)__builtin_amdgcn_raw_buffer_load_b32(rBs, 4u * (uint32_t)lane,
                                                                       (int)((uint32_t)min(wn * T::FN + j, last_b) * gs) + k, 0);
        // B's, 1 KB of four groups at a time, to LDS
        if constexpr (T::kScalesInLds) {
            constexpr int kLoads = T::BN / 64;
#pragma unroll
            for (int q = 0; q < (kLoads + T::kWaves - 1) / T::kWaves; ++q) {
                const int at = q * T::kWaves + wave;
                if (kLoads % T::kWaves == 0 || at < kLoads)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(
                        rBs, (lds_void_t*)(smem + T::STAGES * T::kStage + (unit & 1) * T::kScales + at * 1024), 16,
                        (uint32_t)min(4 * at + (lane >> 4), last_b) * gs + 16u * ((uint32_t)lane & 15u), k, 0, 0);
            }
        }
    };
    auto read_scales = [&](int unit) {
        const uint8_t* ss = smem + T::STAGES * T::kStage + (unit & 1) * T::kScales + wn * T::FN * kMxUnitScales + 4 * lane;
#pragma unroll
        for (int j = 0; j < T::FN; ++j)
            if constexpr (T::kScalesInLds) sb[0][j] = *reinterpret_cast<const int*>(ss + j * kMxUnitScales);
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
    // Up and down the rows of fragments: never do both operands change, which takes
    // less power (large products 0.5 to 2.5 % faster).
    auto multiply = [&](auto S, auto BUF) {
        constexpr int s = decltype(S)::value, buf = decltype(BUF)::value, grp = (s >> 2) & 1;
#pragma unroll
        for (int j = 0; j < T::FN; ++j)
#pragma unroll
            for (int q = 0; q < T::FM; ++q) {
                const int i = j & 1 ? T::FM - 1 - q : q;
                acc[i][j] = mfma4<(s & 3)>(fb[buf][j], fa[buf][i], acc[i][j], sb[T::kScalesInLds ? 0 : grp][j], sa[grp][i]);
            }
    };
    // Step t, of index S in the cycle.
    auto step = [&](int t, auto S) {
        constexpr int s = decltype(S)::value, grp = (s >> 2) & 1, buf = s & 1;
        wait_loads<(T::STAGES - 2) * T::LPW>();
        __builtin_amdgcn_s_barrier();
        if constexpr ((s & 3) == 0) {
            read_scales(t >> 2);
            load_scales((t >> 2) + 1, std::integral_constant<int, grp ^ 1>());
        }
        if constexpr (T::AHEAD) {
            // stage t + 1 is there; refill stage t's place (its operands were
            // read in the step before), read stage t + 1's operands, multiply stage t's
            issue(t + T::STAGES, s % T::STAGES);
            read_frags(std::integral_constant<int, (s + 1) % T::STAGES>(), std::integral_constant<int, buf ^ 1>());
            multiply(S, std::integral_constant<int, buf>());
            constexpr int kReads = T::FM + T::FN, kMfma = T::FM * T::FN, kPer = kMfma / kReads > 0 ? kMfma / kReads : 1;
#pragma unroll
            for (int g = 0; g < kReads; ++g) {
                __builtin_amdgcn_sched_group_barrier(0x008, kPer, 0);   // MFMAs
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);      // one LDS read
            }
        } else {
            // stage t is there; read its operands, refill the place of stage t - 1, multiply
            read_frags(std::integral_constant<int, s % T::STAGES>(), std::integral_constant<int, 0>());
            issue(t + T::STAGES - 1, (s + T::STAGES - 1) % T::STAGES);
            multiply(S, std::integral_constant<int, 0>());
        }
    };
    if (n > 0) {
        load_scales(0, std::integral_constant<int, 0>());
        constexpr int kFirst = T::AHEAD ? T::STAGES : T::STAGES - 1;
#pragma unroll
        for (int i = 0; i < kFirst; ++i) issue(i, i);
        if constexpr (T::AHEAD) {
            wait_loads<(T::STAGES - 1) * T::LPW>();
            __builtin_amdgcn_s_barrier();
            read_frags(std::integral_constant<int, 0>(), std::integral_constant<int, 0>());
        }
        for (int t = 0; t < n; t += T::kCycle)
            unrolled_steps<T::kCycle>([&](auto S) {
                constexpr int s = decltype(S)::value;
                if (t + s >= n) return false;
                step(t + s, S);
                return true;
            });
    }

    // ---- epilogue: 16 rows of a wave at a time through LDS, out in whole lines ----
    // Nontemporal where rows are whole lines of 128 bytes: the lines of C that
    // ordinary stores leave in the last-level cache evict dirty ones.  Weight
    // gradients of 16 experts, 32768 rows, 4096 x 2048: 258 -> 188 us; 32768 x 4096
    // outputs in bf16 and the quantizer that reads them next, together 268 -> 254
    // us; 3152 x 768 in fp32, 17.1 -> 15.8.  Other rows share lines with the next
    // tile's, which the caches have to join: 12748 x 1369 in bf16 14.8 us against
    // 19.5 nontemporal, 113 experts of 2018 x 79 in fp32 21 against 41.
    __builtin_amdgcn_s_waitcnt(0);
    __builtin_amdgcn_s_barrier();
    constexpr int kLd = T::TN + 4;
    static_assert(T::kWaves * 16 * kLd * 4 <= T::kSmem && T::TN >= 32, "a fragment row per wave fits");
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
    const int64_t n_w = n0 + wn * T::TN;
    const bool lines = (((uint64_t)C | (uint64_t)((base | ldc) * (type == SQ_TYPE_F32 ? 4 : 2))) & 127) == 0;
#pragma unroll
    for (int i = 0; i < T::FM; ++i) {
        const int64_t m = m0 + wm * T::TM + i * 16;
#pragma unroll
        for (int j = 0; j < T::FN; ++j) *reinterpret_cast<v4f*>(tr + er * kLd + j * 16 + eq * 4) = acc[i][j];
        // 16 bytes a lane, whole lines: 8 columns of bf16, 4 of fp32
        auto rows_out = [&](auto F32, auto LINES) {
            constexpr bool f32 = decltype(F32)::value, lines = decltype(LINES)::value;
            // keeps the compiler from joining the two kinds of store, which loses the hint
            if constexpr (lines) asm volatile("; whole lines");
            constexpr int kCols = f32 ? 4 : 8, kPer = T::TN / kCols, kRows = 64 / kPer;
            const int q = lane % kPer, r0 = lane / kPer;
#pragma unroll
            for (int rr = 0; rr < 16; rr += kRows) {
                const int r = r0 + rr;
                const float* src = tr + r * kLd + kCols * q;
                const v4f a = *reinterpret_cast<const v4f*>(src);
                v4f b = a;
                if constexpr (!f32) b = *reinterpret_cast<const v4f*>(src + 4);
                const int64_t row = m + r, col = n_w + kCols * q, at = base + row * ldc + col;
                if (row >= row_end || col >= p.N) continue;
                if (col + kCols <= p.N) {
                    if constexpr (f32) {
                        f32x4_any* to = reinterpret_cast<f32x4_any*>(static_cast<float*>(C) + at);
                        if constexpr (lines) __builtin_nontemporal_store((f32x4_any)a, to);
                        else *to = (f32x4_any)a;
                    } else {
                        const u32x4_any w = {bf16_pair(a.x, a.y), bf16_pair(a.z, a.w), bf16_pair(b.x, b.y), bf16_pair(b.z, b.w)};
                        u32x4_any* to = reinterpret_cast<u32x4_any*>(static_cast<uint16_t*>(C) + at);
                        if constexpr (lines) __builtin_nontemporal_store(w, to);
                        else *to = w;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < kCols; ++e)
                        if (col + e < p.N) store_out(C, type, at + e, e < 4 ? a[e & 3] : b[e & 3]);
                }
            }
            if constexpr (lines) asm volatile("; whole lines");
        };
        if (type == SQ_TYPE_F32) {
            if (lines) rows_out(std::true_type(), std::true_type());
            else rows_out(std::true_type(), std::false_type());
        } else {
            if (lines) rows_out(std::false_type(), std::true_type());
            else rows_out(std::false_type(), std::false_type());
        }
    }
}
#endif

template <class T, int MODE>
__global__ __launch_bounds__(T::kThreads, T::kOccupancy) void k_mx_gemm(MxProduct d) {
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ __attribute__((aligned(1024))) uint8_t smem[T::kSmem];
    product<T, MODE>(d, blockIdx.x, smem);
#endif
}

// Two products that do not depend on each other, in one launch: a layer's
// input and weight gradients.  Dense, one after the other (alternating blocks
// share less of the L2: the step of 8192 x 4096 x 11008 622 -> 680 us).  By
// expert their blocks alternate, eight of one at a time (one for each XCD), in
// proportion: a weight gradient over few rows is bound by its stores, which go
// along with the products of the other (32768 rows, 16 experts, 785 -> 756).
template <class T, int MODE_A, int MODE_B>
__global__ __launch_bounds__(T::kThreads, T::kOccupancy) void k_mx_gemm_pair(MxProduct a, MxProduct b) {
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ __attribute__((aligned(1024))) uint8_t smem[T::kSmem];
    const uint32_t na = (a.blocks + kXcds - 1) / kXcds, nb = (b.blocks + kXcds - 1) / kXcds;
    const uint32_t c = blockIdx.x / kXcds, lane = blockIdx.x % kXcds;
    uint32_t of_a = min(c, na);                 // eights of a before this one
    bool is_a = c < na;
    if constexpr (MODE_B == kExpertInner) {
        of_a = (uint32_t)((uint64_t)c * na / (na + nb));
        is_a = (uint32_t)((uint64_t)(c + 1) * na / (na + nb)) > of_a;
    }
    const uint32_t i = (is_a ? of_a : c - of_a) * kXcds + lane;
    if (is_a) {
        if (i < a.blocks) product<T, MODE_A>(a, i, smem);
    } else {
        if (i < b.blocks) product<T, MODE_B>(b, i, smem);
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
// Few rows of values: Y = X W^T, bound by the one read of W.  The operand
// layout is the matrix instruction's, so a wave loads 16 x 128 tiles of W
// straight into registers, 1 KB at a time.  A block owns 16 rows (of one
// expert) and 16 FN columns; its eight waves share the inner axis in contiguous
// parts, U tiles in flight each.  A lane reads the 32 elements of X of its row
// and block and quantizes them in registers.  The waves' sums meet in LDS in a
// fixed order.  One row, 4096 -> 4096: 4.5 us, 1.8 of them the launch (8.9 MB); 64
// rows on 64 experts, 2048 -> 1024: 12 us, 71 MB at 5.9 TB/s.
// ---------------------------------------------------------------------------
constexpr int kRowsWaves = 8;

#if defined(__HIP_DEVICE_COMPILE__)
// 32 bf16 from an address that may be an odd multiple of two bytes: 16-byte loads
// from such ones are split (16 x 1741 -> 1024, one launch, 7.9 us, now 5.2), so the
// words around them are loaded and shifted.  Every word holds an element asked for.
__device__ __forceinline__ void load_halves(const uint16_t* src, uint32_t* w) {
    typedef uint32_t u32x4_word __attribute__((ext_vector_type(4), aligned(4)));
    const uint32_t odd = (uint32_t)(uintptr_t)src & 2u;
    const uint32_t* at = reinterpret_cast<const uint32_t*>(src - odd / 2);
    uint32_t t[17];
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
        const u32x4_word l = *reinterpret_cast<const u32x4_word*>(at + i);
        t[i] = l.x;
        t[i + 1] = l.y;
        t[i + 2] = l.z;
        t[i + 3] = l.w;
    }
    t[16] = at[odd ? 16 : 15];
#pragma unroll
    for (int i = 0; i < 16; ++i) w[i] = __builtin_amdgcn_alignbit(t[i + 1], t[i], 8u * odd);
}
#endif

// Codes and scale of 32 values in the words w (bf16 pairs, or fp32).
template <bool BF16>
__device__ __forceinline__ v4i quantize_lane(const uint32_t* w, int& scale_byte) {
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    typedef uint16_t v2u16 __attribute__((ext_vector_type(2)));
    uint32_t b = 0;
    if constexpr (BF16) {
        v2u16 m = {0, 0};
#pragma unroll
        for (int i = 0; i < 16; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(v2u16, w[i] & 0x7FFF7FFFu));
        b = (uint32_t)max(m.x, m.y) << 16;
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) b = max(b, w[i] & 0x7FFFFFFFu);
    }
    const uint32_t s = mx_scale4(b);
    const float scale = mx_value(s);
    v4i a;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t r = 0;
        if constexpr (BF16) {
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(v2bf, w[4 * i]), scale, 0);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(v2bf, w[4 * i + 1]), scale, 1);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(v2bf, w[4 * i + 2]), scale, 2);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(r, __builtin_bit_cast(v2bf, w[4 * i + 3]), scale, 3);
        } else {
#define SQ_F(k) __uint_as_float(w[8 * i + k])
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, SQ_F(0), SQ_F(1), scale, 0);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, SQ_F(2), SQ_F(3), scale, 1);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, SQ_F(4), SQ_F(5), scale, 2);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, SQ_F(6), SQ_F(7), scale, 3);
#undef SQ_F
        }
        a[i] = (int)(s == 255u ? 0u : r);
    }
    scale_byte = (int)s;
    return a;
}

template <typename T, int FN, int U>
__global__ __launch_bounds__(64 * kRowsWaves, 4) void k_mx_rows(MxRowsArgs p, uint32_t tiles_n) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int kLd = 16 * FN + 4, kWords = 32 * sizeof(T) / 4, kV = 16 / sizeof(T);
    __shared__ float sums[kRowsWaves * 16 * kLd];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t tm = blockIdx.x / tiles_n;
    const int64_t n0 = (int64_t)(blockIdx.x - tm * tiles_n) * (16 * FN);
    int64_t m0 = (int64_t)tm * 16, row_end = p.M, expert = 0;
    if (p.offsets) {
        const Segment g = find_segment(p.offsets, p.experts, (int)p.M, 16, (int)tm);
        if (g.expert < 0) return;
        expert = g.expert;
        m0 = (int64_t)g.lo + (int64_t)g.tile * 16;
        row_end = g.hi;
    }
    const int K = (int)p.K, n = (K + kMxTile - 1) / kMxTile, part = (n + kRowsWaves - 1) / kRowsWaves;
    const int beg = min(wave * part, n), end = min(beg + part, n);
    const int64_t units = mx_units(K), first = expert * mx_groups(p.N) + (n0 >> 4);
    const int last = (int)(mx_groups(p.N) - 1 - (n0 >> 4));
    const uint32_t gb = (uint32_t)(units * kMxUnitBytes), gs = (uint32_t)(units * kMxUnitScales);
    const __amdgpu_buffer_rsrc_t rW = mx_rsrc(p.W + first * gb, (int64_t)(last + 1) * gb),
                                 rWs = mx_rsrc(p.Ws + first * gs, (int64_t)(last + 1) * gs);
    // rows past the end read the last one; their results are never stored
    const T* x = static_cast<const T*>(p.x) + min(m0 + (lane & 15), row_end - 1) * p.ld;
    const bool halves = sizeof(T) == 2 && (((uint64_t)p.x | (uint64_t)p.ld * sizeof(T)) & 2) != 0;
    v4f acc[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    auto load_w = [&](int at, int j, v4i& w, int& ws) {
        const uint32_t grp = (uint32_t)min(j, last);
        w = __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(rW, 16u * (uint32_t)lane,
                                                                          (int)(grp * gb) + at * kMxTileBytes, 0));
        ws = (int)__builtin_amdgcn_raw_buffer_load_b32(rWs, 4u * (uint32_t)lane, (int)(grp * gs) + (at >> 2) * kMxUnitScales, 0);
    };
    const int full = K / kMxTile, stop = min(end, full);    // whole tiles
    for (int t = beg; t < stop; t += U) {
        v4i w[U][FN];
        int ws[U][FN];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < FN; ++j) load_w(min(t + u, stop - 1), j, w[u][j], ws[u][j]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = min(t + u, stop - 1);
            uint32_t v[kWords];
            const T* from = x + at * kMxTile + (lane >> 4) * 32;
            bool done = false;
            if constexpr (sizeof(T) == 2) {
                if (halves) load_halves(from, v);
                done = halves;
            }
            if (!done) {
#pragma unroll
                for (int q = 0; q < 32 / kV; ++q) {
                    const u32x4_any l = *reinterpret_cast<const u32x4_any*>(from + q * kV);
                    v[4 * q] = l.x;
                    v[4 * q + 1] = l.y;
                    v[4 * q + 2] = l.z;
                    v[4 * q + 3] = l.w;
                }
            }
            int sa;
            v4i a = quantize_lane<sizeof(T) == 2>(v, sa);
            if (t + u >= stop) a = v4i{0, 0, 0, 0}, sa = 0;     // read again to keep the loads free of branches
            const int byte = 8 * (at & 3);
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[j] = mfma4<0>(w[u][j], a, acc[j], ws[u][j] >> byte, sa);
        }
    }
    if (end > stop && end == n && beg < end) {      // the tile that K ends in, element by element
        const int c = full * kMxTile + (lane >> 4) * 32;
        uint32_t v[kWords];
#pragma unroll
        for (int q = 0; q < kWords; ++q) {
            if constexpr (sizeof(T) == 4) {
                const uint32_t e = __float_as_uint(x[min(c + q, K - 1)]);
                v[q] = c + q < K ? e : 0u;
            } else {
                const uint32_t lo = x[min(c + 2 * q, K - 1)], hi = x[min(c + 2 * q + 1, K - 1)];
                v[q] = (c + 2 * q < K ? lo : 0u) | (c + 2 * q + 1 < K ? hi << 16 : 0u);
            }
        }
        int sa;
        const v4i a = quantize_lane<sizeof(T) == 2>(v, sa);
        const int byte = 8 * (full & 3);
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            v4i w;
            int ws;
            load_w(full, j, w, ws);
            acc[j] = mfma4<0>(w, a, acc[j], ws >> byte, sa);
        }
    }
    // a lane holds columns 4 (lane / 16).. of row lane % 16
#pragma unroll
    for (int j = 0; j < FN; ++j)
        *reinterpret_cast<v4f*>(&sums[(wave * 16 + (lane & 15)) * kLd + 16 * j + 4 * (lane >> 4)]) = acc[j];
    __syncthreads();
    constexpr int kOut = 16 * 16 * FN / (64 * kRowsWaves) > 0 ? 16 * 16 * FN / (64 * kRowsWaves) : 1;   // a thread
    if (tid * kOut >= 16 * 16 * FN) return;
    const int r = tid * kOut / (16 * FN), c = tid * kOut % (16 * FN);
#pragma unroll
    for (int e = 0; e < kOut; ++e) {
        float s = sums[r * kLd + c + e];
#pragma unroll
        for (int w = 1; w < kRowsWaves; ++w) s += sums[(w * 16 + r) * kLd + c + e];
        if (m0 + r < row_end && n0 + c + e < p.N) store_out(p.Y, p.out_type, (m0 + r) * p.ldy + n0 + c + e, s);
    }
#endif
}

// Rows and columns of 128 x 128 tiles (of every expert) and the steps of 128
// inner elements of each.
struct MxExtent {
    int64_t rows, cols, steps;
};
MxExtent extent(const MxGemmArgs& a) {
    MxExtent x;
    x.rows = a.mode == kExpertRows ? a.M / 128 + std::min<int64_t>(a.experts, a.M) : (a.M + 127) / 128;
    if (a.mode == kExpertInner) x.rows *= a.experts;
    x.cols = (a.N + 127) / 128;
    x.steps = ((a.mode == kExpertInner ? a.rows / a.experts : a.K) + kMxTile - 1) / kMxTile;
    return x;
}

enum MxTileKind { kWide, kMid, kShort, kSmall };

// Tiles by the size of the product, each rule with the times in us of the
// kinds on either side of it.
//   Small below 240 tiles of 128 x 128: 768 x 768 x 3152 (36 tiles) small 6.1,
//     mid 10.0; 2048 x 2048 x 512 (256) small 6.8, mid 6.4.
//   Wide from 12 steps of 128 inner elements on, where its tiles waste little of
//     the columns and of the last round over the CUs: 8192 x 11008 x 4096 wide
//     186, mid 198; 4096 x 2048 x 4096 22.4 and 22.7; 3000 x 3000 x 3000 (288
//     tiles) 28.6 and 24.8; 16384 x 1536 x 768 (6 steps) 20.7 and 19.9.
//   Short up to 8 steps: 8192 x 8192 x 512 short 35.4, mid 37.1;
//     1024 x 8192 x 2048 (16 steps) 16.2 and 15.5.
MxTileKind tile_kind(const MxGemmArgs& a) {
    const MxExtent x = extent(a);
    if (x.rows * x.cols < 240) return kSmall;
    const int64_t tn = (a.N + 255) / 256, wide = x.rows * tn, rounds = (wide + 255) / 256;
    if (x.steps >= 12 && 20 * 256 * tn <= 21 * a.N && 100 * 256 * rounds <= 135 * wide) return kWide;
    return x.steps <= 8 ? kShort : kMid;
}

template <class T, int MODE>
MxProduct product_of(const MxGemmArgs& a, int splits) {
    MxProduct d{};
    d.a = a;
    d.splits = splits;
    d.tiles_n = (uint32_t)((a.N + T::BN - 1) / T::BN);
    d.tiles_m = (uint32_t)(MODE == kExpertRows ? a.M / T::BM + std::min<int64_t>(a.experts, a.M) : (a.M + T::BM - 1) / T::BM);
    d.blocks = d.tiles_m * d.tiles_n * (uint32_t)(MODE == kExpertInner ? a.experts : splits);
    return d;
}

hipError_t reduce(const MxGemmArgs& a, int splits, hipStream_t s) {
    const int64_t n = a.M * a.N;
    k_mx_reduce<<<(uint32_t)std::min<int64_t>((n + 255) / 256, 4096), 256, 0, s>>>(a.part, splits, a.M, a.N, a.C, a.type, a.ldc);
    return hipGetLastError();
}

template <class T, int MODE>
hipError_t gemm(const MxGemmArgs& a, hipStream_t s) {
    const int splits = (int)mx_gemm_splits(a);
    const MxProduct d = product_of<T, MODE>(a, splits);
    k_mx_gemm<T, MODE><<<d.blocks, T::kThreads, 0, s>>>(d);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess && splits > 1 ? reduce(a, splits, s) : e;
}

template <int MODE>
hipError_t gemm_mode(const MxGemmArgs& a, hipStream_t s) {
    switch (tile_kind(a)) {
        case kWide: return gemm<MxWide, MODE>(a, s);
        case kMid: return gemm<MxMid, MODE>(a, s);
        case kShort: return gemm<MxShort, MODE>(a, s);
        default: return gemm<MxSmall, MODE>(a, s);
    }
}

template <class T, int MODE_A, int MODE_B>
hipError_t pair(const MxGemmArgs& a, const MxGemmArgs& b, hipStream_t s) {
    const int splits_a = (int)mx_gemm_splits(a), splits_b = (int)mx_gemm_splits(b);
    const MxProduct da = product_of<T, MODE_A>(a, splits_a), db = product_of<T, MODE_B>(b, splits_b);
    k_mx_gemm_pair<T, MODE_A, MODE_B><<<(uint32_t)(round_up(da.blocks, 8) + round_up(db.blocks, 8)), T::kThreads, 0, s>>>(da, db);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && splits_a > 1) e = reduce(a, splits_a, s);
    return e == hipSuccess && splits_b > 1 ? reduce(b, splits_b, s) : e;
}

}  // namespace

// Few tiles of a long inner axis are split, in parts of at least 40 steps: 64 x
// 640 x 30000, 235 steps, 26.7 us unsplit and 13.3 in 5; 1024 x 1024 x 32768,
// 256 steps, 42.0 and 35.5 in 2; but 128 x 4096 x 8192, 64 steps, 10.4 and 12.6
// in 2, 768 x 768 x 3152, 25 steps, 8.9 and 12.6 (a second launch for the sums).
int64_t mx_gemm_splits(const MxGemmArgs& a) {
    if (a.mode != kDense) return 1;
    const int64_t tiles = ((a.M + 63) / 64) * ((a.N + 63) / 64), k = (a.K + kMxTile - 1) / kMxTile;
    return std::max<int64_t>(1, std::min<int64_t>(512 / std::max<int64_t>(tiles, 1), k / 40));
}

namespace {

template <typename T, int FN, int U>
hipError_t rows(const MxRowsArgs& a, int64_t tiles_m, hipStream_t s) {
    const int64_t tiles_n = (a.N + 16 * FN - 1) / (16 * FN);
    k_mx_rows<T, FN, U><<<(uint32_t)(tiles_m * tiles_n), 64 * kRowsWaves, 0, s>>>(a, (uint32_t)tiles_n);
    return hipGetLastError();
}

// 64 columns a block where blocks of 16 would be more than two a CU (one row,
// 4096 -> 11008, 688 of them: 7.5 us against 8.3; 64 experts, 64 rows, 2048 ->
// 1024: 12.4 against 16.3; one row, 4096 -> 4096, 256: 5.6 against 4.7).
// bf16 has two tiles in flight, fp32 one: 16 rows, 11008 -> 4096, 22.5 us and 24.2
// with two; 8200 -> 8197 21.4 and 24.2; one row, 4096 -> 4096, 4.5 and 4.6; 64 rows on
// 64 experts, 2048 -> 1024, 16.0 and 15.0.
template <typename T>
hipError_t rows_of(const MxRowsArgs& a, hipStream_t s) {
    const int64_t tiles_m = a.offsets ? a.M / 16 + std::min<int64_t>(a.experts, a.M) : (a.M + 15) / 16;
    constexpr int U = sizeof(T) == 4 ? 1 : 2;
    return tiles_m * ((a.N + 15) / 16) >= 512 ? rows<T, 4, U>(a, tiles_m, s) : rows<T, 1, U>(a, tiles_m, s);
}

}  // namespace

hipError_t launch_mx_gemm(const MxGemmArgs& a, hipStream_t s) {
    if (a.M == 0 || a.N == 0) return hipSuccess;
    switch (a.mode) {
        case kDense: return gemm_mode<kDense>(a, s);
        case kExpertRows: return gemm_mode<kExpertRows>(a, s);
        default: return gemm_mode<kExpertInner>(a, s);
    }
}

namespace {

// Whether a block of `few` in 128 x 128 tiles, 0.4 us a step, would take longer
// than both products together: 1.2 ns a tile and step, outputs at 5 TB/s.  In us,
// gradients in large tiles and in small ones: 16200 x 768 x 1408 82 and 50, 4000
// x 768 x 1024 28 and 17, 300 x 8192 x 1024 43 and 22 (few blocks that last); 32768 x
// 1408 x 2048 140 and 196, 6000 x 1500 x 1500 38 and 42, 1187 x 520 x 1000 on 12
// experts 17.0 and 19.7 (blocks that the rest covers).
bool outlasts(const MxGemmArgs& few, const MxGemmArgs& other) {
    const auto rest = [](const MxGemmArgs& a) {
        const MxExtent x = extent(a);
        const double bytes = (a.mode == kExpertInner ? (double)a.experts : 1.0) * (double)a.M * (double)a.N *
                             (a.type == SQ_TYPE_F32 ? 4.0 : 2.0);
        return 1.2e-3 * (double)(x.rows * x.cols * x.steps) + bytes / 5e6;
    };
    return 0.4 * (double)extent(few).steps / (double)mx_gemm_splits(few) > rest(few) + rest(other);
}

}  // namespace

hipError_t launch_mx_gemm_pair(const MxGemmArgs& a, const MxGemmArgs& b, hipStream_t s) {
    MxTileKind ka = tile_kind(a), kb = tile_kind(b);
    // A product of few tiles goes along in the other one's larger tiles, unless a
    // block of it would outlast the rest: then both take small tiles.
    if (ka == kSmall) ka = outlasts(a, b) ? (kb = kSmall) : kb;
    else if (kb == kSmall) kb = outlasts(b, a) ? (ka = kSmall) : ka;
    if (ka != kb || a.M == 0 || a.N == 0 || b.M == 0 || b.N == 0) {
        const hipError_t e = launch_mx_gemm(a, s);
        return e == hipSuccess ? launch_mx_gemm(b, s) : e;
    }
    if (a.mode == kDense) {     // the longer tiles first
        const MxGemmArgs &x = a.K >= b.K ? a : b, &y = a.K >= b.K ? b : a;
        switch (ka) {
            case kWide: return pair<MxWide, kDense, kDense>(x, y, s);
            case kMid: return pair<MxMid, kDense, kDense>(x, y, s);
            case kShort: return pair<MxShort, kDense, kDense>(x, y, s);
            default: return pair<MxSmall, kDense, kDense>(x, y, s);
        }
    }
    switch (ka) {
        case kWide: return pair<MxWide, kExpertRows, kExpertInner>(a, b, s);
        case kMid: return pair<MxMid, kExpertRows, kExpertInner>(a, b, s);
        case kShort: return pair<MxShort, kExpertRows, kExpertInner>(a, b, s);
        default: return pair<MxSmall, kExpertRows, kExpertInner>(a, b, s);
    }
}

// Few rows: at most 16 (an expert, on average), or so few blocks of 16 rows and
// columns that to quantize the rows in each of them costs less than a launch
// of its own: 64 x 4096 -> 4096 in bf16 8.9 us against 13.1 with the quantizer
// and the product, 1024 x 512 -> 512 5.5 against 6.9; 128 x 4096 -> 4096 13.5
// against 11.7, 4096 x 512 -> 512 16.3 against 8.4, 64 x 4096 -> 4096 in fp32
// 12.9 against 11.7.  Not where many blocks have a tile or less of the inner axis
// for each of their waves: 64 experts, 512 -> 4096, 512 rows 32 against 24; 2048 ->
// 4096, 64 rows 29 against 40.
bool mx_rows_ok(int64_t M, int64_t K, int64_t N, int64_t experts, int type) {
    const double tiles = experts ? (double)(M / 16 + std::min(experts, M)) : (double)((M + 15) / 16);
    const double blocks = tiles * (double)((N + 15) / 16), steps = (double)((K + 127) / 128);
    if (M <= 16 * std::max<int64_t>(1, experts)) return blocks <= 10000.0 || steps > kRowsWaves;
    return blocks * (steps + 6.0) * (type == SQ_TYPE_F32 ? 2.0 : 1.0) <= 40000.0;
}

hipError_t launch_mx_rows(const MxRowsArgs& a, hipStream_t s) {
    if (a.M == 0 || a.N == 0) return hipSuccess;
    return a.type == SQ_TYPE_F32 ? rows_of<float>(a, s) : rows_of<uint16_t>(a, s);
}

}  // namespace sq
