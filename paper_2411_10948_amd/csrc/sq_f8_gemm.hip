// Products of matrices in 8-bit floating point for gfx950,
//     C[i, j] = sum_k A(i, k) B(j, k).
//
// v_mfma_scale_f32_32x32x64_f8f6f4 takes 32 x 64 codes of either operand (32 bytes
// a lane) and one scale a lane and accumulates in fp32; the blocks' scales are powers
// of two, which the instruction applies.  The operands lie in memory as it takes
// them (sq_f8.h): half a tile is 1 KB, from memory to LDS and from LDS to registers
// in contiguous pieces.
//
// The instruction adds the products of 16 elements at the largest one's exponent and
// drops what lies more than 13 bits below (measured: 2^16 - 2^16 + p keeps p down to
// 2^3).  Sums of 4096 products of normal values are off by 1.5e-5 of their size so,
// 6.5e-5 where channels differ in size: nothing next to the 2^-9 of a result in
// bf16 (1024 x 4096 x 2048 is 1.6548e-3 off 64 bits, where one rounding of these is
// 1.6547e-3; 1.5 % of the values take their other neighbour), but too much for one in
// fp32.  Those (EXACT) take the codes' values in bf16, which holds code and scale
// together, and v_mfma_f32_32x32x16_bf16, whose sums keep 24 bits: 1e-8 to 1e-7, at
// 1.8 instead of 4.0 PFLOP/s (register loops on random codes).
// Large ones are bound by the matrix instructions, at what power leaves of the clock and
// where the waves keep these fed: 8192 x 11008 x 4096 with bf16 results (300 us, 2.5 PFLOP/s) has
// them busy for 73 % of the cycles at 1.9 GHz, on zeros for 72 % at 2.4 (218 us); with fp32
// results for 79 % at 1.8 and 78 % at 2.4 GHz (534 and 395 us).  A bf16 library product of 8192^3 runs
// at 1.25 PFLOP/s.  Small ones are bound by the launch and the first loads.
#include <algorithm>
#include <type_traits>

#include "sq_f8.h"

namespace sq {

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void lds_void_t;

#if defined(__HIP_DEVICE_COMPILE__)
constexpr int kE4m3 = 0;    // the instructions' code of E4M3 operands

__device__ __forceinline__ v8i join(v4i a, v4i b) { return v8i{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}; }

// c + a b^T over 64 or 128 inner elements; byte `S` of each lane's scale words.
template <int S>
__device__ __forceinline__ v16f mfma32(v8i a, v8i b, v16f c, int sa, int sb) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, kE4m3, kE4m3, S, sa, S, sb);
}
// bf16 values of 8 codes in two words
__device__ __forceinline__ v8bf values8(int lo, int hi, float scale) {
    const v2bf a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)lo, scale, true),
               c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((unsigned)hi, scale, true);
    return v8bf{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}
__device__ __forceinline__ v4f mfma16(v8i a, v8i b, v4f c, int sa, int sb) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, kE4m3, kE4m3, 0, sa, 0, sb);
}
#endif

// s_waitcnt vmcnt(n) lgkmcnt(0) (gfx9 encoding): at most n loads in flight, and
// every LDS read of this wave done, so that the stage it read may be refilled
// once all waves have passed the barrier that follows.
template <int N>
__device__ __forceinline__ void wait_loads() {
    __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | (0x7 << 4));
}

// Block tile BM x BN of WM x WN waves, a ring of STAGES stages of half a tile (64 inner
// elements) in LDS; operands are read into registers while those before them are
// multiplied.
template <int BM_, int BN_, int WM_, int WN_, int STAGES_, int BLOCKS>
struct F8Cfg {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_;
    static constexpr int kWaves = WM * WN, kThreads = 64 * kWaves, kOccupancy = BLOCKS * kWaves / 4;
    static constexpr int TM = BM / WM, TN = BN / WN, FM = TM / 32, FN = TN / 32;
    static constexpr int kGroups = (BM + BN) / 16;            // 16-row operand groups of a stage
    static constexpr int LPW = kGroups / kWaves;              // 1 KB loads per wave per stage
    static constexpr int kStage = kGroups * kF8HalfBytes;
    static constexpr int kCols = TN < 64 ? TN : 64;           // columns of the epilogue's pieces
    static constexpr int kLd = kCols + 4;
    static constexpr int kSmem = std::max(STAGES * kStage, kWaves * 32 * kLd * 4);
    static constexpr int kCycle = 8;                          // stages of a unit: scale bytes are part of the instruction
    static_assert(BM / 16 % kWaves == 0 && BN / 16 % kWaves == 0, "a wave's i-th loads are all of A or all of B");
    static_assert(STAGES >= 3 && BLOCKS * kSmem <= 160 * 1024, "ring");
};
using F8Wide = F8Cfg<128, 256, 2, 2, 3, 2>;     // waves of 64 x 128
using F8Mid = F8Cfg<128, 128, 2, 2, 4, 2>;      // waves of 64 x 64
using F8Small = F8Cfg<64, 64, 2, 2, 4, 4>;      // waves of 32 x 32

__device__ __forceinline__ void store_out(void* C, int type, int64_t at, float v) {
    if (type == SQ_TYPE_F32) static_cast<float*>(C)[at] = v;
    else static_cast<uint16_t*>(C)[at] = (uint16_t)bf16_bits(v);
}

#if defined(__HIP_DEVICE_COMPILE__)   // buffer resources exist in the device pass only
__device__ __forceinline__ __amdgpu_buffer_rsrc_t f8_rsrc(const uint8_t* base, int64_t bytes) {
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

constexpr int64_t kSplit = 20, kSplitExact = 16;

// A product, its tiles and K splits, and how many blocks it takes.
struct F8Product {
    F8GemmArgs a;
    uint32_t tiles_m, tiles_n, blocks;
    int splits;
};

#if defined(__HIP_DEVICE_COMPILE__)
template <class T, bool EXACT>
__device__ __forceinline__ void product(const F8Product& d, uint32_t block, uint8_t* smem) {
    const F8GemmArgs& p = d.a;
    const uint32_t tiles_m = d.tiles_m, tiles_n = d.tiles_n;
    const int splits = d.splits;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / T::WN, wn = wave % T::WN;

    // ---- which tile, which half tiles of the inner axis ----
    int64_t split = 0, t0 = 0, n_tiles = (p.K + kMxTile - 1) / kMxTile;
    uint32_t item = xcd_item(block, d.blocks);
    if (splits > 1) {       // whole units, for the scales' words
        const uint32_t sp = item / (tiles_m * tiles_n);
        item -= sp * tiles_m * tiles_n;
        split = sp;
        const int64_t per = ((n_tiles + splits - 1) / splits + 3) & ~(int64_t)3;
        t0 = min(split * per, n_tiles);
        n_tiles = min(per, n_tiles - t0);
    }
    // kGroupM tile rows at a time, so that an XCD's blocks share panels of B in its L2
    const uint32_t per_group = kGroupM * tiles_n, grp0 = item / per_group, first = grp0 * kGroupM;
    const uint32_t gsz = min(tiles_m - first, kGroupM), u = item - grp0 * per_group, un = u / gsz;
    const int64_t m0 = (int64_t)(first + u - un * gsz) * T::BM, n0 = (int64_t)un * T::BN;

    // ---- operand loads: a fixed offset per lane, the group and the inner axis in a scalar ----
    // Group g of a stage: rows 16 g.. of A (g < BM / 16), then of B; groups past the
    // last one read it again, their results are never stored.
    const int64_t units = mx_units(p.K), gbytes = units * kF8UnitBytes, sbytes = units * kF8UnitScales;
    const int last_a = (int)(mx_groups(p.M) - 1 - (m0 >> 4)), last_b = (int)(mx_groups(p.N) - 1 - (n0 >> 4));
    const __amdgpu_buffer_rsrc_t rA = f8_rsrc(p.A + (m0 >> 4) * gbytes, (last_a + 1) * gbytes),
                                 rB = f8_rsrc(p.B + (n0 >> 4) * gbytes, (last_b + 1) * gbytes),
                                 rAs = f8_rsrc(p.As + (m0 >> 4) * sbytes, (last_a + 1) * sbytes),
                                 rBs = f8_rsrc(p.Bs + (n0 >> 4) * sbytes, (last_b + 1) * sbytes);
    const uint32_t gb = (uint32_t)gbytes, gs = (uint32_t)sbytes;
    // Stages past the last one read it again (never multiplied), so that every
    // step issues the same loads and the waits below are fixed counts.
    const int n = 2 * (int)n_tiles;
    auto issue = [&](int t, int stage) {
        const int k = (2 * (int)t0 + min(t, n - 1)) * kF8HalfBytes;
#pragma unroll
        for (int i = 0; i < T::LPW; ++i) {
            const int g = i * T::kWaves + wave;
            const bool isa = i * T::kWaves < T::BM / 16;
            const int grp = min(isa ? g : g - T::BM / 16, isa ? last_a : last_b);
            __builtin_amdgcn_raw_ptr_buffer_load_lds(isa ? rA : rB, (lds_void_t*)(smem + stage * T::kStage + g * kF8HalfBytes), 16,
                                                     16u * (uint32_t)lane, (int)((uint32_t)grp * gb) + k, 0, 0);
        }
    };

    v16f acc[T::FM][T::FN];
#pragma unroll
    for (int i = 0; i < T::FM; ++i)
#pragma unroll
        for (int j = 0; j < T::FN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    // The scales of a unit, one word a lane's row, and those of the next one on their way.
    int sa[T::FM], sb[T::FN], na[T::FM], nb[T::FN];
    const uint32_t row16 = ((uint32_t)lane & 15u) * 4u;
    const int upper = (lane >> 4) & 1;      // which 16-row group of a fragment's two
    auto load_scales = [&](int unit) {
        const int k = ((int)(t0 >> 2) + min(unit, (n - 1) >> 3)) * kF8UnitScales;
#pragma unroll
        for (int i = 0; i < T::FM; ++i)
            na[i] = (int)__builtin_amdgcn_raw_buffer_load_b32(
                rAs, row16 + (uint32_t)min(wm * T::TM / 16 + 2 * i + upper, last_a) * gs, k, 0);
#pragma unroll
        for (int j = 0; j < T::FN; ++j)
            nb[j] = (int)__builtin_amdgcn_raw_buffer_load_b32(
                rBs, row16 + (uint32_t)min(wn * T::TN / 16 + 2 * j + upper, last_b) * gs, k, 0);
    };
    // lane l: row l % 32, 16-element pieces 2 (l / 32) and 2 (l / 32) + 1 of a half tile
    const uint32_t frag = (uint32_t)upper * kF8HalfBytes + ((uint32_t)lane >> 5) * 512u + ((uint32_t)lane & 15u) * 16u;
    auto next_unit = [&]() {
#pragma unroll
        for (int i = 0; i < T::FM; ++i) sa[i] = na[i];
#pragma unroll
        for (int j = 0; j < T::FN; ++j) sb[j] = nb[j];
    };
    auto piece_a = [&](int stg, int i, int piece) {
        return *reinterpret_cast<const v4i*>(smem + stg * T::kStage + frag + (wm * T::TM / 16 + 2 * i) * kF8HalfBytes + piece * 256);
    };
    auto piece_b = [&](int stg, int j, int piece) {
        return *reinterpret_cast<const v4i*>(smem + stg * T::kStage + frag + (T::BM / 16 + wn * T::TN / 16 + 2 * j) * kF8HalfBytes +
                                             piece * 256);
    };
    // Operands of the 8-bit instructions, a half tile of them, two buffers; up and down the
    // rows of fragments: never do both operands change, which takes less power.
    v8i fa[2][T::FM], fb[2][T::FN];
    auto read_stage = [&](int stg, auto BUF) {
        constexpr int buf = decltype(BUF)::value;
#pragma unroll
        for (int i = 0; i < T::FM; ++i) fa[buf][i] = join(piece_a(stg, i, 0), piece_a(stg, i, 1));
#pragma unroll
        for (int j = 0; j < T::FN; ++j) fb[buf][j] = join(piece_b(stg, j, 0), piece_b(stg, j, 1));
    };
    auto multiply_stage = [&](auto S, auto BUF) {
        constexpr int s = decltype(S)::value, buf = decltype(BUF)::value;
#pragma unroll
        for (int j = 0; j < T::FN; ++j)
#pragma unroll
            for (int q = 0; q < T::FM; ++q) {
                const int i = j & 1 ? T::FM - 1 - q : q;
                acc[i][j] = mfma32<(s >> 1)>(fb[buf][j], fa[buf][i], acc[i][j], sb[j], sa[i]);
            }
    };
    // And of the bf16 ones, 16 bytes a lane of a half tile, two buffers.  One fragment a wave: two
    // sums of its own, so that an instruction does not wait for the one before.
    constexpr bool TWO = EXACT && T::FM * T::FN == 1;
    v16f other;
#pragma unroll
    for (int e = 0; e < 16; ++e) other[e] = 0.0f;
    v4i pa[2][T::FM], pb[2][T::FN];
    float va[T::FM], vb[T::FN];     // the tile's scales
    auto read_piece = [&](int stg, auto PIECE) {
        constexpr int piece = decltype(PIECE)::value;
#pragma unroll
        for (int i = 0; i < T::FM; ++i) pa[piece][i] = piece_a(stg, i, piece);
#pragma unroll
        for (int j = 0; j < T::FN; ++j) pb[piece][j] = piece_b(stg, j, piece);
    };
    auto multiply_piece = [&](auto PIECE) {
        constexpr int buf = decltype(PIECE)::value;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            v8bf xa[T::FM];
#pragma unroll
            for (int i = 0; i < T::FM; ++i) xa[i] = values8(pa[buf][i][2 * h], pa[buf][i][2 * h + 1], va[i]);
#pragma unroll
            for (int j = 0; j < T::FN; ++j) {
                const v8bf xb = values8(pb[buf][j][2 * h], pb[buf][j][2 * h + 1], vb[j]);
#pragma unroll
                for (int q = 0; q < T::FM; ++q) {
                    const int i = j & 1 ? T::FM - 1 - q : q;
                    v16f& to = TWO && h ? other : acc[i][j];
                    to = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xb, xa[i], to, 0, 0, 0);
                }
            }
        }
    };
    // A whole stage's operands in registers ahead: step t, of index S in its unit and in place
    // `stg`, has stage t + 1 there; refills its own place (its operands were read in the step
    // before), reads stage t + 1's, multiplies its own.
    auto step_fast = [&](int t, int stg, auto S) {
        constexpr int s = decltype(S)::value, buf = s & 1;
        wait_loads<(T::STAGES - 2) * T::LPW>();
        __builtin_amdgcn_s_barrier();
        if constexpr (s == 0) {
            next_unit();
            load_scales((t >> 3) + 1);
        }
        issue(t + T::STAGES, stg);
        read_stage(stg + 1 == T::STAGES ? 0 : stg + 1, std::integral_constant<int, buf ^ 1>());
        multiply_stage(S, std::integral_constant<int, buf>());
        constexpr int kReads = 2 * (T::FM + T::FN), kMfma = T::FM * T::FN, kPer = (kReads + kMfma - 1) / kMfma;
#pragma unroll
        for (int g = 0; g < kMfma; ++g) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);          // an MFMA
            __builtin_amdgcn_sched_group_barrier(0x100, kPer, 0);       // LDS reads
        }
    };
    // In bf16 a stage's two pieces one by one, the first in registers: stage t + 1 is there;
    // refill the place of stage t - 1, read the second piece, multiply the first, read stage
    // t + 1's first, multiply the second.
    auto step_exact = [&](int t, int stg, auto S) {
        constexpr int s = decltype(S)::value;
        typedef std::integral_constant<int, 0> First;
        typedef std::integral_constant<int, 1> Second;
        wait_loads<(T::STAGES - 3) * T::LPW>();
        __builtin_amdgcn_s_barrier();
        if constexpr (s == 0) {
            next_unit();
            load_scales((t >> 3) + 1);
        }
        issue(t + T::STAGES - 1, stg == 0 ? T::STAGES - 1 : stg - 1);
        if constexpr ((s & 1) == 0) {
#pragma unroll
            for (int i = 0; i < T::FM; ++i) va[i] = mx_value((uint32_t)sa[i] >> (4 * s) & 255u);
#pragma unroll
            for (int j = 0; j < T::FN; ++j) vb[j] = mx_value((uint32_t)sb[j] >> (4 * s) & 255u);
        }
        read_piece(stg, Second());
        multiply_piece(First());
        read_piece(stg + 1 == T::STAGES ? 0 : stg + 1, First());
        multiply_piece(Second());
    };
    if (n > 0) {
        constexpr int kFirst = EXACT ? T::STAGES - 1 : T::STAGES;
        load_scales(0);
#pragma unroll
        for (int i = 0; i < kFirst; ++i) issue(i, i);
        wait_loads<(kFirst - 1) * T::LPW>();
        __builtin_amdgcn_s_barrier();
        typedef std::integral_constant<int, 0> First;
        if constexpr (EXACT) read_piece(0, First());
        else read_stage(0, First());
        int place = 0;
        for (int t = 0; t < n; t += T::kCycle)
            unrolled_steps<T::kCycle>([&](auto S) {
                constexpr int s = decltype(S)::value;
                if (t + s >= n) return false;
                const int stg = T::kCycle % T::STAGES == 0 ? s % T::STAGES : place;     // known where the ring fits a unit
                if constexpr (EXACT) step_exact(t + s, stg, S);
                else step_fast(t + s, stg, S);
                place = place + 1 == T::STAGES ? 0 : place + 1;
                return true;
            });
    }
    if constexpr (TWO) {
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[0][0][e] += other[e];
    }

    // ---- epilogue: kCols columns of a wave's 32 rows at a time through LDS, out in whole lines ----
    // Nontemporal where rows are whole lines of 128 bytes: ordinary stores leave the
    // lines of C in the last-level cache, where they evict dirty ones.
    __builtin_amdgcn_s_waitcnt(0);
    __builtin_amdgcn_s_barrier();
    float* tr = reinterpret_cast<float*>(smem) + wave * 32 * T::kLd;
    const int er = lane & 31, eq = lane >> 5;
    void* C = p.C;
    int64_t ldc = p.ldc, base = 0;
    int type = p.type;
    if (splits > 1) {
        C = p.part;
        type = SQ_TYPE_F32;
        ldc = p.N;
        base = split * p.M * p.N;
    }
    const bool lines = (((uint64_t)C | (uint64_t)((base | ldc) * (type == SQ_TYPE_F32 ? 4 : 2))) & 127) == 0;
#pragma unroll
    for (int i = 0; i < T::FM; ++i)
#pragma unroll
        for (int h = 0; h < T::TN / T::kCols; ++h) {
            const int64_t m = m0 + wm * T::TM + i * 32, n_w = n0 + wn * T::TN + h * T::kCols;
            // a lane holds columns 8 q + 4 (lane / 32).. of row lane % 32
#pragma unroll
            for (int j = 0; j < T::kCols / 32; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const v16f& a = acc[i][h * (T::kCols / 32) + j];
                    *reinterpret_cast<v4f*>(tr + er * T::kLd + j * 32 + q * 8 + eq * 4) = v4f{a[4 * q], a[4 * q + 1], a[4 * q + 2], a[4 * q + 3]};
                }
            // 16 bytes a lane, whole lines: 8 columns of bf16, 4 of fp32
            auto rows_out = [&](auto F32, auto LINES) {
                constexpr bool f32 = decltype(F32)::value, lines = decltype(LINES)::value;
                // keeps the compiler from joining the two kinds of store, which loses the hint
                if constexpr (lines) asm volatile("; whole lines");
                constexpr int kPiece = f32 ? 4 : 8, kPer = T::kCols / kPiece, kRows = 64 / kPer;
                const int q = lane % kPer, r0 = lane / kPer;
#pragma unroll
                for (int rr = 0; rr < 32; rr += kRows) {
                    const int r = r0 + rr;
                    const float* src = tr + r * T::kLd + kPiece * q;
                    const v4f a = *reinterpret_cast<const v4f*>(src);
                    v4f b = a;
                    if constexpr (!f32) b = *reinterpret_cast<const v4f*>(src + 4);
                    const int64_t row = m + r, col = n_w + kPiece * q, at = base + row * ldc + col;
                    if (row >= p.M || col >= p.N) continue;
                    if (col + kPiece <= p.N) {
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
                        for (int e = 0; e < kPiece; ++e)
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

template <class T, bool EXACT>
__global__ __launch_bounds__(T::kThreads, T::kOccupancy) void k_f8_gemm(F8Product d) {
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ __attribute__((aligned(1024))) uint8_t smem[T::kSmem];
    product<T, EXACT>(d, blockIdx.x, smem);
#endif
}

// Two products that do not depend on each other, in one launch, one after the other:
// a layer's input and weight gradients.
template <class T, bool EXACT_A, bool EXACT_B>
__global__ __launch_bounds__(T::kThreads, T::kOccupancy) void k_f8_gemm_pair(F8Product a, F8Product b) {
#if defined(__HIP_DEVICE_COMPILE__)
    __shared__ __attribute__((aligned(1024))) uint8_t smem[T::kSmem];
    const uint32_t past = (a.blocks + kXcds - 1) / kXcds * kXcds;
    if (blockIdx.x < past) {
        if (blockIdx.x < a.blocks) product<T, EXACT_A>(a, blockIdx.x, smem);
    } else {
        product<T, EXACT_B>(b, blockIdx.x - past, smem);
    }
#endif
}

// Sum of the split-K partials, in the order of the splits, four columns a thread.
__global__ __launch_bounds__(256) void k_f8_reduce(const float* part, int splits, int64_t M, int64_t N, void* C, int type, int64_t ldc) {
    const int64_t n = M * N, per = (N + 3) / 4;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < M * per; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / per, c = (i - r * per) * 4;
        const float* src = part + r * N + c;
        v4f s = {0.0f, 0.0f, 0.0f, 0.0f};
        if (c + 4 <= N) {
            for (int k = 0; k < splits; ++k) s += *reinterpret_cast<const f32x4_any*>(src + k * n);
        } else {
            for (int k = 0; k < splits; ++k)
                for (int e = 0; e < 4 && c + e < N; ++e) s[e] += src[k * n + e];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < N) store_out(C, type, r * ldc + c + e, s[e]);
    }
}

// ---------------------------------------------------------------------------
// Few rows of values: Y = X W^T, bound by the one read of W.  A wave loads 16 x 128
// tiles of W straight into registers; a block owns 16 rows and 16 FN columns, its
// waves share the inner axis in contiguous parts, U tiles in flight each.  Four lanes hold the 128
// elements of X of a row and tile and quantize them in registers.  The waves' sums
// meet in LDS in a fixed order.
// ---------------------------------------------------------------------------
// Codes of 32 values in the words w (bf16 pairs, or fp32), with the block's scale byte.
template <bool BF16>
__device__ __forceinline__ v8i quantize_lane(const uint32_t* w, int& scale_byte) {
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    typedef uint16_t v2u16 __attribute__((ext_vector_type(2)));
    typedef short v2i16 __attribute__((ext_vector_type(2)));
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
    b = max(b, (uint32_t)__shfl_xor((int)b, 16));
    b = max(b, (uint32_t)__shfl_xor((int)b, 32));
    const uint32_t s = f8_scale(b);
    const float scale = mx_value(s);
    v8i a;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v2i16 r = {0, 0};
        if constexpr (BF16) {
            r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(v2bf, w[2 * i]), scale, false);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(v2bf, w[2 * i + 1]), scale, true);
        } else {
            r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, __uint_as_float(w[4 * i]), __uint_as_float(w[4 * i + 1]), scale, false);
            r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, __uint_as_float(w[4 * i + 2]), __uint_as_float(w[4 * i + 3]), scale, true);
        }
        a[i] = s == 255u ? 0 : __builtin_bit_cast(int, r);
    }
    scale_byte = (int)s;
    return a;
}

template <typename T, int FN, int U, int kRowsWaves, bool EXACT>
__global__ __launch_bounds__(64 * kRowsWaves, 4) void k_f8_rows(F8RowsArgs p, uint32_t tiles_n) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr int kLd = 16 * FN + 4, kWords = 32 * sizeof(T) / 4, kHalf = kWords / 2, kV = 16 / sizeof(T);
    __shared__ float sums[kRowsWaves * 16 * kLd];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t tm = blockIdx.x / tiles_n;
    const int64_t n0 = (int64_t)(blockIdx.x - tm * tiles_n) * (16 * FN), m0 = (int64_t)tm * 16;
    const int K = (int)p.K, n = (K + kMxTile - 1) / kMxTile, part = (n + kRowsWaves - 1) / kRowsWaves;
    const int beg = min(wave * part, n), end = min(beg + part, n);
    const int64_t units = mx_units(K), first = n0 >> 4;
    const int last = (int)(mx_groups(p.N) - 1 - first);
    const uint32_t gb = (uint32_t)(units * kF8UnitBytes), gs = (uint32_t)(units * kF8UnitScales);
    const __amdgpu_buffer_rsrc_t rW = f8_rsrc(p.W + first * gb, (int64_t)(last + 1) * gb),
                                 rWs = f8_rsrc(p.Ws + first * gs, (int64_t)(last + 1) * gs);
    // rows past the end read the last one; their results are never stored
    const T* x = static_cast<const T*>(p.x) + min(m0 + (lane & 15), p.M - 1) * p.ld;
    v4f acc[FN];
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[j] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    auto multiply = [&](const v8i& w, int ws, const v8i& a, int sa, v4f c) {
        if constexpr (EXACT) {
            const float fw = mx_value((uint32_t)ws & 255u), fa = mx_value((uint32_t)sa);
#pragma unroll
            for (int i = 0; i < 8; i += 2)
                c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(values8(w[i], w[i + 1], fw), values8(a[i], a[i + 1], fa), c, 0, 0, 0);
            return c;
        } else {
            return mfma16(w, a, c, ws, sa);
        }
    };
    // lane l: row l % 16, 16-element pieces l / 16 and 4 + l / 16 of the tile
    auto load_w = [&](int at, int j, v8i& w, int& ws) {
        const uint32_t grp = (uint32_t)min(j, last);
        const int off = (int)(grp * gb) + at * kF8TileBytes;
        w = join(__builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(rW, 16u * (uint32_t)lane, off, 0)),
                 __builtin_bit_cast(v4i, __builtin_amdgcn_raw_buffer_load_b128(rW, 16u * (uint32_t)lane, off + 1024, 0)));
        ws = (int)__builtin_amdgcn_raw_buffer_load_b32(rWs, 4u * ((uint32_t)lane & 15u), (int)(grp * gs) + (at >> 2) * kF8UnitScales, 0);
    };
    const int full = K / kMxTile, stop = min(end, full);    // whole tiles
    for (int t = beg; t < stop; t += U) {
        v8i w[U][FN];
        int ws[U][FN];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < FN; ++j) load_w(min(t + u, stop - 1), j, w[u][j], ws[u][j]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // read again to keep the loads free of branches: not multiplied, or times zeros, which a value that is Inf
            // in bf16 would make NaN
            if (EXACT && t + u >= stop) break;
            const int at = min(t + u, stop - 1);
            uint32_t v[kWords];
            const T* from = x + at * kMxTile + (lane >> 4) * 16;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int q = 0; q < 16 / kV; ++q) {
                    const u32x4_any l = *reinterpret_cast<const u32x4_any*>(from + 64 * h + q * kV);
                    v[kHalf * h + 4 * q] = l.x;
                    v[kHalf * h + 4 * q + 1] = l.y;
                    v[kHalf * h + 4 * q + 2] = l.z;
                    v[kHalf * h + 4 * q + 3] = l.w;
                }
            int sa;
            v8i a = quantize_lane<sizeof(T) == 2>(v, sa);
            if (t + u >= stop) a = v8i{0, 0, 0, 0, 0, 0, 0, 0}, sa = 0;
            const int byte = 8 * (at & 3);
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[j] = multiply(w[u][j], ws[u][j] >> byte, a, sa, acc[j]);
        }
    }
    if (end > stop && end == n && beg < end) {      // the tile that K ends in, element by element
        uint32_t v[kWords];
#pragma unroll
        for (int q = 0; q < kWords; ++q) {
            const int c = full * kMxTile + (lane >> 4) * 16 + (q >= kHalf ? 64 : 0) + (q % kHalf) * (4 / (int)sizeof(T));
            if constexpr (sizeof(T) == 4) {
                const uint32_t e = __float_as_uint(x[min(c, K - 1)]);
                v[q] = c < K ? e : 0u;
            } else {
                const uint32_t lo = x[min(c, K - 1)], hi = x[min(c + 1, K - 1)];
                v[q] = (c < K ? lo : 0u) | (c + 1 < K ? hi << 16 : 0u);
            }
        }
        int sa;
        const v8i a = quantize_lane<sizeof(T) == 2>(v, sa);
        const int byte = 8 * (full & 3);
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            v8i w;
            int ws;
            load_w(full, j, w, ws);
            acc[j] = multiply(w, ws >> byte, a, sa, acc[j]);
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
        if (m0 + r < p.M && n0 + c + e < p.N) store_out(p.Y, p.out_type, (m0 + r) * p.ldy + n0 + c + e, s);
    }
#endif
}

enum F8TileKind { kWide, kMid, kSmall };

// Tiles by the size of the product.  us in bf16 / fp32:
//   128 x 256 and 128 x 128: 4096^3 (512 large tiles) 58 / 107 and 62 / 117, 8192 x 8192 x 512 48 / 76 and 55 / 85,
//     3000^3 (288) 38 / 67 and 34 / 63;
//   128 x 128 and 64 x 64: 2048^3 (256) 10.7 / 20.9 and 14.1 / 21.5, 1024 x 4096 x 1024 (256) 7.8 / 13.4 and 9.5 / 12.9,
//     1500^3 (144) 9.6 / 16.2 and 9.7 / 14.0, 512 x 4096 x 4096 (128) 16 / 33 and 14 / 24.
F8TileKind tile_kind(const F8GemmArgs& a) {
    const auto tiles = [&](int64_t m, int64_t n) { return ((a.M + m - 1) / m) * ((a.N + n - 1) / n); };
    if (tiles(128, 256) >= 400) return kWide;
    return tiles(128, 128) >= 240 ? kMid : kSmall;
}

template <class T>
F8Product product_of(const F8GemmArgs& a) {
    F8Product d{};
    d.a = a;
    d.splits = (int)f8_gemm_splits(a.M, a.N, a.K, a.type);
    d.tiles_n = (uint32_t)((a.N + T::BN - 1) / T::BN);
    d.tiles_m = (uint32_t)((a.M + T::BM - 1) / T::BM);
    d.blocks = d.tiles_m * d.tiles_n * (uint32_t)d.splits;
    return d;
}

hipError_t reduce(const F8Product& d, hipStream_t s) {
    if (d.splits == 1) return hipSuccess;
    const F8GemmArgs& a = d.a;
    k_f8_reduce<<<(uint32_t)std::min<int64_t>((a.M * ((a.N + 3) / 4) + 255) / 256, 4096), 256, 0, s>>>(a.part, d.splits, a.M, a.N, a.C, a.type, a.ldc);
    return hipGetLastError();
}

template <class T>
hipError_t gemm(const F8GemmArgs& a, hipStream_t s) {
    const F8Product d = product_of<T>(a);
    if (a.type == SQ_TYPE_F32) k_f8_gemm<T, true><<<d.blocks, T::kThreads, 0, s>>>(d);
    else k_f8_gemm<T, false><<<d.blocks, T::kThreads, 0, s>>>(d);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? reduce(d, s) : e;
}

template <class T>
hipError_t pair(const F8GemmArgs& a, const F8GemmArgs& b, hipStream_t s) {
    const F8Product da = product_of<T>(a), db = product_of<T>(b);
    const uint32_t blocks = (uint32_t)round_up(da.blocks, 8) + db.blocks;
    if (a.type == SQ_TYPE_F32 && b.type == SQ_TYPE_F32) k_f8_gemm_pair<T, true, true><<<blocks, T::kThreads, 0, s>>>(da, db);
    else if (a.type == SQ_TYPE_F32) k_f8_gemm_pair<T, true, false><<<blocks, T::kThreads, 0, s>>>(da, db);
    else k_f8_gemm_pair<T, false, true><<<blocks, T::kThreads, 0, s>>>(da, db);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess) e = reduce(da, s);
    return e == hipSuccess ? reduce(db, s) : e;
}

template <typename T, int FN, int U, int WAVES>
hipError_t rows(const F8RowsArgs& a, hipStream_t s) {
    const int64_t tiles_n = (a.N + 16 * FN - 1) / (16 * FN);
    const uint32_t blocks = (uint32_t)((a.M + 15) / 16 * tiles_n);
    if (a.out_type == SQ_TYPE_F32) k_f8_rows<T, FN, U, WAVES, true><<<blocks, 64 * WAVES, 0, s>>>(a, (uint32_t)tiles_n);
    else k_f8_rows<T, FN, U, WAVES, false><<<blocks, 64 * WAVES, 0, s>>>(a, (uint32_t)tiles_n);
    return hipGetLastError();
}

}  // namespace

// Few tiles of a long inner axis are split, in parts of at least 20 tiles (16 where
// these take the slower instruction): the sum of the parts is a launch more, 5 to 6 us.
// fp32 results: 300 x 300 x 8192 (64 tiles) whole 29 us, in parts of 20 16.9, of 16
// 13.4; 768 x 768 x 3152 (25) whole 14, in halves 15.8; 1024^3 (8) 7.0 and 13.9.
int64_t f8_gemm_splits(int64_t M, int64_t N, int64_t K, int type) {
    const int64_t tiles = ((M + 63) / 64) * ((N + 63) / 64), k = (K + kMxTile - 1) / kMxTile, least = type == SQ_TYPE_F32 ? kSplitExact : kSplit;
    return std::max<int64_t>(1, std::min<int64_t>(512 / std::max<int64_t>(tiles, 1), k / least));
}

hipError_t launch_f8_gemm(const F8GemmArgs& a, hipStream_t s) {
    if (a.M == 0 || a.N == 0) return hipSuccess;
    switch (tile_kind(a)) {
        case kWide: return gemm<F8Wide>(a, s);
        case kMid: return gemm<F8Mid>(a, s);
        default: return gemm<F8Small>(a, s);
    }
}

hipError_t launch_f8_gemm_pair(const F8GemmArgs& a, const F8GemmArgs& b, hipStream_t s) {
    if (a.M == 0 || a.N == 0 || b.M == 0 || b.N == 0 || tile_kind(a) != tile_kind(b) || (a.type != SQ_TYPE_F32 && b.type != SQ_TYPE_F32)) {
        const hipError_t e = launch_f8_gemm(a, s);
        return e == hipSuccess ? launch_f8_gemm(b, s) : e;
    }
    // the longer tiles first
    const auto length = [](const F8GemmArgs& g) { return (double)g.K * (g.type == SQ_TYPE_F32 ? 2.0 : 1.0); };
    const F8GemmArgs &x = length(a) >= length(b) ? a : b, &y = length(a) >= length(b) ? b : a;
    switch (tile_kind(a)) {
        case kWide: return pair<F8Wide>(x, y, s);
        case kMid: return pair<F8Mid>(x, y, s);
        default: return pair<F8Small>(x, y, s);
    }
}

// Few rows, for which the products' tiles would be mostly empty.  bf16, and the quantizer
// with the product, one W over and over: 64 x 4096 -> 4096 (38912 of the 40000) 9.3 us, 13.5; 96 rows of it
// (58368) 14.4, 14.0; 512 x 1024 -> 1024 (28672) 6.1, 8.7; fp32: 512 x 768 -> 768
// (36864) 7.1, 9.5, 32 x 4096 -> 4096 (38912) 11.3, 15.5.
bool f8_rows_ok(int64_t M, int64_t K, int64_t N, int type) {
    const double blocks = (double)((M + 15) / 16) * (double)((N + 15) / 16), steps = (double)((K + 127) / 128);
    return M <= 16 || blocks * (steps + 6.0) * (type == SQ_TYPE_F32 ? 2.0 : 1.0) <= 40000.0;
}

hipError_t launch_f8_rows(const F8RowsArgs& a, hipStream_t s) {
    if (a.M == 0 || a.N == 0) return hipSuccess;
    // One tile of rows: as many blocks as there are (1 x 4096 -> 11008 in bf16 11.6 us, with 32 columns a block 12.3), fp32
    // rows with twice the waves where these have two tiles each (1 x 4096 -> 4096 6.8 us, 7.9 with eight).  More rows:
    // columns that share the rows' codes (64 x 4096 -> 4096 10.5 us with 64 columns a block, 12.8 with 32, 19.6 with 16;
    // 128 x 1024 -> 1024, 512 tiles, 3.9 with 32 and 4.2 with 64).  All with 12 or more W in turn.
    const int64_t tiles_m = (a.M + 15) / 16, tiles = tiles_m * ((a.N + 15) / 16);
    if (tiles_m > 1 && tiles >= 512) {
        if (a.type == SQ_TYPE_F32) return tiles >= 1024 ? rows<float, 4, 1, 8>(a, s) : rows<float, 2, 1, 8>(a, s);
        return tiles >= 1024 ? rows<uint16_t, 4, 1, 8>(a, s) : rows<uint16_t, 2, 1, 8>(a, s);
    }
    if (a.type == SQ_TYPE_F32) return a.K >= 32 * kMxTile ? rows<float, 1, 1, 16>(a, s) : rows<float, 1, 1, 8>(a, s);
    return rows<uint16_t, 1, 2, 8>(a, s);
}

}  // namespace sq
