// Matrix products D[i][j] = sum_r A[i][r] * B[j][r] out of tiles in LDS, as the cross entropy and the layers' gradients take them: 16-bit operands
// (fp16, or fp32 numbers as three bf16) that lie as the product wants them, r contiguous, or turned.
#pragma once
#include <math.h>

#include "dcnv4_common.h"

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// One operand of a product: `count` rows i (or j) and a sum over `length` numbers r, in planes.  As it is: row i at base + i * row_bytes, r
// contiguous, length a multiple of eight.  Turned: row r at base + r * row_bytes, i contiguous, count a multiple of eight.
struct Operand {
    const char *base;
    long long row_bytes;
    int count, length, plane_bytes;
};

struct Product {
    Operand a, b;
    int steps, steps_per_split;
    int a_tiles, b_tiles, all, per_xcd;   // all: tiles times splits
    FastDiv div_tiles, div_band, div_3;   // by the tiles, those of a band of four, and three
};

typedef short s16x4 __attribute__((ext_vector_type(4)));

// The LDS read that turns.  (Its pointer is `restrict`: without that mark the compiler lets every such read wait for all loads into LDS,
// those of the next step among them.)
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
__device__ __forceinline__ s16x4 read_turned(const lds_s16x4 *__restrict p)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16(const_cast<lds_s16x4 *>(p));
}

// PL planes: 1 (fp16) or 3 (fp32 as three bf16).  A step is R numbers r of each plane, of which STAGES are in LDS or on their way.  TA, TB:
// A, B turned.  PAIRS: A (as it is) has 2 * count rows, and a tile's 32 rows are 16 of the first half and the same 16 of the second, so that a lane gets both
// results of a pair: those of row i in acc[..][4 * a + c], a < 2, and of row count + i in acc[..][4 * (a + 2) + c].
template <int PL, int WR, int WC, int WM, int WN, int R, int STAGES, bool TA = false, bool TB = false, bool PAIRS = false> struct Tile {
    static constexpr int kWaves = WR * WC, kThreads = kWaves * 64;
    static constexpr int BM = WR * 32 * WM, BN = WC * 32 * WN;
    static constexpr int STEP = 2 * R;                                     // a step in bytes
    static constexpr int LOAD = kWaves * 1024;                             // bytes that all waves' load brings
    static constexpr int LA = BM * STEP / LOAD, LB = BN * STEP / LOAD, LOADS = (LA + LB) * PL;
    static_assert(LA * LOAD == BM * STEP && LB * LOAD == BN * STEP);
    static constexpr int PLANE = (BM + BN) * STEP, STAGE = PL * PLANE;
    static constexpr int OUT = kWaves * 32 * (32 * WM * 4 + 16);           // rows of results on their way out, at most
    static constexpr int LDS = STAGES * STAGE > OUT ? STAGES * STAGE : OUT;
    static constexpr int kWavesPerSimd = kWaves / 4 * (LDS > 80 * 1024 ? 1 : 2);     // that registers have to leave room for

    // Where things lie in LDS, so that what is read in one pass falls on all 64 banks.  As it is: rows of STEP bytes; a pass of a 16-byte
    // read is 16 lanes (of the first 32: 0-3, 12-15, 20-27, and the others), so rows two apart (128-byte rows; four, 64-byte rows) take
    // other units.  Turned: rows (r) of 2 * COUNT bytes; a pass of a turning read is 32 lanes, 64 bytes of four rows, which take
    // other 64-byte pieces.  (Units by row % 8: half the cycles of the reads were conflicts; 8192 x
    // 1024 x 8192 forward took 1.5 % longer, as power is what it waits for.)
    static __device__ __forceinline__ int swizzle(int row) { return R == 64 ? row >> 1 & 7 : row >> 2 & 3; }
    template <int COUNT> static __device__ __forceinline__ int swizzle_turned(int r)     // in pieces of 32 bytes
    {
        return COUNT >= 128 ? (r & 3) << 1 : r & 2;
    }

    // An operand's loads: what a lane asks for, load after load, of COUNT rows from i0 on.
    template <bool TURNED, int COUNT, int LOADS_, bool PAIRED = false> struct Source {
        const Operand &o;
        int from[LOADS_], at0;                             // byte offsets; as it is: the lane's first r, in bytes
        int rows;
        const char *base;
        __device__ __forceinline__ Source(const Operand &op, int i0, int wave, int lane) : o(op)
        {
            constexpr int UNITS = (TURNED ? 2 * COUNT : STEP) / 16, ROWS = 64 / UNITS;      // of a row; rows of a wave's load
            static_assert(64 % UNITS == 0);
            const int first = wave * ROWS + lane / UNITS, unit = lane % UNITS;
            if constexpr (TURNED) {
                base = o.base + i0 * 2;
                at0 = 0;
                rows = 0;
#pragma unroll
                for (int i = 0; i < LOADS_; ++i) {
                    const int r = i * kWaves * ROWS + first;
                    from[i] = (int)(r * o.row_bytes) + (unit ^ swizzle_turned<COUNT>(r) << 1) * 16;
                }
            } else {
                // rows past the last are the last once more
                rows = min(PAIRED ? COUNT / 2 : COUNT, o.count - i0);
                base = o.base + i0 * o.row_bytes;
                at0 = (unit ^ swizzle(first)) * 16;
#pragma unroll
                for (int i = 0; i < LOADS_; ++i) {
                    const int row = i * kWaves * ROWS + first;
                    if constexpr (PAIRED)
                        from[i] = (int)((min(row / 32 * 16 + row % 16, rows - 1) + (row & 16 ? o.count : 0)) * o.row_bytes) + at0;
                    else
                        from[i] = (int)(min(row, rows - 1) * o.row_bytes) + at0;
                }
                if (PAIRED)
                    rows += o.count;                       // (that the descriptor reaches)
            }
        }
        // Step t: past t1 nothing is read and zeros are written, likewise past the sum's length.
        rsrc_t r;
        unsigned out;
        int at;
        __device__ __forceinline__ void step(int t, int t1)
        {
            if constexpr (TURNED) {
                // (from row t * R on; what lies past a row's end is the next one's, for rows of the result that are dropped)
                const int left = t < t1 ? min(R, o.length - t * R) : 0;
                r = make_rsrc(base + (long long)t * R * o.row_bytes, left <= 0 ? 0u : (unsigned)(left * o.row_bytes - (base - o.base)));
                out = 0u;
                at = 0;
            } else {
                r = make_rsrc(base, (unsigned)(rows * o.row_bytes));
                at = t * STEP;
                out = t < t1 && at + at0 < 2 * o.length ? 0u : (unsigned)kOutside;
            }
        }
        __device__ __forceinline__ void load(char *to, int p, int i) const
        {
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)(to + p * PLANE + i * LOAD), 16,
                                                     (int)((unsigned)(from[i] + at + p * o.plane_bytes) | out), 0, 0, 0);
        }
    };

    // Fragment g (16 numbers r) of rows first to first + 31 of an operand's tile: lane l gets eight r of row l % 32.
    template <bool TURNED, int COUNT> static __device__ __forceinline__ u32x4 fragment(const char *tile, int first, int g, int lane)
    {
        const int row = lane & 31, kb = lane >> 5;
        if constexpr (!TURNED) {
            return *reinterpret_cast<const u32x4 *>(tile + (first + row) * STEP + (((2 * g + kb) ^ swizzle(row)) << 4));
        } else {
            // 16 lanes: four r, four lanes to the 32 bytes of one; the lane gets four r of its own row
            const int r = 8 * kb + (lane >> 2 & 3), piece = first / 16 + (lane >> 4 & 1);
            const char *p = tile + (16 * g + r) * (2 * COUNT) + ((piece ^ swizzle_turned<COUNT>(r)) << 5) + (lane & 3) * 8;
            const char *q = tile + (16 * g + r + 4) * (2 * COUNT) + ((piece ^ swizzle_turned<COUNT>(r + 4)) << 5) + (lane & 3) * 8;
            const s16x4 lo = read_turned((const lds_s16x4 *)p);
            const s16x4 hi = read_turned((const lds_s16x4 *)q);
            const u32x2 a = __builtin_bit_cast(u32x2, lo), b = __builtin_bit_cast(u32x2, hi);
            return u32x4{a[0], a[1], b[0], b[1]};
        }
    }

    static_assert(!PAIRS || !TA);
    // Three planes: the five products with small parts are summed apart where a wave has the registers (one wave to a SIMD).  In one sum each of six
    // products is rounded to the large one's step: the gated layer of 2000 numbers, 1 x 2000, 2 x 4000, was 1.1e-6 off, and is 4.3e-7 so (a library's
    // sums in parts: 5.8e-7), in the same 46 us.
    static constexpr bool kApart = PAIRS && PL == 3 && kWavesPerSimd == 1;
    // acc[m][n]: rows a0 + (wr * WM + m) * 32 of A (pairs: from pair a0 + (wr * WM + m) * 16 on), rows b0 + (wc * WN + n) * 32 of B, steps t0 to t1 - 1
    static __device__ __forceinline__ void multiply(char *smem, const Operand &a, const Operand &b, int a0, int b0, int t0, int t1,
                                                    f32x16 (&acc)[WM][WN])
    {
        const int tid = (int)threadIdx.x, lane = tid & 63;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int wr = wave / WC, wc = wave % WC;
        Source<TA, BM, LA, PAIRS> sa(a, a0, wave, lane);
        Source<TB, BN, LB> sb(b, b0, wave, lane);
        auto load = [&](int j, int stage) {               // load j of the step that sa and sb are at
            char *to = smem + stage * STAGE + wave * 1024;
            const int p = j / (LA + LB), i = j % (LA + LB);
            if (i < LA)
                sa.load(to, p, i);
            else
                sb.load(to + BM * STEP, p, i - LA);
        };
        u32x4 af[2][PL][WM], bf[2][PL][WN];
        f32x16 small[kApart ? WM : 1][kApart ? WN : 1];
        if constexpr (kApart) {
#pragma unroll
            for (int m = 0; m < WM; ++m)
#pragma unroll
                for (int n = 0; n < WN; ++n)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        small[m][n][r] = 0.f;
        }
        auto fetch = [&](const char *stage, int g, int f) {      // fragment f of group g
            const int p = f / (WM + WN), i = f % (WM + WN);
            if (i < WM)
                af[g & 1][p][i] = fragment<TA, BM>(stage + p * PLANE, (wr * WM + i) * 32, g, lane);
            else
                bf[g & 1][p][i - WM] = fragment<TB, BN>(stage + p * PLANE + BM * STEP, (wc * WN + i - WM) * 32, g, lane);
        };
        // The products of group g.  Among them: the fragments of the next group (`next` of `ahead`), as early as two to a product, and loads
        // j0 to j1 - 1 of a later step into stage `to`.  (Before the products they would hold the wave up: eight waves' loads take
        // the unit 29 clocks a KiB, and more than 15 LDS reads on their way are waited for.)
        auto products = [&](int g, const char *ahead, int next, int j0, int j1, int to) {
            // (three planes: small parts first)
            constexpr int pa[6] = {0, 2, 1, 0, 1, 0}, pb[6] = {2, 0, 1, 1, 0, 0}, Q = PL == 1 ? 1 : 6, ALL = Q * WM * WN, ALL_F = PL * (WM + WN);
            int j = j0, f = 0;
#pragma unroll
            for (int q = 6 - Q; q < 6; ++q)
#pragma unroll
                for (int m = 0; m < WM; ++m)
#pragma unroll
                    for (int n = 0; n < WN; ++n) {
                        const int k = ((q - 6 + Q) * WM + m) * WN + n;
                        const u32x4 x = af[g & 1][pa[q]][m], y = bf[g & 1][pb[q]][n];
                        if constexpr (PL == 1)
                            acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y),
                                                                               acc[m][n], 0, 0, 0);
                        else if (kApart && q < 5)
                            small[kApart ? m : 0][kApart ? n : 0] =
                                __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y),
                                                                        small[kApart ? m : 0][kApart ? n : 0], 0, 0, 0);
                        else
                            acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y),
                                                                                acc[m][n], 0, 0, 0);
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int e = 0; e < (ALL_F + ALL - 1) / ALL + 1; ++e)
                            if (f < ALL_F)
                                fetch(ahead, next, f++);
#pragma unroll
                        for (int e = 0; e < LOADS; ++e)
                            if (j < j1 && (k + 1) * (j1 - j0) >= (j - j0 + 1) * ALL)
                                load(j++, to);
                        __builtin_amdgcn_sched_barrier(0);
                    }
        };
        // Fragments are read while the products of the group before them run, across steps too: where the last group of a step is in
        // registers, the next step's loads have to have landed and the step's stage is free.  Three stages and more: a step
        // issues the loads of the step STAGES - 1 later, a part with each group, into the stage that the step before has freed.  Two stages:
        // its last group issues those of the step after the next, into its own.
        constexpr int GROUPS = R / 16, AHEAD = STAGES > 2 ? STAGES - 1 : 2;
        constexpr int EARLY = STAGES > 2 ? LOADS * (GROUPS - 1) / GROUPS : 0;          // of a step's loads, before its last group
        constexpr int FLYING = STAGES > 2 ? (STAGES - 3) * LOADS + EARLY : 0;          // that need not have landed there
        static_assert(GROUPS % 2 == 0 && STAGES > 1 && (AHEAD - 1) * LOADS < 64 && FLYING < 64);
#pragma unroll
        for (int s = 0; s < AHEAD; ++s) {
            sa.step(t0 + s, t1);
            sb.step(t0 + s, t1);
#pragma unroll
            for (int j = 0; j < LOADS; ++j)
                load(j, s);
        }
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"((AHEAD - 1) * LOADS) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int f = 0; f < PL * (WM + WN); ++f)
            fetch(smem, 0, f);
        int at = 0;
#pragma unroll 1
        for (int t = t0; t < t1; ++t) {
            const int to = STAGES == 2 ? at : at == 0 ? STAGES - 1 : at - 1;
            sa.step(t + AHEAD, t1);
            sb.step(t + AHEAD, t1);
            const char *stage = smem + at * STAGE;
#pragma unroll
            for (int g = 0; g + 1 < GROUPS; ++g)
                products(g, stage, g + 1, EARLY * g / (GROUPS - 1), EARLY * (g + 1) / (GROUPS - 1), to);
            // the next step's loads have landed, for every wave, and all have read this stage
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(FLYING) : "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            at = at + 1 == STAGES ? 0 : at + 1;
            products(GROUPS - 1, smem + at * STAGE, 0, EARLY, LOADS, to);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (results go where the last loads write)
        __syncthreads();
        if constexpr (kApart) {
#pragma unroll
            for (int m = 0; m < WM; ++m)
#pragma unroll
                for (int n = 0; n < WN; ++n)
                    acc[m][n] += small[m][n];
        }
    }
};

// The tile and split of workgroup `block`: consecutive ones to one XCD, split after split (the tiles of a split read the same part of both
// operands), in the order of bands of four tiles of B and along A within a band, so that the 32 tiles that an XCD has at once
// read eight tiles of A and four of B into its L2, not 32 and one.  False: none.
__device__ __forceinline__ bool tile_of(const Product &q, int block, int &a_tile, int &b_tile, int &split)
{
    const int at = (block & (kXcds - 1)) * q.per_xcd + (block >> 3);
    if ((block >> 3) >= q.per_xcd || at >= q.all)
        return false;
    split = fdiv(at, q.div_tiles);
    const int tile = at - split * q.a_tiles * q.b_tiles;
    const int band = fdiv(tile, q.div_band), rest = tile - band * 4 * q.a_tiles, wide = min(4, q.b_tiles - band * 4);
    a_tile = wide == 4 ? rest >> 2 : wide == 2 ? rest >> 1 : wide == 1 ? rest : fdiv(rest, q.div_3);
    b_tile = band * 4 + rest - a_tile * wide;
    return true;
}

__device__ __forceinline__ float other_half(float v)       // of the lane 32 away
{
    float a = v, b = v;
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b));
    return (threadIdx.x & 32) ? a : b;
}

template <int CTRL> __device__ __forceinline__ float dpp(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float sum_of_32(float v)        // over the lane's half of the wave, in every lane of it
{
    v += dpp<0xB1>(v);                                     // quad_perm [1,0,3,2], [2,3,0,1], row_half_mirror, row_mirror
    v += dpp<0x4E>(v);
    v += dpp<0x141>(v);
    v += dpp<0x140>(v);
    float a = v, b = v;
    asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(a), "+v"(b));
    return a + b;
}


// grad_b: the pixel runs' sums, added up.
struct Bias {
    const float *sums;                // [runs][count]
    int runs, count, blocks;          // blocks: workgroups, none for no grad_b
    void *grad_b;
};

// 16 classes to a workgroup of 256, 16 runs side by side.
// (Of more threads the others do the same.  `part` is the caller's: with a second LDS object in a kernel this compiler lets the LDS reads of Tile::multiply
// wait for all loads.)
template <typename T> __device__ __forceinline__ void bias_of(const Bias &b, int block, float (*part)[17])
{
    const int i = (int)threadIdx.x & 15, slice = (int)threadIdx.x >> 4 & 15, c = block * 16 + i;
    float s = 0.f;
    if (c < b.count)
#pragma unroll 8
        for (int r = slice; r < b.runs; r += 16)
            s += b.sums[(long long)r * b.count + c];
    part[slice][i] = s;
    __syncthreads();
    if (slice != 0 || c >= b.count)
        return;
#pragma unroll
    for (int k = 1; k < 16; ++k)
        s += part[k][i];
    ((T *)b.grad_b)[c] = (T)s;
}
// Tiles by number: classes (or columns of a result) x pixels (or its rows).  fp16: 64x64, 128x128, 256x256; fp32: 64x64, 128x128, 256x128.
enum { kSmall, kMiddle, kLarge };

// The work is planned for this many compute units (the plan gives the size of the workspace, without a device).
constexpr int kUnits = 256;

struct Shape {
    int bm, bn, r;                     // classes (or columns of a result), pixels (or its rows), numbers of a step
    int slots;                         // tiles of a compute unit side by side
    float step, fixed, alone, gen;
};
// Estimated times (us): a unit works through its share of the tiles, `slots` of them side by side, where half the difference between the
// fullest unit and the mean is felt, and a part (`gen`) of the idle slots of the last round.  A tile takes `step` for a step, a lone
// one `alone` at least, and `fixed` for its first loads and its results.  Fitted to products of 17 sizes (16 to 51200 rows, 30 to 40000 classes,
// K 128 to 1024, every tile, 1 to 64 splits; rms 12 %): the choice costs 2.5 % (fp16) and 0.9 % (fp32) on average.  16384 rows, 512 -> 1000,
// forward: 45 (64x64), 29, 25 us, fp32 of 8192: 65, 52, 44; 1000, 256 -> 1000: 5.6, 9.0, 14, fp32: 8.2, 16, 20.
inline const Shape &shape_of(int pl, int i)
{
    static const Shape f16[] = {{64, 64, 64, 2, .204f, .75f, .263f, .5f}, {128, 128, 32, 2, .273f, 1.44f, .273f, 0.f}, {256, 256, 32, 1, .562f, 5.9f, 0.f, 0.f}};
    static const Shape f32[] = {{64, 64, 64, 1, .719f, 1.44f, 0.f, 0.f}, {128, 128, 32, 1, 1.01f, 2.6f, 0.f, 0.f}, {256, 128, 32, 1, 1.73f, 3.7f, 0.f, 0.f}};
    return (pl == 1 ? f16 : f32)[i];
}

struct Choice {
    int shape, splits;
};

// Estimated time (us) of m x n results over `length` numbers, each sum in `splits` parts.
float estimate(const Shape &s, long long m, long long n, int length, int splits)
{
    const int steps = (length + s.r - 1) / s.r;
    const long long tiles = ((m + s.bm - 1) / s.bm) * ((n + s.bn - 1) / s.bn);
    const float x = (float)(tiles * splits) / (float)kUnits, full = ceilf(x), slots = (float)s.slots;
    const float rounds = x > slots ? slots * ceilf(x / slots) : full, even = s.slots > 1 && x > 1.f ? .5f * (x + full) : full;
    const float share = even + s.gen * (rounds - even);
    const float step = s.step * share > s.alone ? s.step * share : s.alone;
    float us = (float)((steps + splits - 1) / splits) * step + s.fixed * share;
    if (splits > 1)                                        // planes written and read once more, by a launch of its own
        us += 2.5f + .09f * (float)splits + (float)(m * n) * (float)splits * 1.2e-6f;
    return us;
}

// The tile, and over how many workgroups a sum is split, with the lowest estimated time.
// Test switches: only the tile `only` (1 + its number; 0: any); `asked` workgroups to a sum, where it may be split (0: any).
Choice choose_product(int pl, long long m, long long n, int length, bool may_split, int only, int asked)
{
    Choice best = {-1, 1};
    float best_us = 0.f;
    for (int i = kSmall; i <= kLarge; ++i) {
        if (only && only != 1 + i)
            continue;
        const Shape &s = shape_of(pl, i);
        const long long tiles = ((m + s.bm - 1) / s.bm) * ((n + s.bn - 1) / s.bn);
        // powers of two, and what fills the units once and twice
        const int fill = tiles < kUnits ? (int)(kUnits / tiles) : 1, tries[] = {1, 2, 4, 8, 16, 32, 64, fill, 2 * fill};
        for (const int splits : tries) {
            if (splits > 1 && (!may_split || splits > 64 || length / splits < 256))
                continue;
            const float us = estimate(s, m, n, length, splits);
            if (best.shape < 0 || us < best_us) {
                best = {i, splits};
                best_us = us;
            }
        }
    }
    if (may_split && asked)
        best.splits = asked;
    return best;
}

long long round_up(long long v, long long to) { return (v + to - 1) / to * to; }

// Rows [rows][PL planes][pad] of 16 bits, `cols` of which count: as they are, or turned.
Operand rows_of(const void *base, int rows, int cols, int pl, int pad)
{
    return {(const char *)base, (long long)pl * pad * 2, rows, cols, pad * 2};
}
Operand turned(const Operand &o) { return {o.base, o.row_bytes, o.length, o.count, o.plane_bytes}; }

// `pairs`: A has 2 * count rows, which the tiles take in pairs.
Product product_of(const Operand &a, const Operand &b, const Shape &s, const Choice &c, bool pairs = false)
{
    Product q;
    q.a = a;
    q.b = b;
    q.steps = (b.length + s.r - 1) / s.r;
    q.steps_per_split = (q.steps + c.splits - 1) / c.splits;
    const int bm = pairs ? s.bm / 2 : s.bm;
    q.a_tiles = (a.count + bm - 1) / bm;
    q.b_tiles = (b.count + s.bn - 1) / s.bn;
    q.all = q.a_tiles * q.b_tiles * c.splits;
    q.per_xcd = (q.all + kXcds - 1) / kXcds;
    q.div_tiles = make_div((unsigned)(q.a_tiles * q.b_tiles));
    q.div_band = make_div(4u * (unsigned)q.a_tiles);
    q.div_3 = make_div(3);
    return q;
}

// Calls f with the tile's parameters (waves, blocks of a wave, stages) as constants.
template <int A, int B, int C, int D, int E, int F> struct TileOf {
    static constexpr int WR = A, WC = B, WM = C, WN = D, R = E, STAGES = F;
};
template <int PL, typename F> int with_tile(int shape, F &&f)
{
    if constexpr (PL == 1) {
        if (shape == kLarge) return f(TileOf<4, 2, 2, 4, 32, 4>());
        if (shape == kMiddle) return f(TileOf<2, 2, 2, 2, 32, 4>());
        return f(TileOf<2, 2, 1, 1, 64, 4>());
    } else {
        if (shape == kLarge) return f(TileOf<4, 2, 2, 2, 32, 2>());
        if (shape == kMiddle) return f(TileOf<2, 2, 2, 2, 32, 3>());
        return f(TileOf<2, 2, 1, 1, 64, 3>());
    }
}

int launched() { return hipGetLastError() == hipSuccess ? DCNV4_OK : DCNV4_ERR_LAUNCH; }

unsigned row_groups(long long rows) { return (unsigned)((rows + 7) / 8 < 8192 ? (rows + 7) / 8 : 8192); }

}  // namespace
