// Softmax cross entropy out of the last linear layer, and its gradient (dcnv4_linear_cross_entropy of include/dcnv4.h):
//     logit[p][v] = sum_k x[p][k] * w[v][k] + b[v],   lse[p] = log sum_v exp(logit[p][v]),   loss[p] = lse[p] - logit[p][target[p]]
// The logits are never stored.  Forward: a workgroup makes a tile of classes x pixels on the matrix cores and reduces it to a
// maximum and a sum of exponentials per pixel; these are joined over the tiles.  Backward, a piece of the classes at a time: the
// tile again, d = softmax - onehot out of it and lse, stored in 16 bits, then the two products
//     grad_x[p][k] = g[p] * sum_v d[p][v] * w[v][k]        grad_w[v][k] = sum_p d[p][v] * (g[p] * x[p][k])
// All products are D[i][j] = sum_r A[i][r] * B[j][r] with the matrix instructions, which want runs of r.  w and x in the gradients' products,
// and d in the second, lie the other way round (r is their row): their tiles come to LDS as they are and are turned by
// the LDS reads that transpose 4 x 16 numbers on their way to the registers, so no tensor is laid out a second time.
// (With copies of w, x and d laid out the other way: 8192 rows, 1024 features, 40009 classes backward 2.3 ms, of which 0.35 in those.)
//
// fp16: d lies in [-1, 1] and a probability of 2^-24 is the least that fp16 holds, so it is stored times 2^15; it is rounded so once, to
// half a step of fp16, for both products.  grad_x takes its row's g afterwards, in fp32.  In grad_w's sum rows meet, so g goes into x, as a part of
// the largest |g|: where g is the same in all rows that leaves x as it is, else it is rounded to fp16 once more.  Rows of less than 2^-8 of the
// largest lie in planes of x of their own, times 2^8, 2^16 or 2^24, so that no more than eight of x's powers of two go (half of fp16's least
// step, 2^-25, is 2^-17 of such an x); the planes' products are added up in the same registers, one plane after the other.  Weights that are alike take
// one plane.  (One plane for all: rows of 10^-6 of the largest kept x to 2 %, of 10^-8 not at all.  51200 x 256, 150 classes backward: one plane 70 us,
// two 81, four 106; 8192 x 1024, 8192 classes 454, 553, 754.)
// fp32: every operand is held as three bf16 numbers (8 + 8 + 8 bits, a = h + m + l) and a product is the sum of h*h, h*m, m*h, m*m,
// h*l, l*h in fp32: what is left out is at most 2^-22 of a product.  (The fp32 matrix instructions have a sixteenth of the bf16 rate.)
//
// What bounds it: many rows and classes, the matrix units and the power they draw: 8192 rows, 1024 features, 40009 classes, fp16, forward 630
// to 740 us, backward 1990 to 2170 (0.93 to 1.1 PFLOP/s; with zeros for numbers, 4096 features, up to 1.73); 2000, 768, 10007, fp32, backward
// 505 (1.1 PFLOP/s of bf16).  Few classes, the seven launches' beginnings and ends: 51200, 256, 150, fp16, 16 and 68.  Few rows, latency:
// 64, 1024, 1000, fp16, 10 and 24.
#include <math.h>
#include <string.h>

#include <type_traits>

#include "dcnv4_common.h"

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kUp = 32768.f, kDown = 1.f / 32768.f;     // what d is stored times, in fp16
constexpr int kBands = 4, kBandBits = 8;                   // planes of x in fp16 grad_w, and the powers of two of each but the last

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
// A, B turned.
template <int PL, int WR, int WC, int WM, int WN, int R, int STAGES, bool TA = false, bool TB = false> struct Tile {
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
    template <bool TURNED, int COUNT, int LOADS_> struct Source {
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
                rows = min(COUNT, o.count - i0);
                base = o.base + i0 * o.row_bytes;
                at0 = (unit ^ swizzle(first)) * 16;
#pragma unroll
                for (int i = 0; i < LOADS_; ++i)
                    from[i] = (int)(min(i * kWaves * ROWS + first, rows - 1) * o.row_bytes) + at0;
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

    // acc[m][n]: rows a0 + (wr * WM + m) * 32 of A, rows b0 + (wc * WN + n) * 32 of B, steps t0 to t1 - 1
    static __device__ __forceinline__ void multiply(char *smem, const Operand &a, const Operand &b, int a0, int b0, int t0, int t1,
                                                    f32x16 (&acc)[WM][WN])
    {
        const int tid = (int)threadIdx.x, lane = tid & 63;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int wr = wave / WC, wc = wave % WC;
        Source<TA, BM, LA> sa(a, a0, wave, lane);
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
    }
};

// The tile and split of this workgroup: consecutive ones to one XCD, split after split (the tiles of a split read the same part of both
// operands), in the order of bands of four tiles of B and along A within a band, so that the 32 tiles that an XCD has at once
// read eight tiles of A and four of B into its L2, not 32 and one.  False: none.
__device__ __forceinline__ bool tile_of(const Product &q, int &a_tile, int &b_tile, int &split)
{
    const int at = ((int)blockIdx.x & (kXcds - 1)) * q.per_xcd + ((int)blockIdx.x >> 3);
    if (((int)blockIdx.x >> 3) >= q.per_xcd || at >= q.all)
        return false;
    split = fdiv(at, q.div_tiles);
    const int tile = at - split * q.a_tiles * q.b_tiles;
    const int band = fdiv(tile, q.div_band), rest = tile - band * 4 * q.a_tiles, wide = min(4, q.b_tiles - band * 4);
    a_tile = wide == 4 ? rest >> 2 : wide == 2 ? rest >> 1 : wide == 1 ? rest : fdiv(rest, q.div_3);
    b_tile = band * 4 + rest - a_tile * wide;
    return true;
}

struct Labels {
    const void *bias;                 // of the layer's type, or null
    const long long *target;
    long long ignore;
    int P, V;                         // V: all classes
    int v0, count;                    // of this launch: first class, how many
};

// The logits of a wave's classes and pixels: acc[m][n][4 * a + c] is class first + 32 * m + 8 * a + 4 * kb + c, pixel n * 32 + lane % 32.
template <typename T, int WM, int WN>
__device__ __forceinline__ void start_with_bias(const Labels &l, int first, int kb, f32x16 (&acc)[WM][WN])
{
    typedef T four __attribute__((ext_vector_type(4)));
    const T *bias = (const T *)l.bias;
    const bool inside = first + 32 * WM <= l.V;
#pragma unroll
    for (int m = 0; m < WM; ++m)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            const int c = first + 32 * m + 8 * a + 4 * kb;
            four b = {};
            if (bias != nullptr) {
                if (inside)
                    b = *reinterpret_cast<const four *>(bias + c);
                else
                    b = four{bias[min(c, l.V - 1)], bias[min(c + 1, l.V - 1)], bias[min(c + 2, l.V - 1)], bias[min(c + 3, l.V - 1)]};
            }
#pragma unroll
            for (int n = 0; n < WN; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc[m][n][4 * a + e] = (float)b[e];
        }
}

// Class of a wave's acc[m][n][r], from its first.
__device__ __forceinline__ int class_of(int m, int r, int kb) { return 32 * m + 8 * (r / 4) + 4 * kb + r % 4; }

// Calls f with the (m, r) of the lane's class `want`, in lanes that have it (-1: none).  Most waves have none: a few of thousands of classes.
template <int WM, typename F> __device__ __forceinline__ void at_class(int want, int kb, F &&f)
{
    if (__builtin_amdgcn_ballot_w64(want >= 0) == 0)
        return;
#pragma unroll
    for (int m = 0; m < WM; ++m)
#pragma unroll
        for (int r = 0; r < 16; ++r)
            if (class_of(m, r, kb) == want)
                f(m, r);
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

}  // namespace

// The loss of a row, from its largest logit, the sum of exponentials beside it, and its target's logit.
__device__ __forceinline__ void finish_row(const Labels &l, int px, float top, float sum, float hit, float *loss, float *lse)
{
    const float all = top + logf(sum);
    const long long t = l.target[px];
    lse[px] = all;
    loss[px] = t == l.ignore ? 0.f : t >= 0 && t < l.V ? all - hit : __builtin_nanf("");
}

// Forward: per pixel and tile of classes the largest logit and the sum of the others' exponentials beside it: partial[a_tile][P];
// the target's logit goes to target_logit[P] (one lane of the grid has it).  One tile of classes (partial null): the loss at once.
template <typename T, int PL, int WR, int WC, int WM, int WN, int R, int STAGES>
__global__ __launch_bounds__(WR * WC * 64, (Tile<PL, WR, WC, WM, WN, R, STAGES>::kWavesPerSimd)) void dcnv4_loss_kernel(Product q, Labels l, float2 *partial, float *target_logit,
                                                                                                                                             float *loss, float *lse)
{
    typedef Tile<PL, WR, WC, WM, WN, R, STAGES> G;
    __shared__ __attribute__((aligned(16))) char smem[G::LDS];
    int at, bt, split;
    if (!tile_of(q, at, bt, split))
        return;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wr = wave / WC, wc = wave % WC, kb = lane >> 5;
    const int first = at * G::BM + wr * 32 * WM;           // this wave's first class, of the launch
    f32x16 acc[WM][WN];
    start_with_bias<T, WM, WN>(l, l.v0 + first, kb, acc);
    G::multiply(smem, q.a, q.b, at * G::BM, bt * G::BN, 0, q.steps, acc);
    float2 *mine = reinterpret_cast<float2 *>(smem);       // [WR][BN]
    float *hits = reinterpret_cast<float *>(mine + WR * G::BN);
#pragma unroll
    for (int n = 0; n < WN; ++n) {
        const int col = (wc * WN + n) * 32 + (lane & 31), px = bt * G::BN + col;
        const long long t = px < l.P ? l.target[px] : -1;
        const int want = t >= l.v0 + first && t < l.v0 + l.count && t < l.v0 + first + 32 * WM ? (int)(t - l.v0 - first) : -1;
        if (first + 32 * WM > l.count)                     // (the same for the whole wave)
#pragma unroll
            for (int m = 0; m < WM; ++m)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    acc[m][n][r] = first + class_of(m, r, kb) < l.count ? acc[m][n][r] : -__builtin_inff();
        at_class<WM>(want, kb, [&](int m, int r) {
            if (partial != nullptr)
                target_logit[px] = acc[m][n][r];
            else
                hits[col] = acc[m][n][r];
        });
        float top = -__builtin_inff();
#pragma unroll
        for (int m = 0; m < WM; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                top = fmaxf(top, acc[m][n][r]);
        top = fmaxf(top, other_half(top));
        // (no class left: a sum of zeros.  The difference comes first: the product of a type's lowest value overflows)
        const float base = top == -__builtin_inff() ? 0.f : top;
        float sum = 0.f;
#pragma unroll
        for (int m = 0; m < WM; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                sum += __builtin_amdgcn_exp2f((acc[m][n][r] - base) * kLog2e);
        sum += other_half(sum);
        if (kb == 0)
            mine[wr * G::BN + col] = make_float2(top, sum);
    }
    __syncthreads();
    for (int col = (int)threadIdx.x; col < G::BN; col += G::kThreads) {
        const int px = bt * G::BN + col;
        if (px >= l.P)
            continue;
        float top = mine[col].x;
#pragma unroll
        for (int w = 1; w < WR; ++w)
            top = fmaxf(top, mine[w * G::BN + col].x);
        const float base = top == -__builtin_inff() ? 0.f : top;
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < WR; ++w)
            sum += mine[w * G::BN + col].y * __builtin_amdgcn_exp2f((mine[w * G::BN + col].x - base) * kLog2e);
        if (partial != nullptr)
            partial[(long long)at * l.P + px] = make_float2(top, sum);
        else
            finish_row(l, px, top, sum, hits[col], loss, lse);
    }
}

// Joins the tiles' maxima and sums: 16 pixels to a workgroup, 16 tiles side by side.  Of a piece of the classes: what the pieces before left in
// `all` (first: nothing) comes in last, and goes there again before the last piece gives the loss.
__global__ __launch_bounds__(256) void dcnv4_loss_join_kernel(const float2 *partial, int tiles, float2 *all, bool first, bool last,
                                                              const float *target_logit, Labels l, float *loss, float *lse)
{
    __shared__ float2 part[16][17];
    const int i = (int)threadIdx.x & 15, slice = (int)threadIdx.x >> 4, px = (int)blockIdx.x * 16 + i;
    float top = -__builtin_inff(), sum = 0.f;
    auto join = [&](float2 v) {
        const float t = fmaxf(top, v.x), base = t == -__builtin_inff() ? 0.f : t;
        sum = sum * __builtin_amdgcn_exp2f((top - base) * kLog2e) + v.y * __builtin_amdgcn_exp2f((v.x - base) * kLog2e);
        top = t;
    };
    if (px < l.P)
#pragma unroll 4
        for (int t = slice; t < tiles; t += 16)
            join(partial[(long long)t * l.P + px]);
    part[slice][i] = make_float2(top, sum);
    __syncthreads();
    if (slice != 0 || px >= l.P)
        return;
#pragma unroll
    for (int s = 1; s < 16; ++s)
        join(part[s][i]);
    if (!first)
        join(all[px]);
    if (last)
        finish_row(l, px, top, sum, target_logit[px], loss, lse);
    else
        all[px] = make_float2(top, sum);
}

// What the backward pass knows of its rows beforehand: g per row (zero where the row is ignored, NaN where its target is no class), and
// the largest and least |g| (of finite ones that are not zero; 0 and infinity where there is none) of each 1024 rows.
__device__ __forceinline__ float row_weight(const float *grad_loss, const Labels &l, long long px)
{
    const long long t = l.target[px];
    return t == l.ignore ? 0.f : t >= 0 && t < l.V ? grad_loss[px] : __builtin_nanf("");
}
// The plane of a row in fp16 grad_w, from its g over the largest: [2^-8, 1], [2^-16, 2^-8), [2^-24, 2^-16), and what is less.  (Infinities and NaN:
// the first.)
__device__ __forceinline__ int band_of(float part)
{
    const int below = -__builtin_amdgcn_frexp_expf(part);  // (the part is less than 2^-below)
    return below > 0 ? min(below / kBandBits, kBands - 1) : 0;
}

struct Sizes {
    float most, least;
    __device__ __forceinline__ void add(float g)
    {
        const float v = fabsf(g);
        if (v > 0.f && v < __builtin_inff()) {
            most = fmaxf(most, v);
            least = fminf(least, v);
        }
    }
    __device__ __forceinline__ void join(Sizes o)
    {
        most = fmaxf(most, o.most);
        least = fminf(least, o.least);
    }
    __device__ __forceinline__ void join_wave()
    {
#pragma unroll
        for (int d = 1; d < 64; d *= 2)
            join({__shfl_xor(most, d), __shfl_xor(least, d)});
    }
};

__global__ __launch_bounds__(1024) void dcnv4_loss_rows_kernel(const float *grad_loss, Labels l, Sizes *sizes, float *g)
{
    __shared__ Sizes part[16];
    const int px = (int)blockIdx.x * 1024 + (int)threadIdx.x;
    Sizes all = {0.f, __builtin_inff()};
    if (px < l.P) {
        const float v = row_weight(grad_loss, l, px);
        g[px] = v;
        all.add(v);
    }
    all.join_wave();
    if ((threadIdx.x & 63) == 0)
        part[threadIdx.x >> 6] = all;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int w = 1; w < 16; ++w)
            all.join(part[w]);
        sizes[blockIdx.x] = all;
    }
}

// What grad_w's product knows of all rows: what its sums are multiplied with in the end, and how many planes of x there are.
struct Scale {
    float by;
    int bands;
};

// Rows as the products take them: in [rows][cols] -> out [rows][PL planes][pad], zeros behind the columns, fp32 numbers split into three.
// Scaled: a row times g / the largest |g|; fp16: out [bands][rows][pad], a row times 2^(kBandBits * band) too, in the plane of its band, zeros in
// the others.  Rows whose g is zero are zeros, whatever they hold.  Few rows (parts = 0): g and the largest are made here too, a launch less.  Eight numbers a lane.
template <typename T, int PL, bool SCALED>
__global__ __launch_bounds__(256) void dcnv4_loss_rows_in_kernel(const T *in, long long rows, int cols, int pad, unsigned short *out,
                                                                 float *g, const Sizes *sizes, int parts, Scale *scale, const float *grad_loss, Labels l)
{
    float inv = 1.f;
    int bands = 1;
    if constexpr (SCALED) {
        __shared__ Sizes part[4];
        Sizes all = {0.f, __builtin_inff()};
        if (parts > 0)
            for (int i = (int)threadIdx.x; i < parts; i += 256)
                all.join(sizes[i]);
        else
            for (int i = (int)threadIdx.x; i < l.P; i += 256)
                all.add(row_weight(grad_loss, l, i));
        all.join_wave();
        if ((threadIdx.x & 63) == 0)
            part[threadIdx.x >> 6] = all;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 4; ++w)
            all.join(part[w]);
        if (all.most > 0.f) {
            inv = all.most;
            if (PL == 1) {
                const float least = all.least / inv;
                bands = least > 0.f ? 1 + band_of(least) : kBands;
            }
        }
        if (blockIdx.x == 0 && threadIdx.x == 0)
            *scale = {PL == 1 ? ldexpf(inv * kDown, (1 - bands) * kBandBits) : inv, bands};
    }
    const int units = pad / 8, unit = (int)threadIdx.x & 31;
    for (long long row = (long long)blockIdx.x * 8 + ((int)threadIdx.x >> 5); row < rows; row += (long long)gridDim.x * 8) {
        float by = 1.f;
        int band = 0;
        if constexpr (SCALED) {
            if (parts > 0) {
                by = g[row];
            } else {
                by = row_weight(grad_loss, l, row);
                if (unit == 0)
                    g[row] = by;
            }
            by /= inv;
            if (PL == 1) {
                band = band_of(by);
                by = ldexpf(by, band * kBandBits);
            }
        }
        for (int u = unit; u < units; u += 32) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] = 0.f;
            if (u * 8 < cols && by != 0.f) {               // (columns come in eights)
                T t[8];
                __builtin_memcpy(t, __builtin_assume_aligned(in + row * cols + u * 8, 16), sizeof(t));
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    v[e] = SCALED ? (float)t[e] * by : (float)t[e];
            }
            unsigned short s[8];
#pragma unroll
            for (int p = 0; p < PL; ++p) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (PL == 1) {
                        s[e] = __builtin_bit_cast(unsigned short, (_Float16)v[e]);
                    } else {
                        const __bf16 h = (__bf16)v[e];
                        v[e] -= (float)h;
                        s[e] = __builtin_bit_cast(unsigned short, h);
                    }
                }
                if constexpr (PL == 1) {
                    u32x4 v4;
                    __builtin_memcpy(&v4, s, sizeof(s));
                    for (int b = 0; b < bands; ++b)
                        *reinterpret_cast<u32x4 *>(out + (b * rows + row) * pad + u * 8) = b == band ? v4 : u32x4{};
                } else {
                    __builtin_memcpy(__builtin_assume_aligned(out + (row * PL + p) * pad + u * 8, 16), s, sizeof(s));
                }
            }
        }
    }
}

struct Deltas {
    const float *lse, *g;
    unsigned short *d;                // [P][PL][v_pad] (fp16: times 2^15), zeros behind the classes
    float *bias_sums;                 // [pixel runs of 32 * WN][count], or null: sums of g * d
    int v_pad;
};

// Backward, first part: the logits of a tile again, and d out of them.
template <typename T, int PL, int WR, int WC, int WM, int WN, int R, int STAGES>
__global__ __launch_bounds__(WR * WC * 64, (Tile<PL, WR, WC, WM, WN, R, STAGES>::kWavesPerSimd)) void dcnv4_loss_delta_kernel(Product q, Labels l, Deltas d)
{
    typedef Tile<PL, WR, WC, WM, WN, R, STAGES> G;
    __shared__ __attribute__((aligned(16))) char smem[G::LDS];
    int at, bt, split;
    if (!tile_of(q, at, bt, split))
        return;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wr = wave / WC, wc = wave % WC, row = lane & 31, kb = lane >> 5;
    const int first = at * G::BM + wr * 32 * WM, px0 = bt * G::BN + wc * 32 * WN;
    f32x16 acc[WM][WN];
    start_with_bias<T, WM, WN>(l, l.v0 + first, kb, acc);
    G::multiply(smem, q.a, q.b, at * G::BM, bt * G::BN, 0, q.steps, acc);
    float g[WN];
#pragma unroll
    for (int n = 0; n < WN; ++n) {
        const int px = px0 + n * 32 + row;
        const bool in = px < l.P;
        g[n] = in ? d.g[px] : 0.f;
        const float lse = in ? d.lse[px] : 0.f;
        const long long t = in ? l.target[px] : -1;
        const int want = t >= l.v0 + first && t < l.v0 + first + 32 * WM ? (int)(t - l.v0 - first) : -1;
#pragma unroll
        for (int m = 0; m < WM; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                acc[m][n][r] = __builtin_amdgcn_exp2f((acc[m][n][r] - lse) * kLog2e);
        at_class<WM>(want, kb, [&](int m, int r) { acc[m][n][r] -= 1.f; });
        if (first + 32 * WM > l.count)
#pragma unroll
            for (int m = 0; m < WM; ++m)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    acc[m][n][r] = first + class_of(m, r, kb) < l.count ? acc[m][n][r] : 0.f;
        if (__builtin_amdgcn_ballot_w64(g[n] == 0.f) != 0)
#pragma unroll
            for (int m = 0; m < WM; ++m)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    acc[m][n][r] = g[n] != 0.f ? acc[m][n][r] : 0.f;
    }
    if (d.bias_sums != nullptr) {
        // over the pixels of a lane, then of 32 lanes; lane i of them stores class i
#pragma unroll
        for (int m = 0; m < WM; ++m) {
            float mine = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                float s = 0.f;
#pragma unroll
                for (int n = 0; n < WN; ++n)
                    s = __builtin_fmaf(acc[m][n][r], g[n], s);
                s = sum_of_32(s);
                mine = (row & 15) == r ? s : mine;
            }
            const int c = first + class_of(m, row & 15, kb);
            if (row < 16 && c < l.count)
                d.bias_sums[(long long)(bt * WC + wc) * l.count + c] = mine;
        }
    }
    // results in 16 bits, PL planes one after the other: 32 pixels at a time, each a run of 32 * WM classes
    char *out = smem + wave * (G::OUT / G::kWaves);
    constexpr int ROW = 32 * WM * 2 + 16, UNITS = 32 * WM * 2 / 16;
#pragma unroll
    for (int n = 0; n < WN; ++n) {
#pragma unroll
        for (int p = 0; p < PL; ++p) {
#pragma unroll
            for (int m = 0; m < WM; ++m)
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    unsigned short s[4];
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const float v = acc[m][n][4 * a + c];
                        if constexpr (PL == 1) {
                            s[c] = __builtin_bit_cast(unsigned short, (_Float16)(v * kUp));
                        } else {
                            const __bf16 h = (__bf16)v;
                            acc[m][n][4 * a + c] = v - (float)h;
                            s[c] = __builtin_bit_cast(unsigned short, h);
                        }
                    }
                    *reinterpret_cast<u32x2 *>(out + row * ROW + (32 * m + 8 * a + 4 * kb) * 2) =
                        u32x2{(unsigned)s[0] | (unsigned)s[1] << 16, (unsigned)s[2] | (unsigned)s[3] << 16};
                }
            // (the same wave wrote and reads)
#pragma unroll
            for (int it = 0; it < UNITS / 2; ++it) {
                const int e = it * 64 + lane, u = e % UNITS, r = e / UNITS;
                const u32x4 v = *reinterpret_cast<const u32x4 *>(out + r * ROW + u * 16);
                const int px = px0 + n * 32 + r, col = first + u * 8;
                if (px < l.P && col < d.v_pad)
                    *reinterpret_cast<u32x4 *>(d.d + ((long long)px * PL + p) * d.v_pad + col) = v;
            }
        }
    }
}

struct Result {
    void *out;                        // [b rows][a rows] of T; or float planes, one per split
    long long plane;                  // floats
    const float *g;                   // of b rows (grad_x), or null
    const Scale *scale;               // of all (grad_w), or null
    int add;                          // planes: to what is there
};

// What a row's sum is multiplied with.
template <int PL> __device__ __forceinline__ float factor_of(const Result &o, float g)
{
    return o.g == nullptr ? o.scale->by : PL == 1 ? g * kDown : g;
}

// Backward, second part: out[j][i] = scale * sum_r A[i][r] * B[j][r], whole (T) or a split of the sum (float planes).
// A turned, B turned in the product over pixels (grad_w).
template <typename T, bool WHOLE, bool PIXELS, int PL, int WR, int WC, int WM, int WN, int R, int STAGES>
__global__ __launch_bounds__(WR * WC * 64, (Tile<PL, WR, WC, WM, WN, R, STAGES>::kWavesPerSimd)) void dcnv4_loss_product_kernel(Product q, Result o)
{
    typedef Tile<PL, WR, WC, WM, WN, R, STAGES, true, PIXELS> G;
    typedef std::conditional_t<WHOLE, T, float> S;
    __shared__ __attribute__((aligned(16))) char smem[G::LDS];
    int at, bt, split;
    if (!tile_of(q, at, bt, split))
        return;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wr = wave / WC, wc = wave % WC, row = lane & 31, kb = lane >> 5;
    f32x16 acc[WM][WN];
#pragma unroll
    for (int m = 0; m < WM; ++m)
#pragma unroll
        for (int n = 0; n < WN; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                acc[m][n][r] = 0.f;
    const int t0 = split * q.steps_per_split, t1 = min(t0 + q.steps_per_split, q.steps);
    G::multiply(smem, q.a, q.b, at * G::BM, bt * G::BN, t0, t1, acc);
    if constexpr (PIXELS && PL == 1) {
        // The other planes of x, each 2^kBandBits times less, in code of their own.  (One loop over the steps of all planes: scalar work between steps
        // and the wait for `bands` in front of the first, 6 % of the time of 8192 x 1024, 13336 classes.)
        const int bands = o.scale->bands;
        Operand a = q.a;
#pragma unroll 1
        for (int band = 1; band < bands; ++band) {
            a.base += a.length * a.row_bytes;
#pragma unroll
            for (int m = 0; m < WM; ++m)
#pragma unroll
                for (int n = 0; n < WN; ++n) {
                    asm volatile("" : "+v"(acc[m][n]));
                    acc[m][n] *= (float)(1 << kBandBits);
                    asm volatile("" : "+v"(acc[m][n]));
                }
            G::multiply(smem, a, q.b, at * G::BM, bt * G::BN, t0, t1, acc);
        }
    }
    char *out = smem + wave * (G::OUT / G::kWaves);
    const int i0 = at * G::BM + wr * 32 * WM, j0 = bt * G::BN + wc * 32 * WN;
    constexpr int ES = (int)sizeof(S), ROW = 32 * WM * ES + 16, UNITS = 32 * WM * ES / 16;
    S *to = (S *)o.out + (WHOLE ? 0 : (long long)split * o.plane);
#pragma unroll
    for (int n = 0; n < WN; ++n) {
        const int j = j0 + n * 32 + row;
        const float by = WHOLE ? factor_of<PL>(o, o.g != nullptr && j < q.b.count ? o.g[j] : 0.f) : 1.f;
#pragma unroll
        for (int m = 0; m < WM; ++m)
#pragma unroll
            for (int a = 0; a < 4; ++a) {
                S s[4];
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    s[c] = (S)(acc[m][n][4 * a + c] * by);
                __builtin_memcpy(out + row * ROW + (32 * m + 8 * a + 4 * kb) * ES, s, sizeof(s));
            }
#pragma unroll
        for (int it = 0; it < UNITS / 2; ++it) {
            const int e = it * 64 + lane, u = e % UNITS, r = e / UNITS, jj = j0 + n * 32 + r, i = i0 + u * (16 / ES);
            u32x4 v = *reinterpret_cast<const u32x4 *>(out + r * ROW + u * 16);
            if (jj < q.b.count && i < q.a.count) {
                u32x4 *p = reinterpret_cast<u32x4 *>(to + (long long)jj * q.a.count + i);
                if (!WHOLE && o.add)
                    v = __builtin_bit_cast(u32x4, __builtin_bit_cast(f32x4, v) + __builtin_bit_cast(f32x4, *p));
                *p = v;
            }
        }
    }
}

// grad_b: the pixel runs' sums, added up.
struct Bias {
    const float *sums;                // [runs][count]
    int runs, count, blocks;          // blocks: workgroups, none for no grad_b
    void *grad_b;
};

// 16 classes to a workgroup of 256, 16 runs side by side.
template <typename T> __device__ __forceinline__ void bias_of(const Bias &b, int block)
{
    __shared__ float part[16][17];
    const int i = (int)threadIdx.x & 15, slice = (int)threadIdx.x >> 4, c = block * 16 + i;
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
template <typename T> __global__ __launch_bounds__(256) void dcnv4_loss_bias_kernel(Bias b) { bias_of<T>(b, (int)blockIdx.x); }

// Adds up the splits' planes [splits][rows][cols] and rounds: four numbers a lane.  The first workgroups make grad_b, where that saves it a
// launch of its own (51200 x 256, 150 classes backward 70.6 -> 68.1 us).
template <typename T>
__global__ __launch_bounds__(256) void dcnv4_loss_sum_kernel(const float *planes, long long plane, int splits, long long n, int cols,
                                                             Result o, Bias b)
{
    if ((int)blockIdx.x < b.blocks) {
        bias_of<T>(b, (int)blockIdx.x);
        return;
    }
    const int units = cols / 4, block = (int)blockIdx.x - b.blocks, blocks = (int)gridDim.x - b.blocks;
    for (long long i = (long long)block * 256 + (int)threadIdx.x; i < n / 4; i += (long long)blocks * 256) {
        f32x4 v = *reinterpret_cast<const f32x4 *>(planes + i * 4);
#pragma unroll 8
        for (int s = 1; s < splits; ++s)
            v += *reinterpret_cast<const f32x4 *>(planes + s * plane + i * 4);
        const float by = factor_of<sizeof(T) == 2 ? 1 : 3>(o, o.g != nullptr ? o.g[i / units] : 0.f);
        T t[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            t[e] = (T)(v[e] * by);
        __builtin_memcpy(__builtin_assume_aligned((T *)o.out + i * 4, 4 * sizeof(T)), t, sizeof(t));
    }
}

namespace {

// Tiles by number: classes (or columns of a result) x pixels (or its rows).  fp16: 64x64, 128x128, 256x256; fp32: 64x64, 128x128, 256x128.
enum { kSmall, kMiddle, kLarge };

// The work is planned for this many compute units (the plan gives the size of the workspace, without a device).
constexpr int kUnits = 256;
constexpr int kFewRows = 512;        // that every workgroup looks through by itself (2000: as long as the launch it saves)
constexpr int kLossMaxRows = 1 << 20, kLossMaxClasses = 1 << 22;
// Classes of a piece: d takes P * classes numbers, this many at most (and P * 256 at least).
constexpr long long kPieceNumbers = 1ll << 27;
constexpr long long kMaxPiece = 1 << 20;                   // (256 rows of d, in three planes, stay below 2 GiB)
// ... and fp32 weights, split, this many
constexpr long long kPieceWeights = 1ll << 27;
// ... and the forward pass leaves a maximum and a sum per row and tile of classes, this many at most, which are joined piece by piece.
constexpr long long kPiecePartials = 1ll << 25;
// Logits of a launch: a grid has fewer than 2^32 lanes, and the smallest tile's make 16 logits each.
constexpr long long kLaunchLogits = 1ll << 35;

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

// Test switches (dcnv4_set_option): 0 = the library's own choice.
struct LossOptions {
    int tile = 0;                      // 1 + the tile's number
    int splits = 0;                    // workgroups to a sum, where it may be split
    int piece = 0;                     // classes of a piece
} g_loss;

struct Choice {
    int shape, splits;
};

// The tile, and over how many workgroups a sum is split, with the lowest estimated time.
Choice choose_product(int pl, long long m, long long n, int length, bool may_split)
{
    Choice best = {-1, 1};
    float best_us = 0.f;
    for (int i = kSmall; i <= kLarge; ++i) {
        if (g_loss.tile && g_loss.tile != 1 + i)
            continue;
        const Shape &s = shape_of(pl, i);
        const int steps = (length + s.r - 1) / s.r;
        const long long tiles = ((m + s.bm - 1) / s.bm) * ((n + s.bn - 1) / s.bn);
        // powers of two, and what fills the units once and twice
        const int fill = tiles < kUnits ? (int)(kUnits / tiles) : 1, tries[] = {1, 2, 4, 8, 16, 32, 64, fill, 2 * fill};
        for (const int splits : tries) {
            if (splits > 1 && (!may_split || splits > 64 || length / splits < 256))
                continue;
            const float x = (float)(tiles * splits) / (float)kUnits, full = ceilf(x), slots = (float)s.slots;
            const float rounds = x > slots ? slots * ceilf(x / slots) : full, even = s.slots > 1 && x > 1.f ? .5f * (x + full) : full;
            const float share = even + s.gen * (rounds - even);
            const float step = s.step * share > s.alone ? s.step * share : s.alone;
            float us = (float)((steps + splits - 1) / splits) * step + s.fixed * share;
            if (splits > 1)                                // planes written and read once more, by a launch of its own
                us += 2.5f + .09f * (float)splits + (float)(m * n) * (float)splits * 1.2e-6f;
            if (best.shape < 0 || us < best_us) {
                best = {i, splits};
                best_us = us;
            }
        }
    }
    if (may_split && g_loss.splits)
        best.splits = g_loss.splits;
    return best;
}

struct Plan {
    int pl, es, K, P, V;
    int kp, vc, vp, pieces;            // padded K (split operands), classes of a piece and padded, pieces
    Choice logits, gx, gw;
    bool gx_planes, gw_planes;
    // bytes from the start of the workspace
    long long scale, sizes, g, d, bias_sums, x_scaled, x_split, w_split, gx_at, gw_at, partial, all, hit, bytes;
};

long long round_up(long long v, long long to) { return (v + to - 1) / to * to; }

int make_plan(Plan *out, long long P, int K, int V, int dtype, bool backward)
{
    if (P < 1 || K < 1 || V < 1)
        return DCNV4_ERR_SHAPE;
    if (dtype != DCNV4_F32 && dtype != DCNV4_F16)
        return DCNV4_ERR_UNSUPPORTED;
    Plan p = {};
    p.es = esize(dtype);
    p.pl = dtype == DCNV4_F16 ? 1 : 3;
    if ((long long)K * p.es % 32 || P > kLossMaxRows || V > kLossMaxClasses || K > (1 << 20))
        return DCNV4_ERR_UNSUPPORTED;
    p.K = K;
    p.P = (int)P;
    p.V = V;
    p.kp = p.pl == 1 ? K : (int)round_up(K, 32);
    const long long most_d = kPieceNumbers / P, most_w = kPieceWeights / p.kp;
    long long most = backward && most_d < most_w ? most_d : most_w;
    if (g_loss.piece)
        most = g_loss.piece;
    most = most < 256 ? 256 : most > kMaxPiece ? kMaxPiece : most;
    if (p.pl == 1 && !backward && !g_loss.piece)
        most = V;                                          // (w is read as it lies, and there is no d)
    most = most < kLaunchLogits / P ? most : kLaunchLogits / P;
    p.logits = choose_product(p.pl, V < most ? V : most, P, p.kp, false);
    const int bm = shape_of(p.pl, p.logits.shape).bm;
    if (!backward && most > kPiecePartials / P * bm)
        most = kPiecePartials / P * bm;
    p.pieces = (int)((V + most - 1) / most);
    p.vc = (int)round_up((V + p.pieces - 1) / p.pieces, 256);
    p.vc = p.vc < V ? p.vc : V;
    p.pieces = (V + p.vc - 1) / p.vc;
    p.vp = (int)round_up(p.vc, 64);
    if (backward)
        p.logits = choose_product(p.pl, p.vc, P, p.kp, false);
    long long at = 0;
    auto take = [&](long long bytes) {
        const long long here = at;
        at += (long long)align256((size_t)bytes);
        return here;
    };
    if (p.pl == 3) {
        p.x_split = take(P * 6 * p.kp);
        p.w_split = take((long long)p.vc * 6 * p.kp);
    }
    if (!backward) {
        p.partial = take((p.vc + bm - 1) / bm * P * 8);
        if (p.pieces > 1)
            p.all = take(P * 8);
        p.hit = take(P * 4);
    } else {
        p.gx = choose_product(p.pl, K, P, p.vp, true);
        p.gw = choose_product(p.pl, K, p.vc, p.P, true);
        p.gx_planes = p.gx.splits > 1 || p.pieces > 1;
        p.gw_planes = p.gw.splits > 1;
        p.scale = take(sizeof(Scale));
        p.sizes = take((P + 1023) / 1024 * (long long)sizeof(Sizes));
        p.g = take(P * 4);
        p.d = take(P * p.pl * p.vp * 2);
        p.x_scaled = take(P * (p.pl == 1 ? kBands : p.pl) * p.kp * 2);
        p.bias_sums = take(round_up(P, 256) / 32 * p.vc * 4);
        if (p.gx_planes)
            p.gx_at = take(p.gx.splits * P * K * 4);
        if (p.gw_planes)
            p.gw_at = take((long long)p.gw.splits * p.vc * K * 4);
    }
    p.bytes = at > 0 ? at : 256;
    *out = p;
    return DCNV4_OK;
}

// Rows [rows][PL planes][pad] of 16 bits, `cols` of which count: as they are, or turned.
Operand rows_of(const void *base, int rows, int cols, int pl, int pad)
{
    return {(const char *)base, (long long)pl * pad * 2, rows, cols, pad * 2};
}
Operand turned(const Operand &o) { return {o.base, o.row_bytes, o.length, o.count, o.plane_bytes}; }

Product product_of(const Operand &a, const Operand &b, int pl, const Choice &c)
{
    const Shape &s = shape_of(pl, c.shape);
    Product q;
    q.a = a;
    q.b = b;
    q.steps = (b.length + s.r - 1) / s.r;
    q.steps_per_split = (q.steps + c.splits - 1) / c.splits;
    q.a_tiles = (a.count + s.bm - 1) / s.bm;
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

void split_rows(const void *in, long long rows, int cols, int pad, void *out, hipStream_t s)
{
    hipLaunchKernelGGL((dcnv4_loss_rows_in_kernel<float, 3, false>), dim3(row_groups(rows)), dim3(256), 0, s, (const float *)in, rows, cols, pad,
                       (unsigned short *)out, (float *)nullptr, (const Sizes *)nullptr, 0, (Scale *)nullptr, (const float *)nullptr, Labels{});
}

template <typename T, int PL> int loss_forward(const Plan &p, const void *x, const void *w, const Labels &labels, float *loss, float *lse, char *ws,
                                               hipStream_t s)
{
    if (PL == 3)
        split_rows(x, p.P, p.K, p.kp, ws + p.x_split, s);
    const Operand b = rows_of(PL == 3 ? (const void *)(ws + p.x_split) : x, p.P, p.kp, PL, p.kp);
    for (int piece = 0; piece < p.pieces; ++piece) {
        Labels l = labels;
        l.v0 = piece * p.vc;
        l.count = p.V - l.v0 < p.vc ? p.V - l.v0 : p.vc;
        const char *rows = (const char *)w + (long long)l.v0 * p.K * p.es;
        if (PL == 3)
            split_rows(rows, l.count, p.K, p.kp, ws + p.w_split, s);
        const Product q = product_of(rows_of(PL == 3 ? ws + p.w_split : rows, l.count, p.kp, PL, p.kp), b, PL, p.logits);
        const bool one = p.pieces == 1 && q.a_tiles == 1;
        with_tile<PL>(p.logits.shape, [&](auto t) {
            typedef decltype(t) G;
            hipLaunchKernelGGL((dcnv4_loss_kernel<T, PL, G::WR, G::WC, G::WM, G::WN, G::R, G::STAGES>), dim3((unsigned)(q.per_xcd * kXcds)),
                               dim3(G::WR * G::WC * 64), 0, s, q, l, one ? nullptr : (float2 *)(ws + p.partial),
                               (float *)(ws + p.hit), loss, lse);
            return 0;
        });
        if (!one)
            hipLaunchKernelGGL(dcnv4_loss_join_kernel, dim3((unsigned)((p.P + 15) / 16)), dim3(256), 0, s, (const float2 *)(ws + p.partial), q.a_tiles,
                               (float2 *)(ws + p.all), piece == 0, piece == p.pieces - 1, (const float *)(ws + p.hit), labels, loss, lse);
    }
    return launched();
}

template <typename T, int PL, bool PIXELS>
void launch_product(const Product &q, const Choice &c, bool planes, const Result &o, hipStream_t s)
{
    with_tile<PL>(c.shape, [&](auto t) {
        typedef decltype(t) G;
        const dim3 grid((unsigned)(q.per_xcd * kXcds)), block(G::WR * G::WC * 64);
        if (planes)
            hipLaunchKernelGGL((dcnv4_loss_product_kernel<T, false, PIXELS, PL, G::WR, G::WC, G::WM, G::WN, G::R, G::STAGES>), grid, block, 0, s, q, o);
        else
            hipLaunchKernelGGL((dcnv4_loss_product_kernel<T, true, PIXELS, PL, G::WR, G::WC, G::WM, G::WN, G::R, G::STAGES>), grid, block, 0, s, q, o);
        return 0;
    });
}

template <typename T> void sum_planes(const void *planes, int splits, long long rows, int cols, const Result &o, const Bias &b, hipStream_t s)
{
    const long long n = rows * cols, groups = (n / 4 + 255) / 256;
    hipLaunchKernelGGL((dcnv4_loss_sum_kernel<T>), dim3((unsigned)((groups < 8192 ? groups : 8192) + b.blocks)), dim3(256), 0, s,
                       (const float *)planes, n, splits, n, cols, o, b);
}

template <typename T, int PL>
int loss_backward(const Plan &p, const void *x, const void *w, const Labels &labels, const float *lse, const float *grad_loss, void *grad_x,
                  void *grad_w, void *grad_b, char *ws, hipStream_t s)
{
    Scale *scale = (Scale *)(ws + p.scale);
    Sizes *sizes = (Sizes *)(ws + p.sizes);
    float *g = (float *)(ws + p.g);
    const int parts = p.P <= kFewRows ? 0 : (p.P + 1023) / 1024;
    if (parts > 0)
        hipLaunchKernelGGL(dcnv4_loss_rows_kernel, dim3((unsigned)parts), dim3(1024), 0, s, grad_loss, labels, sizes, g);
    hipLaunchKernelGGL((dcnv4_loss_rows_in_kernel<T, PL, true>), dim3(row_groups(p.P)), dim3(256), 0, s, (const T *)x, (long long)p.P, p.K, p.kp,
                       (unsigned short *)(ws + p.x_scaled), g, (const Sizes *)sizes, parts, scale, grad_loss, labels);
    if (PL == 3)
        split_rows(x, p.P, p.K, p.kp, ws + p.x_split, s);
    const Operand xo = rows_of(PL == 3 ? (const void *)(ws + p.x_split) : x, p.P, p.kp, PL, p.kp);
    const Operand xg = turned(rows_of(ws + p.x_scaled, p.P, p.K, PL, p.kp));
    for (int piece = 0; piece < p.pieces; ++piece) {
        Labels l = labels;
        l.v0 = piece * p.vc;
        l.count = p.V - l.v0 < p.vc ? p.V - l.v0 : p.vc;
        const char *rows = (const char *)w + (long long)l.v0 * p.K * p.es;
        const int vp = (int)round_up(l.count, 64);         // (nothing behind them is written or read)
        if (PL == 3)
            split_rows(rows, l.count, p.K, p.kp, ws + p.w_split, s);
        const void *wrows = PL == 3 ? (const void *)(ws + p.w_split) : rows;
        // d
        const Deltas d = {lse, g, (unsigned short *)(ws + p.d), grad_b != nullptr ? (float *)(ws + p.bias_sums) : nullptr, vp};
        const Product q = product_of(rows_of(wrows, l.count, p.kp, PL, p.kp), xo, PL, p.logits);
        int runs = 0;
        with_tile<PL>(p.logits.shape, [&](auto t) {
            typedef decltype(t) G;
            runs = q.b_tiles * G::WC;
            hipLaunchKernelGGL((dcnv4_loss_delta_kernel<T, PL, G::WR, G::WC, G::WM, G::WN, G::R, G::STAGES>), dim3((unsigned)(q.per_xcd * kXcds)),
                               dim3(G::WR * G::WC * 64), 0, s, q, l, d);
            return 0;
        });
        Bias bias = {};
        if (grad_b != nullptr)
            bias = {d.bias_sums, runs, l.count, (l.count + 15) / 16, (T *)grad_b + l.v0};
        if (bias.blocks > 0 && !p.gw_planes)
            hipLaunchKernelGGL((dcnv4_loss_bias_kernel<T>), dim3((unsigned)bias.blocks), dim3(256), 0, s, bias);
        // grad_x, over the pieces
        const Result ox = {grad_x, 0, g, nullptr, 0};
        const Product qx = product_of(turned(rows_of(wrows, l.count, p.K, PL, p.kp)), rows_of(d.d, p.P, vp, PL, vp), PL, p.gx);
        if (p.gx_planes) {
            const Result o = {ws + p.gx_at, (long long)p.P * p.K, nullptr, nullptr, piece > 0};
            launch_product<T, PL, false>(qx, p.gx, true, o, s);
            if (piece == p.pieces - 1)
                sum_planes<T>(ws + p.gx_at, p.gx.splits, p.P, p.K, ox, Bias{}, s);
        } else {
            launch_product<T, PL, false>(qx, p.gx, false, ox, s);
        }
        // grad_w of the piece
        const Result ow = {(char *)grad_w + (long long)l.v0 * p.K * p.es, 0, nullptr, scale, 0};
        const Product qw = product_of(xg, turned(rows_of(d.d, p.P, l.count, PL, vp)), PL, p.gw);
        if (p.gw_planes) {
            const Result o = {ws + p.gw_at, (long long)l.count * p.K, nullptr, scale, 0};
            launch_product<T, PL, true>(qw, p.gw, true, o, s);
            sum_planes<T>(ws + p.gw_at, p.gw.splits, l.count, p.K, ow, bias, s);
        } else {
            launch_product<T, PL, true>(qw, p.gw, false, ow, s);
        }
    }
    return launched();
}

bool off16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

}  // namespace

int loss_set_option(const char *key, int value)
{
    if (!strcmp(key, "reset"))
        g_loss = LossOptions();
    else if (!strcmp(key, "loss_tile") && value >= 0 && value <= 3)
        g_loss.tile = value;
    else if (!strcmp(key, "loss_splits") && value >= 0 && value <= 64)
        g_loss.splits = value;
    else if (!strcmp(key, "loss_piece") && value >= 0)
        g_loss.piece = value;
    else
        return DCNV4_ERR_UNSUPPORTED;
    return DCNV4_OK;
}

extern "C" {

long long dcnv4_linear_cross_entropy_workspace_bytes(long long P, int K, int V, int dtype, int backward)
{
    Plan p;
    return make_plan(&p, P, K, V, dtype, backward != 0) == DCNV4_OK ? p.bytes : -1;
}

int dcnv4_linear_cross_entropy(const void *x, const void *w, const void *b, const long long *target, float *loss, float *lse, void *workspace,
                               long long workspace_bytes, long long P, int K, int V, long long ignore_index, int dtype, void *stream)
{
    if (!x || !w || !target || !loss || !lse || !workspace)
        return DCNV4_ERR_NULL;
    Plan p;
    const int rc = make_plan(&p, P, K, V, dtype, false);
    if (rc)
        return rc;
    if (workspace_bytes < p.bytes)
        return DCNV4_ERR_SHAPE;
    if (off16(x) || off16(w) || off16(b) || off16(target) || off16(loss) || off16(lse) || off16(workspace))
        return DCNV4_ERR_ALIGN;
    const Labels l = {b, target, ignore_index, p.P, V, 0, V};
    hipStream_t s = (hipStream_t)stream;
    return dtype == DCNV4_F16 ? loss_forward<_Float16, 1>(p, x, w, l, loss, lse, (char *)workspace, s)
                              : loss_forward<float, 3>(p, x, w, l, loss, lse, (char *)workspace, s);
}

int dcnv4_linear_cross_entropy_backward(const void *x, const void *w, const void *b, const long long *target, const float *lse,
                                        const float *grad_loss, void *grad_x, void *grad_w, void *grad_b, void *workspace,
                                        long long workspace_bytes, long long P, int K, int V, long long ignore_index, int dtype, void *stream)
{
    if (!x || !w || !target || !lse || !grad_loss || !grad_x || !grad_w || !workspace)
        return DCNV4_ERR_NULL;
    Plan p;
    const int rc = make_plan(&p, P, K, V, dtype, true);
    if (rc)
        return rc;
    if (workspace_bytes < p.bytes)
        return DCNV4_ERR_SHAPE;
    if (off16(x) || off16(w) || off16(b) || off16(target) || off16(lse) || off16(grad_loss) || off16(grad_x) || off16(grad_w) || off16(grad_b) ||
        off16(workspace))
        return DCNV4_ERR_ALIGN;
    const Labels l = {b, target, ignore_index, p.P, V, 0, V};
    hipStream_t s = (hipStream_t)stream;
    return dtype == DCNV4_F16 ? loss_backward<_Float16, 1>(p, x, w, l, lse, grad_loss, grad_x, grad_w, grad_b, (char *)workspace, s)
                              : loss_backward<float, 3>(p, x, w, l, lse, grad_loss, grad_x, grad_w, grad_b, (char *)workspace, s);
}

}  // extern "C"
