// Softmax cross entropy out of the last linear layer, and its gradient (dcnv4_linear_cross_entropy of include/dcnv4.h):
//     logit[p][v] = sum_k x[p][k] * w[v][k] + b[v],   lse[p] = log sum_v exp(logit[p][v]),   loss[p] = lse[p] - logit[p][target[p]]
// The logits are never stored.  Forward: a workgroup makes a tile of classes x pixels on the matrix cores and reduces it to a
// maximum and a sum of exponentials per pixel; these are joined over the tiles.  Backward, a piece of the classes at a time: the
// tile again, d = softmax - onehot out of it and lse, stored in 16 bits (pixel-major and class-major), then the two products
//     grad_x[p][k] = g[p] * sum_v d[p][v] * w[v][k]        grad_w[v][k] = sum_p g[p] * d[p][v] * x[p][k]
// All products are D[i][j] = sum_r A[i][r] * B[j][r] with r contiguous in both operands, so w and x are laid out
// once more with rows and columns exchanged.
//
// fp16: d lies in [-1, 1] and a probability of 2^-24 is the least that fp16 holds, so it is stored times 2^15; for grad_w the row's g goes
// into it, as a part of the largest |g| (a power of two above it), so that any loss scale keeps its bits.
// fp32: every operand is held as three bf16 numbers (8 + 8 + 8 bits, a = h + m + l) and a product is the sum of h*h, h*m, m*h, m*m,
// h*l, l*h in fp32: what is left out is at most 2^-24 of a product.  (The fp32 matrix instructions have a sixteenth of the bf16 rate.)
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

// One operand: rows of `kbytes` bytes (a multiple of 16) in each of the planes.
struct Operand {
    const char *base;
    long long row_bytes;
    int rows, plane_bytes, kbytes;
};

struct Product {
    Operand a, b;
    int steps, steps_per_split;
    int a_tiles, tiles, tiles_per_xcd;
    FastDiv div_a;
};

// PL planes: 1 (fp16) or 3 (fp32 as three bf16).  A step is 128 bytes of a row of one plane, or 64 of each of three.
template <int PL, int WR, int WC, int WM, int WN, int STAGES> struct Tile {
    static constexpr int kWaves = WR * WC, kThreads = kWaves * 64;
    static constexpr int BM = WR * 32 * WM, BN = WC * 32 * WN;
    static constexpr int STEP = PL == 1 ? 128 : 64, UPR = STEP / 16, LANE_ROWS = 64 / UPR;
    static constexpr int LOAD_ROWS = kWaves * LANE_ROWS;
    static constexpr int LA = BM / LOAD_ROWS, LB = BN / LOAD_ROWS, LOADS = (LA + LB) * PL;
    static_assert(LA * LOAD_ROWS == BM && LB * LOAD_ROWS == BN);
    static constexpr int PLANE = (BM + BN) * STEP, STAGE = PL * PLANE;
    static constexpr int OUT_A = 32 * WM * 4 + 16, OUT_B = 32 * WN * 4 + 16;   // rows of results on their way out, at most
    static constexpr int OUT = kWaves * 32 * (OUT_A > OUT_B ? OUT_A : OUT_B);
    static constexpr int LDS = STAGES * STAGE > OUT ? STAGES * STAGE : OUT;
    static constexpr int kWavesPerSimd = kWaves / 4 * (LDS > 80 * 1024 ? 1 : 2);     // that registers have to leave room for

    // 16-byte units of a row are permuted in LDS so that a fragment's reads, 16 rows at a time, fall on all banks
    static __device__ __forceinline__ int swizzle(int row) { return PL == 1 ? row & 7 : (row >> 2) & 3; }

    // acc[m][n]: rows a0 + (wr * WM + m) * 32 of A, rows b0 + (wc * WN + n) * 32 of B, steps t0 to t1 - 1
    static __device__ __forceinline__ void multiply(char *smem, const Operand &a, const Operand &b, int a0, int b0, int t0, int t1,
                                                    f32x16 (&acc)[WM][WN])
    {
        const int tid = (int)threadIdx.x, lane = tid & 63;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int wr = wave / WC, wc = wave % WC, row = lane & 31, kb = lane >> 5;
        // rows past the last are the last once more; units past the end of K lie past the descriptor and read zero
        const int a_rows = min(BM, a.rows - a0), b_rows = min(BN, b.rows - b0);
        const rsrc_t ra = make_rsrc(a.base + a0 * a.row_bytes, (unsigned)(a_rows * a.row_bytes));
        const rsrc_t rb = make_rsrc(b.base + b0 * b.row_bytes, (unsigned)(b_rows * b.row_bytes));
        const int lrow = wave * LANE_ROWS + lane / UPR;
        const int unit = (lane % UPR) ^ swizzle(lrow);
        int ao[LA], bo[LB];
#pragma unroll
        for (int i = 0; i < LA; ++i)
            ao[i] = (int)(min(i * LOAD_ROWS + lrow, a_rows - 1) * a.row_bytes) + unit * 16;
#pragma unroll
        for (int i = 0; i < LB; ++i)
            bo[i] = (int)(min(i * LOAD_ROWS + lrow, b_rows - 1) * b.row_bytes) + unit * 16;
        auto load = [&](int t, int stage) {               // past the last step: nothing is read, zeros are written
            char *to = smem + stage * STAGE + wave * 1024;
            const int at = t * STEP;
            const unsigned a_out = t < t1 && at + unit * 16 < a.kbytes ? 0u : (unsigned)kOutside;
            const unsigned b_out = t < t1 && at + unit * 16 < b.kbytes ? 0u : (unsigned)kOutside;
#pragma unroll
            for (int p = 0; p < PL; ++p) {
#pragma unroll
                for (int i = 0; i < LA; ++i)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(
                        ra, (__attribute__((address_space(3))) void *)(to + p * PLANE + i * (kWaves * 1024)), 16,
                        (int)((unsigned)(ao[i] + at + p * a.plane_bytes) | a_out), 0, 0, 0);
#pragma unroll
                for (int i = 0; i < LB; ++i)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(
                        rb, (__attribute__((address_space(3))) void *)(to + p * PLANE + (LA + i) * (kWaves * 1024)), 16,
                        (int)((unsigned)(bo[i] + at + p * b.plane_bytes) | b_out), 0, 0, 0);
            }
        };
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s)
            load(t0 + s, s);
        const int a_at = (wr * 32 * WM + row) * STEP, b_at = (BM + wc * 32 * WN + row) * STEP, sw = swizzle(row);
        int at = 0;
#pragma unroll 1
        for (int t = t0; t < t1; ++t) {
            // this step's loads have landed, for every wave, and all are done with the stage of the step before
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((STAGES - 2) * LOADS) : "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            load(t + STAGES - 1, at == 0 ? STAGES - 1 : at - 1);
            const char *stage = smem + at * STAGE;
            at = at + 1 == STAGES ? 0 : at + 1;
            auto fetch_a = [&](int p, int g, int m) {
                return *reinterpret_cast<const u32x4 *>(stage + p * PLANE + a_at + m * 32 * STEP + (((2 * g + kb) ^ sw) << 4));
            };
            auto fetch_b = [&](int p, int g, int n) {
                return *reinterpret_cast<const u32x4 *>(stage + p * PLANE + b_at + n * 32 * STEP + (((2 * g + kb) ^ sw) << 4));
            };
            if constexpr (PL == 1) {
                // fragments are read while the products of the group before them run
                u32x4 af[2][WM], bf[2][WN];
                auto fetch = [&](int g) {
#pragma unroll
                    for (int m = 0; m < WM; ++m)
                        af[g & 1][m] = fetch_a(0, g, m);
#pragma unroll
                    for (int n = 0; n < WN; ++n)
                        bf[g & 1][n] = fetch_b(0, g, n);
                };
                fetch(0);
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    if (g + 1 < 4)
                        fetch(g + 1);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int m = 0; m < WM; ++m)
#pragma unroll
                        for (int n = 0; n < WN; ++n)
                            acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, af[g & 1][m]),
                                                                               __builtin_bit_cast(f16x8, bf[g & 1][n]), acc[m][n], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                }
            } else {
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    u32x4 af[3][WM], bf[3][WN];
#pragma unroll
                    for (int p = 0; p < 3; ++p) {
#pragma unroll
                        for (int m = 0; m < WM; ++m)
                            af[p][m] = fetch_a(p, g, m);
#pragma unroll
                        for (int n = 0; n < WN; ++n)
                            bf[p][n] = fetch_b(p, g, n);
                    }
                    // small parts first
                    constexpr int pa[6] = {0, 2, 1, 0, 1, 0}, pb[6] = {2, 0, 1, 1, 0, 0};
#pragma unroll
                    for (int q = 0; q < 6; ++q)
#pragma unroll
                        for (int m = 0; m < WM; ++m)
#pragma unroll
                            for (int n = 0; n < WN; ++n)
                                acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, af[pa[q]][m]),
                                                                                    __builtin_bit_cast(bf16x8, bf[pb[q]][n]), acc[m][n], 0, 0, 0);
                }
            }
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (results go where the last loads write)
        __syncthreads();
    }
};

// The tile of this workgroup: consecutive ones to one XCD.  False: none.
__device__ __forceinline__ bool tile_of(const Product &q, int &a_tile, int &b_tile)
{
    const int tile = ((int)blockIdx.x & (kXcds - 1)) * q.tiles_per_xcd + ((int)blockIdx.x >> 3);
    if (((int)blockIdx.x >> 3) >= q.tiles_per_xcd || tile >= q.tiles)
        return false;
    b_tile = fdiv(tile, q.div_a);
    a_tile = tile - b_tile * q.a_tiles;
    return true;
}

struct Labels {
    const void *bias;                 // of the layer's type, or null
    const long long *target;
    long long ignore;
    int P, V;                         // V: all classes
    int v0, count;                    // of this launch: first class, how many
};

template <typename T> __device__ __forceinline__ float bias_of(const Labels &l, int v)
{
    return l.bias != nullptr ? (float)((const T *)l.bias)[min(v, l.V - 1)] : 0.f;
}

// The logits of a wave's classes and pixels: acc[m][n][4 * a + c] is class first + 32 * m + 8 * a + 4 * kb + c, pixel n * 32 + lane % 32.
template <typename T, int WM, int WN>
__device__ __forceinline__ void start_with_bias(const Labels &l, int first, int kb, f32x16 (&acc)[WM][WN])
{
#pragma unroll
    for (int m = 0; m < WM; ++m)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float b = bias_of<T>(l, first + 32 * m + 8 * (r / 4) + 4 * kb + r % 4);
#pragma unroll
            for (int n = 0; n < WN; ++n)
                acc[m][n][r] = b;
        }
}

__device__ __forceinline__ float other_half(float v)       // of the lane 32 away
{
    float a = v, b = v;
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b));
    return (threadIdx.x & 32) ? a : b;
}

}  // namespace

// Forward: per pixel and tile of classes the largest logit and the sum of the others' exponentials beside it: partial[a_tile][P];
// the target's logit goes to target_logit[P] (one lane of the grid has it).
template <typename T, int PL, int WR, int WC, int WM, int WN, int STAGES>
__global__ __launch_bounds__(WR * WC * 64, (Tile<PL, WR, WC, WM, WN, STAGES>::kWavesPerSimd)) void dcnv4_loss_kernel(Product q, Labels l, float2 *partial, float *target_logit)
{
    typedef Tile<PL, WR, WC, WM, WN, STAGES> G;
    __shared__ __attribute__((aligned(16))) char smem[G::LDS];
    int at, bt;
    if (!tile_of(q, at, bt))
        return;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wr = wave / WC, wc = wave % WC, kb = lane >> 5;
    const int first = at * G::BM + wr * 32 * WM;           // this wave's first class, of the launch
    f32x16 acc[WM][WN];
    start_with_bias<T, WM, WN>(l, l.v0 + first, kb, acc);
    G::multiply(smem, q.a, q.b, at * G::BM, bt * G::BN, 0, q.steps, acc);
    float2 *mine = reinterpret_cast<float2 *>(smem);       // [WR][BN]
#pragma unroll
    for (int n = 0; n < WN; ++n) {
        const int col = (wc * WN + n) * 32 + (lane & 31), px = bt * G::BN + col;
        const long long t = px < l.P ? l.target[px] : -1;
        const int want = t >= l.v0 + first && t < l.v0 + l.count && t < l.v0 + first + 32 * WM ? (int)(t - l.v0 - first) : -1;
        float top = -__builtin_inff(), hit = 0.f;
        bool have = false;
#pragma unroll
        for (int m = 0; m < WM; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int c = 32 * m + 8 * (r / 4) + 4 * kb + r % 4;
                if (first + c >= l.count)
                    acc[m][n][r] = -__builtin_inff();
                if (c == want) {
                    hit = acc[m][n][r];
                    have = true;
                }
                top = fmaxf(top, acc[m][n][r]);
            }
        if (have)
            target_logit[px] = hit;
        top = fmaxf(top, other_half(top));
        const float base = top == -__builtin_inff() ? 0.f : top;       // (no class left: a sum of zeros)
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
        partial[(long long)at * l.P + px] = make_float2(top, sum);
    }
}

// Joins the tiles' maxima and sums: 16 pixels to a workgroup, 16 tiles side by side.
__global__ __launch_bounds__(256) void dcnv4_loss_join_kernel(const float2 *partial, int tiles, const float *target_logit, Labels l, float *loss,
                                                              float *lse)
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
    const float all = top + logf(sum);
    const long long t = l.target[px];
    lse[px] = all;
    loss[px] = t == l.ignore ? 0.f : t >= 0 && t < l.V ? all - target_logit[px] : __builtin_nanf("");
}

// What the backward pass knows of its rows beforehand: scale[0], a power of two no less than the largest |g| (of finite ones), and per row
// its g: zero where the row is ignored, NaN where its target is no class.
__global__ __launch_bounds__(1024) void dcnv4_loss_rows_kernel(const float *grad_loss, Labels l, float *scale, float *g)
{
    __shared__ float most[16];
    float top = 0.f;
    for (int px = (int)threadIdx.x; px < l.P; px += 1024) {
        const long long t = l.target[px];
        const float v = t == l.ignore ? 0.f : t >= 0 && t < l.V ? grad_loss[px] : __builtin_nanf("");
        g[px] = v;
        const float size = fabsf(v);
        if (size < __builtin_inff())
            top = fmaxf(top, size);
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2)
        top = fmaxf(top, __shfl_xor(top, d));
    if ((threadIdx.x & 63) == 0)
        most[threadIdx.x >> 6] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 16; ++w)
            top = fmaxf(top, most[w]);
        int e = 0;
        frexpf(top, &e);                                   // top < 2^e
        scale[0] = top > 0.f ? ldexpf(1.f, e < -100 ? -100 : e > 127 ? 127 : e) : 1.f;
    }
}

// Rows to columns: in [rows][cols] -> out [cols][PL planes][pad], zeros behind the rows; rows whose g is zero are zeros, whatever they hold
// (g null: every row counts).  fp32 numbers are split into three on their way.  64 x 64 to a workgroup.
template <typename T, int PL>
__global__ __launch_bounds__(256) void dcnv4_loss_turn_kernel(const T *in, const float *g, int rows, int cols, int pad, unsigned short *out)
{
    __shared__ T tile[64][65];
    const int r0 = (int)blockIdx.x * 64, c0 = (int)blockIdx.y * 64, i = (int)threadIdx.x & 63, j = (int)threadIdx.x >> 6;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const int r = r0 + k * 4 + j, c = c0 + i;
        T v = (T)0.f;
        if (r < rows && c < cols && (g == nullptr || g[r] != 0.f))
            v = in[(long long)r * cols + c];
        tile[k * 4 + j][i] = v;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k) {
        const int c = c0 + k * 4 + j;
        if (c >= cols || r0 + i >= pad)
            continue;
        unsigned short *to = out + (long long)c * PL * pad + r0 + i;
        if constexpr (PL == 1) {
            to[0] = __builtin_bit_cast(unsigned short, (_Float16)tile[i][k * 4 + j]);
        } else {
            float rest = tile[i][k * 4 + j];
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                const __bf16 h = (__bf16)rest;
                rest -= (float)h;
                to[(long long)p * pad] = __builtin_bit_cast(unsigned short, h);
            }
        }
    }
}

// fp32 rows as three planes of bf16: in [rows][cols] -> out [rows][3][pad], zeros behind the columns.
__global__ __launch_bounds__(256) void dcnv4_loss_split_kernel(const float *in, long long rows, int cols, int pad, unsigned short *out)
{
    const int c = ((int)blockIdx.x * 64 + ((int)threadIdx.x & 63)) * 4;
    const long long r = (long long)blockIdx.y * 4 + ((int)threadIdx.x >> 6);
    for (long long row = r; row < rows && c < pad; row += (long long)gridDim.y * 4) {
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        if (c < cols)                                      // (columns come in eights)
            v = *reinterpret_cast<const f32x4 *>(in + row * cols + c);
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            unsigned short s[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const __bf16 h = (__bf16)v[e];
                v[e] -= (float)h;
                s[e] = __builtin_bit_cast(unsigned short, h);
            }
            *reinterpret_cast<u32x2 *>(out + (row * 3 + p) * pad + c) =
                u32x2{(unsigned)s[0] | (unsigned)s[1] << 16, (unsigned)s[2] | (unsigned)s[3] << 16};
        }
    }
}

struct Deltas {
    const float *lse, *g, *scale;
    unsigned short *by_pixel;         // [P][PL][v_pad]: d (fp16: times 2^15)
    unsigned short *by_class;         // [count][PL][p_pad]: d * g / scale (fp16: times 2^15)
    float *bias_sums;                 // [pixel runs of 32 * WN][count], or null: sums of what by_class holds
    int v_pad, p_pad;
};

// Backward, first part: the logits of a tile again, and d out of them in both layouts.
template <typename T, int PL, int WR, int WC, int WM, int WN, int STAGES>
__global__ __launch_bounds__(WR * WC * 64, (Tile<PL, WR, WC, WM, WN, STAGES>::kWavesPerSimd)) void dcnv4_loss_delta_kernel(Product q, Labels l, Deltas d)
{
    typedef Tile<PL, WR, WC, WM, WN, STAGES> G;
    __shared__ __attribute__((aligned(16))) char smem[G::LDS];
    int at, bt;
    if (!tile_of(q, at, bt))
        return;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wr = wave / WC, wc = wave % WC, row = lane & 31, kb = lane >> 5;
    const int first = at * G::BM + wr * 32 * WM, px0 = bt * G::BN + wc * 32 * WN;
    f32x16 acc[WM][WN];
    start_with_bias<T, WM, WN>(l, l.v0 + first, kb, acc);
    G::multiply(smem, q.a, q.b, at * G::BM, bt * G::BN, 0, q.steps, acc);
    const float up = PL == 1 ? kUp : 1.f, inv = 1.f / d.scale[0];
    float part[WN];                                        // of the row's g, as by_class holds it
#pragma unroll
    for (int n = 0; n < WN; ++n) {
        const int px = px0 + n * 32 + row;
        const bool in = px < l.P;
        const float g = in ? d.g[px] : 0.f, lse = in ? d.lse[px] : 0.f;
        const long long t = in ? l.target[px] : -1;
        const int want = t >= l.v0 + first && t < l.v0 + first + 32 * WM ? (int)(t - l.v0 - first) : -1;
        part[n] = g * inv;
#pragma unroll
        for (int m = 0; m < WM; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int c = 32 * m + 8 * (r / 4) + 4 * kb + r % 4;
                float v = __builtin_amdgcn_exp2f((acc[m][n][r] - lse) * kLog2e);
                if (c == want)
                    v -= 1.f;
                acc[m][n][r] = g != 0.f && first + c < l.count ? v * up : 0.f;
            }
    }
    // results in 16 bits, PL planes one after the other
    char *out = smem + wave * (G::OUT / G::kWaves);
    auto bits = [&](float &v) {
        if constexpr (PL == 1)
            return __builtin_bit_cast(unsigned short, (_Float16)v);
        const __bf16 h = (__bf16)v;
        v -= (float)h;
        return __builtin_bit_cast(unsigned short, h);
    };
    // by pixel: 32 pixels at a time, each a run of 32 * WM classes
    constexpr int ROW_P = 32 * WM * 2 + 16, UNITS_P = 32 * WM * 2 / 16;
#pragma unroll
    for (int n = 0; n < WN; ++n) {
        f32x16 rest[WM];
#pragma unroll
        for (int m = 0; m < WM; ++m)
            rest[m] = acc[m][n];
#pragma unroll
        for (int p = 0; p < PL; ++p) {
#pragma unroll
            for (int m = 0; m < WM; ++m)
#pragma unroll
                for (int a = 0; a < 4; ++a) {
                    unsigned short s[4];
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        float v = rest[m][4 * a + c];
                        s[c] = bits(v);
                        rest[m][4 * a + c] = v;
                    }
                    *reinterpret_cast<u32x2 *>(out + row * ROW_P + (32 * m + 8 * a + 4 * kb) * 2) =
                        u32x2{(unsigned)s[0] | (unsigned)s[1] << 16, (unsigned)s[2] | (unsigned)s[3] << 16};
                }
            // (the same wave wrote and reads)
#pragma unroll
            for (int it = 0; it < UNITS_P / 2; ++it) {
                const int e = it * 64 + lane, u = e % UNITS_P, r = e / UNITS_P;
                const u32x4 v = *reinterpret_cast<const u32x4 *>(out + r * ROW_P + u * 16);
                const int px = px0 + n * 32 + r, col = first + u * 8;
                if (px < l.P && col < d.v_pad)
                    *reinterpret_cast<u32x4 *>(d.by_pixel + ((long long)px * PL + p) * d.v_pad + col) = v;
            }
        }
    }
    // by class: 32 classes at a time, each a run of 32 * WN pixels
    constexpr int ROW_C = 32 * WN * 2 + 16, UNITS_C = 32 * WN * 2 / 16;
#pragma unroll
    for (int m = 0; m < WM; ++m) {
#pragma unroll
        for (int n = 0; n < WN; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r)                   // (a zero stays one, also beside an infinite g)
                acc[m][n][r] = acc[m][n][r] == 0.f ? 0.f : acc[m][n][r] * part[n];
        float sums[UNITS_C / 2];
#pragma unroll
        for (int it = 0; it < UNITS_C / 2; ++it)
            sums[it] = 0.f;
#pragma unroll
        for (int p = 0; p < PL; ++p) {
#pragma unroll
            for (int n = 0; n < WN; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    float v = acc[m][n][r];
                    *reinterpret_cast<unsigned short *>(out + (8 * (r / 4) + 4 * kb + r % 4) * ROW_C + (32 * n + row) * 2) = bits(v);
                    acc[m][n][r] = v;
                }
#pragma unroll
            for (int it = 0; it < UNITS_C / 2; ++it) {
                const int e = it * 64 + lane, u = e % UNITS_C, r = e / UNITS_C;
                const u32x4 v = *reinterpret_cast<const u32x4 *>(out + r * ROW_C + u * 16);
                const int c = first + 32 * m + r, px = px0 + u * 8;
                if (c < l.count && px < d.p_pad)
                    *reinterpret_cast<u32x4 *>(d.by_class + ((long long)c * PL + p) * d.p_pad + px) = v;
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    sums[it] += PL == 1 ? (float)__builtin_bit_cast(f16x8, v)[k] : (float)__builtin_bit_cast(bf16x8, v)[k];
            }
        }
        if (d.bias_sums != nullptr)
#pragma unroll
            for (int it = 0; it < UNITS_C / 2; ++it) {
                const int e = it * 64 + lane, u = e % UNITS_C, r = e / UNITS_C, c = first + 32 * m + r;
                float s = sums[it];
#pragma unroll
                for (int k = 1; k < UNITS_C; k *= 2)
                    s += __shfl_xor(s, k);
                if (u == 0 && c < l.count)
                    d.bias_sums[(long long)(bt * WC + wc) * l.count + c] = s;
            }
    }
}

struct Result {
    void *out;                        // [b rows][a rows] of T; or float planes, one per split
    long long plane;                  // floats
    const float *row_scale;           // by b row, or null
    const float *scale;               // one number, or null
    float factor;
    int add;                          // planes: to what is there
};

// Backward, second part: out[j][i] = scale * sum_r A[i][r] * B[j][r], whole (T) or a split of the sum (float planes).
template <typename T, bool WHOLE, int PL, int WR, int WC, int WM, int WN, int STAGES>
__global__ __launch_bounds__(WR * WC * 64, (Tile<PL, WR, WC, WM, WN, STAGES>::kWavesPerSimd)) void dcnv4_loss_product_kernel(Product q, Result o)
{
    typedef Tile<PL, WR, WC, WM, WN, STAGES> G;
    typedef std::conditional_t<WHOLE, T, float> S;
    __shared__ __attribute__((aligned(16))) char smem[G::LDS];
    int at, bt;
    if (!tile_of(q, at, bt))
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
    const int t0 = (int)blockIdx.y * q.steps_per_split, t1 = min(t0 + q.steps_per_split, q.steps);
    G::multiply(smem, q.a, q.b, at * G::BM, bt * G::BN, t0, t1, acc);
    char *out = smem + wave * (G::OUT / G::kWaves);
    const int i0 = at * G::BM + wr * 32 * WM, j0 = bt * G::BN + wc * 32 * WN;
    constexpr int ES = (int)sizeof(S), ROW = 32 * WM * ES + 16, UNITS = 32 * WM * ES / 16;
    S *to = (S *)o.out + (WHOLE ? 0 : (long long)blockIdx.y * o.plane);
    const float scale = WHOLE ? o.factor * (o.scale != nullptr ? o.scale[0] : 1.f) : 1.f;
#pragma unroll
    for (int n = 0; n < WN; ++n) {
        const int j = j0 + n * 32 + row;
        const float by = WHOLE && o.row_scale != nullptr && j < q.b.rows ? scale * o.row_scale[j] : scale;
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
            if (jj < q.b.rows && i < q.a.rows) {
                u32x4 *p = reinterpret_cast<u32x4 *>(to + (long long)jj * q.a.rows + i);
                if (!WHOLE && o.add)
                    v = __builtin_bit_cast(u32x4, __builtin_bit_cast(f32x4, v) + __builtin_bit_cast(f32x4, *p));
                *p = v;
            }
        }
    }
}

// Adds up the splits' planes [splits][rows][cols] and rounds: four numbers a lane.
template <typename T>
__global__ __launch_bounds__(256) void dcnv4_loss_sum_kernel(const float *planes, long long plane, int splits, long long n, int cols,
                                                             Result o)
{
    const float scale = o.factor * (o.scale != nullptr ? o.scale[0] : 1.f);
    const int units = cols / 4;
    for (long long i = (long long)blockIdx.x * 256 + (int)threadIdx.x; i < n / 4; i += (long long)gridDim.x * 256) {
        f32x4 v = *reinterpret_cast<const f32x4 *>(planes + i * 4);
        for (int s = 1; s < splits; ++s)
            v += *reinterpret_cast<const f32x4 *>(planes + s * plane + i * 4);
        const float by = o.row_scale != nullptr ? scale * o.row_scale[i / units] : scale;
        T t[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            t[e] = (T)(v[e] * by);
        __builtin_memcpy(__builtin_assume_aligned((T *)o.out + i * 4, 4 * sizeof(T)), t, sizeof(t));
    }
}

// grad_b: the pixel runs' sums, added up and scaled: 64 classes to a workgroup, 16 runs side by side.
template <typename T>
__global__ __launch_bounds__(1024) void dcnv4_loss_bias_kernel(const float *sums, int runs, int count, const float *scale, float factor, T *grad_b)
{
    __shared__ float part[16][64];
    const int i = (int)threadIdx.x & 63, slice = (int)threadIdx.x >> 6, c = (int)blockIdx.x * 64 + i;
    float s = 0.f;
    if (c < count)
#pragma unroll 8
        for (int r = slice; r < runs; r += 16)
            s += sums[(long long)r * count + c];
    part[slice][i] = s;
    __syncthreads();
    if (slice != 0 || c >= count)
        return;
#pragma unroll
    for (int k = 1; k < 16; ++k)
        s += part[k][i];
    grad_b[c] = (T)(s * factor * scale[0]);
}

namespace {

// Tiles by number: classes (or columns of a result) x pixels (or its rows).
enum { kSmall, kMiddle, kLarge };                          // fp16: 64x64, 128x128, 256x256; fp32: 64x64, 128x128, 256x128

// The work is planned for this many compute units (the plan gives the size of the workspace, without a device).
constexpr int kUnits = 256;
constexpr int kLossMaxRows = 1 << 20, kLossMaxClasses = 1 << 22;
// Classes of a piece: d takes P * classes numbers in each layout, this many at most.
constexpr long long kPieceNumbers = 1ll << 27;
constexpr long long kMaxPiece = 1 << 20;                   // (256 rows of d, in three planes, stay below 2 GiB)
// ... and fp32 weights, split, this many
constexpr long long kPieceWeights = 1ll << 27;

struct Shape {
    int bm, bn;
    float step, fixed, alone;          // us: a step of all tiles that a unit has at once, a tile's beginning and end, a lone tile's step
    int slots;                         // tiles of a unit side by side
};
inline const Shape &shape_of(int pl, int i)
{
    static const Shape f16[] = {{64, 64, .17f, 1.2f, .25f, 2}, {128, 128, .55f, 1.9f, .55f, 2}, {256, 256, 1.15f, 8.6f, 1.15f, 1}};
    static const Shape f32[] = {{64, 64, .45f, 1.2f, .55f, 2}, {128, 128, .85f, 2.5f, .85f, 1}, {256, 128, 1.5f, 5.f, 1.5f, 1}};
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
Choice choose_product(int pl, long long m, long long n, int steps, bool may_split)
{
    Choice best = {-1, 1};
    float best_us = 0.f;
    for (int i = kSmall; i <= kLarge; ++i) {
        if (g_loss.tile && g_loss.tile != 1 + i)
            continue;
        const Shape &s = shape_of(pl, i);
        const long long tiles = ((m + s.bm - 1) / s.bm) * ((n + s.bn - 1) / s.bn);
        for (int splits = 1; splits == 1 || (may_split && splits <= 64 && steps / splits >= 4); splits *= 2) {
            const float full = ceilf((float)(tiles * splits) / (float)kUnits);
            const int each = (steps + splits - 1) / splits;
            float us = (float)each * (s.step * full > s.alone ? s.step * full : s.alone) + s.fixed * full;
            if (splits > 1)                                // planes written and read once more, by a launch of its own
                us += 3.f + (float)(m * n) * 8e-6f * (float)splits / 4.f;
            if (best.shape < 0 || us < best_us) {
                best = {i, splits};
                best_us = us;
            }
        }
    }
    if (may_split && g_loss.splits)
        best.splits = g_loss.splits < steps ? g_loss.splits : steps;
    return best;
}

struct Plan {
    int pl, es, K, P, V;
    int kp, pp, vc, vp, pieces;        // padded K (split operands), padded P, classes of a piece and padded, pieces
    int k_steps, v_steps, p_steps;
    Choice logits, gx, gw;
    bool gx_planes, gw_planes;
    // bytes from the start of the workspace
    long long scale, g, x_turned, w_turned, by_pixel, by_class, bias_sums, x_split, w_split, gx_at, gw_at, partial, hit, bytes;
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
    p.pp = (int)round_up(P, 64);
    const long long most_d = kPieceNumbers / p.pp, most_w = kPieceWeights / p.kp;
    long long most = backward && most_d < most_w ? most_d : most_w;
    if (g_loss.piece)
        most = g_loss.piece;
    most = most < 256 ? 256 : most > kMaxPiece ? kMaxPiece : most;
    if (p.pl == 1 && !backward)
        most = V;                                          // (nothing of a piece is kept)
    p.pieces = (int)((V + most - 1) / most);
    p.vc = (int)round_up((V + p.pieces - 1) / p.pieces, 256);
    p.vc = p.vc < V ? p.vc : V;
    p.pieces = (V + p.vc - 1) / p.vc;
    p.vp = (int)round_up(p.vc, 64);
    const int step = p.pl == 1 ? 64 : 32;                  // numbers of a step
    p.k_steps = (p.kp + step - 1) / step;
    p.v_steps = p.vp / step;
    p.p_steps = p.pp / step;
    p.logits = choose_product(p.pl, p.vc, P, p.k_steps, false);
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
        const int bm = shape_of(p.pl, p.logits.shape).bm;
        const long long tiles = (long long)(p.pieces - 1) * ((p.vc + bm - 1) / bm) + (V - (p.pieces - 1) * p.vc + bm - 1) / bm;
        p.partial = take(tiles * P * 8);
        p.hit = take(P * 4);
    } else {
        p.gx = choose_product(p.pl, K, P, p.v_steps, true);
        p.gw = choose_product(p.pl, K, p.vc, p.p_steps, true);
        p.gx_planes = p.gx.splits > 1 || p.pieces > 1;
        p.gw_planes = p.gw.splits > 1;
        p.scale = take(256);
        p.g = take(P * 4);
        p.x_turned = take((long long)K * p.pl * p.pp * 2);
        p.w_turned = take((long long)K * p.pl * p.vp * 2);
        p.by_pixel = take(P * p.pl * p.vp * 2);
        p.by_class = take((long long)p.vc * p.pl * p.pp * 2);
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

Operand rows_of(const void *base, int rows, int pl, int pad)
{
    Operand o;
    o.base = (const char *)base;
    o.row_bytes = (long long)pl * pad * 2;
    o.rows = rows;
    o.plane_bytes = pad * 2;
    o.kbytes = pad * 2;
    return o;
}

Product product_of(const Operand &a, const Operand &b, int pl, const Choice &c, int steps)
{
    const Shape &s = shape_of(pl, c.shape);
    Product q;
    q.a = a;
    q.b = b;
    q.steps = steps;
    q.steps_per_split = (steps + c.splits - 1) / c.splits;
    q.a_tiles = (a.rows + s.bm - 1) / s.bm;
    q.tiles = q.a_tiles * ((b.rows + s.bn - 1) / s.bn);
    q.tiles_per_xcd = (q.tiles + kXcds - 1) / kXcds;
    q.div_a = make_div((unsigned)q.a_tiles);
    return q;
}

// Calls f with the tile's parameters (waves, blocks of a wave, stages) as constants.
template <int A, int B, int C, int D, int E> struct TileOf {
    static constexpr int WR = A, WC = B, WM = C, WN = D, STAGES = E;
};
template <int PL, typename F> int with_tile(int shape, F &&f)
{
    if constexpr (PL == 1) {
        if (shape == kLarge) return f(TileOf<4, 2, 2, 4, 2>());
        if (shape == kMiddle) return f(TileOf<2, 2, 2, 2, 2>());
        return f(TileOf<2, 2, 1, 1, 4>());
    } else {
        if (shape == kLarge) return f(TileOf<4, 2, 2, 2, 2>());
        if (shape == kMiddle) return f(TileOf<2, 2, 2, 2, 3>());
        return f(TileOf<2, 2, 1, 1, 3>());
    }
}

int launched() { return hipGetLastError() == hipSuccess ? DCNV4_OK : DCNV4_ERR_LAUNCH; }

void split_rows(const void *in, long long rows, int cols, int pad, void *out, hipStream_t s)
{
    const long long y = (rows + 3) / 4;
    hipLaunchKernelGGL(dcnv4_loss_split_kernel, dim3((unsigned)((pad + 255) / 256), (unsigned)(y < 65535 ? y : 65535)), dim3(256), 0, s,
                       (const float *)in, rows, cols, pad, (unsigned short *)out);
}

template <typename T, int PL> int loss_forward(const Plan &p, const void *x, const void *w, const Labels &labels, float *loss, float *lse, char *ws,
                                               hipStream_t s)
{
    if (PL == 3)
        split_rows(x, p.P, p.K, p.kp, ws + p.x_split, s);
    const Operand b = rows_of(PL == 3 ? (const void *)(ws + p.x_split) : x, p.P, PL, p.kp);
    int tiles = 0;
    for (int piece = 0; piece < p.pieces; ++piece) {
        Labels l = labels;
        l.v0 = piece * p.vc;
        l.count = p.V - l.v0 < p.vc ? p.V - l.v0 : p.vc;
        const char *rows = (const char *)w + (long long)l.v0 * p.K * p.es;
        if (PL == 3)
            split_rows(rows, l.count, p.K, p.kp, ws + p.w_split, s);
        const Product q = product_of(rows_of(PL == 3 ? ws + p.w_split : rows, l.count, PL, p.kp), b, PL, p.logits, p.k_steps);
        with_tile<PL>(p.logits.shape, [&](auto t) {
            typedef decltype(t) G;
            hipLaunchKernelGGL((dcnv4_loss_kernel<T, PL, G::WR, G::WC, G::WM, G::WN, G::STAGES>), dim3((unsigned)(q.tiles_per_xcd * kXcds)),
                               dim3(G::WR * G::WC * 64), 0, s, q, l, (float2 *)(ws + p.partial) + (long long)tiles * p.P, (float *)(ws + p.hit));
            return 0;
        });
        tiles += q.a_tiles;
    }
    hipLaunchKernelGGL(dcnv4_loss_join_kernel, dim3((unsigned)((p.P + 15) / 16)), dim3(256), 0, s, (const float2 *)(ws + p.partial), tiles,
                       (const float *)(ws + p.hit), labels, loss, lse);
    return launched();
}

template <typename T, int PL>
void launch_product(const Product &q, const Choice &c, bool planes, const Result &o, hipStream_t s)
{
    with_tile<PL>(c.shape, [&](auto t) {
        typedef decltype(t) G;
        const dim3 grid((unsigned)(q.tiles_per_xcd * kXcds), (unsigned)c.splits), block(G::WR * G::WC * 64);
        if (planes)
            hipLaunchKernelGGL((dcnv4_loss_product_kernel<T, false, PL, G::WR, G::WC, G::WM, G::WN, G::STAGES>), grid, block, 0, s, q, o);
        else
            hipLaunchKernelGGL((dcnv4_loss_product_kernel<T, true, PL, G::WR, G::WC, G::WM, G::WN, G::STAGES>), grid, block, 0, s, q, o);
        return 0;
    });
}

template <typename T> void sum_planes(const void *planes, int splits, long long rows, int cols, const Result &o, hipStream_t s)
{
    const long long n = rows * cols, groups = (n / 4 + 255) / 256;
    hipLaunchKernelGGL((dcnv4_loss_sum_kernel<T>), dim3((unsigned)(groups < 8192 ? groups : 8192)), dim3(256), 0, s, (const float *)planes, n, splits,
                       n, cols, o);
}

template <typename T, int PL>
int loss_backward(const Plan &p, const void *x, const void *w, const Labels &labels, const float *lse, const float *grad_loss, void *grad_x,
                  void *grad_w, void *grad_b, char *ws, hipStream_t s)
{
    float *scale = (float *)(ws + p.scale), *g = (float *)(ws + p.g);
    unsigned short *x_turned = (unsigned short *)(ws + p.x_turned), *w_turned = (unsigned short *)(ws + p.w_turned);
    hipLaunchKernelGGL(dcnv4_loss_rows_kernel, dim3(1), dim3(1024), 0, s, grad_loss, labels, scale, g);
    hipLaunchKernelGGL((dcnv4_loss_turn_kernel<T, PL>), dim3((unsigned)(p.pp / 64), (unsigned)((p.K + 63) / 64)), dim3(256), 0, s, (const T *)x,
                       (const float *)g, p.P, p.K, p.pp, x_turned);
    if (PL == 3)
        split_rows(x, p.P, p.K, p.kp, ws + p.x_split, s);
    const Operand xo = rows_of(PL == 3 ? (const void *)(ws + p.x_split) : x, p.P, PL, p.kp);
    const float down = PL == 1 ? kDown : 1.f;
    for (int piece = 0; piece < p.pieces; ++piece) {
        Labels l = labels;
        l.v0 = piece * p.vc;
        l.count = p.V - l.v0 < p.vc ? p.V - l.v0 : p.vc;
        const char *rows = (const char *)w + (long long)l.v0 * p.K * p.es;
        const int vp = (int)round_up(l.count, 64), v_steps = vp / (PL == 1 ? 64 : 32);      // (nothing behind them is written or read)
        hipLaunchKernelGGL((dcnv4_loss_turn_kernel<T, PL>), dim3((unsigned)(vp / 64), (unsigned)((p.K + 63) / 64)), dim3(256), 0, s, (const T *)rows,
                           (const float *)nullptr, l.count, p.K, vp, w_turned);
        if (PL == 3)
            split_rows(rows, l.count, p.K, p.kp, ws + p.w_split, s);
        // d
        Deltas d;
        d.lse = lse;
        d.g = g;
        d.scale = scale;
        d.by_pixel = (unsigned short *)(ws + p.by_pixel);
        d.by_class = (unsigned short *)(ws + p.by_class);
        d.bias_sums = grad_b != nullptr ? (float *)(ws + p.bias_sums) : nullptr;
        d.v_pad = vp;
        d.p_pad = p.pp;
        const Product q = product_of(rows_of(PL == 3 ? ws + p.w_split : rows, l.count, PL, p.kp), xo, PL, p.logits, p.k_steps);
        int runs = 0;
        with_tile<PL>(p.logits.shape, [&](auto t) {
            typedef decltype(t) G;
            runs = q.tiles / q.a_tiles * G::WC;
            hipLaunchKernelGGL((dcnv4_loss_delta_kernel<T, PL, G::WR, G::WC, G::WM, G::WN, G::STAGES>), dim3((unsigned)(q.tiles_per_xcd * kXcds)),
                               dim3(G::WR * G::WC * 64), 0, s, q, l, d);
            return 0;
        });
        if (grad_b != nullptr)
            hipLaunchKernelGGL((dcnv4_loss_bias_kernel<T>), dim3((unsigned)((l.count + 63) / 64)), dim3(1024), 0, s, (const float *)d.bias_sums, runs,
                               l.count, (const float *)scale, down, (T *)grad_b + l.v0);
        // grad_x, over the pieces
        const Operand wt = rows_of(w_turned, p.K, PL, vp), dp = rows_of(d.by_pixel, p.P, PL, vp);
        Result ox = {grad_x, 0, g, nullptr, down, 0};
        const Product qx = product_of(wt, dp, PL, p.gx, v_steps);
        if (p.gx_planes) {
            Result o = {ws + p.gx_at, (long long)p.P * p.K, nullptr, nullptr, 1.f, piece > 0};
            launch_product<T, PL>(qx, p.gx, true, o, s);
            if (piece == p.pieces - 1)
                sum_planes<T>(ws + p.gx_at, p.gx.splits, p.P, p.K, ox, s);
        } else {
            launch_product<T, PL>(qx, p.gx, false, ox, s);
        }
        // grad_w of the piece
        const Operand xt = rows_of(x_turned, p.K, PL, p.pp), dc = rows_of(d.by_class, l.count, PL, p.pp);
        Result ow = {(char *)grad_w + (long long)l.v0 * p.K * p.es, 0, nullptr, scale, down, 0};
        const Product qw = product_of(xt, dc, PL, p.gw, p.p_steps);
        if (p.gw_planes) {
            Result o = {ws + p.gw_at, (long long)l.count * p.K, nullptr, nullptr, 1.f, 0};
            launch_product<T, PL>(qw, p.gw, true, o, s);
            sum_planes<T>(ws + p.gw_at, p.gw.splits, l.count, p.K, ow, s);
        } else {
            launch_product<T, PL>(qw, p.gw, false, ow, s);
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
