// Layers of a network's blocks and their gradients (dcnv4_gated_linear, its backward pass and that of dcnv4_linear, of include/dcnv4.h).
//
// The gated layer: a = x Wg^T + bg, u = x Wu^T + bu, h = act(a) * u, in one kernel: a workgroup makes a tile of pairs (a, u) x pixels on the matrix cores,
// where a lane has both numbers of a pair, and stores h alone.  Backward: the tile again, out of it and grad_h
//     da = grad_h * u * act'(a),   du = grad_h * act(a)
// stored in 16 bits as d [P][2F], and the two products
//     grad_x[p] = sum_j d[p][j] * w[j],    grad_w[j] = sum_p d[p][j] * x[p]
// whose operands lie as they are and are turned on the way from LDS to registers where the product wants them turned.  grad_b's sums are of d before it
// is rounded.  a and u are not kept from the forward pass: that would hold 2F numbers a row from there to here, twice h's memory, and in fp16 round both once
// more before anything is made of them.  It would not be slower: making them again is a third of the step's products, for 12544 x 512, 2 x 2048, fp16
// 53 GFLOP, 75 us at the rate below, where 205 MB written and read are 41 us of a copy.
//
// fp16: d is rounded to fp16 once, for both products, times a power of two that puts the largest |grad_h| into [2, 4): u * act'(a) and act(a) may be as
// large as 16000 before d is infinite, and d of down to 2^-15 of the largest grad_h keeps all bits (2^-14, fp16's least normal number, is 2^-15 of what
// lies at 2); from 2^-27 on it is zero.  fp32: operands as three bf16 numbers, six products.
//
// What bounds it: large layers the matrix units, under the card's power limit, and the results of tiles; small ones the steps of a tile one after the
// other.  fp16, 12544 x 512, 2 x 2048: h 68 + 7 us (700 TFLOP/s; a library's product with K = 512 reaches 680), d 92 + 8 (with 102 MB written), both
// gradients 119 (890 TFLOP/s, matrix units busy 48 % of the time), the sums' planes 10; 12544 x 2048 -> 512, backward: 69 (770 TFLOP/s) + 11.
// fp32, 3001 x 256, 2 x 680: 23, 30, 29 and 16 (140 TFLOP/s of fp32 in the gradients, six times that in bf16).  49 x 1024, 2 x 2728: 7.7 us, 16 steps.
#include <math.h>
#include <string.h>

#include <type_traits>

#include "dcnv4_product.h"

namespace {

constexpr float kLog2e = 1.44269504088896340736f;

// act(a) and its derivative.  EXACT (fp32): by the library's functions.  Else, for results of 11 bits: the hardware's exp2 and reciprocal, and
// the normal distribution function of -|a| as exp(-a^2 / 2) * t * p(t), t = 1 / (1 + 0.43 |a| / sqrt 2), p of degree 7: erfc(z) exp(z^2) is
// smooth in such a t; the coefficients are a minimax fit of it, 1.8e-7 relative, made for this for z up to 12.
struct Act {
    float value, slope;
};
template <int ACT, bool EXACT> __device__ __forceinline__ Act activation(float a)
{
    if constexpr (ACT == DCNV4_SILU) {
        const float s = EXACT ? 1.f / (1.f + expf(-a)) : __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(a * -kLog2e));
        const float v = a * s;
        return {v, __builtin_fmaf(v, 1.f - s, s)};
    } else {
        const float square = a * a;
        float lower, bell;                                 // the distribution function at -|a|, exp(-a^2 / 2)
        if constexpr (EXACT) {
            bell = expf(-.5f * square);
            lower = .5f * erfcf(fabsf(a) * .70710678118654752440f);
        } else {
            bell = __builtin_amdgcn_exp2f(square * (-.5f * kLog2e));
            const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(fabsf(a), .43f * .70710678118654752440f, 1.f));
            float p = .0709221512f;
            p = __builtin_fmaf(p, t, -.299080256f);
            p = __builtin_fmaf(p, t, .364815278f);
            p = __builtin_fmaf(p, t, -.0688891833f);
            p = __builtin_fmaf(p, t, .238243611f);
            p = __builtin_fmaf(p, t, .207459638f);
            p = __builtin_fmaf(p, t, .243989955f);
            p = __builtin_fmaf(p, t, .242538629f);
            lower = .5f * t * p * bell;
        }
        const float phi = a < 0.f ? lower : 1.f - lower;
        return {a * phi, __builtin_fmaf(a * .39894228040143267794f, bell, phi)};
    }
}

// Sixteen numbers of each lane summed over the lane's half of the wave: lane i gets the sum of number i % 16.  Lanes whose numbers differ in a bit exchange
// halves of what they still have: 15 additions and one, where each number's own sum would take five.
__device__ __forceinline__ float sums_of_32(float (&v)[16])
{
    const int lane = (int)threadIdx.x & 63;
    auto halve = [&](auto ctrl, int bit, int left) {
        const bool up = (lane & bit) != 0;
#pragma unroll
        for (int i = 0; i < left; ++i) {
            const float keep = up ? v[i + left] : v[i], give = up ? v[i] : v[i + left];
            v[i] = keep + dpp<decltype(ctrl)::value>(give);
        }
    };
    // (mirrors change more bits than one: the lane on the other side has the other half, and the same numbers of the halves before)
    halve(std::integral_constant<int, 0x140>(), 8, 8);     // row_mirror: lane 15 - i
    halve(std::integral_constant<int, 0x141>(), 4, 4);     // row_half_mirror: lane 7 - i of eight
    halve(std::integral_constant<int, 0x4E>(), 2, 2);      // quad_perm [2,3,0,1]
    halve(std::integral_constant<int, 0xB1>(), 1, 1);      // quad_perm [1,0,3,2]
    float a = v[0], b = v[0];
    asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(a), "+v"(b));
    return a + b;
}

struct Pairs {
    const void *bias;                                      // [2][F] of the layer's type, or null
    int F, P;
};

// Pair of a wave's acc[m][n][4 * a + c] (a < 2), from its first.
__device__ __forceinline__ int pair_of(int m, int a, int kb) { return 16 * m + 8 * a + 4 * kb; }

template <typename T, int WM, int WN>
__device__ __forceinline__ void start_with_bias(const Pairs &l, int first, int kb, f32x16 (&acc)[WM][WN])
{
    typedef T four __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int m = 0; m < WM; ++m)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            four b = {};
            if (l.bias != nullptr)                         // (F is a multiple of eight: four are inside or outside)
                b = *reinterpret_cast<const four *>((const T *)l.bias + min(first + pair_of(m, a & 1, kb), l.F - 4) + (a < 2 ? 0 : l.F));
#pragma unroll
            for (int n = 0; n < WN; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    acc[m][n][4 * a + e] = (float)b[e];
        }
}

}  // namespace

// h of a tile.
template <typename T, int PL, int ACT, int WR, int WC, int WM, int WN, int R, int STAGES>
__global__ __launch_bounds__(WR * WC * 64, (Tile<PL, WR, WC, WM, WN, R, STAGES>::kWavesPerSimd)) void dcnv4_gated_kernel(Product q, Pairs l, T *h)
{
    typedef Tile<PL, WR, WC, WM, WN, R, STAGES, false, false, true> G;
    __shared__ __attribute__((aligned(16))) char smem[G::LDS];
    int at, bt, split;
    if (!tile_of(q, (int)blockIdx.x, at, bt, split))
        return;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wr = wave / WC, wc = wave % WC, row = lane & 31, kb = lane >> 5;
    const int first = at * (G::BM / 2) + wr * 16 * WM, px0 = bt * G::BN + wc * 32 * WN;
    f32x16 acc[WM][WN];
    start_with_bias<T, WM, WN>(l, first, kb, acc);
    G::multiply(smem, q.a, q.b, at * (G::BM / 2), bt * G::BN, 0, q.steps, acc);
    // 32 pixels at a time, each a run of 16 * WM numbers
    char *out = smem + wave * (G::OUT / G::kWaves);
    constexpr int ES = (int)sizeof(T), ROW = 16 * WM * ES + 16, UNITS = 16 * WM * ES / 16;
#pragma unroll
    for (int n = 0; n < WN; ++n) {
#pragma unroll
        for (int m = 0; m < WM; ++m)
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                T t[4];
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    t[c] = (T)(activation<ACT, PL == 3>(acc[m][n][4 * a + c]).value * acc[m][n][4 * (a + 2) + c]);
                __builtin_memcpy(out + row * ROW + pair_of(m, a, kb) * ES, t, sizeof(t));
            }
        // (the same wave wrote and reads)
#pragma unroll
        for (int it = 0; it < (UNITS + 1) / 2; ++it) {
            const int e = it * 64 + lane, u = e % UNITS, r = e / UNITS, px = px0 + n * 32 + r, f = first + u * (16 / ES);
            const u32x4 v = *reinterpret_cast<const u32x4 *>(out + r * ROW + u * 16);
            if (px < l.P && f < l.F)
                *reinterpret_cast<u32x4 *>(h + (long long)px * l.F + f) = v;
        }
    }
}

namespace {

// What a product's result is multiplied with in the end, where its operand was scaled.
struct Scale {
    float by;
};

struct Deltas {
    const void *grad_h;
    unsigned short *d;                                     // [P][PL planes][2F]
    float *bias_sums;                                      // [pixel runs of 32 * WN][2F], or null
    const float *most;                                     // fp16: largest |grad_h| of `parts` parts; no parts: grad_h (of the one launch) has `few` numbers
    int parts, few;
    Scale *scale;                                          // fp16: what undoes d's factor
};

// Four numbers at a byte offset.
template <typename T> __device__ __forceinline__ auto load_four(rsrc_t r, int at)
{
    typedef T four __attribute__((ext_vector_type(4)));
    if constexpr (sizeof(T) == 2)
        return __builtin_bit_cast(four, __builtin_amdgcn_raw_buffer_load_b64(r, at, 0, 0));
    else
        return __builtin_bit_cast(four, __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0));
}

struct Result {
    void *out;                                             // [b rows][a rows] of T; or float planes, one per split
    long long plane;                                       // floats
    const Scale *scale;                                    // or null
};

}  // namespace

namespace {

// The largest finite magnitude of a lane's fp16 numbers.
struct Most {
    typedef unsigned short eight __attribute__((ext_vector_type(8)));
    eight top = {};
    __device__ __forceinline__ void add(eight v)
    {
        v &= (unsigned short)0x7fff;                       // (fp16's bits without the sign are in the numbers' order)
        top = __builtin_elementwise_max(top, v < (unsigned short)0x7c00 ? v : eight{});
    }
    __device__ __forceinline__ float value() const
    {
        int v = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v = max(v, (int)top[e]);
        return (float)__builtin_bit_cast(_Float16, (unsigned short)v);
    }
};

}  // namespace

// The largest finite |grad_h| of a workgroup's part of n numbers (a multiple of eight).
__global__ __launch_bounds__(256) void dcnv4_gated_most_kernel(const unsigned short *g, long long n, float *most)
{
    __shared__ float part[4];
    Most top;
    const long long units = n / 8, stride = (long long)gridDim.x * 256;
    const Most::eight *p = reinterpret_cast<const Most::eight *>(g);
    long long i = (long long)blockIdx.x * 256 + (int)threadIdx.x;
    for (; i + 3 * stride < units; i += 4 * stride) {
        const Most::eight a = p[i], b = p[i + stride], c = p[i + 2 * stride], d = p[i + 3 * stride];
        top.add(a);
        top.add(b);
        top.add(c);
        top.add(d);
    }
    for (; i < units; i += stride)
        top.add(p[i]);
    float v = top.value();
#pragma unroll
    for (int d = 1; d < 64; d *= 2)
        v = fmaxf(v, __shfl_xor(v, d));
    if ((threadIdx.x & 63) == 0)
        part[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0)
        most[blockIdx.x] = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
}

// The tile again, and d out of it.
template <typename T, int PL, int ACT, int WR, int WC, int WM, int WN, int R, int STAGES>
__global__ __launch_bounds__(WR * WC * 64, (Tile<PL, WR, WC, WM, WN, R, STAGES>::kWavesPerSimd)) void dcnv4_gated_delta_kernel(Product q, Pairs l, Deltas d)
{
    typedef Tile<PL, WR, WC, WM, WN, R, STAGES, false, false, true> G;
    typedef T four __attribute__((ext_vector_type(4)));
    __shared__ __attribute__((aligned(16))) char smem[G::LDS];
    int at, bt, split;
    if (!tile_of(q, (int)blockIdx.x, at, bt, split))
        return;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wr = wave / WC, wc = wave % WC, row = lane & 31, kb = lane >> 5;
    const int first = at * (G::BM / 2) + wr * 16 * WM, px0 = bt * G::BN + wc * 32 * WN;
    float top = 0.f;                                       // (asked for here, joined after the products)
    if constexpr (PL == 1) {
        for (int i = (int)threadIdx.x; i < d.parts; i += G::kThreads)
            top = fmaxf(top, d.most[i]);
        if (d.parts == 0) {                                // few numbers: all of them, a launch less
            Most most;
            for (int i = (int)threadIdx.x; i < d.few / 8; i += G::kThreads)
                most.add(reinterpret_cast<const Most::eight *>(d.grad_h)[i]);
            top = most.value();
        }
    }
    f32x16 acc[WM][WN];
    start_with_bias<T, WM, WN>(l, first, kb, acc);
    G::multiply(smem, q.a, q.b, at * (G::BM / 2), bt * G::BN, 0, q.steps, acc);
    // (all asked for at once; outside the tensor, which a wave's pixels may be altogether: zeros.  128 pixels of 2^19 numbers at most: 2^28 bytes)
    four g[WN][WM][2];
    const int pixels = max(min(l.P - px0, 32 * WN), 0);
    const rsrc_t from = make_rsrc((const T *)d.grad_h + (long long)px0 * l.F, (unsigned)(pixels * l.F * (int)sizeof(T)));
#pragma unroll
    for (int n = 0; n < WN; ++n)
#pragma unroll
        for (int m = 0; m < WM; ++m)
#pragma unroll
            for (int a = 0; a < 2; ++a) {
                const int f = first + pair_of(m, a, kb);
                g[n][m][a] = load_four<T>(from, f < l.F ? ((n * 32 + row) * l.F + f) * (int)sizeof(T) : kOutside);
            }
    float up = 1.f, down = 1.f;
    if constexpr (PL == 1) {
#pragma unroll
        for (int s = 1; s < 64; s *= 2)
            top = fmaxf(top, __shfl_xor(top, s));
        // (the products are through with the LDS.  An object of its own: every LDS read of the loop would wait for all loads)
        float *tops = reinterpret_cast<float *>(smem);
        if (lane == 0)
            tops[wave] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < G::kWaves; ++w)
            top = fmaxf(top, tops[w]);
        __syncthreads();                                   // (results go there)
        const int e = top > 0.f ? 2 - __builtin_amdgcn_frexp_expf(top) : 0;
        up = ldexpf(1.f, e);
        down = ldexpf(1.f, -e);
        if (at == 0 && bt == 0 && threadIdx.x == 0)
            d.scale->by = down;
    }
#pragma unroll
    for (int n = 0; n < WN; ++n)
#pragma unroll
        for (int m = 0; m < WM; ++m)
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const Act v = activation<ACT, PL == 3>(acc[m][n][4 * a + c]);
                    const float gh = (float)g[n][m][a][c] * up;     // (exact: a power of two)
                    acc[m][n][4 * a + c] = gh * acc[m][n][4 * (a + 2) + c] * v.slope;
                    acc[m][n][4 * (a + 2) + c] = gh * v.value;
                }
    if (d.bias_sums != nullptr) {
#pragma unroll
        for (int m = 0; m < WM; ++m) {
            float v[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                v[r] = acc[m][0][r];
#pragma unroll
                for (int n = 1; n < WN; ++n)
                    v[r] += acc[m][n][r];
            }
            const float sum = sums_of_32(v);               // lane i: of number i % 16
            const int r = row & 15, f = first + pair_of(m, r >> 2 & 1, kb) + (r & 3);
            if (row < 16 && f < l.F)
                d.bias_sums[((long long)(bt * WC + wc) * 2 + (r >> 3)) * l.F + f] = sum * down;
        }
    }
    // results in 16 bits, PL planes one after the other: 32 pixels at a time, each 16 * WM numbers of da and as many of du
    char *out = smem + wave * (G::OUT / G::kWaves);
    constexpr int HALF = 16 * WM * 2, ROW = 2 * HALF + 16, UNITS = 2 * HALF / 16;
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
                            s[c] = __builtin_bit_cast(unsigned short, (_Float16)v);
                        } else {
                            const __bf16 b = (__bf16)v;
                            acc[m][n][4 * a + c] = v - (float)b;
                            s[c] = __builtin_bit_cast(unsigned short, b);
                        }
                    }
                    *reinterpret_cast<u32x2 *>(out + row * ROW + (a < 2 ? 0 : HALF) + pair_of(m, a & 1, kb) * 2) =
                        u32x2{(unsigned)s[0] | (unsigned)s[1] << 16, (unsigned)s[2] | (unsigned)s[3] << 16};
                }
            // (the same wave wrote and reads)
#pragma unroll
            for (int it = 0; it < UNITS / 2; ++it) {
                const int e = it * 64 + lane, u = e % UNITS, r = e / UNITS, px = px0 + n * 32 + r;
                const int half = u >= UNITS / 2 ? 1 : 0, f = first + (u - half * (UNITS / 2)) * 8;
                const u32x4 v = *reinterpret_cast<const u32x4 *>(out + r * ROW + u * 16);
                if (px < l.P && f < l.F)
                    *reinterpret_cast<u32x4 *>(d.d + (((long long)px * PL + p) * 2 + half) * l.F + f) = v;
            }
        }
    }
}

// out[j][i] = scale * sum_r A[i][r] * B[j][r] of a tile, whole (T) or a split of the sum (float planes).  A turned; B turned in the product over
// pixels (grad_w).
template <typename G, typename S, int WR, int WC, int WM, int WN>
__device__ __forceinline__ void store_tile(char *smem, const Product &q, S *to, float by, int at, int bt, f32x16 (&acc)[WM][WN])
{
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wr = wave / WC, wc = wave % WC, row = lane & 31, kb = lane >> 5;
    char *out = smem + wave * (G::OUT / G::kWaves);
    const int i0 = at * G::BM + wr * 32 * WM, j0 = bt * G::BN + wc * 32 * WN;
    constexpr int ES = (int)sizeof(S), ROW = 32 * WM * ES + 16, UNITS = 32 * WM * ES / 16;
#pragma unroll
    for (int n = 0; n < WN; ++n) {
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
        // (the same wave wrote and reads)
#pragma unroll
        for (int it = 0; it < UNITS / 2; ++it) {
            const int e = it * 64 + lane, u = e % UNITS, r = e / UNITS, j = j0 + n * 32 + r, i = i0 + u * (16 / ES);
            const u32x4 v = *reinterpret_cast<const u32x4 *>(out + r * ROW + u * 16);
            if (j < q.b.count && i < q.a.count)
                *reinterpret_cast<u32x4 *>(to + (long long)j * q.a.count + i) = v;
        }
    }
}

// grad_x, or grad_w (PIXELS).
template <typename T, bool PIXELS, int PL, int WR, int WC, int WM, int WN, int R, int STAGES>
__device__ __forceinline__ void product_tile(char *smem, const Product &q, const Result &o, int block)
{
    typedef Tile<PL, WR, WC, WM, WN, R, STAGES, true, PIXELS> G;
    int at, bt, split;
    if (!tile_of(q, block, at, bt, split))
        return;
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
    if (o.plane > 0)
        store_tile<G, float, WR, WC, WM, WN>(smem, q, (float *)o.out + (long long)split * o.plane, 1.f, at, bt, acc);
    else
        store_tile<G, T, WR, WC, WM, WN>(smem, q, (T *)o.out, o.scale != nullptr ? o.scale->by : 1.f, at, bt, acc);
}

// Both gradients of a layer, and grad_b: workgroups of grad_x, of grad_w (in front of the others where they take longer, so that what is left in the end is
// short), then of grad_b.  One launch, so that the two fill the units together (5883 x 352 -> 1872 fp16: 39 us one after the other, 30 so).
namespace {

struct Gradients {
    Product x, w;
    Result to_x, to_w;
    int x_blocks, w_blocks, w_first;
    Bias bias;
};

}  // namespace

template <typename T, int PL, int WR, int WC, int WM, int WN, int R, int STAGES>
__global__ __launch_bounds__(WR * WC * 64, (Tile<PL, WR, WC, WM, WN, R, STAGES>::kWavesPerSimd)) void dcnv4_layer_gradients_kernel(Gradients q)
{
    // (the only LDS object: see bias_of)
    __shared__ __attribute__((aligned(16))) char smem[Tile<PL, WR, WC, WM, WN, R, STAGES>::LDS];
    const int block = (int)blockIdx.x, both = q.x_blocks + q.w_blocks;
    if (block >= both)
        bias_of<T>(q.bias, block - both, reinterpret_cast<float(*)[17]>(smem));
    else if (q.w_first ? block >= q.w_blocks : block < q.x_blocks)
        product_tile<T, false, PL, WR, WC, WM, WN, R, STAGES>(smem, q.x, q.to_x, q.w_first ? block - q.w_blocks : block);
    else
        product_tile<T, true, PL, WR, WC, WM, WN, R, STAGES>(smem, q.w, q.to_w, q.w_first ? block : block - q.x_blocks);
}

namespace {

struct Sum {
    const float *planes;                                   // [splits][n]
    int splits, blocks;                                    // blocks: workgroups, none for no sum
    long long n;
    Result o;
};

}  // namespace

// Adds up the splits' planes of both gradients and rounds: four numbers a lane.  The last workgroups make grad_b.
template <typename T> __global__ __launch_bounds__(256) void dcnv4_layer_sum_kernel(Sum x, Sum w, Bias b)
{
    __shared__ float part[16][17];
    int block = (int)blockIdx.x;
    if (block >= x.blocks + w.blocks) {
        bias_of<T>(b, block - x.blocks - w.blocks, part);
        return;
    }
    const bool second = block >= x.blocks;
    const Sum &q = second ? w : x;
    block -= second ? x.blocks : 0;
    const float by = q.o.scale != nullptr ? q.o.scale->by : 1.f;
    const long long n = q.n;
    for (long long i = (long long)block * 256 + (int)threadIdx.x; i < n / 4; i += (long long)q.blocks * 256) {
        f32x4 v = *reinterpret_cast<const f32x4 *>(q.planes + i * 4);
#pragma unroll 8
        for (int s = 1; s < q.splits; ++s)
            v += *reinterpret_cast<const f32x4 *>(q.planes + s * n + i * 4);
        T t[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            t[e] = (T)(v[e] * by);
        __builtin_memcpy(__builtin_assume_aligned((T *)q.o.out + i * 4, 4 * sizeof(T)), t, sizeof(t));
    }
}
template <typename T> __global__ __launch_bounds__(256) void dcnv4_layer_bias_kernel(Bias b)
{
    __shared__ float part[16][17];
    bias_of<T>(b, (int)blockIdx.x, part);
}

namespace {

// What is made in front of the products, in one launch: sums over runs of rows of g, and fp32 tensors as the products take them.
struct Ahead {
    const void *g;                                         // [P][N], N a multiple of eight; sums [runs][N]
    float *sums;
    int P, N, lanes_log, run_rows, across, blocks;         // workgroups: `across` to a run, none for no sums
    struct {
        const float *in;                                   // [rows][cols] -> out [rows][3 planes][pad] of bf16, zeros behind the columns
        unsigned short *out;
        long long rows;
        int cols, pad, blocks;
    } split[3];
};

}  // namespace

// Sums: eight columns a lane, 2^lanes_log of them side by side and 256 >> lanes_log rows.  Splits: eight numbers a lane.
// (One launch where there were four: 2047 x 384 -> 1000 fp32 backward 45 -> 38 us)
template <typename T> __global__ __launch_bounds__(256) void dcnv4_layer_ahead_kernel(Ahead q)
{
    typedef T eight __attribute__((ext_vector_type(8)));
    __shared__ float part[256][9];
    int block = (int)blockIdx.x;
    if (block < q.blocks) {
        const int run = block / q.across, lanes = 1 << q.lanes_log, side = 256 >> q.lanes_log, l = (int)threadIdx.x & (lanes - 1);
        const int c0 = (block - run * q.across) * lanes * 8, c = c0 + l * 8, r0 = run * q.run_rows, r1 = min(r0 + q.run_rows, q.P);
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (c < q.N)
#pragma unroll 4
            for (int r = r0 + ((int)threadIdx.x >> q.lanes_log); r < r1; r += side) {
                const eight t = *reinterpret_cast<const eight *>((const T *)q.g + (long long)r * q.N + c);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    v[e] += (float)t[e];
            }
#pragma unroll
        for (int e = 0; e < 8; ++e)
            part[threadIdx.x][e] = v[e];
        __syncthreads();
        // eight lanes' numbers side by side: a lane a column, over the rows in order
        for (int i = (int)threadIdx.x; i < lanes * 8; i += 256) {
            float sum = 0.f;
            for (int k = 0; k < side; ++k)
                sum += part[k * lanes + (i >> 3)][i & 7];
            if (c0 + i < q.N)
                q.sums[(long long)run * q.N + c0 + i] = sum;
        }
        return;
    }
    block -= q.blocks;
    if constexpr (sizeof(T) == 4) {
        int k = 0;
        while (k < 2 && block >= q.split[k].blocks)
            block -= q.split[k++].blocks;
        const auto &t = q.split[k];
        const int units = t.pad / 8;
        const long long all = t.rows * units;
        for (long long i = (long long)block * 256 + (int)threadIdx.x; i < all; i += (long long)t.blocks * 256) {
            const long long row = i / units;
            const int u = (int)(i - row * units);
            float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (u * 8 < t.cols)                            // (columns come in eights)
                __builtin_memcpy(v, __builtin_assume_aligned(t.in + row * t.cols + u * 8, 16), sizeof(v));
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                unsigned short s[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const __bf16 b = (__bf16)v[e];
                    v[e] -= (float)b;
                    s[e] = __builtin_bit_cast(unsigned short, b);
                }
                __builtin_memcpy(__builtin_assume_aligned(t.out + (row * 3 + p) * t.pad + u * 8, 16), s, sizeof(s));
            }
        }
    }
}

namespace {

struct LayerOptions {
    int tile = 0, splits = 0;          // as loss_tile and loss_splits
} g_layers;

constexpr int kFewNumbers = 1 << 15;                       // of grad_h, which every workgroup looks through by itself
constexpr int kLayerMaxRows = 1 << 24, kLayerMaxWidth = 1 << 20;

bool fits(const Shape &s, const Choice &c, long long m, long long n)
{
    return ((m + s.bm - 1) / s.bm) * ((n + s.bn - 1) / s.bn) * c.splits < (1 << 22);     // (a grid has fewer than 2^32 lanes)
}

// A product over pixels in one launch, or in two: as many pixels as give whole rounds of large tiles, and the others in the tile that suits them.
struct Parts {
    int count, pixels[2];
    Choice choice[2];
};

struct LayerPlan {
    int pl, es, P, K, N, kp, np;       // N: results of the layer (gated: 2F); padded in split operands
    Parts forward;
    Choice gx, gw;                     // (of one shape)
    int w_first;
    int most_parts, columns_runs, columns_rows;
    // bytes from the start of the workspace
    long long x_split, w_split, g_split, d, scale, most, bias_sums, gx_at, gw_at, bytes;
};

int check_layer(long long P, int K, int N, int dtype)
{
    if (P < 1 || K < 1 || N < 1)
        return DCNV4_ERR_SHAPE;
    if ((dtype != DCNV4_F32 && dtype != DCNV4_F16) || K % 8 || N % 8 || P > kLayerMaxRows || K > kLayerMaxWidth ||
        N > kLayerMaxWidth)
        return DCNV4_ERR_UNSUPPORTED;
    return DCNV4_OK;
}

struct Room {
    long long at = 0;
    long long take(long long bytes)
    {
        const long long here = at;
        at += (long long)align256((size_t)bytes);
        return here;
    }
};

// Tiles of pairs and pixels: the products', and in fp16 one more, half a large one by four waves, two workgroups to a unit, where one's products go on while the other
// makes its results: with few features that is most of a tile's time.  What `estimate` makes of these figures ranks the tiles: they were
// fitted to the forward kernel and the one that makes d together, of 31 layers (49 to 134400 pixels, K 32 to 2048, F 128 to 4096) in every tile, so that the
// choice costs least (0.4 % in fp16, 0 in fp32, on average), not so that it is the time, of which it is 0.5 (three rounds of large tiles: 88 for 160 us) to 0.9 (half a
// round: 47 for 53).
// Forward and d, 50176 x 256, 2 x 1024: 400, 238, 259 and 225 us by the four tiles; 8192 x 1024, 2 x 2816: 390, 268, 229, 250; 1000 x 1024, 2 x 1024: 25, 28, 53, 39.
enum { kTall = kLarge + 1, kGatedTiles };
const Shape &gated_shape(int pl, int i)
{
    static const Shape f16[] = {{64, 64, 64, 2, .347f, 1.77f, .476f, .067f}, {128, 128, 32, 2, .552f, 1.65f, .552f, 0.f},
                                {256, 256, 32, 1, 1.105f, 11.7f, 1.105f, 0.f}, {256, 128, 32, 2, .901f, 2.01f, .901f, 0.f}};
    static const Shape f32[] = {{64, 64, 64, 1, 1.68f, 2.46f, 1.68f, 0.f}, {128, 128, 32, 1, 2.38f, 4.83f, 2.38f, 0.f}, {256, 128, 32, 1, 3.85f, 1.54f, 3.85f, 0.f}};
    return (pl == 1 ? f16 : f32)[i];
}
int gated_tiles(int pl) { return pl == 1 ? kGatedTiles : kLarge + 1; }
template <int PL, typename F> int with_gated_tile(int shape, F &&f)
{
    if constexpr (PL == 1)
        if (shape == kTall) return f(TileOf<4, 1, 2, 4, 32, 3>());
    return with_tile<PL>(shape, f);
}

Choice choose_gated(int pl, int m, long long pixels, int length, int only)
{
    Choice best = {-1, 1};
    float least = 0.f;
    for (int i = 0; i < gated_tiles(pl); ++i) {
        if (only && only <= gated_tiles(pl) && only != 1 + i)
            continue;
        const float us = estimate(gated_shape(pl, i), m, pixels, length, 1);
        if (best.shape < 0 || us < least) {
            best.shape = i;
            least = us;
        }
    }
    return best;
}

// (12544 x 512, 2 x 2048, fp16: 784 large tiles for 256 units; forward and d 190 us in one launch each, 174 in two)
Parts parts_of(int pl, int m, int P, int length)
{
    Parts best = {1, {P, 0}, {choose_gated(pl, m, P, length, g_layers.tile), {0, 1}}};
    const Shape &s = gated_shape(pl, kLarge);
    const long long across = (m + s.bm - 1) / s.bm, rounds = across * ((P + s.bn - 1) / s.bn) / kUnits;
    const long long first = rounds * kUnits / across * s.bn;
    if (g_layers.tile || first <= 0 || first >= P)
        return best;
    const Choice rest = choose_gated(pl, m, P - first, length, 0);
    // (6: two launches more, in units of the estimate, which are up to two us)
    if (estimate(s, m, first, length, 1) + estimate(gated_shape(pl, rest.shape), m, P - first, length, 1) + 6.f <
        estimate(gated_shape(pl, best.choice[0].shape), m, P, length, 1))
        best = {2, {(int)first, P - (int)first}, {{kLarge, 1}, rest}};
    return best;
}

// The two products of a gradient, [P][K] over N numbers and [N][K] over P, in one launch: the tile and over how many workgroups each sum is split, with the
// lowest estimate (which is 0.7 to 0.9 of the time in us: 91 for 129, 54 for 75, 30 for 34; it is made to rank).  Workgroups that are all there at once take as long as the longest, `share` to a unit; more of them share the units, which feel a
// part (`tail`) of one of the shorter kind in the end.  A tile takes `step` for a step (alone on its unit `alone`) and `fixed`.  Planes are written and read once
// more, by a launch of its own.  Fitted to 34 layers (23 to 50176 rows, K 32 to 2048, 40 to 4096 results; every tile, 1 to 64 splits of either sum, 1950
// measurements) so that the choice costs least: 1.8 % (fp16) and 1.4 % (fp32) on average, 8 % at most.  12544, 512 -> 4096: 107 us with large tiles and 4 parts of
// grad_w, 143 with middle ones and no parts; 3001, 256 -> 1360 fp32: 42 with middle ones, 2 and 6 parts, 51 with small ones and no parts.
void choose_gradients(LayerPlan &p)
{
    struct Times {
        float step, fixed, alone;
    };
    static const Times f16[] = {{.171f, 1.08f, .336f}, {.176f, 2.24f, .275f}, {.387f, 5.46f, .592f}};
    static const Times f32[] = {{.551f, 2.33f, .652f}, {.835f, 4.81f, .835f}, {1.585f, 6.41f, 1.585f}};
    static const int tries[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};
    const bool half = p.pl == 1;
    const float tail = half ? 1.38f : .59f, per_split = half ? .144f : .09f, per_number = half ? .77e-6f : .48e-6f, sum = half ? 3.1f : 0.f;
    float best = -1.f;
    auto may = [&](int splits, int length) { return g_layers.splits ? splits == g_layers.splits : splits == 1 || length / splits >= 256; };
    auto planes = [&](int splits, long long n) { return splits > 1 ? per_split * (float)splits + (float)n * (float)splits * per_number : 0.f; };
    for (int i = kSmall; i <= kLarge; ++i) {
        if (g_layers.tile && g_layers.tile <= kLarge + 1 && g_layers.tile != 1 + i)
            continue;
        const Shape &s = shape_of(p.pl, i);
        const Times &t = (half ? f16 : f32)[i];
        const long long across = (p.K + s.bm - 1) / s.bm, x_tiles = across * ((p.P + s.bn - 1) / s.bn), w_tiles = across * ((p.N + s.bn - 1) / s.bn);
        const int x_steps = (p.np + s.r - 1) / s.r, w_steps = (p.P + s.r - 1) / s.r;
        for (const int sx : tries) {
            if (!may(sx, p.np))
                continue;
            const int nx = (x_steps + sx - 1) / sx;
            const float x = (float)nx * t.step + t.fixed;
            for (const int sw : tries) {
                if (!may(sw, p.P))
                    continue;
                const int nw = (w_steps + sw - 1) / sw;
                const float w = (float)nw * t.step + t.fixed;
                const long long all = x_tiles * sx + w_tiles * sw;
                const float full = (float)((all + kUnits - 1) / kUnits), share = full < (float)s.slots ? full : (float)s.slots;
                float us = (float)(nx > nw ? nx : nw) * (t.step * share > t.alone ? t.step * share : t.alone) + t.fixed * share;
                if (all > (long long)kUnits * s.slots) {
                    const float shared = ((float)(x_tiles * sx) * x + (float)(w_tiles * sw) * w) / (float)kUnits + tail * (x < w ? x : w);
                    us = shared > us ? shared : us;
                }
                us += planes(sx, (long long)p.P * p.K) + planes(sw, (long long)p.N * p.K) + (sx > 1 || sw > 1 ? sum : 0.f);
                if (best < 0.f || us < best) {
                    best = us;
                    p.gx = {i, sx};
                    p.gw = {i, sw};
                    p.w_first = w > x;
                }
            }
        }
    }
}

bool plan_gradients(LayerPlan &p, Room &room)
{
    choose_gradients(p);
    if (!fits(shape_of(p.pl, p.gx.shape), p.gx, p.K, p.P) || !fits(shape_of(p.pl, p.gw.shape), p.gw, p.K, p.N))
        return false;
    if (p.gx.splits > 1)
        p.gx_at = room.take((long long)p.gx.splits * p.P * p.K * 4);
    if (p.gw.splits > 1)
        p.gw_at = room.take((long long)p.gw.splits * p.N * p.K * 4);
    return true;
}

int plan_gated(LayerPlan *out, long long P, int K, int F, int dtype, bool backward)
{
    if (F < 1)
        return DCNV4_ERR_SHAPE;
    if (F > kLayerMaxWidth / 2)
        return DCNV4_ERR_UNSUPPORTED;
    if (const int rc = check_layer(P, K, F, dtype))
        return rc;
    LayerPlan p = {};
    p.es = esize(dtype);
    p.pl = dtype == DCNV4_F16 ? 1 : 3;
    p.P = (int)P;
    p.K = K;
    p.N = p.np = 2 * F;
    p.kp = p.pl == 1 ? K : (int)round_up(K, 32);
    // one more limit than the products': byte offsets inside the weights are 32 bits (fp32: of three planes of 16 bits)
    if ((long long)p.N * p.pl * p.kp * 2 >= 0x7fffffffLL)
        return DCNV4_ERR_UNSUPPORTED;
    p.forward = parts_of(p.pl, p.N, p.P, p.kp);
    for (int i = 0; i < p.forward.count; ++i)
        if (!fits(gated_shape(p.pl, p.forward.choice[i].shape), p.forward.choice[i], p.N, p.forward.pixels[i]))
            return DCNV4_ERR_UNSUPPORTED;
    Room room;
    if (p.pl == 3) {
        p.x_split = room.take(P * 6 * p.kp);
        p.w_split = room.take((long long)p.N * 6 * p.kp);
    }
    if (backward) {
        // (0: workgroups look through all of grad_h, from where their launch's rows begin, so there may be one launch only)
        p.most_parts = P * F <= kFewNumbers && p.forward.count == 1 ? 0 : (int)(P * F / 8 / 1024 < 512 ? P * F / 8 / 1024 + 1 : 512);
        p.scale = room.take(sizeof(Scale));
        p.most = room.take((p.most_parts + 1) * 4);
        p.d = room.take(P * p.pl * p.N * 2);
        p.bias_sums = room.take(round_up(P, 256) / 32 * p.N * 4);
        if (!plan_gradients(p, room))
            return DCNV4_ERR_UNSUPPORTED;
    }
    p.bytes = room.at;
    *out = p;
    return DCNV4_OK;
}

// Lanes side by side over N columns, eight each, in the sums over runs of rows.
constexpr int kChain = 256;
int lanes_log_of(int N)
{
    int log = 0;
    while (log < 6 && (8 << log) < N)
        ++log;
    return log;
}

int plan_linear_backward(LayerPlan *out, long long P, int K, int N, int dtype)
{
    if (const int rc = check_layer(P, K, N, dtype))
        return rc;
    LayerPlan p = {};
    p.es = esize(dtype);
    p.pl = dtype == DCNV4_F16 ? 1 : 3;
    p.P = (int)P;
    p.K = K;
    p.N = N;
    p.kp = p.pl == 1 ? K : (int)round_up(K, 32);
    p.np = N;
    Room room;
    if (p.pl == 3) {
        p.x_split = room.take(P * 6 * p.kp);
        p.w_split = room.take((long long)N * 6 * p.kp);
        p.g_split = room.take(P * 6 * p.np);
    }
    // runs of rows: two workgroups to a unit, 32 rows at least, and no more than give a lane kChain numbers to add up one after the other (fp32 sums of one sign
    // lose as many halves of a step: 131080 outputs and 8192 rows, in one run until then, were 2^-15 off)
    const long long across = (N / 8 + 63) / 64, chain = (long long)kChain * (256 >> lanes_log_of(N));
    const long long runs = across < 512 ? 512 / across : 1, rows = round_up((P + runs - 1) / runs, 32);
    p.columns_rows = (int)(rows < chain ? rows : chain);
    p.columns_runs = (int)((P + p.columns_rows - 1) / p.columns_rows);
    p.bias_sums = room.take((long long)p.columns_runs * N * 4);
    if (!plan_gradients(p, room))
        return DCNV4_ERR_UNSUPPORTED;
    p.bytes = room.at;
    *out = p;
    return DCNV4_OK;
}

void add_split(Ahead &q, const void *in, long long rows, int cols, int pad, void *out)
{
    int k = 0;
    while (q.split[k].blocks > 0)
        ++k;
    const long long groups = (rows * (pad / 8) + 255) / 256;
    q.split[k] = {(const float *)in, (unsigned short *)out, rows, cols, pad, (int)(groups < 4096 ? groups : 4096)};
}

template <typename T> void launch_ahead(const Ahead &q, hipStream_t s)
{
    const int blocks = q.blocks + q.split[0].blocks + q.split[1].blocks + q.split[2].blocks;
    if (blocks > 0)
        hipLaunchKernelGGL((dcnv4_layer_ahead_kernel<T>), dim3((unsigned)blocks), dim3(256), 0, s, q);
}

// grad_x, grad_w and, out of the runs' sums, grad_b (each may be null) of a layer with rows w [N][K], x [P][K], d [P][N] as operands.
template <typename T, int PL>
void gradients(const LayerPlan &p, const Operand &x, const Operand &w, const Operand &d, const Scale *scale, Bias b, void *grad_x, void *grad_w, char *ws,
               hipStream_t s)
{
    const bool x_planes = grad_x && p.gx.splits > 1, w_planes = grad_w && p.gw.splits > 1;
    const Result ox = {grad_x, 0, scale}, ow = {grad_w, 0, scale};
    Sum sx = {}, sw = {};
    auto sum_of = [&](Sum &q, const Choice &c, long long at, long long n, const Result &o) {
        const long long groups = (n / 4 + 255) / 256;
        q = {(const float *)(ws + at), c.splits, (int)(groups < 8192 ? groups : 8192), n, o};
        return Result{ws + at, n, nullptr};
    };
    const Result to_x = x_planes ? sum_of(sx, p.gx, p.gx_at, (long long)p.P * p.K, ox) : ox;
    const Result to_w = w_planes ? sum_of(sw, p.gw, p.gw_at, (long long)p.N * p.K, ow) : ow;
    // (grad_b goes with a launch that is there anyway)
    const bool sums = x_planes || w_planes, with_products = b.blocks > 0 && !sums && (grad_x || grad_w);
    if (grad_x || grad_w) {
        Gradients q = {product_of(turned(w), d, shape_of(PL, p.gx.shape), p.gx), product_of(turned(x), turned(d), shape_of(PL, p.gw.shape), p.gw),
                       to_x, to_w, 0, 0, p.w_first, with_products ? b : Bias{}};
        q.x_blocks = grad_x ? q.x.per_xcd * kXcds : 0;
        q.w_blocks = grad_w ? q.w.per_xcd * kXcds : 0;
        with_tile<PL>(p.gx.shape, [&](auto t) {
            typedef decltype(t) G;
            hipLaunchKernelGGL((dcnv4_layer_gradients_kernel<T, PL, G::WR, G::WC, G::WM, G::WN, G::R, G::STAGES>),
                               dim3((unsigned)(q.x_blocks + q.w_blocks + q.bias.blocks)), dim3(G::WR * G::WC * 64), 0, s, q);
            return 0;
        });
    }
    if (sums)
        hipLaunchKernelGGL((dcnv4_layer_sum_kernel<T>), dim3((unsigned)(sx.blocks + sw.blocks + b.blocks)), dim3(256), 0, s, sx, sw, b);
    else if (b.blocks > 0 && !with_products)
        hipLaunchKernelGGL((dcnv4_layer_bias_kernel<T>), dim3((unsigned)b.blocks), dim3(256), 0, s, b);
}

template <typename F> void by_activation(int act, F &&f)
{
    if (act == DCNV4_SILU)
        f(std::integral_constant<int, DCNV4_SILU>());
    else
        f(std::integral_constant<int, DCNV4_GELU>());
}

// x and w as the products take them
template <int PL> void operands(const LayerPlan &p, const void *x, const void *w, char *ws, bool with_x, bool with_w, Operand *xo, Operand *wo, Ahead &q)
{
    if (PL == 3) {
        if (with_x)
            add_split(q, x, p.P, p.K, p.kp, ws + p.x_split);
        if (with_w)
            add_split(q, w, p.N, p.K, p.kp, ws + p.w_split);
    }
    *xo = rows_of(PL == 3 ? (const void *)(ws + p.x_split) : x, p.P, p.kp, PL, p.kp);
    *wo = rows_of(PL == 3 ? (const void *)(ws + p.w_split) : w, p.N, p.kp, PL, p.kp);
}

// The operand's rows of K numbers (its planes are kp apart).
Operand narrowed(Operand o, int K)
{
    o.length = K;
    return o;
}

// The rows of an operand from `first` on.
Operand rows_from(Operand o, int first, int count)
{
    o.base += first * o.row_bytes;
    o.count = count;
    return o;
}

template <typename T, int PL>
int gated_forward(const LayerPlan &p, const void *x, const void *w, const void *bias, int F, int act, T *h, char *ws, hipStream_t s)
{
    Operand xo, wo;
    Ahead ahead = {};
    operands<PL>(p, x, w, ws, true, true, &xo, &wo, ahead);
    launch_ahead<T>(ahead, s);
    wo.count = F;
    int first = 0;
    for (int i = 0; i < p.forward.count; ++i) {
        const Choice &c = p.forward.choice[i];
        const Pairs l = {bias, F, p.forward.pixels[i]};
        const Product q = product_of(wo, rows_from(xo, first, l.P), gated_shape(PL, c.shape), c, true);
        by_activation(act, [&](auto A) {
            with_gated_tile<PL>(c.shape, [&](auto t) {
                typedef decltype(t) G;
                hipLaunchKernelGGL((dcnv4_gated_kernel<T, PL, A(), G::WR, G::WC, G::WM, G::WN, G::R, G::STAGES>), dim3((unsigned)(q.per_xcd * kXcds)),
                                   dim3(G::WR * G::WC * 64), 0, s, q, l, h + (long long)first * F);
                return 0;
            });
        });
        first += l.P;
    }
    return launched();
}

template <typename T, int PL>
int gated_backward(const LayerPlan &p, const void *x, const void *w, const void *bias, int F, int act, const T *grad_h, void *grad_x, void *grad_w, void *grad_b,
                   char *ws, hipStream_t s)
{
    if (PL == 1 && p.most_parts > 0)
        hipLaunchKernelGGL(dcnv4_gated_most_kernel, dim3((unsigned)p.most_parts), dim3(256), 0, s, (const unsigned short *)grad_h, (long long)p.P * F,
                           (float *)(ws + p.most));
    Operand xo, wo;
    Ahead ahead = {};
    operands<PL>(p, x, w, ws, true, true, &xo, &wo, ahead);
    launch_ahead<T>(ahead, s);
    Operand pairs = wo;
    pairs.count = F;
    Scale *scale = PL == 1 ? (Scale *)(ws + p.scale) : nullptr;
    unsigned short *d = (unsigned short *)(ws + p.d);
    float *bias_sums = (float *)(ws + p.bias_sums);
    int first = 0, runs = 0;
    for (int i = 0; i < p.forward.count; ++i) {
        const Choice &c = p.forward.choice[i];
        const Pairs l = {bias, F, p.forward.pixels[i]};
        const Product q = product_of(pairs, rows_from(xo, first, l.P), gated_shape(PL, c.shape), c, true);
        const Deltas e = {grad_h + (long long)first * F, d + (long long)first * PL * p.N, grad_b ? bias_sums + (long long)runs * p.N : nullptr,
                          (const float *)(ws + p.most), p.most_parts, p.most_parts > 0 ? 0 : p.P * F, scale};
        by_activation(act, [&](auto A) {
            with_gated_tile<PL>(c.shape, [&](auto t) {
                typedef decltype(t) G;
                runs += q.b_tiles * G::WC;
                hipLaunchKernelGGL((dcnv4_gated_delta_kernel<T, PL, A(), G::WR, G::WC, G::WM, G::WN, G::R, G::STAGES>), dim3((unsigned)(q.per_xcd * kXcds)),
                                   dim3(G::WR * G::WC * 64), 0, s, q, l, e);
                return 0;
            });
        });
        first += l.P;
    }
    Bias b = {};
    if (grad_b)
        b = {bias_sums, runs, p.N, (p.N + 15) / 16, grad_b};
    gradients<T, PL>(p, narrowed(xo, p.K), narrowed(wo, p.K), rows_of(d, p.P, p.N, PL, p.N), scale, b, grad_x, grad_w, ws, s);
    return launched();
}

template <typename T, int PL>
int linear_backward(const LayerPlan &p, const void *x, const void *w, const void *grad_y, void *grad_x, void *grad_w, void *grad_b, char *ws, hipStream_t s)
{
    Operand xo, wo;
    Ahead ahead = {};
    operands<PL>(p, x, w, ws, grad_w != nullptr, grad_x != nullptr, &xo, &wo, ahead);
    if (PL == 3 && (grad_x || grad_w))
        add_split(ahead, grad_y, p.P, p.N, p.np, ws + p.g_split);
    Bias b = {};
    if (grad_b) {
        b = {(const float *)(ws + p.bias_sums), p.columns_runs, p.N, (p.N + 15) / 16, grad_b};
        const int log = lanes_log_of(p.N);
        const int across = (p.N / 8 + (1 << log) - 1) >> log;
        ahead.g = grad_y;
        ahead.sums = (float *)(ws + p.bias_sums);
        ahead.P = p.P;
        ahead.N = p.N;
        ahead.lanes_log = log;
        ahead.run_rows = p.columns_rows;
        ahead.across = across;
        ahead.blocks = across * p.columns_runs;
    }
    launch_ahead<T>(ahead, s);
    gradients<T, PL>(p, narrowed(xo, p.K), narrowed(wo, p.K), rows_of(PL == 3 ? (const void *)(ws + p.g_split) : grad_y, p.P, p.N, PL, p.np), nullptr, b, grad_x,
                     grad_w, ws, s);
    return launched();
}

bool off16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

}  // namespace

int layers_set_option(const char *key, int value)
{
    if (!strcmp(key, "reset"))
        g_layers = LayerOptions();
    else if (!strcmp(key, "layer_tile") && value >= 0 && value <= kGatedTiles)
        g_layers.tile = value;
    else if (!strcmp(key, "layer_splits") && (value == 0 || value == 1 || value == 2 || value == 3 || value == 8 || value == 64))
        g_layers.splits = value;
    else
        return DCNV4_ERR_UNSUPPORTED;
    return DCNV4_OK;
}

extern "C" {

long long dcnv4_gated_linear_workspace_bytes(long long P, int K, int F, int dtype, int backward)
{
    LayerPlan p;
    return plan_gated(&p, P, K, F, dtype, backward != 0) == DCNV4_OK ? p.bytes : -1;
}

int dcnv4_gated_linear(const void *x, const void *w, const void *b, void *h, void *workspace, long long workspace_bytes, long long P, int K, int F,
                       int activation, int dtype, void *stream)
{
    if (!x || !w || !h)
        return DCNV4_ERR_NULL;
    LayerPlan p;
    const int rc = plan_gated(&p, P, K, F, dtype, false);
    if (rc)
        return rc;
    if (activation != DCNV4_SILU && activation != DCNV4_GELU)
        return DCNV4_ERR_UNSUPPORTED;
    if (p.bytes > 0 && !workspace)
        return DCNV4_ERR_NULL;
    if (p.bytes > 0 && workspace_bytes < p.bytes)
        return DCNV4_ERR_SHAPE;
    if (off16(x) || off16(w) || off16(b) || off16(h) || off16(workspace))
        return DCNV4_ERR_ALIGN;
    hipStream_t s = (hipStream_t)stream;
    return dtype == DCNV4_F16 ? gated_forward<_Float16, 1>(p, x, w, b, F, activation, (_Float16 *)h, (char *)workspace, s)
                              : gated_forward<float, 3>(p, x, w, b, F, activation, (float *)h, (char *)workspace, s);
}

int dcnv4_gated_linear_backward(const void *x, const void *w, const void *b, const void *grad_h, void *grad_x, void *grad_w, void *grad_b, void *workspace,
                                long long workspace_bytes, long long P, int K, int F, int activation, int dtype, void *stream)
{
    if (!x || !w || !grad_h || (!grad_x && !grad_w && !grad_b) || !workspace)
        return DCNV4_ERR_NULL;
    LayerPlan p;
    const int rc = plan_gated(&p, P, K, F, dtype, true);
    if (rc)
        return rc;
    if (activation != DCNV4_SILU && activation != DCNV4_GELU)
        return DCNV4_ERR_UNSUPPORTED;
    if (workspace_bytes < p.bytes)
        return DCNV4_ERR_SHAPE;
    if (off16(x) || off16(w) || off16(b) || off16(grad_h) || off16(grad_x) || off16(grad_w) || off16(grad_b) || off16(workspace))
        return DCNV4_ERR_ALIGN;
    hipStream_t s = (hipStream_t)stream;
    return dtype == DCNV4_F16 ? gated_backward<_Float16, 1>(p, x, w, b, F, activation, (const _Float16 *)grad_h, grad_x, grad_w, grad_b, (char *)workspace, s)
                              : gated_backward<float, 3>(p, x, w, b, F, activation, (const float *)grad_h, grad_x, grad_w, grad_b, (char *)workspace, s);
}

long long dcnv4_linear_backward_workspace_bytes(long long P, int K, int Nout, int dtype)
{
    LayerPlan p;
    return plan_linear_backward(&p, P, K, Nout, dtype) == DCNV4_OK ? p.bytes : -1;
}

int dcnv4_linear_backward(const void *x, const void *w, const void *grad_y, void *grad_x, void *grad_w, void *grad_b, void *workspace,
                          long long workspace_bytes, long long P, int K, int Nout, int dtype, void *stream)
{
    if (!grad_y || (!grad_x && !grad_w && !grad_b) || (grad_x && !w) || (grad_w && !x) || !workspace)
        return DCNV4_ERR_NULL;
    LayerPlan p;
    const int rc = plan_linear_backward(&p, P, K, Nout, dtype);
    if (rc)
        return rc;
    if (workspace_bytes < p.bytes)
        return DCNV4_ERR_SHAPE;
    if (off16(x) || off16(w) || off16(grad_y) || off16(grad_x) || off16(grad_w) || off16(grad_b) || off16(workspace))
        return DCNV4_ERR_ALIGN;
    hipStream_t s = (hipStream_t)stream;
    return dtype == DCNV4_F16 ? linear_backward<_Float16, 1>(p, x, w, grad_y, grad_x, grad_w, grad_b, (char *)workspace, s)
                              : linear_backward<float, 3>(p, x, w, grad_y, grad_x, grad_w, grad_b, (char *)workspace, s);
}

}  // extern "C"
