// Layer norm, dropout, and the end of a residual branch (dropout, add, layer norm in one pass), each with its gradient, on
// rows of C channels: the C ABI entry points of include/dcnv4.h and their kernels.
//
// All of it is bound by memory: a kernel reads each input once, keeps a row in registers while its statistics are made, and
// writes each output once.  A lane holds runs of eight channels (16 bytes in fp16, 32 in fp32).  A row belongs to L lanes: as
// few of a wave as its runs need, whole waves for wide rows.  A workgroup stays for many rows and asks for the next ones before it
// deals with the present ones: a wave's loads alone, some KiB, do not cover the memory's latency (65536 x 256 fp16 norm: forward 15.8
// -> 15.0 us, backward 32.5 -> 23.8).
//
// Rates (16.8 million elements, 128 to 4096 channels; a copy of as much: 6.5 TB/s in fp16, which the caches hold in part, 5.2 in fp32):
// norm 4.2 to 4.8 TB/s forward and 3.5 to 4.3 backward in fp16, 4.5 to 4.8 and 4.1 to 4.7 in fp32; branch ends 4.5 to 4.9 and 4.0 to 4.3, 4.8
// to 5.2 and 4.4 to 4.9; rows of odd lengths 55 to 75 % of that in fp16, 75 to 95 % in fp32.
#include <math.h>

#include <initializer_list>
#include <type_traits>

#include "dcnv4_common.h"

// Products and sums are fused where the code says so and nowhere else, so that kernels that share a formula give the same bits.
#pragma clang fp contract(off)

namespace {

// ------------------------------------------------------------------------------------------
// Dropout's decisions: Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2,
// 3", 2011).  Key: the seed; counter: (block, offset), 64 bits each.  A block serves eight elements, 16 bits each, so that a
// run of eight takes one block: with 32 bits an element the generator, and not memory, would bound fp16 tensors (20 products
// of 32 x 32 bits at a quarter of the rate, 80 clocks of a lane, for eight elements or for four).
// ------------------------------------------------------------------------------------------
struct Drop {
    unsigned limit;                   // an element goes where its 16 bits are below
    float scale;                      // of those that stay
    unsigned long long seed, offset;
    const unsigned long long *more;   // null, or where a number to be added to the offset lies
};

struct Bits8 {
    unsigned w[4];
};

__device__ __forceinline__ unsigned long long drop_offset(const Drop &d)
{
    return d.offset + (d.more != nullptr ? *d.more : 0ull);
}

__device__ __forceinline__ Bits8 philox(unsigned long long block, unsigned long long offset, unsigned long long seed)
{
    unsigned c0 = (unsigned)block, c1 = (unsigned)(block >> 32), c2 = (unsigned)offset, c3 = (unsigned)(offset >> 32);
    unsigned k0 = (unsigned)seed, k1 = (unsigned)(seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const unsigned long long a = (unsigned long long)c0 * 0xD2511F53u, b = (unsigned long long)c2 * 0xCD9E8D57u;
        c0 = (unsigned)(b >> 32) ^ c1 ^ k0;
        c1 = (unsigned)b;
        c2 = (unsigned)(a >> 32) ^ c3 ^ k1;
        c3 = (unsigned)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
}

// The decisions of a block's eight elements, a bit each: set where the element goes.
__device__ __forceinline__ unsigned gone_of(const Bits8 &b, const Drop &d)
{
    unsigned m = 0u;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        m |= ((b.w[e / 2] >> (16 * (e & 1))) & 0xffffu) < d.limit ? 1u << e : 0u;
    return m;
}

// Element e of the eight: r + v scaled, or r alone whatever v is.  WHOLE: by the block's bits; else by decisions (in w[0]).
template <bool WHOLE> __device__ __forceinline__ float drop_apply(const Bits8 &b, int e, const Drop &d, float v, float r)
{
    const bool gone = WHOLE ? ((b.w[e / 2] >> (16 * (e & 1))) & 0xffffu) < d.limit : (b.w[0] >> e & 1u) != 0u;
    float sum = __builtin_fmaf(v, d.scale, r);
    asm("" : "+v"(sum));                                   // (an fp32 number here: not one instruction with a store's rounding)
    return gone ? r : sum;
}

// ------------------------------------------------------------------------------------------
// Runs of eight channels.  WHOLE: C is a multiple of eight, so that every run is whole and aligned; otherwise rows start at any
// element (memory instructions of 16 bytes take any address), and the last run of a row may be short.
// ------------------------------------------------------------------------------------------
template <typename T> struct Run {                         // as they lie in memory, aligned to 16 bytes or to an element
    typedef T type __attribute__((ext_vector_type(8)));
    typedef type aligned __attribute__((aligned(16)));
    typedef type any __attribute__((aligned(sizeof(T))));
};
template <typename T> using Raw8 = typename Run<T>::type;

// n channels of a row (none for n <= 0), and what follows them where n < 8.  `safe`: eight from the row's last channel on are memory of
// the tensor; otherwise no more than the n are read.
template <typename T, bool WHOLE> __device__ __forceinline__ Raw8<T> load8(const T *p, int n, bool safe)
{
    Raw8<T> r = {};
    if (WHOLE) {
        if (n > 0)
            r = *reinterpret_cast<const typename Run<T>::aligned *>(p);
    } else if (n >= 8 || (n > 0 && safe)) {
        r = *reinterpret_cast<const typename Run<T>::any *>(p);
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n)
                r[e] = p[e];
    }
    return r;
}
// The bits of the first n of eight (which a lane's runs keep from row to row).
template <typename T> struct Mask8 {
    unsigned w[2 * sizeof(T)];
    __device__ __forceinline__ explicit Mask8(int n)
    {
#pragma unroll
        for (int k = 0; k < (int)(2 * sizeof(T)); ++k) {
            if constexpr (sizeof(T) == 2)
                w[k] = n >= 2 * k + 2 ? ~0u : n == 2 * k + 1 ? 0xffffu : 0u;
            else
                w[k] = n >= k + 1 ? ~0u : 0u;
        }
    }
    __device__ __forceinline__ Mask8() {}
};
// As fp32, zeros behind the first n whatever lies there.
template <typename T, bool WHOLE> __device__ __forceinline__ void unpack(Raw8<T> r, const Mask8<T> &m, float (&v)[8])
{
    if constexpr (!WHOLE) {
        typedef unsigned words __attribute__((ext_vector_type(2 * sizeof(T))));
        words u = __builtin_bit_cast(words, r);
#pragma unroll
        for (int k = 0; k < (int)(2 * sizeof(T)); ++k)
            u[k] &= m.w[k];
        r = __builtin_bit_cast(Raw8<T>, u);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] = (float)r[e];
}

template <typename T, bool WHOLE> __device__ __forceinline__ void store8(T *p, int n, const float (&v)[8])
{
    if (n <= 0)
        return;
    Raw8<T> t;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        t[e] = (T)v[e];                                    // one rounding to nearest even
    if (WHOLE) {
        *reinterpret_cast<typename Run<T>::aligned *>(p) = t;
    } else if (n >= 8) {
        *reinterpret_cast<typename Run<T>::any *>(p) = t;
    } else {
        typedef T four __attribute__((ext_vector_type(4)));
        typedef T two __attribute__((ext_vector_type(2)));
        typedef four any_four __attribute__((aligned(sizeof(T))));
        typedef two any_two __attribute__((aligned(sizeof(T))));
        if (n & 4)
            *reinterpret_cast<any_four *>(p) = four{t[0], t[1], t[2], t[3]};
        if (n & 2)
            *reinterpret_cast<any_two *>(p + (n & 4)) = n & 4 ? two{t[4], t[5]} : two{t[0], t[1]};
        if (n & 1)
            p[n - 1] = n == 1 ? t[0] : n == 3 ? t[2] : n == 5 ? t[4] : t[6];
    }
}

// Sums over the L lanes of a row, in every one of them.  Lanes of a wave: exchanges within quads, mirrored halves and rows
// of 16, then rows and halves of the wave swapped.  Wider rows: the waves' sums through LDS, in the order of the waves.
template <int CTRL> __device__ __forceinline__ float dpp(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, false));
}
// (In assembly: the builtins of these swaps give the first register twice in this compiler.  The two idle slots are what
// a swap needs after its operands are written.)
__device__ __forceinline__ float add_rows(float v)         // the other row of 16 of its pair
{
    float a = v, b = v;
    asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(a), "+v"(b));
    return a + b;
}
__device__ __forceinline__ float add_halves(float v)       // the other half of the wave
{
    float a = v, b = v;
    asm("s_nop 1\n\tv_permlane32_swap_b32 %0, %1" : "+v"(a), "+v"(b));
    return a + b;
}
template <int L> __device__ __forceinline__ float wave_sum(float v)
{
    static_assert(L >= 1 && L <= 64);
    if constexpr (L >= 2)
        v += dpp<0xB1>(v);                                 // quad_perm [1,0,3,2]
    if constexpr (L >= 4)
        v += dpp<0x4E>(v);                                 // quad_perm [2,3,0,1]
    if constexpr (L >= 8)
        v += dpp<0x141>(v);                                // row_half_mirror
    if constexpr (L >= 16)
        v += dpp<0x140>(v);                                // row_mirror
    if constexpr (L >= 32)
        v = add_rows(v);
    if constexpr (L >= 64)
        v = add_halves(v);
    return v;
}
template <int L, int N> __device__ __forceinline__ void row_sums(float (&v)[N], float (*lds)[N])
{
#pragma unroll
    for (int k = 0; k < N; ++k)
        v[k] = wave_sum<(L < 64 ? L : 64)>(v[k]);
    if constexpr (L > 64) {
        constexpr int W = L / 64;
        const int wave = (int)threadIdx.x >> 6, first = wave / W * W;
        __syncthreads();                                   // all have read the sums before these
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < N; ++k)
                lds[wave][k] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = lds[first][k];
#pragma unroll
            for (int w = 1; w < W; ++w)
                v[k] += lds[first + w][k];
        }
    }
}

constexpr int norm_threads(int L) { return L >= 256 ? 512 : 256; }

// Where a lane's run j lies in its row, in runs: side by side in a wave, then run after run, then the next wave's.
template <int L, int NV> __device__ __forceinline__ int run_of(int l, int j)
{
    constexpr int G = L < 64 ? L : 64;
    return (l / G * NV + j) * G + l % G;
}

// What drop_apply takes for a lane's runs, `first` being the first element of the row.  Rows that start inside a block share each block
// between two neighbouring runs: a lane makes one block's decisions and takes those of the second from the next lane (the
// last lane of a wave makes its last ones itself).  Both blocks made by each lane: fp16 branch ends of 52265 x 321 72 us, 49 so.
template <int L, int NV, bool WHOLE>
__device__ __forceinline__ void row_bits(Bits8 (&b)[NV], unsigned long long first, int C, int l, unsigned long long offset, const Drop &d)
{
#pragma unroll
    for (int j = 0; j < NV; ++j)
        b[j] = philox((first >> 3) + (unsigned)run_of<L, NV>(l, j), offset, d.seed);
    if constexpr (!WHOLE) {
        constexpr int G = L < 64 ? L : 64;
        const unsigned skip = (unsigned)first & 7u;
        const bool last = l % G == G - 1;
        unsigned end = 0u, mine[NV], beside[NV];
        if (last && run_of<L, NV>(l, NV - 1) * 8 < C)
            end = gone_of(philox((first >> 3) + (unsigned)run_of<L, NV>(l, NV - 1) + 1u, offset, d.seed), d);
        const int next = ((int)(threadIdx.x & 63) / G * G + (l + 1) % G) * 4;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            mine[j] = gone_of(b[j], d);
            beside[j] = (unsigned)__builtin_amdgcn_ds_bpermute(next, (int)mine[j]);
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const unsigned second = last ? (j + 1 < NV ? beside[j + 1 < NV ? j + 1 : j] : end) : beside[j];
            b[j].w[0] = (mine[j] | second << 8) >> skip;
        }
    }
}

struct NormArgs {
    const void *x, *residual, *gamma, *beta;   // gamma, beta: null for ones and zeros
    void *z, *y;
    float *mean, *rstd;                        // null: not asked for
    long long P;
    int C;
    float inv_c, eps;
    Drop drop;
};

struct NormBackArgs {
    const void *x, *gamma;                     // x: what the norm read
    const float *mean, *rstd;
    const void *grad_y, *grad_z;               // grad_z: null, or what comes down the residual path
    void *grad_x, *grad_residual;
    float *partial;                            // [workgroup][2][C], null: no gradients of gamma and beta
    long long P;
    int C;
    float inv_c;
    Drop drop;
};

}  // namespace

// y = (x - mean) / sqrt(var + eps) * gamma + beta, a row of x at a time; BRANCH: of z = residual + dropout(x), rounded as it is
// stored.  The variance is summed from centred values, which are in registers anyway: no cancellation for rows far from zero.
template <typename T, int L, int NV, bool BRANCH, bool WHOLE>
__global__ __launch_bounds__(norm_threads(L)) void dcnv4_norm_kernel(NormArgs a)
{
    constexpr int R = norm_threads(L) / L;                 // rows of a workgroup
    __shared__ float lds[norm_threads(L) / 64][1];
    const int l = (int)threadIdx.x % L, first = (int)threadIdx.x / L;
    const T *gamma = (const T *)a.gamma, *beta = (const T *)a.beta;
    const unsigned long long offset = BRANCH ? drop_offset(a.drop) : 0ull;
    const long long all = a.P * a.C, stride = (long long)gridDim.x * R;
    constexpr bool AHEAD = NV <= 2;                        // (else no registers for two rows)
    Raw8<T> x[NV], res[BRANCH ? NV : 1], gm[NV], bt[NV];
    Mask8<T> mask[NV];
    auto load = [&](long long row) {                       // (a row past the last: nothing)
        const bool safe = (row + 1) * a.C + 7 <= all;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = run_of<L, NV>(l, j) * 8, n = row < a.P ? a.C - c : 0;
            x[j] = load8<T, WHOLE>((const T *)a.x + row * a.C + c, n, safe);
            if constexpr (BRANCH)
                res[j] = load8<T, WHOLE>((const T *)a.residual + row * a.C + c, n, safe);
        }
    };
    long long base = (long long)blockIdx.x * R;
    if (AHEAD)
        load(base + first);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = run_of<L, NV>(l, j) * 8, n = a.C - c;
        mask[j] = Mask8<T>(n);
        if (gamma != nullptr)
            gm[j] = load8<T, WHOLE>(gamma + c, n, false);
        if (beta != nullptr)
            bt[j] = load8<T, WHOLE>(beta + c, n, false);
    }
    for (; base < a.P; base += stride) {                   // (the whole workgroup, for the barriers of wide rows)
        const long long row = base + first, at = row * a.C;
        const bool live = row < a.P;
        if (!AHEAD)
            load(row);
        float v[NV][8], s[1] = {0.f};
        float r[BRANCH ? NV : 1][8];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            unpack<T, WHOLE>(x[j], mask[j], v[j]);
            if constexpr (BRANCH)
                unpack<T, WHOLE>(res[j], mask[j], r[j]);
        }
        if (AHEAD)
            load(row + stride);
        if constexpr (BRANCH) {
            Bits8 bits[NV];
            row_bits<L, NV, WHOLE>(bits, (unsigned long long)at, a.C, l, offset, a.drop);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = run_of<L, NV>(l, j) * 8;
#pragma unroll
                for (int e = 0; e < 8; ++e)                // (zeros behind the row: of the sum of two of them)
                    v[j][e] = (float)(T)drop_apply<WHOLE>(bits[j], e, a.drop, v[j][e], r[j][e]);
                store8<T, WHOLE>((T *)a.z + at + c, live ? a.C - c : 0, v[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                s[0] += v[j][e];
        row_sums<L, 1>(s, lds);
        const float mean = s[0] / (float)a.C;              // (divided: the mean of equal numbers that add up exactly is that number)
        s[0] = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int n = a.C - run_of<L, NV>(l, j) * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[j][e] -= mean;
                if (WHOLE ? n > 0 : e < n)
                    s[0] = __builtin_fmaf(v[j][e], v[j][e], s[0]);
            }
        }
        row_sums<L, 1>(s, lds);
        const float rstd = 1.f / __builtin_sqrtf(__builtin_fmaf(s[0], a.inv_c, a.eps));
        if (l == 0 && live) {
            if (a.mean != nullptr)
                a.mean[row] = mean;
            if (a.rstd != nullptr)
                a.rstd[row] = rstd;
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = run_of<L, NV>(l, j) * 8;
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                y[e] = v[j][e] * rstd;
                if (gamma != nullptr)
                    y[e] = beta != nullptr ? __builtin_fmaf(y[e], (float)gm[j][e], (float)bt[j][e]) : y[e] * (float)gm[j][e];
                else if (beta != nullptr)
                    y[e] += (float)bt[j][e];
            }
            store8<T, WHOLE>((T *)a.y + at + c, live ? a.C - c : 0, y);
        }
    }
}

// With xhat = (x - mean) * rstd and g = grad_y * gamma:
//     grad_x = rstd * (g - avg(g) - xhat * avg(g * xhat)),  grad_gamma = sum over rows of grad_y * xhat,  grad_beta = of grad_y
// A lane meets the same channels in every row of its workgroup, so the sums over rows stay in its registers until the last
// row; then the workgroup's rows side by side are added up through LDS and go out as its partial sums, which
// dcnv4_norm_join_kernel adds up in the order of the workgroups (no atomics: results do not change from run to run).
// BRANCH: grad_residual = that + grad_z, grad_x = dropout's gradient of it, from the number before its rounding.
template <typename T, int L, int NV, bool BRANCH, bool WHOLE>
__global__ __launch_bounds__(norm_threads(L)) void dcnv4_norm_backward_kernel(NormBackArgs a)
{
    constexpr int R = norm_threads(L) / L;
    __shared__ float lds[norm_threads(L) / 64][2];
    __shared__ float sums[R > 1 ? norm_threads(L) * 8 : 1];
    const int l = (int)threadIdx.x % L, first = (int)threadIdx.x / L;
    const T *gamma = (const T *)a.gamma;
    const unsigned long long offset = BRANCH ? drop_offset(a.drop) : 0ull;
    float dg[NV][8], db[NV][8];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            dg[j][e] = db[j][e] = 0.f;
    const long long all = a.P * a.C, stride = (long long)gridDim.x * R;
    constexpr bool AHEAD = NV <= 2;                        // (else no registers for two rows, gamma and grad_z)
    Raw8<T> x[NV], gy[NV], gz[BRANCH && AHEAD ? NV : 1], gm[AHEAD ? NV : 1];
    Mask8<T> mask[NV];
    float mean = 0.f, rstd = 0.f;
    auto load = [&](long long row) {                       // (a row past the last: nothing)
        const bool safe = (row + 1) * a.C + 7 <= all;
        mean = row < a.P ? a.mean[row] : 0.f;
        rstd = row < a.P ? a.rstd[row] : 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = run_of<L, NV>(l, j) * 8, n = row < a.P ? a.C - c : 0;
            const long long at = row * a.C + c;
            x[j] = load8<T, WHOLE>((const T *)a.x + at, n, safe);
            gy[j] = load8<T, WHOLE>((const T *)a.grad_y + at, n, safe);
            if constexpr (BRANCH && AHEAD)
                if (a.grad_z != nullptr)
                    gz[j] = load8<T, WHOLE>((const T *)a.grad_z + at, n, safe);
        }
    };
    long long base = (long long)blockIdx.x * R;
    if (AHEAD)
        load(base + first);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = run_of<L, NV>(l, j) * 8, n = a.C - c;
        mask[j] = Mask8<T>(n);
        if (AHEAD && gamma != nullptr)
            gm[AHEAD ? j : 0] = load8<T, WHOLE>(gamma + c, n, false);
    }
    for (; base < a.P; base += stride) {                   // (the whole workgroup, for the barriers of wide rows)
        const long long row = base + first, at = row * a.C;
        const bool live = row < a.P;
        if constexpr (!AHEAD) {
            load(row);
            asm volatile("" : "+s"(a.C));                  // (what follows from C is worked out again: kept, it would fill the registers)
        }
        const float scale = rstd;
        float xh[NV][8], g[NV][8], r[BRANCH && AHEAD ? NV : 1][8], s[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = run_of<L, NV>(l, j) * 8, n = a.C - c;
            unpack<T, WHOLE>(x[j], mask[j], xh[j]);
            unpack<T, WHOLE>(gy[j], mask[j], g[j]);
            if constexpr (BRANCH && AHEAD) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    r[j][e] = 0.f;
                if (a.grad_z != nullptr)
                    unpack<T, WHOLE>(gz[j], mask[j], r[j]);
            }
            if (!AHEAD && gamma != nullptr)
                gm[0] = load8<T, WHOLE>(gamma + c, n, false);
            // (behind the row both are zero, and so is every sum's term: mean * rstd may be more than fp32 holds)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                xh[j][e] = (WHOLE ? n > 0 : e < n) ? (xh[j][e] - mean) * rstd : 0.f;
                dg[j][e] = __builtin_fmaf(g[j][e], xh[j][e], dg[j][e]);
                db[j][e] += g[j][e];
                if (gamma != nullptr)
                    g[j][e] *= (float)gm[AHEAD ? j : 0][e];
                s[0] += g[j][e];
                s[1] = __builtin_fmaf(g[j][e], xh[j][e], s[1]);
            }
        }
        if (AHEAD)
            load(row + stride);
        row_sums<L, 2>(s, lds);
        const float m0 = s[0] * a.inv_c, m1 = s[1] * a.inv_c;
        Bits8 bits[BRANCH && AHEAD ? NV : 1];
        if constexpr (BRANCH && AHEAD)
            row_bits<L, NV, WHOLE>(bits, (unsigned long long)at, a.C, l, offset, a.drop);
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            if constexpr (!AHEAD)
                __builtin_amdgcn_sched_barrier(0);         // (one run after the other)
            const int c = run_of<L, NV>(l, j) * 8, n = live ? a.C - c : 0;
            float out[8];
            if constexpr (BRANCH && !AHEAD) {
                const unsigned long long i = (unsigned long long)(at + c);
                bits[0] = philox(i >> 3, offset, a.drop.seed);
                if constexpr (!WHOLE)
                    bits[0].w[0] = (gone_of(bits[0], a.drop) | gone_of(philox((i >> 3) + 1, offset, a.drop.seed), a.drop) << 8) >> ((unsigned)i & 7u);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    r[0][e] = 0.f;
                if (a.grad_z != nullptr)
                    unpack<T, WHOLE>(load8<T, WHOLE>((const T *)a.grad_z + at + c, n, (row + 1) * a.C + 7 <= all), mask[j], r[0]);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                out[e] = scale * __builtin_fmaf(-xh[j][e], m1, g[j][e] - m0);
                asm("" : "+v"(out[e]));                    // (as in drop_apply)
            }
            if constexpr (BRANCH) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    out[e] += r[AHEAD ? j : 0][e];
                store8<T, WHOLE>((T *)a.grad_residual + at + c, n, out);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    out[e] = drop_apply<WHOLE>(bits[AHEAD ? j : 0], e, a.drop, out[e], 0.f);
            }
            store8<T, WHOLE>((T *)a.grad_x + at + c, n, out);
        }
    }
    if (a.partial == nullptr)
        return;
    float *to = a.partial + (long long)blockIdx.x * 2 * a.C;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = run_of<L, NV>(l, j) * 8;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] = k == 0 ? dg[j][e] : db[j][e];
            if constexpr (R > 1) {
                // rows side by side in a wave first: lanes 8, 4, 2, 1 further round (of 16), then rows of 16 and halves
                constexpr int G = L < 64 ? L : 64, W = norm_threads(L) / 64;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if constexpr (G < 16) v[e] += dpp<0x128>(v[e]);
                    if constexpr (G < 8) v[e] += dpp<0x124>(v[e]);
                    if constexpr (G < 4) v[e] += dpp<0x122>(v[e]);
                    if constexpr (G < 2) v[e] += dpp<0x121>(v[e]);
                    if constexpr (G < 32) v[e] = add_rows(v[e]);
                    if constexpr (G < 64) v[e] = add_halves(v[e]);
                }
                // then the waves: all of them (rows of a wave and less), or those with the same part of a row
                constexpr int PARTS = L < 64 ? 1 : L / 64;
                const int wave = (int)threadIdx.x >> 6, in = l % G;
                __syncthreads();                           // all have read what was there before
                if ((int)(threadIdx.x & 63) < G)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        sums[(wave * 8 + e) * G + in] = v[e];
                __syncthreads();
                if (first == 0)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
#pragma unroll
                        for (int w = PARTS; w < W; w += PARTS)
                            v[e] += sums[((w + wave) * 8 + e) * G + in];
            }
            if (first == 0)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (c + e < a.C)
                        to[k * a.C + c + e] = v[e];
        }
    }
}

// Adds up partial sums [count][2 * C]: 16 columns to a workgroup, 64 of the rows side by side.
template <typename T>
__global__ __launch_bounds__(1024) void dcnv4_norm_join_kernel(const float *__restrict__ partial, int count, int C, T *grad_gamma, T *grad_beta)
{
    __shared__ float sums[16][16];
    const int col = (int)blockIdx.x * 16 + ((int)threadIdx.x & 15), slice = (int)threadIdx.x >> 4;
    float s = 0.f;
    if (col < 2 * C)
#pragma unroll 8
        for (int r = slice; r < count; r += 64)
            s += partial[(long long)r * 2 * C + col];
    s = add_halves(add_rows(s));
    if ((threadIdx.x & 63) < 16)
        sums[threadIdx.x >> 6][threadIdx.x & 15] = s;
    __syncthreads();
    if (threadIdx.x < 16 && col < 2 * C) {
        s = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r)
            s += sums[r][threadIdx.x];
        T *to = col < C ? grad_gamma : grad_beta;
        if (to != nullptr)
            to[col < C ? col : col - C] = (T)s;
    }
}

// out = [residual +] dropout(x): eight elements of each of two stretches a lane, whose loads go out together.
template <typename T, bool ADD>
__global__ __launch_bounds__(256) void dcnv4_dropout_kernel(const T *__restrict__ x, const T *__restrict__ residual, T *__restrict__ y, long long n,
                                                            Drop d)
{
    const unsigned long long offset = drop_offset(d);
    const long long half = (long long)gridDim.x * 2048;
    for (long long i0 = ((long long)blockIdx.x * 256 + (int)threadIdx.x) * 8; i0 < n; i0 += 2 * half) {
        Raw8<T> v[2], r[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const long long i = i0 + k * half, left = n - i;
            if (left >= 8) {
                v[k] = load8<T, true>(x + i, 8, false);
                if (ADD)
                    r[k] = load8<T, true>(residual + i, 8, false);
            } else if (left > 0) {
                v[k] = load8<T, false>(x + i, (int)left, false);
                if (ADD)
                    r[k] = load8<T, false>(residual + i, (int)left, false);
            }
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const long long i = i0 + k * half, left = n - i;
            if (left <= 0)
                continue;
            const Bits8 b = philox((unsigned long long)i >> 3, offset, d.seed);
            float out[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                out[e] = drop_apply<true>(b, e, d, (float)v[k][e], ADD ? (float)r[k][e] : 0.f);
            if (left >= 8)
                store8<T, true>(y + i, 8, out);
            else
                store8<T, false>(y + i, (int)left, out);
        }
    }
}

namespace {

// Rows wider than this are refused: 512 lanes with four runs of eight each.
constexpr int kNormMaxChannels = 16384;
// Workgroups of the backward pass, each of which leaves partial sums of 2 * C: as many as memory needs for its rate, fewer for
// wide rows, where the partial sums would be a good part of what is moved (8192 fp16 channels, 2048 rows: 94 us with 1024 workgroups, 38 so).
int norm_back_most(int C) { return C <= 512 ? 1024 : C <= 2048 ? 512 : 256; }

bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

int fill_drop(Drop *d, float p, unsigned long long seed, unsigned long long offset, const void *more)
{
    if (!(p >= 0.f && p <= 1.f))
        return DCNV4_ERR_UNSUPPORTED;
    if (reinterpret_cast<uintptr_t>(more) & 7u)
        return DCNV4_ERR_ALIGN;
    d->limit = (unsigned)floor((double)p * 65536.0 + 0.5);
    d->scale = d->limit < 65536u ? (float)(65536.0 / (65536.0 - d->limit)) : 0.f;
    d->seed = seed;
    d->offset = offset;
    d->more = (const unsigned long long *)more;
    return DCNV4_OK;
}

int check_rows(long long P, int C, int dtype)
{
    if (P < 1 || C < 1)
        return DCNV4_ERR_SHAPE;
    if ((dtype != DCNV4_F32 && dtype != DCNV4_F16) || C > kNormMaxChannels || P > (1LL << 40))
        return DCNV4_ERR_UNSUPPORTED;
    return DCNV4_OK;
}

// Calls f with the lanes of a row and a lane's runs of eight channels, as constants: the fewest lanes that hold the row with one run each,
// up to a wave; with two up to 1024 channels, then two, four and eight waves.  (Two rows side by side in a workgroup of four
// waves each rather than eight waves with one run: twice the loads on their way.)  Both sides of the two exceptions, in us for 16.8 million elements:
// Forward, up to 1536 channels: three runs and no barriers.  1032, 1280 and 1536 channels in fp16 norm 17.8, 14.1, 13.2 (by two waves 20.7, 17.4, 15.1),
// branch end 29, 27, 27 (37, 32, 29); 1100 and 1499, 20 and 17 (27, 22); in fp32 0 to 6 % less.  Backward, whose sums leave it no registers
// to load ahead: 16368 x 1025 fp16 41 (44 by two waves), 11184 x 1500 42 and 35.
// fp32, 2049 to 4096 channels: eight waves with one run.  Norms forward and backward together at 2056, 2816, 3584 and 4096 channels 88, 78, 78, 78 (with
// two 80, 77, 82, 79), branch ends 135, 123, 124, 121 (132, 130, 136, 133).  fp16, with one run: norms 65, 54, 48, 46 (as it is 54, 45, 46, 45), branch
// ends 90, 74, 68, 69 (89, 74, 73, 71).
template <typename T, bool BACK, typename F> int by_width(int C, F &&f)
{
    const int runs = (C + 7) / 8;
    if (runs <= 1) return f(std::integral_constant<int, 1>(), std::integral_constant<int, 1>());
    if (runs <= 2) return f(std::integral_constant<int, 2>(), std::integral_constant<int, 1>());
    if (runs <= 4) return f(std::integral_constant<int, 4>(), std::integral_constant<int, 1>());
    if (runs <= 8) return f(std::integral_constant<int, 8>(), std::integral_constant<int, 1>());
    if (runs <= 16) return f(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
    if (runs <= 32) return f(std::integral_constant<int, 32>(), std::integral_constant<int, 1>());
    if (runs <= 64) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
    if (runs <= 128) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
    if constexpr (!BACK)
        if (runs <= 192) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 3>());
    if (runs <= 256) return f(std::integral_constant<int, 128>(), std::integral_constant<int, 2>());
    if (runs <= 512) return f(std::integral_constant<int, sizeof(T) == 2 ? 256 : 512>(), std::integral_constant<int, sizeof(T) == 2 ? 2 : 1>());
    if (runs <= 1024) return f(std::integral_constant<int, 512>(), std::integral_constant<int, 2>());
    return f(std::integral_constant<int, 512>(), std::integral_constant<int, 4>());
}

template <typename T> int norm_back_groups(long long P, int C)
{
    int groups = 0;
    by_width<T, true>(C, [&](auto L, auto) {
        const long long rows = norm_threads(L()) / L(), n = (P + rows - 1) / rows;
        // (four rows a lane at least, where that leaves every unit two workgroups)
        const long long enough = n / 4 > 512 ? n / 4 : 512, most = norm_back_most(C);
        groups = (int)(n < enough ? n : enough < most ? enough : most);
        return 0;
    });
    return groups;
}

template <typename T, bool BRANCH> int launch_norm(const NormArgs &a, hipStream_t s)
{
    const int cus = device_cus();
    if (cus <= 0)
        return DCNV4_ERR_LAUNCH;
    return by_width<T, false>(a.C, [&](auto L, auto NV) {
        constexpr int threads = norm_threads(L());
        const long long rows = threads / L(), groups = (a.P + rows - 1) / rows, most = (long long)(2048 / threads) * cus;
        const dim3 grid((unsigned)(groups < most ? groups : most));
        if (a.C % 8 == 0)
            hipLaunchKernelGGL((dcnv4_norm_kernel<T, L(), NV(), BRANCH, true>), grid, dim3(threads), 0, s, a);
        else
            hipLaunchKernelGGL((dcnv4_norm_kernel<T, L(), NV(), BRANCH, false>), grid, dim3(threads), 0, s, a);
        return hipGetLastError() == hipSuccess ? DCNV4_OK : DCNV4_ERR_LAUNCH;
    });
}

template <typename T, bool BRANCH> int launch_norm_backward(const NormBackArgs &a, void *grad_gamma, void *grad_beta, hipStream_t s)
{
    const int groups = norm_back_groups<T>(a.P, a.C);
    const int rc = by_width<T, true>(a.C, [&](auto L, auto NV) {
        constexpr int threads = norm_threads(L());
        if (a.C % 8 == 0)
            hipLaunchKernelGGL((dcnv4_norm_backward_kernel<T, L(), NV(), BRANCH, true>), dim3((unsigned)groups), dim3(threads), 0, s, a);
        else
            hipLaunchKernelGGL((dcnv4_norm_backward_kernel<T, L(), NV(), BRANCH, false>), dim3((unsigned)groups), dim3(threads), 0, s, a);
        return hipGetLastError() == hipSuccess ? DCNV4_OK : DCNV4_ERR_LAUNCH;
    });
    if (rc || a.partial == nullptr)
        return rc;
    hipLaunchKernelGGL((dcnv4_norm_join_kernel<T>), dim3((unsigned)((2 * a.C + 15) / 16)), dim3(1024), 0, s, a.partial, groups, a.C,
                       (T *)grad_gamma, (T *)grad_beta);
    return hipGetLastError() == hipSuccess ? DCNV4_OK : DCNV4_ERR_LAUNCH;
}

int norm_impl(NormArgs &a, float eps, int dtype, bool branch, void *stream)
{
    if (!a.x || !a.y || (branch && (!a.residual || !a.z)))
        return DCNV4_ERR_NULL;
    const int rc = check_rows(a.P, a.C, dtype);
    if (rc)
        return rc;
    if (!(eps >= 0.f && eps <= 3.0e38f))
        return DCNV4_ERR_UNSUPPORTED;
    for (const void *p : {a.x, a.residual, a.gamma, a.beta, (const void *)a.z, (const void *)a.y, (const void *)a.mean, (const void *)a.rstd})
        if (misaligned(p))
            return DCNV4_ERR_ALIGN;
    a.eps = eps;
    a.inv_c = 1.f / (float)a.C;
    hipStream_t s = (hipStream_t)stream;
    if (branch)
        return dtype == DCNV4_F16 ? launch_norm<_Float16, true>(a, s) : launch_norm<float, true>(a, s);
    return dtype == DCNV4_F16 ? launch_norm<_Float16, false>(a, s) : launch_norm<float, false>(a, s);
}

int norm_backward_impl(NormBackArgs &a, void *grad_gamma, void *grad_beta, void *workspace, long long workspace_bytes, int dtype, bool branch,
                       void *stream)
{
    const bool sums = grad_gamma != nullptr || grad_beta != nullptr;
    if (!a.x || !a.mean || !a.rstd || !a.grad_y || !a.grad_x || (branch && !a.grad_residual) || (sums && !workspace))
        return DCNV4_ERR_NULL;
    const int rc = check_rows(a.P, a.C, dtype);
    if (rc)
        return rc;
    if (sums && workspace_bytes < dcnv4_layer_norm_workspace_bytes(a.P, a.C))
        return DCNV4_ERR_SHAPE;
    for (const void *p : {a.x, a.gamma, (const void *)a.mean, (const void *)a.rstd, a.grad_y, a.grad_z, (const void *)a.grad_x,
                          (const void *)a.grad_residual, (const void *)grad_gamma, (const void *)grad_beta, (const void *)workspace})
        if (misaligned(p))
            return DCNV4_ERR_ALIGN;
    a.inv_c = 1.f / (float)a.C;
    a.partial = sums ? (float *)workspace : nullptr;
    hipStream_t s = (hipStream_t)stream;
    if (branch)
        return dtype == DCNV4_F16 ? launch_norm_backward<_Float16, true>(a, grad_gamma, grad_beta, s)
                                  : launch_norm_backward<float, true>(a, grad_gamma, grad_beta, s);
    return dtype == DCNV4_F16 ? launch_norm_backward<_Float16, false>(a, grad_gamma, grad_beta, s)
                              : launch_norm_backward<float, false>(a, grad_gamma, grad_beta, s);
}

template <typename T>
int launch_dropout(const void *x, const void *residual, void *y, long long n, const Drop &d, hipStream_t s)
{
    const int cus = device_cus();
    if (cus <= 0)
        return DCNV4_ERR_LAUNCH;
    const long long groups = (n + 4095) / 4096, most = 64LL * cus;
    const dim3 grid((unsigned)(groups < most ? groups : most));
    if (residual != nullptr)
        hipLaunchKernelGGL((dcnv4_dropout_kernel<T, true>), grid, dim3(256), 0, s, (const T *)x, (const T *)residual, (T *)y, n, d);
    else
        hipLaunchKernelGGL((dcnv4_dropout_kernel<T, false>), grid, dim3(256), 0, s, (const T *)x, (const T *)nullptr, (T *)y, n, d);
    return hipGetLastError() == hipSuccess ? DCNV4_OK : DCNV4_ERR_LAUNCH;
}

}  // namespace

extern "C" {

int dcnv4_layer_norm(const void *x, const void *gamma, const void *beta, void *y, float *mean, float *rstd, long long P, int C,
                     float eps, int dtype, void *stream)
{
    NormArgs a = {};
    a.x = x;
    a.gamma = gamma;
    a.beta = beta;
    a.y = y;
    a.mean = mean;
    a.rstd = rstd;
    a.P = P;
    a.C = C;
    return norm_impl(a, eps, dtype, false, stream);
}

int dcnv4_layer_norm_backward(const void *x, const void *gamma, const float *mean, const float *rstd, const void *grad_y,
                              void *grad_x, void *grad_gamma, void *grad_beta, void *workspace, long long workspace_bytes,
                              long long P, int C, int dtype, void *stream)
{
    NormBackArgs a = {};
    a.x = x;
    a.gamma = gamma;
    a.mean = mean;
    a.rstd = rstd;
    a.grad_y = grad_y;
    a.grad_x = grad_x;
    a.P = P;
    a.C = C;
    return norm_backward_impl(a, grad_gamma, grad_beta, workspace, workspace_bytes, dtype, false, stream);
}

long long dcnv4_layer_norm_workspace_bytes(long long P, int C)
{
    if (P < 1 || C < 1 || C > kNormMaxChannels)
        return -1;
    // (either type's)
    const int f32 = norm_back_groups<float>(P, C), f16 = norm_back_groups<_Float16>(P, C);
    return (long long)align256((size_t)(f32 > f16 ? f32 : f16) * 2 * (size_t)C * 4);
}

int dcnv4_dropout(const void *x, const void *residual, void *y, long long n, float p, unsigned long long seed,
                  unsigned long long offset, const void *offset_on_device, int dtype, void *stream)
{
    if (!x || !y)
        return DCNV4_ERR_NULL;
    if (n < 1)
        return DCNV4_ERR_SHAPE;
    if ((dtype != DCNV4_F32 && dtype != DCNV4_F16) || n > (1LL << 48))
        return DCNV4_ERR_UNSUPPORTED;
    Drop d;
    const int rc = fill_drop(&d, p, seed, offset, offset_on_device);
    if (rc)
        return rc;
    if (misaligned(x) || misaligned(residual) || misaligned(y))
        return DCNV4_ERR_ALIGN;
    return dtype == DCNV4_F16 ? launch_dropout<_Float16>(x, residual, y, n, d, (hipStream_t)stream)
                              : launch_dropout<float>(x, residual, y, n, d, (hipStream_t)stream);
}

int dcnv4_dropout_backward(const void *grad_y, void *grad_x, long long n, float p, unsigned long long seed,
                           unsigned long long offset, const void *offset_on_device, int dtype, void *stream)
{
    return dcnv4_dropout(grad_y, nullptr, grad_x, n, p, seed, offset, offset_on_device, dtype, stream);
}

int dcnv4_dropout_add_layer_norm(const void *x, const void *residual, const void *gamma, const void *beta, void *z, void *y,
                                 float *mean, float *rstd, long long P, int C, float p, unsigned long long seed,
                                 unsigned long long offset, const void *offset_on_device, float eps, int dtype, void *stream)
{
    NormArgs a = {};
    a.x = x;
    a.residual = residual;
    a.gamma = gamma;
    a.beta = beta;
    a.z = z;
    a.y = y;
    a.mean = mean;
    a.rstd = rstd;
    a.P = P;
    a.C = C;
    const int rc = fill_drop(&a.drop, p, seed, offset, offset_on_device);
    return rc ? rc : norm_impl(a, eps, dtype, true, stream);
}

int dcnv4_dropout_add_layer_norm_backward(const void *z, const void *gamma, const float *mean, const float *rstd,
                                          const void *grad_y, const void *grad_z, void *grad_x, void *grad_residual,
                                          void *grad_gamma, void *grad_beta, void *workspace, long long workspace_bytes,
                                          long long P, int C, float p, unsigned long long seed, unsigned long long offset,
                                          const void *offset_on_device, int dtype, void *stream)
{
    NormBackArgs a = {};
    a.x = z;
    a.gamma = gamma;
    a.mean = mean;
    a.rstd = rstd;
    a.grad_y = grad_y;
    a.grad_z = grad_z;
    a.grad_x = grad_x;
    a.grad_residual = grad_residual;
    a.P = P;
    a.C = C;
    const int rc = fill_drop(&a.drop, p, seed, offset, offset_on_device);
    return rc ? rc : norm_backward_impl(a, grad_gamma, grad_beta, workspace, workspace_bytes, dtype, true, stream);
}

}  // extern "C"
