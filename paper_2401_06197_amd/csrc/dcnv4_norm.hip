// Layer norm, dropout, and the end of a residual branch (dropout, add, layer norm in one pass), each with its gradient, on
// rows of C channels: the C ABI entry points of include/dcnv4.h and their kernels.
//
// All of it is bound by memory: a kernel reads each input once, keeps a row in registers while its statistics are made, and
// writes each output once.  A lane holds runs of eight channels (16 bytes in fp16, 32 in fp32).  A row belongs to L lanes: as
// few of a wave as its runs need, whole waves for wide rows.
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

// The bits of eight elements from element i on.  WHOLE: i is a multiple of eight.
template <bool WHOLE>
__device__ __forceinline__ Bits8 drop_bits(unsigned long long i, unsigned long long offset, unsigned long long seed)
{
    const Bits8 lo = philox(i >> 3, offset, seed);
    if constexpr (WHOLE)
        return lo;
    const Bits8 hi = philox((i >> 3) + 1, offset, seed);
    const unsigned words = (unsigned)(i >> 1) & 3u, half = ((unsigned)i & 1u) * 16u;
    unsigned c[8], s[5];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        c[k] = lo.w[k];
        c[4 + k] = hi.w[k];
    }
#pragma unroll
    for (int k = 0; k < 5; ++k) {                          // (word k + words: at most 7)
        const unsigned even = words & 2u ? c[k + 2] : c[k], odd = words & 2u ? c[k + 3] : c[k + 1];
        s[k] = words & 1u ? odd : even;
    }
    Bits8 out;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        out.w[k] = __builtin_amdgcn_alignbit(s[k + 1], s[k], half);
    return out;
}

// Element e of the eight: r + v scaled, or r alone whatever v is.
__device__ __forceinline__ float drop_apply(const Bits8 &b, int e, const Drop &d, float v, float r)
{
    const unsigned half = (b.w[e / 2] >> (16 * (e & 1))) & 0xffffu;
    return half < d.limit ? r : __builtin_fmaf(v, d.scale, r);
}

// ------------------------------------------------------------------------------------------
// Runs of eight channels.  WHOLE: C is a multiple of eight, so that every run is whole and aligned; otherwise rows start at any
// element (memory instructions of 16 bytes take any address), and the last run of a row may be short.
// ------------------------------------------------------------------------------------------
template <typename T> struct __attribute__((packed, aligned(sizeof(T)))) Run8 {
    T e[8];
};

template <typename T, bool WHOLE> __device__ __forceinline__ void load8(const T *p, int n, bool past, float (&v)[8])
{
    // n channels of the row; `past`: eight would reach past the end of the tensor
    if (n <= 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = 0.f;
    } else if (WHOLE) {
        const T *q = (const T *)__builtin_assume_aligned(p, 16);
        T t[8];
        __builtin_memcpy(t, q, sizeof(t));
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = (float)t[e];
    } else if (n >= 8 || !past) {
        const Run8<T> t = *reinterpret_cast<const Run8<T> *>(p);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = e < n ? (float)t.e[e] : 0.f;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = e < n ? (float)p[e] : 0.f;
    }
}

template <typename T, bool WHOLE> __device__ __forceinline__ void store8(T *p, int n, const float (&v)[8])
{
    if (n <= 0)
        return;
    T t[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        t[e] = (T)v[e];                                    // one rounding to nearest even
    if (WHOLE) {
        __builtin_memcpy(__builtin_assume_aligned(p, 16), t, sizeof(t));
    } else if (n >= 8) {
        Run8<T> r;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            r.e[e] = t[e];
        *reinterpret_cast<Run8<T> *>(p) = r;
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n)
                p[e] = t[e];
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
    static_assert(L >= 8 && L <= 64);
    v += dpp<0xB1>(v);                                     // quad_perm [1,0,3,2]
    v += dpp<0x4E>(v);                                     // quad_perm [2,3,0,1]
    v += dpp<0x141>(v);                                    // row_half_mirror
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
        const int wave = (int)threadIdx.x >> 6;
        __syncthreads();                                   // all have read the sums before these
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int k = 0; k < N; ++k)
                lds[wave][k] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = lds[0][k];
#pragma unroll
            for (int w = 1; w < W; ++w)
                v[k] += lds[w][k];
        }
    }
}

constexpr int norm_threads(int L) { return L > 256 ? L : 256; }

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
    __shared__ float lds[L > 64 ? L / 64 : 1][1];
    const int l = (int)threadIdx.x % L;
    const T *gamma = (const T *)a.gamma, *beta = (const T *)a.beta;
    const unsigned long long offset = BRANCH ? drop_offset(a.drop) : 0ull;
    const long long all = a.P * a.C;
    for (long long row = (long long)blockIdx.x * R + (int)threadIdx.x / L; row < a.P; row += (long long)gridDim.x * R) {
        const long long at = row * a.C;
        float v[NV][8], s[1] = {0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * L + l) * 8, n = a.C - c;
            load8<T, WHOLE>((const T *)a.x + at + c, n, all - at - c < 8, v[j]);
            if constexpr (BRANCH) {
                float r[8];
                load8<T, WHOLE>((const T *)a.residual + at + c, n, all - at - c < 8, r);
                if (n > 0) {
                    const Bits8 b = drop_bits<WHOLE>((unsigned long long)(at + c), offset, a.drop.seed);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        v[j][e] = WHOLE || e < n ? (float)(T)drop_apply(b, e, a.drop, v[j][e], r[e]) : 0.f;
                    store8<T, WHOLE>((T *)a.z + at + c, n, v[j]);
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
                s[0] += v[j][e];
        }
        row_sums<L, 1>(s, lds);
        const float mean = s[0] / (float)a.C;              // (divided: the mean of equal numbers that add up exactly is that number)
        s[0] = 0.f;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int n = a.C - (j * L + l) * 8;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = v[j][e] - mean;
                if (WHOLE ? n > 0 : e < n)
                    s[0] = __builtin_fmaf(d, d, s[0]);
            }
        }
        row_sums<L, 1>(s, lds);
        const float rstd = 1.f / __builtin_sqrtf(__builtin_fmaf(s[0], a.inv_c, a.eps));
        if (l == 0) {
            if (a.mean != nullptr)
                a.mean[row] = mean;
            if (a.rstd != nullptr)
                a.rstd[row] = rstd;
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * L + l) * 8, n = a.C - c;
            float g[8], b[8], y[8];
            if (gamma != nullptr)
                load8<T, WHOLE>(gamma + c, n, true, g);
            if (beta != nullptr)
                load8<T, WHOLE>(beta + c, n, true, b);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                y[e] = (v[j][e] - mean) * rstd;
                if (gamma != nullptr)
                    y[e] = beta != nullptr ? __builtin_fmaf(y[e], g[e], b[e]) : y[e] * g[e];
                else if (beta != nullptr)
                    y[e] += b[e];
            }
            store8<T, WHOLE>((T *)a.y + at + c, n, y);
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
    __shared__ float lds[L > 64 ? L / 64 : 1][2];
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
    const long long all = a.P * a.C;
    for (long long row = (long long)blockIdx.x * R + first; row < a.P; row += (long long)gridDim.x * R) {
        const long long at = row * a.C;
        const float mean = a.mean[row], rstd = a.rstd[row];
        float xh[NV][8], g[NV][8], s[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * L + l) * 8, n = a.C - c;
            load8<T, WHOLE>((const T *)a.x + at + c, n, all - at - c < 8, xh[j]);
            load8<T, WHOLE>((const T *)a.grad_y + at + c, n, all - at - c < 8, g[j]);
            float gm[8];
            if (gamma != nullptr)
                load8<T, WHOLE>(gamma + c, n, true, gm);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                xh[j][e] = (WHOLE ? n > 0 : e < n) ? (xh[j][e] - mean) * rstd : 0.f;
                dg[j][e] = __builtin_fmaf(g[j][e], xh[j][e], dg[j][e]);
                db[j][e] += g[j][e];
                if (gamma != nullptr)
                    g[j][e] *= gm[e];
                s[0] += g[j][e];
                s[1] = __builtin_fmaf(g[j][e], xh[j][e], s[1]);
            }
        }
        row_sums<L, 2>(s, lds);
        const float m0 = s[0] * a.inv_c, m1 = s[1] * a.inv_c;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = (j * L + l) * 8, n = a.C - c;
            float out[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                out[e] = rstd * __builtin_fmaf(-xh[j][e], m1, g[j][e] - m0);
                asm("" : "+v"(out[e]));                    // (an fp32 number here: not one instruction with the store's rounding)
            }
            if constexpr (BRANCH) {
                if (a.grad_z != nullptr) {
                    float r[8];
                    load8<T, WHOLE>((const T *)a.grad_z + at + c, n, all - at - c < 8, r);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        out[e] += r[e];
                }
                store8<T, WHOLE>((T *)a.grad_residual + at + c, n, out);
                if (n > 0) {
                    const Bits8 b = drop_bits<WHOLE>((unsigned long long)(at + c), offset, a.drop.seed);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        out[e] = drop_apply(b, e, a.drop, out[e], 0.f);
                }
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
            const int c = (j * L + l) * 8;
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] = k == 0 ? dg[j][e] : db[j][e];
            if constexpr (R > 1) {
                __syncthreads();                           // all have read what was there before
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    sums[(first * 8 + e) * L + l] = v[e];
                __syncthreads();
                if (first == 0)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
#pragma unroll 4
                        for (int r = 1; r < R; ++r)
                            v[e] += sums[(r * 8 + e) * L + l];
            }
            if (first == 0)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (c + e < a.C)
                        to[k * a.C + c + e] = v[e];
        }
    }
}

// Adds up partial sums [count][2 * C]: 16 columns to a workgroup, 64 of the rows side by side, joined through LDS.
template <typename T>
__global__ __launch_bounds__(1024) void dcnv4_norm_join_kernel(const float *__restrict__ partial, int count, int C, T *grad_gamma, T *grad_beta)
{
    __shared__ float sums[64][17];
    const int col = (int)blockIdx.x * 16 + ((int)threadIdx.x & 15), slice = (int)threadIdx.x >> 4;
    float s = 0.f;
    if (col < 2 * C)
#pragma unroll 8
        for (int r = slice; r < count; r += 64)
            s += partial[(long long)r * 2 * C + col];
    sums[slice][threadIdx.x & 15] = s;
    __syncthreads();
    if (threadIdx.x < 16 && col < 2 * C) {
        s = 0.f;
#pragma unroll 8
        for (int r = 0; r < 64; ++r)
            s += sums[r][threadIdx.x];
        T *to = col < C ? grad_gamma : grad_beta;
        if (to != nullptr)
            to[col < C ? col : col - C] = (T)s;
    }
}

// out = [residual +] dropout(x), eight elements a lane.
template <typename T, bool ADD>
__global__ __launch_bounds__(256) void dcnv4_dropout_kernel(const T *__restrict__ x, const T *__restrict__ residual, T *__restrict__ y, long long n,
                                                            Drop d)
{
    const unsigned long long offset = drop_offset(d);
    for (long long i = ((long long)blockIdx.x * 256 + (int)threadIdx.x) * 8; i < n; i += (long long)gridDim.x * 2048) {
        float v[8], r[8];
        const int left = (int)(n - i < 8 ? n - i : 8);
        if (left == 8) {
            load8<T, true>(x + i, 8, false, v);
            if (ADD)
                load8<T, true>(residual + i, 8, false, r);
        } else {
            load8<T, false>(x + i, left, true, v);
            if (ADD)
                load8<T, false>(residual + i, left, true, r);
        }
        const Bits8 b = drop_bits<true>((unsigned long long)i, offset, d.seed);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = drop_apply(b, e, d, v[e], ADD ? r[e] : 0.f);
        if (left == 8)
            store8<T, true>(y + i, 8, v);
        else
            store8<T, false>(y + i, left, v);
    }
}

namespace {

// Rows wider than this are refused: 512 lanes with four runs of eight each.
constexpr int kNormMaxChannels = 16384;
// Workgroups of the backward pass, each of which leaves partial sums of 2 * C.
constexpr int kNormBackGroups = 1024;

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

// Calls f with the lanes of a row and a lane's runs of eight channels, as constants.
template <typename F> int by_width(int C, F &&f)
{
    const int runs = (C + 7) / 8;
    if (runs <= 8) return f(std::integral_constant<int, 8>(), std::integral_constant<int, 1>());
    if (runs <= 16) return f(std::integral_constant<int, 16>(), std::integral_constant<int, 1>());
    if (runs <= 32) return f(std::integral_constant<int, 32>(), std::integral_constant<int, 1>());
    if (runs <= 64) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 1>());
    if (runs <= 128) return f(std::integral_constant<int, 64>(), std::integral_constant<int, 2>());
    if (runs <= 256) return f(std::integral_constant<int, 256>(), std::integral_constant<int, 1>());
    if (runs <= 512) return f(std::integral_constant<int, 256>(), std::integral_constant<int, 2>());
    if (runs <= 1024) return f(std::integral_constant<int, 256>(), std::integral_constant<int, 4>());
    return f(std::integral_constant<int, 512>(), std::integral_constant<int, 4>());
}

int norm_back_groups(long long P, int C)
{
    int groups = 0;
    by_width(C, [&](auto L, auto) {
        const long long rows = norm_threads(L()) / L(), n = (P + rows - 1) / rows;
        groups = (int)(n < kNormBackGroups ? n : kNormBackGroups);
        return 0;
    });
    return groups;
}

template <typename T, bool BRANCH> int launch_norm(const NormArgs &a, hipStream_t s)
{
    const int cus = device_cus();
    if (cus <= 0)
        return DCNV4_ERR_LAUNCH;
    return by_width(a.C, [&](auto L, auto NV) {
        constexpr int threads = norm_threads(L());
        const long long rows = threads / L(), groups = (a.P + rows - 1) / rows, most = 64LL * cus;
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
    const int groups = norm_back_groups(a.P, a.C);
    const int rc = by_width(a.C, [&](auto L, auto NV) {
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
    const long long groups = (n + 2047) / 2048, most = 64LL * cus;
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
    return (long long)align256((size_t)norm_back_groups(P, C) * 2 * (size_t)C * 4);
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
