// What the operators on rows and on lists of tensors share: the counter-based generator, runs of eight elements, sums over lanes.
#pragma once
#include "dcnv4_common.h"

// Products and sums are fused where the code says so and nowhere else, so that kernels that share a formula give the same bits.
#pragma clang fp contract(off)

namespace {

// Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011).  Key: the seed; counter:
// (block, offset), 64 bits each.  A block serves eight elements, 16 bits each.
struct Bits8 {
    unsigned w[4];
};

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

// Eight numbers of each lane summed over the rows that THREADS lanes hold side by side, L lanes a row, in the lanes of the first row.
// `sums`: THREADS * 8 numbers.
template <int L, int THREADS> __device__ __forceinline__ void add_rows_of_workgroup(float (&v)[8], float *sums)
{
    // rows side by side in a wave first: lanes 8, 4, 2, 1 further round (of 16), then rows of 16 and halves
    constexpr int G = L < 64 ? L : 64, W = THREADS / 64;
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
    const int wave = (int)threadIdx.x >> 6, in = (int)threadIdx.x % L % G;
    __syncthreads();                                       // all have read what was there before
    if ((int)(threadIdx.x & 63) < G)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            sums[(wave * 8 + e) * G + in] = v[e];
    __syncthreads();
    if ((int)threadIdx.x < L)
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int w = PARTS; w < W; w += PARTS)
                v[e] += sums[((w + wave) * 8 + e) * G + in];
}

constexpr int norm_threads(int L) { return L >= 256 ? 512 : 256; }

// Where a lane's run j lies in its row, in runs: side by side in a wave, then run after run, then the next wave's.
template <int L, int NV> __device__ __forceinline__ int run_of(int l, int j)
{
    constexpr int G = L < 64 ? L : 64;
    return (l / G * NV + j) * G + l % G;
}

}  // namespace
