// A step of AdamW over many tensors at once (dcnv4_adamw of include/dcnv4.h; Loshchilov, Hutter, "Decoupled weight decay regularization", 2019):
//     m = b1 m + (1 - b1) g,   v = b2 v + (1 - b2) g^2,   p = p (1 - lr wd) - lr / (1 - b1^t) * m / (sqrt(v / (1 - b2^t)) + eps)
// with m and v in fp32, or m and r = sqrt(v) in 8 bits (e4m3: 3 bits behind the point) times an fp32 scale per block of 256 elements.  The root is
// kept, and not v, since e4m3 reaches from 448 down to 2^-9: 18 powers of two of r are 36 of v.  m is rounded to nearest.  r is rounded
// to either neighbour, with the probability that keeps its mean: with b2 = 0.999 a step moves r by less than a thousandth, and rounding to the nearest (up
// to 1/16 away) would take it back to where it was, for good.  r above zero does not become zero, which would leave eps alone to divide by, but in blocks
// whose largest is below 2^-75 (as v in fp32 is zero below 2^-150): r is the root of v in 64 bits, not of v in fp32, which a small r beside larger ones has not.
//
// Memory bounds it: an element is read and written once.  The moments are made in 64 bits (their rate leaves room for it), so that what is rounded to 8 bits
// does not hang on the order of operations.  A launch takes up to kRecords tensors, whose addresses travel with its
// arguments: nothing has to be copied to the device first, so a captured step needs no memory of its own.
// A lane takes one run of eight and ends: two or four of them one after the other, the next asked for early, take longer wherever it was
// measured (55 million parameters in 54 tensors, fp16 gradients and copies, states of 32 bits: 285 us, 292 by two, 299 by four; 78 million in 314,
// states of 8 bits: 264, 282, 296; 65536 in one: 5.6, 5.6, 7.1).  That is 5.35 TB/s and 4.8, where a large copy has 4.98.
#include <float.h>
#include <math.h>

#include <type_traits>

#include "dcnv4_rows.h"

namespace {

constexpr int kAdamBlock = 256;                            // elements that share a scale
constexpr int kPart = 256 * 8;                             // elements of a workgroup: a run of eight to a lane
constexpr int kRecords = 56;                               // of a launch: its arguments are 4 KiB at most
constexpr float kTop = 448.f;                              // e4m3's largest number
constexpr float kNoM = 0x1p-100f, kNoR = 0x1p-75f;         // a block whose largest is less is stored as zeros

struct AdamTensor {
    long long n;
    float *p;
    const void *g;
    void *m, *v;
    float2 *scales;
    _Float16 *copy;
    float lr, decay;                                       // decay: lr * wd
};

struct AdamArgs {
    AdamTensor t[kRecords];
    int first[kRecords];                                   // each tensor's first workgroup
    int count, number;                                     // tensors of this launch; number of the first one in the call
    double b1, b2, log_b1, log_b2;                         // logarithms: where the step's number is on the device
    double unbias1;                                        // 1 / (1 - b1^t)
    float unbias2, eps;                                    // 1 / sqrt(1 - b2^t)
    long long step;
    unsigned long long seed;
    const long long *more;                                 // null, or a number that is added to the step's
    const float *factors;                                  // null, or what gradients and learning rates are multiplied with
};
static_assert(sizeof(AdamArgs) <= 4096);

// Runs of eight elements, aligned to their size (16 bytes at most); `left` of them are there.
template <typename T> __device__ __forceinline__ Raw8<T> take(const T *p, long long left)
{
    typedef Raw8<T> whole __attribute__((aligned(sizeof(T) == 1 ? 8 : 16)));
    Raw8<T> r = {};
    if (left >= 8) {
        r = *reinterpret_cast<const whole *>(p);
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < left)
                r[e] = p[e];
    }
    return r;
}
template <typename T> __device__ __forceinline__ void put(T *p, long long left, Raw8<T> r)
{
    typedef Raw8<T> whole __attribute__((aligned(sizeof(T) == 1 ? 8 : 16)));
    if (left >= 8) {
        *reinterpret_cast<whole *>(p) = r;
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < left)
                p[e] = r[e];
    }
}

typedef unsigned char Byte;

// Eight numbers of e4m3, and back (to nearest even; what is more than 448 is the caller's).
__device__ __forceinline__ void from_8_bits(Raw8<Byte> r, float (&f)[8])
{
    const u32x2 w = __builtin_bit_cast(u32x2, r);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[k], true);
        f[4 * k] = lo[0];
        f[4 * k + 1] = lo[1];
        f[4 * k + 2] = hi[0];
        f[4 * k + 3] = hi[1];
    }
}
__device__ __forceinline__ Raw8<Byte> to_8_bits(const float (&f)[8])
{
    u32x2 w;
#pragma unroll
    for (int k = 0; k < 2; ++k)
        w[k] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * k + 2], f[4 * k + 3], __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * k], f[4 * k + 1], 0, false), true);
    return __builtin_bit_cast(Raw8<Byte>, w);
}

// The largest of a block, in each of its 32 lanes.
__device__ __forceinline__ float block_max(float v)
{
    v = fmaxf(v, dpp<0xB1>(v));                            // (exchanges as in wave_sum)
    v = fmaxf(v, dpp<0x4E>(v));
    v = fmaxf(v, dpp<0x141>(v));
    v = fmaxf(v, dpp<0x140>(v));
    float a = v, b = v;
    asm("s_nop 1\n\tv_permlane16_swap_b32 %0, %1" : "+v"(a), "+v"(b));
    return fmaxf(a, b);
}

// The root of a number of 64 bits in fp32, below fp32's range too: its bits, where v has a square there, are those of (float)v's root.
__device__ __forceinline__ float root_of(double v)
{
    const bool small = v < 0x1p-100;
    return __builtin_sqrtf((float)(small ? v * 0x1p200 : v)) * (small ? 0x1p-100f : 1.f);
}

// A number t from 0 to 448 to one of its neighbours in e4m3, up with probability (missing part) by 16 bits; what is above zero, whatever t is, not to zero.
__device__ __forceinline__ float round_by(float t, bool above_zero, unsigned bits)
{
    const float fine = __builtin_bit_cast(float, (__builtin_bit_cast(unsigned, t) + (bits << 4)) & ~0xFFFFFu);
    const float coarse = (float)(((int)(t * 0x1p25f) + (int)bits) >> 16) * 0x1p-9f;      // numbers below 2^-6 are 2^-9 apart
    float q = t < 0x1p-6f ? coarse : fine;
    q = q < 0x1p-9f ? 0x1p-9f : q;
    return above_zero ? q : 0.f;
}

}  // namespace

template <typename T, bool EIGHT> __global__ __launch_bounds__(256) void dcnv4_adamw_kernel(AdamArgs a)
{
    typedef std::conditional_t<EIGHT, Byte, float> S;
    const int lane = (int)threadIdx.x & 63;
    // the tensor that this workgroup is in: how many of the launch's begin before or with it
    const int before = lane < a.count ? a.first[lane] : 0x7fffffff;
    const int at = __builtin_popcountll(__builtin_amdgcn_ballot_w64(before <= (int)blockIdx.x)) - 1;
    const AdamTensor &t = a.t[at];
    const long long i = (long long)((int)blockIdx.x - a.first[at]) * kPart + (int)threadIdx.x * 8, left = t.n - i;
    if (i - (i & (kAdamBlock - 1)) >= t.n)                 // (all lanes of a block or none, for the exchanges between them)
        return;
    const Raw8<float> p = take(t.p + i, left);
    const Raw8<T> grad = take((const T *)t.g + i, left);
    const Raw8<S> m0 = take((const S *)t.m + i, left), v0 = take((const S *)t.v + i, left);
    const float2 s = EIGHT ? t.scales[i / kAdamBlock] : float2{};
    double by = 1.0, lr = (double)t.lr, unbias1 = a.unbias1;
    float decay = t.decay, unbias2 = a.unbias2;
    long long step = a.step;
    if (a.factors != nullptr) {
        const float f0 = a.factors[0], f1 = a.factors[1];
        if (!(fabsf(f0) < __builtin_inff()))
            return;                                        // (the whole grid)
        by = (double)f0;
        lr *= (double)f1;
        decay *= f1;
    }
    if (a.more != nullptr) {
        step += *a.more;
        step = step < 1 ? 1 : step;
        unbias1 = -1.0 / expm1((double)step * a.log_b1);
        unbias2 = (float)(1.0 / sqrt(-expm1((double)step * a.log_b2)));
    }
    const float rate = (float)(lr * unbias1);
    const double c1 = 1.0 - a.b1, c2 = 1.0 - a.b2;
    float m[8], r[8], v[8];
    bool some[8];                                          // of v
    double sm = 1.0, sr = 1.0;
    if constexpr (EIGHT) {
        from_8_bits(m0, m);
        from_8_bits(v0, v);
        sm = (double)s.x;
        sr = (double)s.y;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            m[e] = m0[e];
            v[e] = v0[e];
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const double g = (double)(float)grad[e] * by;
        double mm = (double)m[e], vv = (double)v[e];
        if constexpr (EIGHT) {
            mm *= sm;
            vv *= sr;
            vv *= vv;
        }
        m[e] = (float)__builtin_fma(a.b1, mm, c1 * g);
        vv = __builtin_fma(a.b2, vv, c2 * (g * g));
        v[e] = (float)vv;
        r[e] = EIGHT ? root_of(vv) : __builtin_sqrtf(v[e]);
        some[e] = vv > 0.;
    }
    Raw8<float> out;
    Raw8<_Float16> half;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float move = rate * m[e] * __builtin_amdgcn_rcpf(__builtin_fmaf(r[e], unbias2, a.eps));
        out[e] = __builtin_fmaf(-decay, p[e], p[e]) - move;
        half[e] = (_Float16)out[e];
    }
    put(t.p + i, left, out);
    if (t.copy != nullptr)
        put(t.copy + i, left, half);
    if constexpr (EIGHT) {
        float tm = 0.f, tr = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {                  // (behind the last element: zeros)
            tm = fmaxf(tm, fabsf(m[e]));
            tr = fmaxf(tr, r[e]);
        }
        tm = block_max(tm);
        tr = block_max(tr);
        tm = tm >= kNoM ? tm : 0.f;
        tr = tr >= kNoR ? tr : 0.f;
        const float im = tm > 0.f ? kTop / tm : 0.f, ir = tr > 0.f ? kTop / tr : 0.f;
        const Bits8 bits = philox((unsigned long long)(i >> 3) + ((unsigned long long)(a.number + at) << 40), (unsigned long long)step, a.seed);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            m[e] *= im;
            m[e] = m[e] > kTop ? kTop : m[e] < -kTop ? -kTop : m[e];
            r[e] *= ir;
            r[e] = round_by(r[e] > kTop ? kTop : r[e], some[e] && tr > 0.f, (bits.w[e / 2] >> (16 * (e & 1))) & 0xffffu);
        }
        put((Byte *)t.m + i, left, to_8_bits(m));
        put((Byte *)t.v + i, left, to_8_bits(r));
        if ((lane & 31) == 0 && left > 0)
            t.scales[i / kAdamBlock] = make_float2(tm * (1.f / kTop), tr * (1.f / kTop));
    } else {
        Raw8<float> mo, vo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            mo[e] = m[e];
            vo[e] = v[e];
        }
        put((float *)t.m + i, left, mo);
        put((float *)t.v + i, left, vo);
    }
}

namespace {

bool aligned_to(const void *p, unsigned bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

int check_tensor(const dcnv4_adamw_tensor &t, bool eight, bool f16)
{
    if (!t.param || !t.grad || !t.m || !t.v || (eight && !t.scales))
        return DCNV4_ERR_NULL;
    if (t.n < 1)
        return DCNV4_ERR_SHAPE;
    // (a launch has fewer than 2^32 lanes; learning rates and decays of any sign are a caller's choice)
    if (t.n > (1LL << 34) || (t.copy && !f16) || !(fabs(t.lr) <= 3e38) || !(fabs(t.lr * t.weight_decay) <= 3e38))
        return DCNV4_ERR_UNSUPPORTED;
    if (!aligned_to(t.param, 16) || !aligned_to(t.grad, 16) || !aligned_to(t.m, 16) || !aligned_to(t.v, 16) || !aligned_to(t.copy, 16) ||
        (eight && !aligned_to(t.scales, 8)))
        return DCNV4_ERR_ALIGN;
    return DCNV4_OK;
}

template <typename T> void launch_adamw(const AdamArgs &a, unsigned groups, bool eight, hipStream_t s)
{
    if (eight)
        hipLaunchKernelGGL((dcnv4_adamw_kernel<T, true>), dim3(groups), dim3(256), 0, s, a);
    else
        hipLaunchKernelGGL((dcnv4_adamw_kernel<T, false>), dim3(groups), dim3(256), 0, s, a);
}

}  // namespace

extern "C" int dcnv4_adamw(const dcnv4_adamw_tensor *tensors, int count, double beta1, double beta2, double eps, long long step,
                           const void *step_on_device, const void *factors_on_device, unsigned long long seed, int state_bits, int dtype,
                           void *stream)
{
    if (!tensors)
        return DCNV4_ERR_NULL;
    if (count < 1)
        return DCNV4_ERR_SHAPE;
    const bool eight = state_bits == 8, f16 = dtype == DCNV4_F16;
    if ((dtype != DCNV4_F32 && !f16) || (!eight && state_bits != 32) || count > (1 << 20))
        return DCNV4_ERR_UNSUPPORTED;
    if (!(beta1 >= 0. && beta1 < 1.) || !(beta2 >= 0. && beta2 < 1.) || !(eps >= (double)FLT_MIN && eps <= 3e38) || step < (step_on_device ? 0 : 1))
        return DCNV4_ERR_UNSUPPORTED;
    if (!aligned_to(step_on_device, 8) || !aligned_to(factors_on_device, 8))
        return DCNV4_ERR_ALIGN;
    for (int i = 0; i < count; ++i)
        if (const int rc = check_tensor(tensors[i], eight, f16))
            return rc;
    AdamArgs a;
    a.b1 = beta1;
    a.b2 = beta2;
    a.log_b1 = log(beta1);                                 // (-infinity for 0: 1 - 0^t = 1)
    a.log_b2 = log(beta2);
    a.unbias1 = step > 0 ? -1. / expm1((double)step * a.log_b1) : 1.;
    a.unbias2 = step > 0 ? (float)(1. / sqrt(-expm1((double)step * a.log_b2))) : 1.f;
    a.eps = (float)eps;
    a.step = step;
    a.seed = seed;
    a.more = (const long long *)step_on_device;
    a.factors = (const float *)factors_on_device;
    for (int from = 0; from < count;) {
        long long groups = 0;
        a.count = 0;
        a.number = from;
        for (; from < count && a.count < kRecords; ++from) {
            const dcnv4_adamw_tensor &t = tensors[from];
            const long long more = (t.n + kPart - 1) / kPart;
            if (groups + more >= 1 << 24)                  // (a tensor has 2^23 at most)
                break;
            a.first[a.count] = (int)groups;
            a.t[a.count++] = {t.n, t.param, t.grad, t.m, t.v, (float2 *)t.scales, (_Float16 *)t.copy, (float)t.lr, (float)(t.lr * t.weight_decay)};
            groups += more;
        }
        if (f16)
            launch_adamw<_Float16>(a, (unsigned)groups, eight, (hipStream_t)stream);
        else
            launch_adamw<float>(a, (unsigned)groups, eight, (hipStream_t)stream);
        if (hipGetLastError() != hipSuccess)
            return DCNV4_ERR_LAUNCH;
    }
    return DCNV4_OK;
}
