// The end of a residual block with its norms, in one pass, and its gradient (dcnv4_norm_scale_add_norm of include/dcnv4.h), on rows of C channels:
//     b = first(x),   z = residual + gate[image] * scale * b,   y = second(z)
// first, second: layer norms, either of which may be missing (then b = x, or there is no y).  Networks of DCNv4 modules have the first (norms
// behind the branch) or the second (in front of the next one), scale per channel, and gate as stochastic depth's 0 or 1 / keep.
//
// Backward, with gz the whole gradient of z (that of y through the second norm, and what comes down the residual path), xh = (x - mean) * rstd (or x):
//     q = gate * gz,  S1 = sum over rows of q * xh,  S0 = of q:   grad_scale = gamma * S1 + beta * S0,   grad_gamma = scale * S1,   grad_beta = scale * S0
//     h = q * scale * gamma:   grad_x = rstd * (h - avg(h) - xh * avg(h * xh)),    grad_gate = sum over an image of gz * scale * b
// so two sums a channel serve the three gradients around the first norm.
//
// Memory bounds it: each tensor is read or written once.  A lane holds one run of eight channels, a row L of them (up to sixteen waves), workgroups are
// persistent and ask for the next row before they deal with the present one, sums over rows stay in registers and are joined in a
// fixed order by a second launch (no atomics).  134400 x 256 fp16, first norm, scale and gate: forward 44 us (207 MB, 4.7 TB/s), backward 43 (212 MB, 4.9) and 5 for
// the join; 5883 x 321 fp32, both norms: 12.2, 15.7 and 4.5 (2.5 and 3.2 TB/s: three rows a lane in one round, rows that end inside a run).
#include <math.h>

#include <initializer_list>
#include <type_traits>

#include "dcnv4_rows.h"

namespace {

constexpr int end_threads(int L) { return L <= 128 ? 256 : L <= 512 ? 512 : 1024; }

struct EndArgs {
    const void *x, *residual;
    const void *gamma1, *beta1, *scale, *gamma2, *beta2;   // null: ones, zeros
    const float *gate;                                     // null: ones
    void *z, *y;
    float *mean1, *rstd1, *mean2, *rstd2;                  // null: not asked for
    long long P;
    FastDiv rows;                                          // of an image
    int C;
    float inv_c, eps;
};

struct EndBackArgs {
    const void *x, *z;
    const void *gamma1, *beta1, *scale, *gamma2;
    const float *gate, *mean1, *rstd1, *mean2, *rstd2;
    const void *grad_y, *grad_z;                           // grad_z: null for zeros
    void *grad_x, *grad_residual;                          // grad_residual: null where grad_z is it
    float *partial;                                        // [workgroup][planes][C]: S1, S0 (of a first norm), then the sums of a second norm
    float *row_sums;                                       // [P], or null: gz * scale * b
    long long P;
    FastDiv rows;
    int C;
    float inv_c;
};

// A lane's eight of a vector over the channels, `other` where there is no vector, zeros behind the row's end.
template <typename T, bool WHOLE> __device__ __forceinline__ Raw8<T> channels(const void *p, int c, int n, float other)
{
    if (p != nullptr)
        return load8<T, WHOLE>((const T *)p + c, n, false);
    Raw8<T> r;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        r[e] = (T)(e < n ? other : 0.f);
    return r;
}

}  // namespace

template <typename T, int L, bool FIRST, bool SECOND, bool WHOLE>
__global__ __launch_bounds__(end_threads(L)) void dcnv4_end_kernel(EndArgs a)
{
    constexpr int R = end_threads(L) / L;                  // rows of a workgroup
    __shared__ float lds[end_threads(L) / 64][1];
    const int l = (int)threadIdx.x % L, first = (int)threadIdx.x / L, c = l * 8, left = a.C - c;
    const long long all = a.P * a.C, stride = (long long)gridDim.x * R;
    Raw8<T> x, res;
    float gate = 1.f;
    auto load = [&](long long row) {                       // (a row past the last: nothing)
        const bool safe = (row + 1) * a.C + 7 <= all;
        const int n = row < a.P ? left : 0;
        x = load8<T, WHOLE>((const T *)a.x + row * a.C + c, n, safe);
        res = load8<T, WHOLE>((const T *)a.residual + row * a.C + c, n, safe);
        if (a.gate != nullptr && row < a.P)
            gate = a.gate[fdiv((int)row, a.rows)];
    };
    long long base = (long long)blockIdx.x * R;
    load(base + first);
    const Mask8<T> mask(left);
    const Raw8<T> sc = channels<T, WHOLE>(a.scale, c, left, 1.f);
    Raw8<T> gm1, bt1, gm2, bt2;
    if constexpr (FIRST) {
        gm1 = channels<T, WHOLE>(a.gamma1, c, left, 1.f);
        bt1 = channels<T, WHOLE>(a.beta1, c, left, 0.f);
    }
    if constexpr (SECOND) {
        gm2 = channels<T, WHOLE>(a.gamma2, c, left, 1.f);
        bt2 = channels<T, WHOLE>(a.beta2, c, left, 0.f);
    }
    // v becomes (v - mean) * rstd; nothing of what lies behind the row's end enters the sums
    float mean, rstd;
    auto norm = [&](float (&v)[8]) {
        float s[1] = {0.f};
#pragma unroll
        for (int e = 0; e < 8; ++e)
            s[0] += v[e];
        row_sums<L, 1>(s, lds);
        mean = s[0] / (float)a.C;
        s[0] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e] = e < left ? v[e] - mean : 0.f;
            s[0] = __builtin_fmaf(v[e], v[e], s[0]);
        }
        row_sums<L, 1>(s, lds);
        rstd = 1.f / __builtin_sqrtf(__builtin_fmaf(s[0], a.inv_c, a.eps));
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] *= rstd;
    };
    for (; base < a.P; base += stride) {                   // (the whole workgroup, for the barriers of wide rows)
        const long long row = base + first, at = row * a.C + c;
        const bool live = row < a.P;
        const float by = gate;
        float v[8], r[8];
        unpack<T, WHOLE>(x, mask, v);
        unpack<T, WHOLE>(res, mask, r);
        load(row + stride);
        if constexpr (FIRST) {
            norm(v);
            if (l == 0 && live) {
                if (a.mean1 != nullptr)
                    a.mean1[row] = mean;
                if (a.rstd1 != nullptr)
                    a.rstd1[row] = rstd;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] = __builtin_fmaf(v[e], (float)gm1[e], (float)bt1[e]);
        }
        // (a gate of zero leaves the residual alone, whatever the branch holds; behind the row: zeros)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float sum = __builtin_fmaf(by * (float)sc[e], v[e], r[e]);
            asm("" : "+v"(sum));                           // (an fp32 number here: not one instruction with the rounding)
            v[e] = (float)(T)(by != 0.f && e < left ? sum : r[e]);
        }
        store8<T, WHOLE>((T *)a.z + at, live ? left : 0, v);
        if constexpr (SECOND) {
            norm(v);
            if (l == 0 && live) {
                if (a.mean2 != nullptr)
                    a.mean2[row] = mean;
                if (a.rstd2 != nullptr)
                    a.rstd2[row] = rstd;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] = __builtin_fmaf(v[e], (float)gm2[e], (float)bt2[e]);
            store8<T, WHOLE>((T *)a.y + at, live ? left : 0, v);
        }
    }
}

template <typename T, int L, bool FIRST, bool SECOND, bool WHOLE>
__global__ __launch_bounds__(end_threads(L)) void dcnv4_end_backward_kernel(EndBackArgs a)
{
    constexpr int R = end_threads(L) / L, K1 = FIRST ? 2 : 1, K = K1 + (SECOND ? 2 : 0);     // planes of sums over rows
    __shared__ float lds1[end_threads(L) / 64][1], lds2[end_threads(L) / 64][2], lds3[end_threads(L) / 64][3];
    __shared__ float sums[R > 1 ? end_threads(L) * 8 : 1];
    const int l = (int)threadIdx.x % L, first = (int)threadIdx.x / L, c = l * 8, left = a.C - c;
    const long long all = a.P * a.C, stride = (long long)gridDim.x * R;
    Raw8<T> x, z, gy, gz = {};
    float gate = 1.f, mean1 = 0.f, rstd1 = 0.f, mean2 = 0.f, rstd2 = 0.f;
    auto load_x = [&](long long row) {                     // (a row past the last: nothing)
        x = load8<T, WHOLE>((const T *)a.x + row * a.C + c, row < a.P ? left : 0, (row + 1) * a.C + 7 <= all);
    };
    auto load = [&](long long row) {
        const bool safe = (row + 1) * a.C + 7 <= all, in = row < a.P;
        const int n = in ? left : 0;
        const long long at = row * a.C + c;
        if (a.grad_z != nullptr)
            gz = load8<T, WHOLE>((const T *)a.grad_z + at, n, safe);
        if constexpr (SECOND) {
            z = load8<T, WHOLE>((const T *)a.z + at, n, safe);
            gy = load8<T, WHOLE>((const T *)a.grad_y + at, n, safe);
            mean2 = in ? a.mean2[row] : 0.f;
            rstd2 = in ? a.rstd2[row] : 0.f;
        }
        if constexpr (FIRST) {
            mean1 = in ? a.mean1[row] : 0.f;
            rstd1 = in ? a.rstd1[row] : 0.f;
        }
        if (a.gate != nullptr)
            gate = in ? a.gate[fdiv((int)row, a.rows)] : 0.f;
    };
    Raw8<T> sc, gm1, bt1, gm2;
    auto load_vectors = [&] {                              // of the branch
        sc = channels<T, WHOLE>(a.scale, c, left, 1.f);
        if constexpr (FIRST) {
            gm1 = channels<T, WHOLE>(a.gamma1, c, left, 1.f);
            bt1 = channels<T, WHOLE>(a.beta1, c, left, 0.f);
        }
    };
    // Sixteen waves have 128 registers each: none for a row ahead, nor for vectors, which are read for each row, the branch's
    // when the second norm is through with its tensors.
    constexpr bool AHEAD = L < 1024;
    long long base = (long long)blockIdx.x * R;
    if (AHEAD) {
        load(base + first);
        load_x(base + first);
        load_vectors();
        if constexpr (SECOND)
            gm2 = channels<T, WHOLE>(a.gamma2, c, left, 1.f);
    }
    const Mask8<T> mask(left);
    // (sixteen waves and both norms: in LDS, where each lane has its own)
    constexpr bool FAR = !AHEAD && FIRST && SECOND;
    __shared__ float far[FAR ? K * 8 * 1024 : 1];
    float near[FAR ? 1 : K][8];
    auto total = [&](int k, int e) -> float & { return FAR ? far[(k * 8 + e) * 1024 + (int)threadIdx.x] : near[FAR ? 0 : k][e]; };
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            total(k, e) = 0.f;
    for (; base < a.P; base += stride) {                   // (the whole workgroup, for the barriers of wide rows)
        const long long row = base + first, at = row * a.C + c;
        const bool live = row < a.P;
        if (!AHEAD) {
            load(row);
            if constexpr (SECOND)
                gm2 = channels<T, WHOLE>(a.gamma2, c, left, 1.f);
            else
                load_x(row);
        }
        const float by = gate, m1 = mean1, s1 = rstd1, m2 = mean2, s2 = rstd2;
        float xh[8], g[8];
        unpack<T, WHOLE>(gz, mask, g);
        if (AHEAD || !SECOND)
            unpack<T, WHOLE>(x, mask, xh);
        if constexpr (SECOND) {
            float zh[8], t[8], s[2] = {0.f, 0.f};
            unpack<T, WHOLE>(z, mask, zh);
            unpack<T, WHOLE>(gy, mask, t);
#pragma unroll
            for (int e = 0; e < 8; ++e) {                  // (behind the row all is zero)
                zh[e] = e < left ? (zh[e] - m2) * s2 : 0.f;
                total(K1, e) = __builtin_fmaf(t[e], zh[e], total(K1, e));
                total(K1 + 1, e) += t[e];
                t[e] *= (float)gm2[e];
                s[0] += t[e];
                s[1] = __builtin_fmaf(t[e], zh[e], s[1]);
            }
            if (AHEAD) {
                load(row + stride);
                load_x(row + stride);
            }
            row_sums<L, 2>(s, lds2);
            const float u0 = s[0] * a.inv_c, u1 = s[1] * a.inv_c;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                g[e] = __builtin_fmaf(s2, __builtin_fmaf(-zh[e], u1, t[e] - u0), g[e]);
                asm("" : "+v"(g[e]));
                g[e] = e < left ? g[e] : 0.f;
            }
            store8<T, WHOLE>((T *)a.grad_residual + at, live ? left : 0, g);
            if (!AHEAD) {
                asm volatile("" ::: "memory");
                load_x(row);
                unpack<T, WHOLE>(x, mask, xh);
            }
        } else if (AHEAD) {
            load(row + stride);
            load_x(row + stride);
        }
        if (!AHEAD)
            load_vectors();
        // a gate of zero: the branch counts for nothing, whatever it holds (but in the gate's own gradient)
        float s[3] = {0.f, 0.f, 0.f}, out[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool on = by != 0.f && e < left;
            if constexpr (FIRST)
                xh[e] = e < left ? (xh[e] - m1) * s1 : 0.f;
            const float gs = g[e] * (float)sc[e];
            if (a.row_sums != nullptr) {
                if constexpr (FIRST)
                    s[2] = __builtin_fmaf(gs, __builtin_fmaf(xh[e], (float)gm1[e], (float)bt1[e]), s[2]);
                else
                    s[2] = __builtin_fmaf(gs, xh[e], s[2]);
            }
            xh[e] = on ? xh[e] : 0.f;
            const float q = on ? by * g[e] : 0.f;
            total(0, e) = __builtin_fmaf(q, xh[e], total(0, e));
            out[e] = on ? by * gs : 0.f;
            if constexpr (FIRST) {
                total(1, e) += q;
                out[e] *= (float)gm1[e];
                s[0] += out[e];
                s[1] = __builtin_fmaf(out[e], xh[e], s[1]);
            }
        }
        if constexpr (FIRST) {
            row_sums<L, 3>(s, lds3);
        } else if (a.row_sums != nullptr) {
            float t[1] = {s[2]};
            row_sums<L, 1>(t, lds1);
            s[2] = t[0];
        }
        if (a.row_sums != nullptr && l == 0 && live)
            a.row_sums[row] = s[2];
        if constexpr (FIRST) {
            const float u0 = s[0] * a.inv_c, u1 = s[1] * a.inv_c;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                out[e] = by != 0.f ? s1 * __builtin_fmaf(-xh[e], u1, out[e] - u0) : 0.f;
        }
        store8<T, WHOLE>((T *)a.grad_x + at, live ? left : 0, out);
    }
    if (a.partial == nullptr)
        return;
    float *to = a.partial + (long long)blockIdx.x * K * a.C;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = total(k, e);
        if constexpr (R > 1)
            add_rows_of_workgroup<L, end_threads(L)>(v, sums);
        if (first == 0)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < left)
                    to[k * a.C + c + e] = v[e];
    }
}

struct EndJoin {
    const float *partial, *row_sums;                       // row_sums: null for no gradient of the gates
    int groups, C;
    const void *gamma1, *beta1, *scale;
    void *grad_scale, *grad_gamma1, *grad_beta1, *grad_gamma2, *grad_beta2;    // null: not asked for
    float *grad_gate;
    int columns;                                           // workgroups that add up columns; the others have an image each
    long long rows;                                        // of an image
};

// Adds up the workgroups' sums (16 channels to a workgroup here, of the branch or of the second norm; 64 of the rows side by side) and an image's row sums.
template <typename T, bool FIRST, bool SECOND> __global__ __launch_bounds__(1024) void dcnv4_end_join_kernel(EndJoin j)
{
    constexpr int K1 = FIRST ? 2 : 1, K = K1 + (SECOND ? 2 : 0);
    __shared__ float part[2][16][16];
    const int in = (int)threadIdx.x & 15, slice = (int)threadIdx.x >> 4, all = SECOND ? 2 * j.columns : j.columns;
    if ((int)blockIdx.x >= all) {
        const int image = (int)blockIdx.x - all;
        const float *from = j.row_sums + (long long)image * j.rows;
        // (in 64 bits: an image's rows may be millions of numbers that cancel)
        __shared__ double waves[16];
        double s = 0.;
#pragma unroll 16
        for (long long r = (int)threadIdx.x; r < j.rows; r += 1024)
            s += (double)from[r];
#pragma unroll
        for (int d = 1; d < 64; d *= 2)
            s += __shfl_xor(s, d);
        if ((threadIdx.x & 63) == 0)
            waves[threadIdx.x >> 6] = s;
        __syncthreads();
        if (threadIdx.x == 0) {
            s = 0.;
#pragma unroll
            for (int w = 0; w < 16; ++w)
                s += waves[w];
            j.grad_gate[image] = (float)s;
        }
        return;
    }
    const bool second = SECOND && (int)blockIdx.x >= j.columns;
    const int col = ((int)blockIdx.x - (second ? j.columns : 0)) * 16 + in, k0 = second ? K1 : 0;
    float s[2] = {0.f, 0.f};                               // (one sum of a branch without a norm, and whatever follows it, which nothing takes)
    if (col < j.C)
#pragma unroll 8
        for (int r = slice; r < j.groups; r += 64)
#pragma unroll
            for (int k = 0; k < (FIRST || SECOND ? 2 : 1); ++k)
                s[k] += j.partial[((long long)r * K + k0 + k) * j.C + col];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        s[k] = add_halves(add_rows(s[k]));
        if ((threadIdx.x & 63) < 16)
            part[k][threadIdx.x >> 6][in] = s[k];
    }
    __syncthreads();
    if (threadIdx.x >= 16 || col >= j.C)
        return;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        s[k] = 0.f;
#pragma unroll
        for (int w = 0; w < 16; ++w)
            s[k] += part[k][w][in];
    }
    auto vector = [&](const void *p, float other) { return p != nullptr ? (float)((const T *)p)[col] : other; };
    auto store = [&](void *p, float v) {
        if (p != nullptr)
            ((T *)p)[col] = (T)v;
    };
    if (second) {
        store(j.grad_gamma2, s[0]);
        store(j.grad_beta2, s[1]);
    } else if constexpr (FIRST) {
        const float scale = vector(j.scale, 1.f);
        store(j.grad_scale, __builtin_fmaf(vector(j.gamma1, 1.f), s[0], vector(j.beta1, 0.f) * s[1]));
        store(j.grad_gamma1, scale * s[0]);
        store(j.grad_beta1, scale * s[1]);
    } else {
        store(j.grad_scale, s[0]);
    }
}

namespace {

// Rows wider than this are refused: sixteen waves with a run of eight each.
constexpr int kEndMaxChannels = 8192;

bool misaligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }

// Calls f with the lanes of a row as a constant: the fewest that hold it with one run of eight channels each.
template <typename F> int by_lanes(int C, F &&f)
{
    const int runs = (C + 7) / 8;
    if (runs <= 1) return f(std::integral_constant<int, 1>());
    if (runs <= 2) return f(std::integral_constant<int, 2>());
    if (runs <= 4) return f(std::integral_constant<int, 4>());
    if (runs <= 8) return f(std::integral_constant<int, 8>());
    if (runs <= 16) return f(std::integral_constant<int, 16>());
    if (runs <= 32) return f(std::integral_constant<int, 32>());
    if (runs <= 64) return f(std::integral_constant<int, 64>());
    if (runs <= 128) return f(std::integral_constant<int, 128>());
    if (runs <= 256) return f(std::integral_constant<int, 256>());
    if (runs <= 512) return f(std::integral_constant<int, 512>());
    return f(std::integral_constant<int, 1024>());
}

// Workgroups of the backward pass, each of which leaves partial sums of up to 4 * C: two to a unit, more only write more sums; one where rows are so wide that
// the sums are much of the traffic.  With both norms, us by 256, 512 and 1024 workgroups: fp16 134400 x 256 88, 87, 98; 50176 x 512 66, 59, 69; 12544 x 1024
// 43, 37, 47; 50176 x 1536 178, 186, 203; 12544 x 2048 64, 72, 90; 4096 x 4096 52, 67, 99; fp32 50176 x 512 117, 122, 125.
int end_back_groups(long long P, int C)
{
    return by_lanes(C, [&](auto L) {
        const long long rows = end_threads(L()) / L(), n = (P + rows - 1) / rows;
        const int most = C <= 1024 ? 512 : 256;
        return n < most ? (int)n : most;
    });
}

template <typename T, bool FIRST, bool SECOND> int launch_end(const EndArgs &a, hipStream_t s)
{
    const int cus = device_cus();
    if (cus <= 0)
        return DCNV4_ERR_LAUNCH;
    return by_lanes(a.C, [&](auto L) {
        constexpr int threads = end_threads(L());
        const long long rows = threads / L(), groups = (a.P + rows - 1) / rows, most = (long long)(2048 / threads) * cus;
        const dim3 grid((unsigned)(groups < most ? groups : most));
        if (a.C % 8 == 0)
            hipLaunchKernelGGL((dcnv4_end_kernel<T, L(), FIRST, SECOND, true>), grid, dim3(threads), 0, s, a);
        else
            hipLaunchKernelGGL((dcnv4_end_kernel<T, L(), FIRST, SECOND, false>), grid, dim3(threads), 0, s, a);
        return hipGetLastError() == hipSuccess ? DCNV4_OK : DCNV4_ERR_LAUNCH;
    });
}

template <typename T, bool FIRST, bool SECOND> int launch_end_backward(const EndBackArgs &a, int groups, const EndJoin &j, hipStream_t s)
{
    const int rc = by_lanes(a.C, [&](auto L) {
        constexpr int threads = end_threads(L());
        if (a.C % 8 == 0)
            hipLaunchKernelGGL((dcnv4_end_backward_kernel<T, L(), FIRST, SECOND, true>), dim3((unsigned)groups), dim3(threads), 0, s, a);
        else
            hipLaunchKernelGGL((dcnv4_end_backward_kernel<T, L(), FIRST, SECOND, false>), dim3((unsigned)groups), dim3(threads), 0, s, a);
        return hipGetLastError() == hipSuccess ? DCNV4_OK : DCNV4_ERR_LAUNCH;
    });
    const long long images = a.row_sums != nullptr ? a.P / j.rows : 0;
    if (rc || j.columns + images == 0)
        return rc;
    hipLaunchKernelGGL((dcnv4_end_join_kernel<T, FIRST, SECOND>), dim3((unsigned)((SECOND ? 2 : 1) * j.columns + images)), dim3(1024), 0, s, j);
    return hipGetLastError() == hipSuccess ? DCNV4_OK : DCNV4_ERR_LAUNCH;
}

template <typename F> int by_form(int norms, int dtype, F &&f)
{
    typedef std::true_type Y;
    typedef std::false_type N;
    auto typed = [&](auto t) {
        return norms == 0 ? f(t, N(), N()) : norms == DCNV4_FIRST_NORM ? f(t, Y(), N()) : norms == DCNV4_SECOND_NORM ? f(t, N(), Y()) : f(t, Y(), Y());
    };
    return dtype == DCNV4_F16 ? typed((_Float16)0) : typed(0.f);
}

int check_end(long long P, int C, int gates, int norms, int dtype)
{
    if (P < 1 || C < 1 || gates < 0 || (gates > 0 && P % gates))
        return DCNV4_ERR_SHAPE;
    // (with gates, rows are counted in 31 bits, and an image of each takes a workgroup of the backward pass)
    if ((dtype != DCNV4_F32 && dtype != DCNV4_F16) || (norms & ~(DCNV4_FIRST_NORM | DCNV4_SECOND_NORM)) || C > kEndMaxChannels || P > (1LL << 40) ||
        (gates > 0 && P > 0x7fffffffLL) || gates > (1 << 20))
        return DCNV4_ERR_UNSUPPORTED;
    return DCNV4_OK;
}

}  // namespace

extern "C" {

long long dcnv4_norm_scale_add_norm_workspace_bytes(long long P, int C, int gates)
{
    if (check_end(P, C, gates, 0, DCNV4_F32))
        return -1;
    const size_t sums = align256((size_t)end_back_groups(P, C) * 4 * (size_t)C * 4);
    return (long long)(sums + (gates > 0 ? align256((size_t)P * 4) : 0));
}

int dcnv4_norm_scale_add_norm(const void *x, const void *residual, const void *gamma1, const void *beta1, const void *scale, const float *gate,
                              const void *gamma2, const void *beta2, void *z, void *y, float *mean1, float *rstd1, float *mean2, float *rstd2,
                              long long P, int C, int gates, int norms, float eps, int dtype, void *stream)
{
    if (!x || !residual || !z || ((norms & DCNV4_SECOND_NORM) && !y) || (gates > 0 && !gate))
        return DCNV4_ERR_NULL;
    const int rc = check_end(P, C, gates, norms, dtype);
    if (rc)
        return rc;
    if (!(eps >= 0.f && eps <= 3.0e38f))
        return DCNV4_ERR_UNSUPPORTED;
    for (const void *p : {x, residual, gamma1, beta1, scale, (const void *)gate, gamma2, beta2, (const void *)z, (const void *)y, (const void *)mean1,
                          (const void *)rstd1, (const void *)mean2, (const void *)rstd2})
        if (misaligned(p))
            return DCNV4_ERR_ALIGN;
    EndArgs a = {x, residual, gamma1, beta1, scale, gamma2, beta2, gates > 0 ? gate : nullptr, z, y, mean1, rstd1, mean2, rstd2, P, {}, C, 1.f / (float)C, eps};
    if (gates > 0)
        a.rows = make_div((unsigned)(P / gates));
    return by_form(norms, dtype, [&](auto t, auto first, auto second) {
        return launch_end<decltype(t), decltype(first)::value, decltype(second)::value>(a, (hipStream_t)stream);
    });
}

int dcnv4_norm_scale_add_norm_backward(const void *x, const void *z, const void *gamma1, const void *beta1, const void *scale, const float *gate,
                                       const void *gamma2, const float *mean1, const float *rstd1, const float *mean2, const float *rstd2,
                                       const void *grad_y, const void *grad_z, void *grad_x, void *grad_residual, void *grad_scale, float *grad_gate,
                                       void *grad_gamma1, void *grad_beta1, void *grad_gamma2, void *grad_beta2, void *workspace,
                                       long long workspace_bytes, long long P, int C, int gates, int norms, int dtype, void *stream)
{
    const bool first = (norms & DCNV4_FIRST_NORM) != 0, second = (norms & DCNV4_SECOND_NORM) != 0;
    const bool sums = grad_scale || (first && (grad_gamma1 || grad_beta1)) || (second && (grad_gamma2 || grad_beta2));
    if (!x || !grad_x || (first && (!mean1 || !rstd1)) || (second ? !z || !mean2 || !rstd2 || !grad_y || !grad_residual : !grad_z) || (gates > 0 && !gate) ||
        ((sums || grad_gate) && !workspace))
        return DCNV4_ERR_NULL;
    const int rc = check_end(P, C, gates, norms, dtype);
    if (rc)
        return rc;
    if ((grad_gate && gates == 0) || ((sums || grad_gate) && workspace_bytes < dcnv4_norm_scale_add_norm_workspace_bytes(P, C, gates)))
        return DCNV4_ERR_SHAPE;
    for (const void *p : {x, z, gamma1, beta1, scale, (const void *)gate, gamma2, (const void *)mean1, (const void *)rstd1, (const void *)mean2,
                          (const void *)rstd2, grad_y, grad_z, (const void *)grad_x, (const void *)grad_residual, (const void *)grad_scale,
                          (const void *)grad_gate, (const void *)grad_gamma1, (const void *)grad_beta1, (const void *)grad_gamma2, (const void *)grad_beta2,
                          (const void *)workspace})
        if (misaligned(p))
            return DCNV4_ERR_ALIGN;
    const int groups = end_back_groups(P, C);
    float *partial = (float *)workspace, *rows = (float *)((char *)workspace + align256((size_t)groups * 4 * (size_t)C * 4));
    EndBackArgs a = {x, z, gamma1, beta1, scale, gamma2, gates > 0 ? gate : nullptr, mean1, rstd1, mean2, rstd2, grad_y, grad_z, grad_x, grad_residual,
                     sums ? partial : nullptr, grad_gate ? rows : nullptr, P, {}, C, 1.f / (float)C};
    if (gates > 0)
        a.rows = make_div((unsigned)(P / gates));
    const EndJoin j = {partial, rows, groups, C, gamma1, beta1, scale, grad_scale, grad_gamma1, grad_beta1, grad_gamma2, grad_beta2, grad_gate,
                 sums ? (C + 15) / 16 : 0, gates > 0 ? P / gates : P};
    return by_form(norms, dtype, [&](auto t, auto one, auto two) {
        return launch_end_backward<decltype(t), decltype(one)::value, decltype(two)::value>(a, groups, j, (hipStream_t)stream);
    });
}

}  // extern "C"
