// What the library's sources share: vector types, buffer descriptors, division by constants, the current device.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dcnv4.h"

// Switches of the cross entropy (dcnv4_loss.hip) and of the layers' gradients (dcnv4_layers.hip); DCNV4_ERR_UNSUPPORTED for a key or value that is
// not one of them.
__attribute__((visibility("hidden"))) int loss_set_option(const char *key, int value);
__attribute__((visibility("hidden"))) int layers_set_option(const char *key, int value);

namespace {

constexpr int kXcds = 8;
// Word 3 of a gfx9-family raw buffer descriptor: 32-bit data format, no swizzle, no stride.
constexpr int kRsrcWord3 = 0x00020000;
// A byte offset no descriptor of ours reaches (images are validated below 2^31 bytes):
// loads through it return zero, atomics through it are dropped.
constexpr int kOutside = (int)0x80000000u;

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __amdgpu_buffer_rsrc_t rsrc_t;

// n / d for 0 <= n < 2^31 as mulhi + add + shift (d >= 1), constants made on the host.
struct FastDiv {
    unsigned mul, shift;
};

__device__ __forceinline__ int fdiv(int n, FastDiv f)
{
    return (int)((__umulhi((unsigned)n, f.mul) + (unsigned)n) >> f.shift);
}

FastDiv make_div(unsigned d)
{
    unsigned s = 0;
    while ((1ull << s) < d)
        ++s;
    FastDiv f;
    f.shift = s;
    f.mul = (unsigned)(((1ull << 32) * ((1ull << s) - d)) / d + 1);
    return f;
}

__device__ __forceinline__ rsrc_t make_rsrc(const void *base, unsigned bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, (int)bytes, kRsrcWord3);
}

int esize(int dtype) { return dtype == DCNV4_F16 ? 2 : 4; }

size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

// Per-device caches (compute-unit count, dynamic-LDS grants) are indexed by the HIP device number.
constexpr int kMaxDevices = 64;
int current_device()
{
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices)
        return -1;
    return dev;
}

// Number of compute units of the current device (persistent kernels launch one workgroup each).
int device_cus()
{
    static int cus[kMaxDevices];
    const int dev = current_device();
    if (dev < 0)
        return 0;
    if (cus[dev] == 0) {
        int n = 0;
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < kXcds)
            return 0;
        cus[dev] = n;
    }
    return cus[dev];
}

}  // namespace
