// What the kernels of the paged key-value cache share (kv_cache.cu, kv_rows.cu).  Device-only, header-only.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "luvc_internal.h"

namespace luvc {
namespace {

__device__ __forceinline__ int status_of(int* status) { return *reinterpret_cast<volatile int*>(status); }

// For a call that has found the status word set and does nothing: rows that a write has skipped become a plain status, at which further
// writes stop too.
__device__ __forceinline__ void stop_writes(int* status, int word) {
    if (word == kRowsSkipped && threadIdx.x == 0) *status = word & kStatusMask;
}

__device__ __forceinline__ int ceil_div(int a, int b) { return (int)(((unsigned)a + (unsigned)b - 1u) / (unsigned)b); }

template <typename T> struct Vec;                           // the elements of 16 input bytes, as floats
template <> struct Vec<float> {
    static constexpr int N = 4;
    static __device__ void unpack(uint4 x, float (&f)[8]) {
        f[0] = __uint_as_float(x.x); f[1] = __uint_as_float(x.y); f[2] = __uint_as_float(x.z); f[3] = __uint_as_float(x.w);
    }
};
template <> struct Vec<__nv_bfloat16> {
    static constexpr int N = 8;
    static __device__ void unpack(uint4 x, float (&f)[8]) {
        const unsigned w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            f[2 * q] = __uint_as_float(w[q] << 16);
            f[2 * q + 1] = __uint_as_float(w[q] & 0xffff0000u);
        }
    }
};

// Last entry of ascending starts[0 .. n] (starts[0] = 0) that is <= t, below n: 32 probes at a time (one warp, one t).
__device__ __forceinline__ int owner_of(const int32_t* starts, int n, int t, int lane) {
    int lo = 0, size = n;                                   // the answer is in [lo, lo + size)
    while (size > 1) {
        const int step = (size + 31) / 32, at = lo + lane * step;
        const unsigned m = __ballot_sync(~0u, lane * step < size && starts[at] <= t);
        const int k = m ? 31 - __clz(m) : 0;
        lo += k * step;
        size = min(step, size - k * step);
    }
    return lo;
}

// Four floats to e4m3, to nearest even, saturated; two e4m3 (the low 16 bits) to floats; four e4m3 times a factor.
__device__ __forceinline__ unsigned e4m3x4(float a, float b, float c, float d) {
    return (unsigned)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3) |
           (unsigned)__nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3) << 16;
}
__device__ __forceinline__ float2 e4m3x2_floats(unsigned two) {
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)two, __NV_E4M3);
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
__device__ __forceinline__ unsigned scaled_e4m3x4(unsigned x, float by) {
    const float2 u = e4m3x2_floats(x & 0xffffu), v = e4m3x2_floats(x >> 16);
    return e4m3x4(u.x * by, u.y * by, v.x * by, v.y * by);
}

}  // namespace
}  // namespace luvc
