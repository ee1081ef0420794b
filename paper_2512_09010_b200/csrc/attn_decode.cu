// Attention of one new token per sequence over its paged key-value cache.
//
// The simplest form: one CTA per (sequence, query head); its warps take every eighth token, keep a running maximum, sum and
// weighted value row (the softmax in one pass: when the maximum grows, what has been summed is scaled down), and
// join them through shared memory.

#include <cuda_bf16.h>
#include <cuda_fp8.h>
#include <math.h>

#include "luvc_internal.h"

namespace luvc {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kMaxD = 256, kPer = kMaxD / 32;

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_float(__nv_fp8_e4m3 x) { return (float)x; }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

template <typename TQ, typename TC>
__global__ void __launch_bounds__(kThreads) attn_decode_kernel(const __grid_constant__ AttnProblem a) {
    __shared__ float part[kWarps][kMaxD], part_m[kWarps], part_s[kWarps];
    const luvc_kv_cache& c = a.c;
    if (__syncthreads_or(*reinterpret_cast<volatile int*>(a.status) != 0)) return;
    const int i = blockIdx.y, hq = blockIdx.x, h = hq / (a.q_heads / c.heads);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, D = c.D, ps = c.page_size;
    const int slot = a.seqs ? a.seqs[i] : i;
    int len = 0;
    if (slot >= 0 && slot < c.slots) len = max(0, min(c.lengths[slot], c.max_pages * ps));
    else if (threadIdx.x == 0) *a.status = LUVC_ERR_SHAPE;
    const float ks = c.k_scale ? c.k_scale[a.layer * c.heads + h] : 1.f;
    const float vs = c.v_scale ? c.v_scale[a.layer * c.heads + h] : 1.f;
    float q[kPer], o[kPer], m = -INFINITY, sum = 0.f;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int d = lane + 32 * j;
        q[j] = d < D ? to_float(static_cast<const TQ*>(a.q)[i * a.q_stride + (long long)hq * D + d]) : 0.f;
        o[j] = 0.f;
    }
    for (int t = warp; t < len; t += kWarps) {
        const int page = c.table[(long long)slot * c.max_pages + t / ps];
        if (page < 0 || page >= c.pages) continue;
        const float bias = t < a.bias_width ? a.bias[i * a.bias_stride + t] : 0.f;
        if (bias == -INFINITY) continue;
        const long long row = ((((long long)a.layer * c.pages + page) * c.heads + h) * ps + t % ps) * D;
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int d = lane + 32 * j;
            if (d < D) s += q[j] * to_float(static_cast<const TC*>(c.k)[row + d]);
        }
#pragma unroll
        for (int x = 16; x; x >>= 1) s += __shfl_xor_sync(~0u, s, x);
        s = s * (a.scale * ks) + bias;
        const float mn = fmaxf(m, s), base = mn == -INFINITY ? 0.f : mn;
        const float f = expf(m - base), w = expf(s - base);
        sum = sum * f + w;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int d = lane + 32 * j;
            if (d < D) o[j] = o[j] * f + w * to_float(static_cast<const TC*>(c.v)[row + d]);
        }
        m = mn;
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) part[warp][lane + 32 * j] = o[j];
    if (lane == 0) { part_m[warp] = m; part_s[warp] = sum; }
    __syncthreads();
    float mt = -INFINITY, st = 0.f;
    for (int w = 0; w < kWarps; ++w) mt = fmaxf(mt, part_m[w]);
    const float base = mt == -INFINITY ? 0.f : mt;
    for (int w = 0; w < kWarps; ++w) st += part_s[w] * expf(part_m[w] - base);
    for (int d = threadIdx.x; d < D; d += kThreads) {
        float x = 0.f;
        for (int w = 0; w < kWarps; ++w) x += part[w][d] * expf(part_m[w] - base);
        put(static_cast<TQ*>(a.out) + ((long long)i * a.q_heads + hq) * D + d, st == 0.f ? 0.f : x * vs / st);
    }
    if (a.lse && threadIdx.x == 0) a.lse[(long long)i * a.q_heads + hq] = st == 0.f ? -INFINITY : base + logf(st);
}

}  // namespace

size_t attn_workspace_bytes() { return 256; }

int attn_decode(const AttnProblem& p) {
    const dim3 grid(p.q_heads, p.n);
    if (p.c.dtype == LUVC_F32) attn_decode_kernel<float, float><<<grid, kThreads, 0, p.stream>>>(p);
    else if (p.c.dtype == LUVC_BF16) attn_decode_kernel<__nv_bfloat16, __nv_bfloat16><<<grid, kThreads, 0, p.stream>>>(p);
    else attn_decode_kernel<__nv_bfloat16, __nv_fp8_e4m3><<<grid, kThreads, 0, p.stream>>>(p);
    count_launch();
    return cudaGetLastError() == cudaSuccess ? LUVC_OK : LUVC_ERR_CUDA;
}

}  // namespace luvc
