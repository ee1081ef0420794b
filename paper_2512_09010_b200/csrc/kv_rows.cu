// Rows in and out of a paged key-value cache: quantised with a scale for each block on the way in, and read back.
//
// Blocks.  Of a cache of type LUVC_E4M3_BLOCK, 16 consecutive tokens of a page share one scale per head, for the keys and for the values,
// and a stored x stands for x * scale.  The scale is the smallest power of two 2^e with max |x| <= 448 2^e: e4m3 is a floating-point type,
// so a scale has only to bring the block into its range; one that is a power of two changes no mantissa, can be applied exactly, and
// lets a block that gets a larger value later be brought to its new scale without a second rounding, but for what falls below 2^-6.
// So a new token of a block that is in use takes the larger of the block's scale and its own, and if that is its own the
// old rows are brought to it.
//
// Bound.  A bf16 row is read once and written with half its bytes, or the other way round: HBM, once there are enough tokens.  Prompts of
// 33947 tokens, 8 heads of 128: 42.5 us with sizes, 39.5 without, 0.75 and 0.80 of the copy rate (issue slots 68 % busy); 37861 read back
// 42.3 us, 0.84.
//
// Split.  A CTA takes up to 32 tokens.  Its first warp finds the blocks that begin among them (a token that is the first of the call in its
// block leads it, wherever the block ends); then each warp takes one (block, head, K or V) after the other, all of it in
// registers: D / 16 pieces of 16 bytes for each lane, whatever D, from which it finds the largest element, then quantises them.

#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "kv_common.cuh"
#include "luvc_internal.h"
#include "sm100_ptx.cuh"

namespace luvc {
namespace {

using namespace ptx;

constexpr int kRowsTokens = 32, kRowsThreads = 256, kRowsWarps = kRowsThreads / 32;
constexpr int kLeast = -60, kMost = 60;         // exponents of scales

struct RowsArgs {
    luvc_kv_cache c;
    int layer, n, tokens, per;                  // per: tokens of a CTA
    const int32_t *seqs, *starts, *sizes, *first;
    const void *k, *v;                          // rows (read: written)
    long long k_stride, v_stride;
    int* status;
};

struct Block {
    long long row;                              // of its first token in head 0 of the layer's pool
    int scale;                                  // index of its scale in head 0 of the layer
    int token, front, count;                    // first row of the call that belongs to it, the place of that row in it, rows
};

// Largest finite |x| as it is among bits of floats >= 0; top: the largest of all.
template <typename Each>
__device__ __forceinline__ float block_top(float top, Each each) {
    unsigned m = __reduce_max_sync(~0u, __float_as_uint(top));
    if (m >= 0x7f800000u) {                     // infinities saturate; they do not set the scale
        float t = 0.f;
        each([&](float x) { t = fabsf(x) < INFINITY ? fmaxf(t, fabsf(x)) : t; });
        m = __reduce_max_sync(~0u, __float_as_uint(t));
    }
    return __uint_as_float(m);
}

// The smallest power of two s with top <= 448 s (448 = 1.75 * 2^8).
__device__ __forceinline__ float scale_for(float top) {
    const unsigned b = __float_as_uint(top);
    const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u);
    return __uint_as_float((unsigned)(min(max(e, kLeast), kMost) + 127) << 23);
}

template <int NC>                               // pieces of a lane: D / 16 at most
__global__ void __launch_bounds__(kRowsThreads, NC > 8 ? 2 : 4) kv_write_block_kernel(const __grid_constant__ RowsArgs a) {
    __shared__ Block blocks[kRowsTokens];
    __shared__ int count;
    const luvc_kv_cache& c = a.c;
    const int t0 = blockIdx.x * a.per, ps = c.page_size, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, tokens = min(a.per, a.tokens - t0);
    pdl_trigger();
    pdl_wait();
    const int word = status_of(a.status);       // (as in luvc_kv_write's other kernel: rows that are skipped stop no other)
    if (__syncthreads_or(word != 0 && word != kRowsSkipped)) return;
    if (warp == 0) {                            // a token per lane, from the owner of the first one on
        int i = a.starts ? owner_of(a.starts, a.n, t0, lane) : t0 + lane;
        bool leads = false;
        Block b = {};
        if (lane < tokens) {
            const int t = t0 + lane;
            int behind = 1, begin = t;          // tokens of the sequence from this one to its end; its first row
            if (a.starts) {
                int end = a.starts[i + 1];
                while (end <= t && i + 1 < a.n) end = a.starts[++i + 1];
                behind = end - t;
                begin = a.starts[i];
            }
            const int slot = a.seqs ? a.seqs[i] : i;
            const int pos = slot >= 0 && slot < c.slots ? c.lengths[slot] - behind : -1;
            int page = -1;
            if (behind >= 1 && pos >= 0 && pos / ps < c.max_pages) page = c.table[(long long)slot * c.max_pages + pos / ps];
            if (page >= 0 && page < c.pages) {
                b.front = pos % kKvBlock;
                b.count = min(min(behind, a.tokens - t), kKvBlock - b.front);        // (starts may say more rows than there are)
                b.token = t;
                b.row = (long long)page * c.heads * ps + pos % ps - b.front;
                b.scale = page * c.heads * (ps / kKvBlock) + pos % ps / kKvBlock;
                leads = t == begin || b.front == 0;
            } else if (blockIdx.y == 0) {
                *a.status = kRowsSkipped;
            }
        }
        const unsigned all = __ballot_sync(~0u, leads);
        if (leads) blocks[__popc(all & ((1u << lane) - 1u))] = b;
        if (lane == 0) count = __popc(all);
    }
    __syncthreads();
    const int heads2 = 2 * c.heads, items = count * heads2, per_row = c.D / 8;
    const unsigned part = 65536 / per_row + 1;  // a piece's row: piece * part / 65536, exact for less than 512 pieces of rows of up to 32
    for (int item = blockIdx.y * kRowsWarps + warp; item < items; item += gridDim.y * kRowsWarps) {
        const Block b = blocks[item / heads2];
        const int rest = item % heads2;
        const bool is_v = rest >= c.heads, enhance = is_v && a.sizes;
        const int h = is_v ? rest - c.heads : rest;
        const long long stride = is_v ? a.v_stride : a.k_stride;
        const __nv_bfloat16* const src = static_cast<const __nv_bfloat16*>(is_v ? a.v : a.k) + b.token * stride + h * c.D;
        float* const scale = (is_v ? c.v_block_scale : c.k_block_scale) + ((size_t)a.layer * c.pages * c.heads * (ps / kKvBlock) + b.scale + (size_t)h * (ps / kKvBlock));
        uint4 x[NC];
        auto row_of = [&](int i) { return (int)(((lane + 32 * i) * part) >> 16); };
        auto live = [&](int i) { return i < c.D / 16 && (unsigned)(row_of(i) - b.front) < (unsigned)b.count; };
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            x[i] = make_uint4(0u, 0u, 0u, 0u);
            const int r = row_of(i);
            if (live(i)) x[i] = __ldcs(reinterpret_cast<const uint4*>(src + (r - b.front) * stride) + (lane + 32 * i - r * per_row));
        }
        const float old = b.front ? *scale : 0.f;
        float bias = 0.f;                       // of the block's row `lane`
        if (enhance && (unsigned)(lane - b.front) < (unsigned)b.count) bias = logf((float)a.sizes[b.token + lane - b.front]);
        // every element of the piece i, as a float, enhanced
        auto piece = [&](int i, float (&f)[8]) {
            Vec<__nv_bfloat16>::unpack(x[i], f);
            if (enhance) {
                const float more = __shfl_sync(~0u, bias, row_of(i) & 15);
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] += more;
            }
        };
        float top;
        if (!enhance) {
            __nv_bfloat162 m = __float2bfloat162_rn(0.f);
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                const unsigned w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) m = __hmax2(m, __habs2(*reinterpret_cast<const __nv_bfloat162*>(&w[e])));    // (a NaN is passed over)
            }
            top = fmaxf(__low2float(m), __high2float(m));
        } else {
            top = 0.f;
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                float f[8];
                piece(i, f);
                if (live(i))
#pragma unroll
                    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(f[e]));
            }
        }
        top = block_top(top, [&](auto see) {
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                float f[8];
                piece(i, f);
                if (live(i))
#pragma unroll
                    for (int e = 0; e < 8; ++e) see(f[e]);
            }
        });
        const float s = fmaxf(old, scale_for(top)), inv = 1.f / s;      // exact: powers of two
        unsigned char* const rows = static_cast<unsigned char*>(is_v ? c.v : c.k) +
                                    ((size_t)a.layer * c.pages * c.heads * ps + b.row + (size_t)h * ps) * c.D;
        if (b.front && s != old) {              // the rows before come to the new scale
            const float f = old / s;
            for (int i = lane; i < b.front * (c.D / 16); i += 32) {
                uint4* const p = reinterpret_cast<uint4*>(rows) + i;
                const uint4 y = *p;
                *p = make_uint4(scaled_e4m3x4(y.x, f), scaled_e4m3x4(y.y, f), scaled_e4m3x4(y.z, f), scaled_e4m3x4(y.w, f));
            }
        }
        if (lane == 0 && s != old) *scale = s;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            float f[8];
            piece(i, f);
            if (live(i))
                __stcs(reinterpret_cast<uint2*>(rows) + lane + 32 * i,
                       make_uint2(e4m3x4(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv), e4m3x4(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv)));
        }
    }
}

// ---- rows back -----------------------------------------------------------------------------------------------------

// 16 bytes of a row that is given out, from the cache's bytes for them.
template <typename TC> struct Stored;
template <> struct Stored<float> {
    using Raw = uint4;
    static __device__ uint4 out(Raw x, float) { return x; }
};
template <> struct Stored<__nv_bfloat16> {
    using Raw = uint4;
    static __device__ uint4 out(Raw x, float) { return x; }
};
template <> struct Stored<__nv_fp8_e4m3> {
    using Raw = uint2;
    static __device__ uint4 out(Raw x, float s) {
        const unsigned w[4] = {x.x & 0xffffu, x.x >> 16, x.y & 0xffffu, x.y >> 16};
        unsigned r[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 u = e4m3x2_floats(w[e]);
            const __nv_bfloat162 two = __floats2bfloat162_rn(u.x * s, u.y * s);
            r[e] = *reinterpret_cast<const unsigned*>(&two);
        }
        return make_uint4(r[0], r[1], r[2], r[3]);
    }
};

// A thread keeps its place in a token's row, as in luvc_kv_write, and takes every `step`-th token of the CTA.
constexpr int kReadBatch = 4;

template <typename TI, typename TC, bool BLOCKS>
__global__ void __launch_bounds__(kRowsThreads, 4) kv_read_kernel(const __grid_constant__ RowsArgs a) {
    constexpr int V = Vec<TI>::N;
    using Raw = typename Stored<TC>::Raw;
    __shared__ long long row_of[kRowsTokens];               // row of head 0 in the layer's pool; -1: zeros, -2: not written
    __shared__ int scale_of[kRowsTokens];
    const luvc_kv_cache& c = a.c;
    const int t0 = blockIdx.x * a.per, ps = c.page_size, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int per_row = c.D / V, per_token = c.heads * per_row, cols = min(per_token, kRowsThreads), step = kRowsThreads / cols;
    const int mine = threadIdx.x / cols, tokens = min(a.per, a.tokens - t0);
    pdl_trigger();
    pdl_wait();
    if (warp == 0) {
        int i = a.starts ? owner_of(a.starts, a.n, t0, lane) : t0 + lane;
        if (lane < tokens) {
            const int t = t0 + lane;
            long long pos = 0;
            bool ours = true;
            if (a.starts) {
                int end = a.starts[i + 1];
                while (end <= t && i + 1 < a.n) end = a.starts[++i + 1];
                ours = t < end;                             // else behind the last sequence
                pos = t - a.starts[i];
            }
            long long row = ours ? -1 : -2;
            if (ours) {
                const int slot = a.seqs ? a.seqs[i] : i;
                if (a.first) pos += a.first[i];
                if (slot >= 0 && slot < c.slots && pos >= 0 && pos < c.lengths[slot] && pos / ps < c.max_pages) {
                    const int page = c.table[(long long)slot * c.max_pages + pos / ps], at = (int)(pos % ps);
                    if (page >= 0 && page < c.pages) {
                        row = (long long)page * c.heads * ps + at;
                        scale_of[lane] = page * c.heads * (ps / kKvBlock) + at / kKvBlock;
                    }
                }
                if (row < 0) *a.status = LUVC_ERR_SHAPE;
            }
            row_of[lane] = row;
        }
    }
    __syncthreads();
    if (mine >= step) return;
    const size_t layer_row = (size_t)a.layer * c.pages * c.heads * ps, layer_scale = (size_t)a.layer * c.pages * c.heads * (ps / kKvBlock);
    for (int col = threadIdx.x - mine * cols; col < per_token; col += cols) {
        const int h = col / per_row;
        const size_t in = (size_t)h * ps * c.D + (size_t)(col - h * per_row) * V;
        float ks = 1.f, vs = 1.f;
        if (!BLOCKS && c.k_scale) { ks = c.k_scale[a.layer * c.heads + h]; vs = c.v_scale[a.layer * c.heads + h]; }
        for (int t = mine; t < tokens; t += kReadBatch * step) {
            Raw kx[kReadBatch], vx[kReadBatch];
            float kf[kReadBatch], vf[kReadBatch];
#pragma unroll
            for (int b = 0; b < kReadBatch; ++b) {
                const int j = t + b * step;
                kx[b] = vx[b] = Raw{};
                kf[b] = ks; vf[b] = vs;
                if (j >= tokens || row_of[j] < 0) continue;
                const size_t src = (layer_row + row_of[j]) * c.D + in;
                kx[b] = __ldcs(reinterpret_cast<const Raw*>(static_cast<const TC*>(c.k) + src));
                vx[b] = __ldcs(reinterpret_cast<const Raw*>(static_cast<const TC*>(c.v) + src));
                if (BLOCKS) {
                    const size_t at = layer_scale + scale_of[j] + (size_t)h * (ps / kKvBlock);
                    kf[b] = c.k_block_scale[at];
                    vf[b] = c.v_block_scale[at];
                }
            }
#pragma unroll
            for (int b = 0; b < kReadBatch; ++b) {
                const int j = t + b * step;
                if (j >= tokens || row_of[j] == -2) continue;
                const long long at = t0 + j;
                __stcs(reinterpret_cast<uint4*>(static_cast<TI*>(const_cast<void*>(a.k)) + at * a.k_stride + col * V), Stored<TC>::out(kx[b], kf[b]));
                __stcs(reinterpret_cast<uint4*>(static_cast<TI*>(const_cast<void*>(a.v)) + at * a.v_stride + col * V), Stored<TC>::out(vx[b], vf[b]));
            }
        }
    }
}

}  // namespace

int kv_write_blocks(const luvc_kv_cache& c, int layer, const int32_t* seqs, int n, const void* k, const void* v, long long k_stride,
                    long long v_stride, int tokens, const int32_t* starts, const int32_t* sizes, int* status, cudaStream_t stream) {
    RowsArgs a = {};
    a.c = c; a.layer = layer; a.n = n; a.tokens = tokens; a.seqs = seqs; a.starts = starts; a.sizes = sizes;
    a.k = k; a.v = v; a.k_stride = k_stride; a.v_stride = v_stride; a.status = status;
    const int sms = sm_count();
    if (!sms) return LUVC_ERR_CUDA;
    // about four CTAs per SM; where there are few tokens the heads of a block go to several CTAs
    const int even = (int)(((long long)tokens + 4 * sms - 1) / (4 * sms));
    a.per = even > kRowsTokens ? kRowsTokens : even;
    const int grid = (tokens - 1) / a.per + 1, rounds = (2 * c.heads + kRowsWarps - 1) / kRowsWarps;
    int across = grid < 4 * sms ? 4 * sms / grid : 1;
    if (across > rounds) across = rounds;
    const dim3 dims(grid, across);
    if (c.D <= 64) return launch_overlapped(kv_write_block_kernel<4>, dims, kRowsThreads, 0, stream, a);
    if (c.D <= 128) return launch_overlapped(kv_write_block_kernel<8>, dims, kRowsThreads, 0, stream, a);
    return launch_overlapped(kv_write_block_kernel<16>, dims, kRowsThreads, 0, stream, a);
}

int kv_read(const luvc_kv_cache& c, int layer, const int32_t* seqs, int n, const int32_t* first, void* k, void* v, long long k_stride,
            long long v_stride, int tokens, const int32_t* starts, int* status, cudaStream_t stream) {
    RowsArgs a = {};
    a.c = c; a.layer = layer; a.n = n; a.tokens = tokens; a.seqs = seqs; a.starts = starts; a.first = first;
    a.k = k; a.v = v; a.k_stride = k_stride; a.v_stride = v_stride; a.status = status;
    const int sms = sm_count();
    if (!sms) return LUVC_ERR_CUDA;
    const int even = (int)(((long long)tokens + 4 * sms - 1) / (4 * sms));
    a.per = even < 4 ? 4 : even > kRowsTokens ? kRowsTokens : even;
    const int grid = (tokens - 1) / a.per + 1;
    if (c.dtype == LUVC_F32) return launch_overlapped(kv_read_kernel<float, float, false>, grid, kRowsThreads, 0, stream, a);
    if (c.dtype == LUVC_BF16) return launch_overlapped(kv_read_kernel<__nv_bfloat16, __nv_bfloat16, false>, grid, kRowsThreads, 0, stream, a);
    if (c.dtype == LUVC_E4M3) return launch_overlapped(kv_read_kernel<__nv_bfloat16, __nv_fp8_e4m3, false>, grid, kRowsThreads, 0, stream, a);
    return launch_overlapped(kv_read_kernel<__nv_bfloat16, __nv_fp8_e4m3, true>, grid, kRowsThreads, 0, stream, a);
}

}  // namespace luvc
