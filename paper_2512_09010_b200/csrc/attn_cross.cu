// Attention of a sequence's tokens to the states of an encoder, which have a length of their own and no order that masks.
//
//   out[t, h] = sum_s p_s V[s] / sum_s p_s,   p_s = exp(scale <q[t, h], K[s]> + bias[s]),   s over the sequence's states
//
// in one pass over the states: a running maximum m, the sum l of the weights so far and their weighted sum O of value rows; when m
// grows, l and O are scaled by exp(m_old - m_new).  Partial results of parts of the states join by the same rule.
//
// Rows.  The query heads of a key head see the same states, so a row of the products is a (token, query head) pair: all rows of a key head
// lie one after another, and a tile of 128 of them is one operand, whether it is 128 tokens of one head or one token of seven.
//
// Split.  The work is the list of all (sequence, key head, block of rows, tile of states); each CTA, one per SM, takes an equal part of it, whatever
// the lengths.  What a CTA has of a (sequence, key head, block of rows) that others share goes through the workspace; the CTA that comes last
// adds the parts, in the order of the list, so that a repeated call gives the same bits.
//
// bf16: tensor cores (attn_cross_tc).  f32: CUDA cores (attn_cross_f32), 32-bit products and sums.

#include <cuda.h>
#include <cuda_bf16.h>
#include <math.h>

#include <algorithm>
#include <atomic>

#include "luvc_internal.h"
#include "sm100_ptx.cuh"

namespace luvc {
namespace {

using namespace ptx;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kMaxCtas = 160;                       // CTAs the workspace has room for
constexpr int kPartFloats = 256 * 130;              // of a partial result: rows of sums, and their (m, l)
constexpr size_t kCounterBytes = 1024;
static_assert(kMaxCtas * sizeof(unsigned) <= kCounterBytes, "room for the counters");
constexpr int kWaitProbes = 1 << 20;                // probes before a wait gives up (seconds)
constexpr int kLeastProbes = 1 << 12;               // and with a limit from the status block (a test's)

struct CrossArgs {
    CrossProblem p;
    int group;                                      // query heads per key head
    // Scores are c <q, k> + bias, weights 2^(unit (score - m)), and a score is worth nat in natural units: with biases c = |scale|, unit = log2(e),
    // nat = 1 (a bias of the lowest value times log2(e) would not be finite), without c = |scale| log2(e), unit = 1, nat = ln(2).
    float c, unit, nat;
    float sign;                                     // of the scale; c has its magnitude
    unsigned* counters;                             // [kMaxCtas] arrivals of parts, by the CTA an item begins in
    float* parts;                                   // [kMaxCtas][2][kPartFloats]
};

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    unsigned long long d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d)
        : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)), "l"(*reinterpret_cast<unsigned long long*>(&c)));
    return *reinterpret_cast<float2*>(&d);
}

// ---- the list of work -----------------------------------------------------------------------------------------------

// A part of one (sequence, key head, block of rows): tiles kb .. kb + count - 1 of its kbs tiles of states.
struct Item {
    int seq, head, rb, kb, count, kbs;
    int q0, rows;                                   // first token of the sequence; rows of the block
    long long k0;                                   // first state
    int klen;
    long long first;                                // its first tile's place in the list
};

template <int BM, int BN>
struct Work {
    const CrossArgs& a;
    long long at = 0, end = 0, per = 0;             // this CTA's part of the list
    int seq = 0, head = 0, rb = 0, kb = 0;
    int q0 = 0, qlen = 0, k0 = 0, klen = 0, rbs = 0, kbs = 0;

    __device__ explicit Work(const CrossArgs& args) : a(args) {}
    __device__ void lengths(int i, int& q0, int& qlen, int& k0, int& klen) const {
        const CrossProblem& p = a.p;
        auto clamped = [](int x, int most) { return min(max(x, 0), most); };
        q0 = p.q_starts ? clamped(p.q_starts[i], p.q_tokens) : i;
        qlen = p.q_starts ? max(clamped(p.q_starts[i + 1], p.q_tokens) - q0, 0) : 1;
        k0 = clamped(p.k_starts[i], p.k_tokens);
        klen = max(clamped(p.k_starts[i + 1], p.k_tokens) - k0, 0);
    }
    __device__ int blocks_of(int qlen) const { return (int)(((long long)qlen * a.group + BM - 1) / BM); }
    __device__ int tiles_of(int klen) const { return (int)(((long long)klen + BN - 1) / BN); }
    __device__ long long units(int i) const {
        int q0, qlen, k0, klen;
        lengths(i, q0, qlen, k0, klen);
        return (long long)a.p.heads * blocks_of(qlen) * tiles_of(klen);
    }
    __device__ void enter(int i) {
        seq = i;
        lengths(i, q0, qlen, k0, klen);
        rbs = blocks_of(qlen);
        kbs = tiles_of(klen);
    }
    // This CTA's part; all NT threads of the CTA call it.
    template <int NT>
    __device__ void begin() {
        __shared__ long long sums[NT / 32 + 1], found_base;
        __shared__ int found;
        const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = a.p.n;
        long long mine = 0;
        for (int i = tid; i < n; i += NT) mine += units(i);
#pragma unroll
        for (int d = 16; d; d >>= 1) mine += __shfl_xor_sync(~0u, mine, d);
        if (lane == 0) sums[warp] = mine;
        if (tid == 0) found = -1;
        __syncthreads();
        long long total = 0;
#pragma unroll
        for (int w = 0; w < NT / 32; ++w) total += sums[w];
        per = (total + gridDim.x - 1) / gridDim.x;
        at = min(total, per * blockIdx.x);
        end = min(total, at + per);
        if (at < end) {                             // (the same in all threads)
            long long base = 0;
            for (int i0 = 0; i0 < n && base <= at; i0 += NT) {
                const long long x = i0 + tid < n ? units(i0 + tid) : 0;
                long long upto = x;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const long long y = __shfl_up_sync(~0u, upto, d);
                    if (lane >= d) upto += y;
                }
                __syncthreads();                    // the sums have been read
                if (lane == 31) sums[warp] = upto;
                __syncthreads();
                long long before = base, all = base;
#pragma unroll
                for (int w = 0; w < NT / 32; ++w) {
                    if (w < warp) before += sums[w];
                    all += sums[w];
                }
                if (before + upto - x <= at && at < before + upto) {
                    found = i0 + tid;
                    found_base = before + upto - x;
                }
                base = all;
            }
            __syncthreads();
            enter(found);
            const long long in = at - found_base, per_head = (long long)rbs * kbs;
            head = (int)(in / per_head);
            rb = (int)((in - head * per_head) / kbs);
            kb = (int)(in % kbs);
        }
    }
    __device__ bool more() const { return at < end; }
    // The next item; the list goes on behind it.
    __device__ Item next() {
        Item it;
        it.seq = seq; it.head = head; it.rb = rb; it.kb = kb; it.kbs = kbs;
        it.count = (int)min((long long)(kbs - kb), end - at);
        it.q0 = q0;
        it.rows = (int)min((long long)qlen * a.group - (long long)rb * BM, (long long)BM);
        it.k0 = k0; it.klen = klen;
        it.first = at - kb;
        at += it.count;
        kb += it.count;
        if (kb == kbs && at < end) {
            kb = 0;
            if (++rb == rbs) {
                rb = 0;
                if (++head == a.p.heads) {
                    head = 0;
                    do { enter(seq + 1); } while (rbs == 0 || kbs == 0);
                }
            }
        }
        return it;
    }
    // Element of q and of out of a row's first column (in units of tokens' rows: see row_of).
    __device__ static long long token_of(const CrossArgs& a, const Item& it, int r, int& h) {
        const long long row = (long long)it.rb * BM + r;
        const long long t = row / a.group;
        h = it.head * a.group + (int)(row - t * a.group);
        return it.q0 + t;
    }
};

template <typename T> __device__ __forceinline__ void put4(T* p, float4 x);
template <> __device__ __forceinline__ void put4<float>(float* p, float4 x) { *reinterpret_cast<float4*>(p) = x; }
template <> __device__ __forceinline__ void put4<__nv_bfloat16>(__nv_bfloat16* p, float4 x) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(x.x, x.y), b = __floats2bfloat162_rn(x.z, x.w);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
__device__ __forceinline__ float lse_of(const CrossArgs& a, float m, float l) { return l == 0.f ? -INFINITY : fmaf(m == -INFINITY ? 0.f : m, a.nat, logf(l)); }

// Sequences without states: rows of zeros.
template <typename T, int BM, int BN, int NT>
__device__ void empty_sequences(const CrossArgs& a, const Work<BM, BN>& w) {
    for (int i = blockIdx.x; i < a.p.n; i += gridDim.x) {
        int q0, qlen, k0, klen;
        w.lengths(i, q0, qlen, k0, klen);
        if (klen > 0) continue;
        const long long row = (long long)a.p.q_heads * a.p.D;
        T* const out = static_cast<T*>(a.p.out) + q0 * row;
        for (long long e = threadIdx.x; e < qlen * row / 4; e += NT) put4(out + 4 * e, make_float4(0.f, 0.f, 0.f, 0.f));
        if (a.p.lse)
            for (long long e = threadIdx.x; e < (long long)qlen * a.p.q_heads; e += NT) a.p.lse[(long long)q0 * a.p.q_heads + e] = -INFINITY;
    }
}

// A partial result in the workspace: four columns of a row at o[column / 4 * BM + row], (m, l) of each row.
template <int BM, int DP>
struct Part {
    float4* o;
    float2* ml;
    __device__ Part(const CrossArgs& a, int cta, int slot) {
        o = reinterpret_cast<float4*>(a.parts + ((size_t)cta * 2 + slot) * kPartFloats);
        ml = reinterpret_cast<float2*>(o + BM * (DP / 4));
        static_assert(BM * (DP + 2) <= kPartFloats, "a part must fit");
    }
};

// Arrival at an item's counter, which is zero before the first and after the last; true for the last.  The summands are 1, and 1 - n for
// the first CTA: their sum is zero whatever comes in between, so calls that overlap on a workspace leave zero behind all the same.
__device__ __forceinline__ bool arrive(unsigned* counter, int i, int n) {
    const unsigned x = i ? 1u : 1u - (unsigned)n;
    return atomicAdd(counter, x) + x == 0u;
}

// Adds the parts of an item, which CTAs c0 .. c1 have written, in order, and writes the result.  NT threads.
template <typename T, int BM, int BN, int DP, int NT>
__device__ void join_parts(const CrossArgs& a, const Item& it, int c0, int c1, int tid) {
    const int cols = a.p.D / 4;
    for (int e = tid; e < it.rows * cols; e += NT) {
        const int r = e % it.rows, c = e / it.rows;
        float m = -INFINITY, l = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k0 = c0; k0 <= c1; k0 += 8) {
            float4 x[8];
            float2 ml[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {                       // past the last part: that one again, not used
                const int cta = min(k0 + k, c1);
                const Part<BM, DP> q(a, cta, cta == c0);
                ml[k] = __ldcg(q.ml + r);
                x[k] = __ldcg(q.o + c * BM + r);
            }
            float top = m;
#pragma unroll
            for (int k = 0; k < 8; ++k) top = fmaxf(top, ml[k].x);
            // o is the mean so far: values near the end of the range stay inside it
            const float base = top == -INFINITY ? 0.f : top, had = l * exp2_fast((m - base) * a.unit);
            m = top;
            l = had;
            float w[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                w[k] = k0 + k > c1 ? 0.f : exp2_fast((ml[k].x - base) * a.unit);
                l = fmaf(w[k], ml[k].y, l);
            }
            const float inv = l == 0.f ? 0.f : 1.f / l, f = had * inv;
            o.x *= f; o.y *= f; o.z *= f; o.w *= f;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (k0 + k > c1) continue;
                const float by = w[k] * inv;
                o.x = fmaf(by, x[k].x, o.x); o.y = fmaf(by, x[k].y, o.y);
                o.z = fmaf(by, x[k].z, o.z); o.w = fmaf(by, x[k].w, o.w);
            }
        }
        int h;
        const long long row = Work<BM, BN>::token_of(a, it, r, h) * a.p.q_heads + h;
        put4(static_cast<T*>(a.p.out) + row * a.p.D + 4 * c, l == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : o);
        if (c == 0 && a.p.lse) a.p.lse[row] = lse_of(a, m, l);
    }
}

// ---- f32 on the CUDA cores --------------------------------------------------------------------------------------------

// Tiles of BM rows by 64 states, 256 threads: a thread has RT = BM / 16 rows (ty) and every 16th state or group of four columns (tx).  Products are
// packed pairs; K and V have one buffer each, and the next tile of K is on its way during the products with V, and the other way round.
template <int BM, int DP>
struct Cores {
    static constexpr int BN = 64, NT = 256, RT = BM / 16, LD = DP + 4, LP = BN + 4;
    static constexpr size_t SMEM = (size_t)(BM * LD + BN * LD + BN * DP + BM * LP) * sizeof(float);
};

template <int BM, int DP>
__global__ void __launch_bounds__(256) attn_cross_f32(const __grid_constant__ CrossArgs a) {
    using C = Cores<BM, DP>;
    constexpr int BN = C::BN, NT = C::NT, RT = C::RT, LD = C::LD, LP = C::LP, CG = DP / 64;
    extern __shared__ __align__(16) float smem[];
    float* const qs = smem;
    float* const ks = qs + BM * LD;
    float* const vs = ks + BN * LD;
    float* const ps = vs + BN * DP;
    __shared__ float sb[BN];
    __shared__ int last;
    const CrossProblem& p = a.p;
    const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4, D = p.D;
    pdl_trigger();
    pdl_wait();
    Work<BM, BN> work(a);
    work.template begin<NT>();
    empty_sequences<float, BM, BN, NT>(a, work);
    for (int e = tid; e < (BM + BN) * (LD / 4); e += NT) reinterpret_cast<float4*>(qs)[e] = make_float4(0.f, 0.f, 0.f, 0.f);   // columns past D
    for (int e = tid; e < BN * (DP / 4); e += NT) reinterpret_cast<float4*>(vs)[e] = make_float4(0.f, 0.f, 0.f, 0.f);
    while (work.more()) {
        const Item it = work.next();
        __syncthreads();                                        // the item before, or the zeros
        // rows past the item's last are left as they are: their results are not written
        auto load = [&](const float* src, long long stride, float* dst, int ld, int kb) {
            const int keys = min(BN, it.klen - kb * BN);
            for (int e = tid; e < BN * (D / 4); e += NT) {
                const int key = e / (D / 4), c = e - key * (D / 4);
                if (key < keys) cp_async16(smem_u32(dst + key * ld + 4 * c), src + (it.k0 + kb * BN + key) * stride + (long long)it.head * D + 4 * c, true);
            }
            cp_async_commit();
        };
        const float* const kg = static_cast<const float*>(p.k);
        const float* const vg = static_cast<const float*>(p.v);
        load(kg, p.k_stride, ks, LD, it.kb);
        load(vg, p.v_stride, vs, DP, it.kb);
        for (int e = tid; e < it.rows * (D / 4); e += NT) {
            const int r = e / (D / 4), c = e - r * (D / 4);
            int h;
            const long long t = Work<BM, BN>::token_of(a, it, r, h);
            const float4 x = *reinterpret_cast<const float4*>(static_cast<const float*>(p.q) + t * p.q_stride + (long long)h * D + 4 * c);
            *reinterpret_cast<float4*>(qs + r * LD + 4 * c) = make_float4(x.x * a.sign, x.y * a.sign, x.z * a.sign, x.w * a.sign);
        }
        float m[RT], l[RT];
        float2 o[RT][CG][2];
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            m[r] = -INFINITY;
            l[r] = 0.f;
#pragma unroll
            for (int g = 0; g < CG; ++g) o[r][g][0] = o[r][g][1] = make_float2(0.f, 0.f);
        }
        for (int j = 0; j < it.count; ++j) {
            const int kb = it.kb + j, keys = min(BN, it.klen - kb * BN);
            cp_async_wait<1>();                                 // K
            bool gone = false;
            if (tid < BN) {
                const float b = tid >= keys ? -INFINITY : p.bias ? p.bias[it.k0 + kb * BN + tid] : 0.f;
                sb[tid] = b;
                gone = b == -INFINITY;
            }
            const bool masked = __syncthreads_or(gone);
            float2 s2[RT][4];
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int x = 0; x < 4; ++x) s2[r][x] = make_float2(0.f, 0.f);
#pragma unroll 4
            for (int c = 0; c < DP / 4; ++c) {
                float4 q[RT], k[4];
#pragma unroll
                for (int r = 0; r < RT; ++r) q[r] = *reinterpret_cast<const float4*>(qs + (ty * RT + r) * LD + 4 * c);
#pragma unroll
                for (int x = 0; x < 4; ++x) k[x] = *reinterpret_cast<const float4*>(ks + (tx + 16 * x) * LD + 4 * c);
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        s2[r][x] = fma2(make_float2(q[r].x, q[r].y), make_float2(k[x].x, k[x].y), s2[r][x]);
                        s2[r][x] = fma2(make_float2(q[r].z, q[r].w), make_float2(k[x].z, k[x].w), s2[r][x]);
                    }
            }
            __syncthreads();                                    // K has been read
            if (j + 1 < it.count) load(kg, p.k_stride, ks, LD, kb + 1);
            else cp_async_commit();
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                float s[4], top = -INFINITY;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const float b = sb[tx + 16 * x];
                    s[x] = b == -INFINITY ? b : fmaf(s2[r][x].x + s2[r][x].y, a.c, b);      // whatever a masked row holds
                    top = fmaxf(top, s[x]);
                }
#pragma unroll
                for (int d = 8; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, d));
                top = fmaxf(top, m[r]);
                const float base = top == -INFINITY ? 0.f : top, f = exp2_fast((m[r] - base) * a.unit);
                m[r] = top;
                l[r] *= f;
#pragma unroll
                for (int g = 0; g < CG; ++g) {
                    o[r][g][0].x *= f; o[r][g][0].y *= f; o[r][g][1].x *= f; o[r][g][1].y *= f;
                }
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const float w = exp2_fast((s[x] - base) * a.unit);
                    l[r] += w;
                    ps[(ty * RT + r) * LP + tx + 16 * x] = w;
                }
            }
            cp_async_wait<1>();                                 // V
            __syncthreads();
            if (masked) {
                for (int e = tid; e < BN * (DP / 4); e += NT)
                    if (sb[e / (DP / 4)] == -INFINITY) reinterpret_cast<float4*>(vs)[e] = make_float4(0.f, 0.f, 0.f, 0.f);
                __syncthreads();
            }
#pragma unroll 2
            for (int k4 = 0; k4 < BN / 4; ++k4) {
                float4 w[RT];
#pragma unroll
                for (int r = 0; r < RT; ++r) w[r] = *reinterpret_cast<const float4*>(ps + (ty * RT + r) * LP + 4 * k4);
#pragma unroll
                for (int x = 0; x < 4; ++x) {
#pragma unroll
                    for (int g = 0; g < CG; ++g) {
                        const float4 v = *reinterpret_cast<const float4*>(vs + (4 * k4 + x) * DP + 64 * g + 4 * tx);
#pragma unroll
                        for (int r = 0; r < RT; ++r) {
                            const float y = x == 0 ? w[r].x : x == 1 ? w[r].y : x == 2 ? w[r].z : w[r].w;
                            o[r][g][0] = fma2(make_float2(y, y), make_float2(v.x, v.y), o[r][g][0]);
                            o[r][g][1] = fma2(make_float2(y, y), make_float2(v.z, v.w), o[r][g][1]);
                        }
                    }
                }
            }
            __syncthreads();                                    // V and the weights have been read
            if (j + 1 < it.count) load(vg, p.v_stride, vs, DP, kb + 1);
            else cp_async_commit();
        }
        const bool whole = it.count == it.kbs;
        const Part<BM, DP> part(a, blockIdx.x, it.kb == 0);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            float sum = l[r];
#pragma unroll
            for (int d = 8; d; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
            const int row = ty * RT + r;
            if (row >= it.rows) continue;
            int h;
            const long long at = Work<BM, BN>::token_of(a, it, row, h) * p.q_heads + h;
            const float f = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
            for (int g = 0; g < CG; ++g) {
                const int d = 64 * g + 4 * tx;
                if (d >= D) continue;
                const float4 x = make_float4(o[r][g][0].x, o[r][g][0].y, o[r][g][1].x, o[r][g][1].y);
                if (whole) put4(static_cast<float*>(p.out) + at * D + d, sum == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(x.x * f, x.y * f, x.z * f, x.w * f));
                else part.o[d / 4 * BM + row] = x;
            }
            if (tx == 0) {
                if (!whole) part.ml[row] = make_float2(m[r], sum);
                else if (p.lse) p.lse[at] = lse_of(a, m[r], sum);
            }
        }
        if (!whole) {
            const int c0 = (int)(it.first / work.per), c1 = (int)((it.first + it.kbs - 1) / work.per);
            __threadfence();
            __syncthreads();
            if (tid == 0) last = arrive(a.counters + c0, blockIdx.x - c0, c1 - c0 + 1);
            __syncthreads();
            if (last) {
                __threadfence();
                join_parts<float, BM, BN, DP, NT>(a, it, c0, c1, tid);
            }
        }
    }
}

// ---- bf16 on the tensor cores -----------------------------------------------------------------------------------------

// DP: columns of a row in shared memory (D, rounded up to 64, 128 or 256).  A CTA has TILES tiles of 128 rows, each with four warps that take
// its weights (a thread has a row), a warp that issues the products and one that brings K and V by TMA.
//
// S = Q K^T lands in tensor memory, the threads read it, and leave the weights, in bf16, in its place, from where they are the first operand of
// O += P V.  While one tile's weights are worked out, the other tile's products run.  Where there are no more than 128 rows both tiles have
// the same rows and every other tile of states, and their results are added at the end.
//
// Roundings.  Scores and sums are fp32; a weight is rounded to bf16 for its product with V, 2^-8 of its size at most: the
// errors of the states' weights are independent, and their mean is below the rounding of the output.  (The pairs of 16-bit floats that the attention
// of one token uses would double the second product, which bounds this one.)
template <int DP_>
struct Tc {
    static constexpr int DP = DP_, TILES = DP <= 128 ? 2 : 1, BN = DP <= 128 ? 128 : 64, ROWS = 128 * TILES;
    static constexpr int Q_BYTES = 128 * DP * 2, STAGE = BN * DP * 2, STAGES = DP == 64 ? 8 : 5;
    static constexpr int THREADS = 320, S_COLS = 128, O_COL = 256, O_COLS = DP <= 128 ? 128 : 256;
    static constexpr size_t SMEM = 1024 + TILES * Q_BYTES + STAGES * STAGE;
    static_assert(TILES == 1 || 2 * Q_BYTES >= 128 * DP * 4, "a tile's result fits the queries' place");
};

// The reference of the weights may lag behind the maximum by this much (in powers of two).
constexpr float kLag = 8.f;

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const void* tmap, uint32_t bar, int x, int y, int z) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(tmap), "r"(bar), "r"(x), "r"(y), "r"(z) : "memory");
}
__device__ __forceinline__ void tmem_ld_wait32(uint32_t (&v)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]), "+r"(v[10]),
                   "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]), "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]),
                   "+r"(v[21]), "+r"(v[22]), "+r"(v[23]), "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31])::"memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&v)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
                   "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t (&v)[32]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
                 "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
                 ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
                   "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]),
                   "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]) : "memory");
}
__device__ __forceinline__ void named_barrier(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// Waits for a phase of a barrier.  When one wait of a CTA gives up, all others do at once: what follows runs through without waiting, so that
// every barrier between threads is still met by all of them, and the results are not to be used.
__device__ __forceinline__ bool wait_phase(uint32_t bar, int parity, volatile int* dead, int* status) {
    if (mbar_try_wait(bar, parity)) return true;
    int limit = kWaitProbes;
    for (int probes = 1; probes < limit; ++probes) {
        if (mbar_try_wait(bar, parity)) return true;
        if (*dead) return false;
        if (probes == kLeastProbes - 1) {
            const int knob = *reinterpret_cast<volatile int*>(status + kStatusProbeLimit);
            if (knob > 0) limit = max(kLeastProbes, knob);
        }
    }
    *dead = 1;
    *status = LUVC_ERR_TIMEOUT;
    return false;
}

// A row of an item once more, by a warp, product by product as the formula has them.  An infinity among the values meets weights that bf16 has
// rounded to 0, and weights above 1, while their reference lags behind, can take values beyond the end of the range; so a
// row that is not finite is worked out again.  It is rare, and need not be fast.
template <int DP>
__device__ __noinline__ void plain_row(const CrossArgs& a, const Item& it, int r) {
    constexpr int ROWS = Tc<DP>::ROWS, BN = Tc<DP>::BN;
    const CrossProblem& p = a.p;
    const int lane = threadIdx.x & 31, D = p.D;
    int h;
    const long long t = Work<ROWS, BN>::token_of(a, it, r, h), row = t * p.q_heads + h;
    const __nv_bfloat16* const qr = static_cast<const __nv_bfloat16*>(p.q) + t * p.q_stride + (long long)h * D;
    float q[DP / 32], o[DP / 32], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int j = 0; j < DP / 32; ++j) {
        q[j] = lane + 32 * j < D ? __bfloat162float(qr[lane + 32 * j]) * a.sign : 0.f;
        o[j] = 0.f;
    }
    const long long k1 = it.k0 + min((long long)(it.kb + it.count) * BN, (long long)it.klen);
    for (long long k = it.k0 + (long long)it.kb * BN; k < k1; ++k) {
        const float bias = p.bias ? p.bias[k] : 0.f;
        if (bias == -INFINITY) continue;
        const __nv_bfloat16* const kr = static_cast<const __nv_bfloat16*>(p.k) + k * p.k_stride + (long long)it.head * D;
        const __nv_bfloat16* const vr = static_cast<const __nv_bfloat16*>(p.v) + k * p.v_stride + (long long)it.head * D;
        float s = 0.f, v[DP / 32];
#pragma unroll
        for (int j = 0; j < DP / 32; ++j) {
            const int d = lane + 32 * j;
            v[j] = 0.f;
            if (d < D) {
                s = fmaf(q[j], __bfloat162float(kr[d]), s);
                v[j] = __bfloat162float(vr[d]);
            }
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
        s = fmaf(s, a.c, bias);
        const float top = fmaxf(m, s), base = top == -INFINITY ? 0.f : top;
        // o is the mean so far: values near the end of the range stay inside it
        const float had = l * exp2_fast((m - base) * a.unit), w = exp2_fast((s - base) * a.unit);
        m = top;
        l = had + w;
        const float inv = l == 0.f ? 0.f : 1.f / l, f = had * inv, by = w * inv;
#pragma unroll
        for (int j = 0; j < DP / 32; ++j) o[j] = lane + 32 * j < D ? fmaf(o[j], f, by * v[j]) : 0.f;
    }
    const bool whole = it.count == it.kbs;
    const Part<ROWS, DP> part(a, blockIdx.x, it.kb == 0);
#pragma unroll
    for (int j = 0; j < DP / 32; ++j) {
        const int d = lane + 32 * j;
        if (d >= D) continue;
        if (whole) static_cast<__nv_bfloat16*>(p.out)[row * D + d] = __float2bfloat16_rn(l == 0.f ? 0.f : o[j]);
        else reinterpret_cast<float*>(part.o + d / 4 * ROWS + r)[d & 3] = o[j];
    }
    if (lane == 0) {
        if (!whole) part.ml[r] = make_float2(l == 0.f ? m : m + __log2f(l) / a.unit, l == 0.f ? 0.f : 1.f);      // weights that sum to one
        else if (p.lse) p.lse[row] = lse_of(a, m, l);
    }
    __syncwarp();
}

template <int DP, bool BIAS>
__global__ void __launch_bounds__(Tc<DP>::THREADS, 1)
attn_cross_tc(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const __grid_constant__ CrossArgs a) {
    using T = Tc<DP>;
    constexpr int TILES = T::TILES, BN = T::BN, ROWS = T::ROWS, STAGES = T::STAGES, CH = BN / 32;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t bars[8 + 2 * STAGES + 1];
    __shared__ __align__(16) float sb[2][128];                  // biases of a tile of states, for each tile of rows; (m, l) of the second one
    __shared__ uint32_t tmem_at;
    __shared__ int dead_flag, last;
    const CrossProblem& p = a.p;
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(~0u, tid >> 5, 0), D = p.D;
    unsigned char* const base = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    const uint32_t qs = smem_u32(base), ring = qs + TILES * T::Q_BYTES, bar0 = smem_u32(bars);
    auto q_full = [&](int t) { return bar0 + 8 * t; };
    auto s_full = [&](int t) { return bar0 + 16 + 8 * t; };
    auto p_ready = [&](int t) { return bar0 + 32 + 8 * t; };
    auto o_full = [&](int t) { return bar0 + 48 + 8 * t; };
    auto kv_full = [&](int s) { return bar0 + 64 + 8 * s; };
    auto kv_free = [&](int s) { return bar0 + 64 + 8 * (STAGES + s); };
    const uint32_t drained = bar0 + 64 + 16 * STAGES;
    volatile int* const dead = &dead_flag;
    const int segs = (D + 63) / 64, ksteps = (D + 15) / 16;

    if (warp == 9) tmem_alloc(smem_u32(&tmem_at), 512);
    if (tid == 0) {
        for (int t = 0; t < 2; ++t) {
            mbar_init(q_full(t), 128);
            mbar_init(s_full(t), 1);
            mbar_init(p_ready(t), 128);
            mbar_init(o_full(t), 1);
        }
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(kv_full(s), 1);
            mbar_init(kv_free(s), 1);
        }
        mbar_init(drained, 1);
        mbar_fence_init();
        dead_flag = 0;
        asm volatile("prefetch.tensormap [%0];" ::"l"(&kmap) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&vmap) : "memory");
    }
    pdl_trigger();
    pdl_wait();
    Work<ROWS, BN> work(a);
    tc_fence_before();
    work.template begin<T::THREADS>();                          // (has barriers of all threads)
    tc_fence_after();
    const uint32_t tmem = tmem_at;
    empty_sequences<__nv_bfloat16, ROWS, BN, T::THREADS>(a, work);

    if (warp == 8) {
        // ---- K and V, tile after tile, through a ring of stages ----
        if (lane == 0) {
            int pos = 0;                                        // K of the n-th tile of this CTA is 2 n, V 2 n + 1
            bool ok = true;
            while (ok && work.more()) {
                const Item it = work.next();
                for (int j = 0; ok && j < 2 * it.count; ++j, ++pos) {
                    const int stage = pos % STAGES, use = pos / STAGES;
                    if (use > 0) ok = wait_phase(kv_free(stage), (use - 1) & 1, dead, p.status);
                    if (!ok) break;
                    // (a test's knob: the first copy of the first CTA is waited for in vain)
                    const uint32_t more = pos == 0 && blockIdx.x == 0 && p.status[kStatusHoldBack] > 0 ? 16 : 0;
                    mbar_arrive_expect_tx(kv_full(stage), segs * BN * 128 + more);
                    for (int s = 0; s < segs; ++s)
                        tma_load_3d(ring + stage * T::STAGE + s * BN * 128, j & 1 ? &vmap : &kmap, kv_full(stage), 64 * s, it.head,
                                    (int)(it.k0 + (long long)(it.kb + j / 2) * BN));
                }
            }
            // the CTA must not end before its copies have landed (they have, unless a wait gave up)
            for (int x = max(0, pos - STAGES); x < pos; ++x)
                for (int probes = 0; !mbar_try_wait(kv_full(x % STAGES), (x / STAGES) & 1) && *dead && probes < kLeastProbes; ++probes) {}
        }
    } else if (warp == 9) {
        // ---- products ----
        const uint32_t idesc_s = make_idesc_bf16(128, BN, false, false), idesc_o = make_idesc_bf16(128, 16 * ksteps, false, true);
        const uint64_t q0 = make_desc_layout(qs, 16, 1024, 2), k0 = make_desc_layout(ring, 16, 1024, 2), v0 = make_desc_layout(ring, BN * 128, 1024, 2);
        auto wait = [&](uint32_t bar, int parity) {
            bool ok = true;
            if (lane == 0) ok = wait_phase(bar, parity, dead, p.status);
            return (bool)__shfl_sync(~0u, (int)ok, 0);
        };
        auto full = [&](int pos) { return wait(kv_full(pos % STAGES), (pos / STAGES) & 1); };
        auto scores = [&](int t, int q_tile, int pos) {         // S of tile t
            if (elect_one()) {
                const uint64_t q = q0 + ((uint32_t)(q_tile * T::Q_BYTES) >> 4), k = k0 + ((uint32_t)(pos % STAGES * T::STAGE) >> 4);
                for (int x = 0; x < ksteps; ++x)
                    umma_bf16(tmem + t * T::S_COLS, q + ((x >> 2) * (128 * 128) + (x & 3) * 32 >> 4), k + ((x >> 2) * (BN * 128) + (x & 3) * 32 >> 4), idesc_s, x ? 1u : 0u);
                umma_commit(s_full(t));
            }
            __syncwarp();
        };
        auto values = [&](int t, int pos, bool first) {         // O of tile t
            if (elect_one()) {
                const uint64_t v = v0 + ((uint32_t)(pos % STAGES * T::STAGE) >> 4);
#pragma unroll
                for (int x = 0; x < BN / 16; ++x)
                    umma_bf16_ts(tmem + T::O_COL + t * T::O_COLS, tmem + t * T::S_COLS + 8 * x, v + (2048 * x >> 4), idesc_o, x || !first ? 1u : 0u);
            }
            __syncwarp();
        };
        auto commit = [&](uint32_t bar) {
            if (elect_one()) umma_commit(bar);
            __syncwarp();
        };
        int n0 = 0, q_used[2] = {0, 0}, p_used[2] = {0, 0};
        bool ok = true;
        while (ok && work.more()) {
            const Item it = work.next();
            const bool two = TILES == 2 && it.rows > 128, both = TILES == 2 && !two;        // two tiles of rows; both take the same rows
            ok = wait(q_full(0), q_used[0]++ & 1);
            if (ok && two) ok = wait(q_full(1), q_used[1]++ & 1);
            if (!ok) break;
            tc_fence_after();
            if (!both) {
                const int tiles = two ? 2 : 1;
                if (!(ok = full(2 * n0))) break;
                for (int t = 0; t < tiles; ++t) scores(t, t, 2 * n0);
                commit(kv_free(2 * n0 % STAGES));
                for (int j = 0; ok && j < it.count; ++j) {
                    const int v = 2 * (n0 + j) + 1;
                    ok = full(v);
                    for (int t = 0; ok && t < tiles; ++t) {
                        if (!(ok = wait(p_ready(t), p_used[t]++ & 1))) break;
                        tc_fence_after();
                        values(t, v, j == 0);
                        if (j + 1 < it.count) {
                            if (t == 0 && !(ok = full(v + 1))) break;
                            scores(t, t, v + 1);
                        } else {
                            commit(o_full(t));
                        }
                    }
                    if (!ok) break;
                    commit(kv_free(v % STAGES));
                    if (j + 1 < it.count) commit(kv_free((v + 1) % STAGES));
                }
            } else {
                for (int s = 0; ok && s < min(2, it.count); ++s) {
                    if (!(ok = full(2 * (n0 + s)))) break;
                    scores(s, 0, 2 * (n0 + s));
                    commit(kv_free(2 * (n0 + s) % STAGES));
                }
                for (int s = 0; ok && s < it.count; ++s) {
                    const int t = s & 1, v = 2 * (n0 + s) + 1;
                    if (!(ok = full(v)) || !(ok = wait(p_ready(t), p_used[t]++ & 1))) break;
                    tc_fence_after();
                    values(t, v, s < 2);
                    commit(kv_free(v % STAGES));
                    if (s + 2 < it.count) {
                        if (!(ok = full(v + 3))) break;
                        scores(t, 0, v + 3);
                        commit(kv_free((v + 3) % STAGES));
                    } else {
                        commit(o_full(t));
                    }
                }
            }
            n0 += it.count;
        }
        if (!ok) {                                              // tensor memory is given back below: products in flight end first
            commit(drained);
            for (int probes = 0; probes < kLeastProbes && !mbar_try_wait(drained, 0); ++probes) {}
        }
    } else {
        // ---- weights ----
        const int t = warp >> 2, r = tid & 127;                 // tile; row of it
        const uint32_t rows_at = tmem + ((uint32_t)((warp & 3) * 32) << 16), s_at = rows_at + t * T::S_COLS, o_at = rows_at + T::O_COL + t * T::O_COLS;
        int n0 = 0, s_used = 0, o_used = 0;
        while (work.more()) {
            const Item it = work.next();
            const bool two = TILES == 2 && it.rows > 128, both = TILES == 2 && !two;
            const int mine = two ? 128 * t + r : r;             // row of the item
            const bool mine_live = mine < it.rows;
            if (t == 0 || two) {                                // queries, in the order the products read them
                int h;
                const long long tok = Work<ROWS, BN>::token_of(a, it, mine_live ? mine : 0, h);
                const uint4* const src = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p.q) + tok * p.q_stride + (long long)h * D);
                const unsigned flip = a.sign < 0.f ? 0x80008000u : 0u;
                unsigned char* const dst = base + t * T::Q_BYTES + r * 128;
#pragma unroll 8
                for (int c = 0; c < 2 * ksteps; ++c) {
                    uint4 x = make_uint4(0u, 0u, 0u, 0u);
                    if (mine_live && 8 * c < D) {
                        x = __ldg(src + c);
                        x.x ^= flip; x.y ^= flip; x.z ^= flip; x.w ^= flip;
                    }
                    *reinterpret_cast<uint4*>(dst + (c >> 3) * (128 * 128) + (((c & 7) ^ (r & 7)) << 4)) = x;
                }
                fence_proxy_async();
                mbar_arrive(q_full(t));
            }
            float m = -INFINITY, l = 0.f;
            int blocks = 0;                                     // tiles of states this tile of rows has had
            const int step = both ? 2 : 1;
            for (int j = both ? t : 0; j < it.count && (t == 0 || TILES == 2); j += step, ++blocks) {
                const int kb = it.kb + j, keys = min(BN, it.klen - kb * BN);
                bool gone = r < BN && r >= keys;
                if (BIAS) {
                    if (r < BN) {
                        const float b = gone ? -INFINITY : p.bias[it.k0 + (long long)kb * BN + r];
                        gone = b == -INFINITY;
                        sb[t][r] = b;
                    }
                    named_barrier(2 + t, 128);
                }
                wait_phase(s_full(t), s_used++ & 1, dead, p.status);
                tc_fence_after();
                uint32_t s[CH][32];
#pragma unroll
                for (int c = 0; c < CH; ++c) tmem_ld32(s_at + 32 * c, s[c]);
#pragma unroll
                for (int c = 0; c < CH; ++c) tmem_ld_wait32(s[c]);
                float top = -INFINITY;
                if (BIAS) {
#pragma unroll
                    for (int c = 0; c < CH; ++c)
#pragma unroll
                        for (int x = 0; x < 32; x += 4) {
                            const float4 b = *reinterpret_cast<const float4*>(&sb[t][32 * c + x]);
                            const float bs[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float y = bs[e] == -INFINITY ? bs[e] : fmaf(__uint_as_float(s[c][x + e]), a.c, bs[e]);
                                s[c][x + e] = __float_as_uint(y);
                            }
                        }
                    named_barrier(2 + t, 128);                  // the biases have been read
                } else if (keys < BN) {
#pragma unroll
                    for (int c = 0; c < CH; ++c)
#pragma unroll
                        for (int x = 0; x < 32; ++x)
                            if (32 * c + x >= keys) s[c][x] = 0xff800000u;
                }
                float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int x = 0; x < 32; x += 2)
                        tops[x >> 1 & 3] = fmaxf(tops[x >> 1 & 3], fmaxf(__uint_as_float(s[c][x]), __uint_as_float(s[c][x + 1])));
                top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
                const float c1 = BIAS ? 1.f : a.c, unit = BIAS ? kLog2e : 1.f;
                top *= c1;
                if (__any_sync(~0u, top > m + kLag / unit)) {
                    const float now = fmaxf(m, top), from = now == -INFINITY ? 0.f : now, f = exp2_fast((m - from) * unit);
                    m = now;
                    l *= f;
                    if (blocks > 0) {                           // the products of the tiles before are done: the scores came after them
                        for (int c = 0; c < 16 * ksteps; c += 32) {
                            uint32_t o[32];
                            tmem_ld32(o_at + c, o);
                            tmem_ld_wait32(o);
#pragma unroll
                            for (int x = 0; x < 32; ++x) o[x] = __float_as_uint(__uint_as_float(o[x]) * f);
                            tmem_st32(o_at + c, o);
                        }
                    }
                }
                const float from = m == -INFINITY ? 0.f : m;
                float2 sums[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    uint32_t w[16];
#pragma unroll
                    for (int x = 0; x < 32; x += 2) {
                        float2 y;
                        if (BIAS) y = make_float2((__uint_as_float(s[c][x]) - from) * kLog2e, (__uint_as_float(s[c][x + 1]) - from) * kLog2e);
                        else y = fma2(make_float2(__uint_as_float(s[c][x]), __uint_as_float(s[c][x + 1])), make_float2(c1, c1), make_float2(-from, -from));
                        y = make_float2(exp2_fast(y.x), exp2_fast(y.y));
                        sums[x >> 1 & 1].x += y.x;
                        sums[x >> 1 & 1].y += y.y;
                        const __nv_bfloat162 two16 = __floats2bfloat162_rn(y.x, y.y);
                        w[x >> 1] = *reinterpret_cast<const uint32_t*>(&two16);
                    }
                    tmem_st16(s_at + 16 * c, w);
                }
                l += (sums[0].x + sums[0].y) + (sums[1].x + sums[1].y);
                if (gone) {                                     // a masked state's values may be anything, and meet a weight of zero
                    const int pos = 2 * (n0 + j) + 1;
                    wait_phase(kv_full(pos % STAGES), (pos / STAGES) & 1, dead, p.status);
                    for (int c = 0; c < 8 * segs; ++c)
                        *reinterpret_cast<uint4*>(base + TILES * T::Q_BYTES + pos % STAGES * T::STAGE + (c >> 3) * (BN * 128) + r * 128 + (c & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                    fence_proxy_async();
                }
                tmem_st_wait();
                tc_fence_before();
                mbar_arrive(p_ready(t));
            }
            n0 += it.count;
            const bool whole = it.count == it.kbs;
            const Part<ROWS, DP> part(a, blockIdx.x, it.kb == 0);
            if (blocks > 0) {
                wait_phase(o_full(t), o_used++ & 1, dead, p.status);
                tc_fence_after();
            }
            // the result of the thread's row: O f0, plus another part's O f1 of columns [d / 4][row] in shared memory
            auto emit = [&](bool add, float f0, float f1) {
                int h;
                const long long row = Work<ROWS, BN>::token_of(a, it, mine_live ? mine : 0, h) * p.q_heads + h;
                float bad = l * 0.f;                            // 0, or NaN
                const float inv = l == 0.f ? 0.f : 1.f / l;
                for (int c = 0; c < D; c += 32) {
                    uint32_t o[32];
                    tmem_ld32(o_at + c, o);
                    tmem_ld_wait32(o);
#pragma unroll
                    for (int x = 0; x < 32; x += 8) {
                        if (c + x >= D) continue;
                        float y[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) y[e] = __uint_as_float(o[x + e]);
                        if (add) {
#pragma unroll
                            for (int e = 0; e < 8; e += 4) {
                                const float4 z = *reinterpret_cast<const float4*>(base + ((size_t)((c + x + e) / 4) * 128 + r) * 16);
                                y[e] = fmaf(z.x, f1, y[e] * f0); y[e + 1] = fmaf(z.y, f1, y[e + 1] * f0);
                                y[e + 2] = fmaf(z.z, f1, y[e + 2] * f0); y[e + 3] = fmaf(z.w, f1, y[e + 3] * f0);
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e) bad = fmaf(y[e], 0.f, bad);
                        if (!mine_live) continue;
                        if (whole) {
                            uint32_t w[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const __nv_bfloat162 two16 = __floats2bfloat162_rn(y[2 * e] * inv, y[2 * e + 1] * inv);
                                w[e] = *reinterpret_cast<const uint32_t*>(&two16);
                            }
                            *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.out) + row * D + c + x) = make_uint4(w[0], w[1], w[2], w[3]);
                        } else {
                            part.o[(c + x) / 4 * ROWS + mine] = make_float4(y[0], y[1], y[2], y[3]);
                            if (c + x + 4 < D) part.o[((c + x) / 4 + 1) * ROWS + mine] = make_float4(y[4], y[5], y[6], y[7]);
                        }
                    }
                }
                if (mine_live) {
                    if (!whole) part.ml[mine] = make_float2(m, l);
                    else if (p.lse) p.lse[row] = lse_of(a, m, l);
                }
                __syncwarp();
                for (unsigned again = __ballot_sync(~0u, mine_live && bad != 0.f && !*dead); again; again &= again - 1)
                    plain_row<DP>(a, it, __shfl_sync(~0u, mine, __ffs(again) - 1));
            };
            if (!both || it.count == 1) {
                if (blocks > 0) emit(false, 1.f, 0.f);
            } else {
                // two results of the same rows: the second one goes through the place of the queries, whose products are done
                named_barrier(1, 256);
                if (t == 1) {
                    for (int c = 0; c < D; c += 32) {
                        uint32_t o[32];
                        tmem_ld32(o_at + c, o);
                        tmem_ld_wait32(o);
#pragma unroll
                        for (int x = 0; x < 32; x += 4)
                            if (c + x < D)
                                *reinterpret_cast<float4*>(base + ((size_t)((c + x) / 4) * 128 + r) * 16) =
                                    make_float4(__uint_as_float(o[x]), __uint_as_float(o[x + 1]), __uint_as_float(o[x + 2]), __uint_as_float(o[x + 3]));
                    }
                    reinterpret_cast<float2*>(&sb[0][0])[r] = make_float2(m, l);
                }
                named_barrier(1, 256);
                if (t == 0) {
                    const float2 ml = reinterpret_cast<const float2*>(&sb[0][0])[r];
                    const float now = fmaxf(m, ml.x), from = now == -INFINITY ? 0.f : now;
                    const float f0 = exp2_fast((m - from) * a.unit), f1 = exp2_fast((ml.x - from) * a.unit);
                    m = now;
                    l = l * f0 + ml.y * f1;
                    emit(true, f0, f1);
                }
                named_barrier(1, 256);
            }
            tc_fence_before();                                  // O has been read before the next item's weights are announced
            if (!whole) {
                const int c0 = (int)(it.first / work.per), c1 = (int)((it.first + it.kbs - 1) / work.per);
                __threadfence();
                named_barrier(1, 256);
                if (tid == 0) last = arrive(a.counters + c0, blockIdx.x - c0, c1 - c0 + 1);
                named_barrier(1, 256);
                if (last) {
                    __threadfence();
                    join_parts<__nv_bfloat16, ROWS, BN, DP, 256>(a, it, c0, c1, tid);
                }
            }
        }
    }
    __syncthreads();
    if (warp == 9) tmem_dealloc(tmem, 512);
}

// ---- launch -----------------------------------------------------------------------------------------------------------

// The kernel may use this much shared memory; once per device.
template <typename K>
bool allow_smem(K kernel, size_t bytes, std::atomic<unsigned long long>& set) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return false;
    if (dev <= 63 && ((set.load(std::memory_order_relaxed) >> dev) & 1)) return true;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    if (dev <= 63) set.fetch_or(1ull << dev, std::memory_order_relaxed);
    return true;
}

template <int BM, int DP>
int launch_f32(const CrossArgs& a) {
    static std::atomic<unsigned long long> set{0};
    const int sms = std::min(sm_count(), kMaxCtas);
    if (!sms || !allow_smem(attn_cross_f32<BM, DP>, Cores<BM, DP>::SMEM, set)) return LUVC_ERR_CUDA;
    return launch_overlapped(attn_cross_f32<BM, DP>, sms, Cores<BM, DP>::NT, Cores<BM, DP>::SMEM, a.p.stream, a);
}

template <int BM>
int launch_f32_wide(const CrossArgs& a) {
    return a.p.D <= 64 ? launch_f32<BM, 64>(a) : a.p.D <= 128 ? launch_f32<BM, 128>(a) : launch_f32<BM, 256>(a);
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_tiled_fn() {
    static EncodeTiledFn fn = nullptr;
    if (!fn) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiledFn>(p);
    }
    return fn;
}

// The states as [k_tokens][heads][D], fetched in boxes of BN states of a head by 64 columns (zeros past the last state and column).
template <int BN>
bool states_map(CUtensorMap* map, const CrossProblem& p, const void* rows, long long stride) {
    EncodeTiledFn encode = encode_tiled_fn();
    if (!encode) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)p.D, (cuuint64_t)p.heads, (cuuint64_t)std::max(p.k_tokens, 1)};
    const cuuint64_t strides[2] = {(cuuint64_t)p.D * 2, (cuuint64_t)stride * 2};
    const cuuint32_t box[3] = {64u, 1u, (cuuint32_t)BN}, ones[3] = {1u, 1u, 1u};
    void* const base = const_cast<void*>(p.k_tokens ? rows : p.q);      // (nothing is read where there are no states)
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, base, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DP, bool BIAS>
int launch_tc(const CrossArgs& a) {
    using T = Tc<DP>;
    static std::atomic<unsigned long long> set{0};
    const int sms = std::min(sm_count(), kMaxCtas);
    CUtensorMap kmap, vmap;
    if (!sms || !states_map<T::BN>(&kmap, a.p, a.p.k, a.p.k_stride) || !states_map<T::BN>(&vmap, a.p, a.p.v, a.p.v_stride) ||
        !allow_smem(attn_cross_tc<DP, BIAS>, T::SMEM, set))
        return LUVC_ERR_CUDA;
    return launch_overlapped(attn_cross_tc<DP, BIAS>, sms, T::THREADS, T::SMEM, a.p.stream, kmap, vmap, a);
}

template <int DP>
int launch_tc_bias(const CrossArgs& a) {
    return a.p.bias ? launch_tc<DP, true>(a) : launch_tc<DP, false>(a);
}

}  // namespace

size_t attn_cross_workspace_bytes() { return kCounterBytes + (size_t)kMaxCtas * 2 * kPartFloats * sizeof(float); }

int attn_cross(const CrossProblem& p) {
    CrossArgs a;
    a.p = p;
    a.group = p.q_heads / p.heads;
    a.c = fabsf(p.scale) * (p.bias ? 1.f : kLog2e);
    a.unit = p.bias ? kLog2e : 1.f;
    a.nat = p.bias ? 1.f : kLn2;
    a.sign = p.scale < 0.f ? -1.f : 1.f;
    a.counters = static_cast<unsigned*>(p.workspace);
    a.parts = reinterpret_cast<float*>(static_cast<unsigned char*>(p.workspace) + kCounterBytes);
    if (p.dtype == LUVC_BF16) return p.D <= 64 ? launch_tc_bias<64>(a) : p.D <= 128 ? launch_tc_bias<128>(a) : launch_tc_bias<256>(a);
    // few rows of a key head: small blocks
    const bool few = (long long)p.q_tokens * a.group <= 16ll * p.n;
    return few ? launch_f32_wide<16>(a) : launch_f32_wide<64>(a);
}

}  // namespace luvc
