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
// Split.  The work is the list of all (sequence, key head, block of rows, tile of states); each CTA takes an equal part of it, whatever the
// lengths.  What a CTA has of a (sequence, key head, block of rows) that others share goes through the workspace; the CTA that comes last
// adds the parts, in the order of the list, so that a repeated call gives the same bits.  Where there is little to do, the parts are whole
// (sequence, key head, block of rows)s: a join costs as much as some tiles (JOIN).
//
// Bound.  4 D flops for each row and state: the tensor pipe, where there are many rows.  Two sequences of 1777 to 2048 tokens to 12001 to 16384
// states, 32 / 8 heads of 128 (970 GFLOP, bf16): 984 us in a short loop, 0.59 of the rate of a large matrix product, 1083 in a long one, where the power
// limit brings the clock down (one of 2048 to 16384: 530 us for 550 GFLOP, 0.62).  Eight questions of 17 to 96 tokens to 1296 states, 28 / 4 heads:
// 26.4 us, a chain of latencies.  A few tokens are a matter of bytes, and go another way (attn_rows).
//
// bf16: tensor cores (attn_cross_tc).  f32: CUDA cores (attn_cross_f32), 32-bit products and sums, 44 TFLOP/s of 73 that packed products reach (a
// choice: pairs of tf32 on the tensor cores are not built).

#include <cuda.h>
#include <cuda_bf16.h>
#include <cmath>

#include <algorithm>
#include <atomic>
#include <type_traits>

#include "luvc_internal.h"
#include "sm100_ptx.cuh"

namespace luvc {
namespace {

using namespace ptx;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kMaxCtas = 320;                       // CTAs there are counters for
constexpr size_t kCounterBytes = 2048, kPartsBytes = (size_t)160 * 2 * 256 * 130 * sizeof(float);      // 160 CTAs' parts of 256 rows of 128 columns
static_assert(kMaxCtas * sizeof(unsigned) <= kCounterBytes, "room for the counters");
constexpr int kWaitProbes = 1 << 20;                // probes before a wait gives up (seconds)
constexpr int kLeastProbes = 1 << 12;               // and with a limit from the status block (a test's)

struct CrossArgs {
    CrossProblem p;
    int group;                                      // query heads per key head
    int block, shift;                               // rows of a block: a power of two
    // Scores are c <q, k> + bias, weights 2^(unit (score - m)), and a score is worth nat in natural units: with biases c = |scale|, unit = log2(e),
    // nat = 1 (a bias of the lowest value times log2(e) would not be finite), without c = |scale| log2(e), unit = 1, nat = ln(2).
    float c, unit, nat;
    float sign;                                     // of the scale; c has its magnitude
    // All weights are multiplied by down = 2^-below, so that the sum of a row's weights stays below 1, and sums of values below the largest value
    // (results below 2^-126 / down lose bits).  up = 1 / down.
    float below, down, up;
    const int* gate;                                // not NULL: attn_rows has done the call where this is 0
    unsigned* counters;                             // [kMaxCtas] arrivals of parts, by the CTA an item begins in
    float* parts;                                   // two for each CTA
};

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    unsigned long long d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)));
    return *reinterpret_cast<float2*>(&d);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    unsigned long long d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d)
        : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)), "l"(*reinterpret_cast<unsigned long long*>(&c)));
    return *reinterpret_cast<float2*>(&d);
}

// a / b of numbers >= 0: 32 bits where they do (a division of 64 bits takes a tenth of a microsecond).
__device__ __forceinline__ long long quotient(long long a, long long b) {
    return ((a | b) >> 32) == 0 ? (long long)((unsigned)a / (unsigned)b) : a / b;
}

// ---- the list of work -----------------------------------------------------------------------------------------------

// A part of one (sequence, key head, block of rows): tiles kb .. kb + count - 1 of its kbs tiles of states.
struct Item {
    int seq, head, rb, kb, count, kbs;
    int q0, rows;                                   // first token of the sequence; rows of the block
    long long k0;                                   // first state
    int klen;
    int first;                                      // its first tile's place in the list
};

template <int BN, int JOIN>                         // states of a tile; tiles that a join costs as much as
struct Work {
    const CrossArgs& a;
    int at = 0, end = 0;                            // this CTA's part of the list
    unsigned per = 1;                               // and of all others
    bool whole = false;                             // the list is of blocks, not of tiles
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
    __device__ int blocks_of(int qlen) const { return (int)(((long long)qlen * a.group + a.block - 1) >> a.shift); }
    __device__ int tiles_of(int klen) const { return (int)(((long long)klen + BN - 1) / BN); }
    __device__ int steps() const { return whole ? min(kbs, 1) : kbs; }          // of the list, of a block
    __device__ void enter(int i) {
        lengths(i, q0, qlen, k0, klen);
        settle(i);
    }
    __device__ void settle(int i) {
        seq = i;
        rbs = blocks_of(qlen);
        kbs = tiles_of(klen);
    }
    // This CTA's part; all NT threads of the CTA call it.  Up to 32 sequences each warp works it out for itself.
    template <int NT>
    __device__ void begin() {
        constexpr int NW = NT / 32;
        __shared__ unsigned sums[NW], blocks[NW], found_in;
        __shared__ float sizes[NW];
        __shared__ int most[NW], found;
        const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = a.p.n;
        // tiles and blocks of 32 or NT sequences at a time, of all before them, and of all
        unsigned tiles = 0, tiles_before = 0, total = 0, blocks_mine = 0, blocks_before = 0, all_blocks = 0;
        float size = 0.f;                           // of the list, which must have less than 2^31 tiles
        int longest = 0;
        auto scan = [&](int i) {
            q0 = qlen = k0 = klen = 0;
            if (i < n) lengths(i, q0, qlen, k0, klen);
            const int t = tiles_of(klen);
            const float b = (float)a.p.heads * blocks_of(qlen);
            blocks_mine = t && b < 2147483648.f ? a.p.heads * (unsigned)blocks_of(qlen) : 0u;
            tiles = blocks_mine * t;
            float x = t ? b * t : 0.f;
            unsigned s = tiles, c = blocks_mine;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const unsigned y = __shfl_up_sync(~0u, s, d), z = __shfl_up_sync(~0u, c, d);
                x += __shfl_xor_sync(~0u, x, d);
                if (lane >= d) { s += y; c += z; }
            }
            const int m = __reduce_max_sync(~0u, t && qlen ? t : 0);
            tiles_before = total + s - tiles;
            blocks_before = all_blocks + c - blocks_mine;
            if (n <= 32) {
                total = __shfl_sync(~0u, s, 31);
                all_blocks = __shfl_sync(~0u, c, 31);
                longest = m;
                size = x;
                return;
            }
            if (lane == 31) { sums[warp] = s; blocks[warp] = c; most[warp] = m; sizes[warp] = x; }
            __syncthreads();
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                if (w < warp) { tiles_before += sums[w]; blocks_before += blocks[w]; }
                total += sums[w];
                all_blocks += blocks[w];
                longest = max(longest, most[w]);
                size += sizes[w];
            }
        };
        scan(n <= 32 ? lane : tid);
        for (int i0 = NT; i0 < n; i0 += NT) {
            __syncthreads();                        // the sums have been read
            scan(i0 + tid);
        }
        if (size >= 2147000000.f) {
            if (tid == 0) *a.p.status = LUVC_ERR_SHAPE;
            return;
        }
        per = (total + gridDim.x - 1) / gridDim.x;
        const unsigned rounds = (all_blocks + gridDim.x - 1) / gridDim.x;
        whole = (float)rounds * longest <= (float)(per + JOIN);
        if (whole) per = rounds;
        unsigned all = whole ? all_blocks : total;
        at = (int)min((unsigned long long)all, (unsigned long long)per * blockIdx.x);
        end = (int)min(all, at + per);
        if (at >= end) return;                      // (the same in all threads)
        unsigned in = 0;
        int which = -1;
        auto look = [&](int i) {
            const unsigned before = whole ? blocks_before : tiles_before, x = whole ? blocks_mine : tiles;
            if (before <= (unsigned)at && (unsigned)at < before + x) {
                which = i;
                in = at - before;
            }
        };
        if (n <= 32) {
            look(lane);
            const int from = __ffs(__ballot_sync(~0u, which >= 0)) - 1;
            which = from;
            in = __shfl_sync(~0u, in, from);
            q0 = __shfl_sync(~0u, q0, from); qlen = __shfl_sync(~0u, qlen, from);
            k0 = __shfl_sync(~0u, k0, from); klen = __shfl_sync(~0u, klen, from);
            settle(from);
        } else {
            if (n <= NT) {
                look(tid);
            } else {
                total = all_blocks = 0;
                for (int i0 = 0; i0 < n && (whole ? all_blocks : total) <= (unsigned)at; i0 += NT) {
                    __syncthreads();
                    scan(i0 + tid);
                    look(i0 + tid);
                }
            }
            if (which >= 0) { found = which; found_in = in; }
            __syncthreads();
            in = found_in;
            enter(found);
        }
        const unsigned per_head = (unsigned)rbs * steps();
        head = in / per_head;
        rb = (in - head * per_head) / steps();
        kb = whole ? 0 : (int)(in - head * per_head - (unsigned)rb * kbs);
    }
    __device__ bool more() const { return at < end; }
    // The next item; the list goes on behind it.
    __device__ Item next() {
        Item it;
        it.seq = seq; it.head = head; it.rb = rb; it.kb = kb; it.kbs = kbs;
        it.count = whole ? kbs : min(kbs - kb, end - at);
        it.q0 = q0;
        it.rows = (int)min((long long)qlen * a.group - (long long)rb * a.block, (long long)a.block);
        it.k0 = k0; it.klen = klen;
        it.first = at - kb;
        at += whole ? 1 : it.count;
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
};

// Token and query head of row r of an item.
__device__ __forceinline__ long long token_of(const CrossArgs& a, const Item& it, int r, int& h) {
    const long long row = (long long)it.rb * a.block + r;
    const long long t = quotient(row, a.group);
    h = it.head * a.group + (int)(row - t * a.group);
    return it.q0 + t;
}

template <typename T> __device__ __forceinline__ void put4(T* p, float4 x);
template <> __device__ __forceinline__ void put4<float>(float* p, float4 x) { *reinterpret_cast<float4*>(p) = x; }
template <> __device__ __forceinline__ void put4<__nv_bfloat16>(__nv_bfloat16* p, float4 x) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(x.x, x.y), b = __floats2bfloat162_rn(x.z, x.w);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
__device__ __forceinline__ float lse_of(const CrossArgs& a, float m, float l) { return l == 0.f ? -INFINITY : fmaf(m == -INFINITY ? 0.f : m, a.nat, logf(l * a.up)); }

// Sequences without states: rows of zeros.  By a warp, or by a CTA of NT threads; where there are fewer sequences than CTAs, several share one (2048 tokens
// of 28 heads of 128 beside a question of 60 to 1296 states: 27 us, a warp for each sequence 306).
template <typename T, int NT, typename W>
__device__ void empty_sequences(const CrossArgs& a, const W& w) {
    const int share = max((int)gridDim.x / a.p.n, 1), mine = blockIdx.x % share * NT + threadIdx.x % NT;
    for (int i = blockIdx.x / share; i < a.p.n; i += gridDim.x) {       // (once only where several share one)
        int q0, qlen, k0, klen;
        w.lengths(i, q0, qlen, k0, klen);
        if (klen > 0) continue;
        const long long row = (long long)a.p.q_heads * a.p.D;
        T* const out = static_cast<T*>(a.p.out) + q0 * row;
        for (long long e = mine; e < qlen * row / 4; e += share * NT) put4(out + 4 * e, make_float4(0.f, 0.f, 0.f, 0.f));
        if (a.p.lse)
            for (long long e = mine; e < (long long)qlen * a.p.q_heads; e += share * NT) a.p.lse[(long long)q0 * a.p.q_heads + e] = -INFINITY;
    }
}

// A partial result in the workspace: four columns of a row at o[column / 4 * BM + row], (m, l) of each row.
template <int BM, int DP>
struct Part {
    static constexpr size_t BYTES = BM * (DP + 2) * sizeof(float);
    float4* o;
    float2* ml;
    __device__ Part(const CrossArgs& a, int cta, int slot) {
        o = reinterpret_cast<float4*>(a.parts + ((size_t)cta * 2 + slot) * (BM * (DP + 2)));
        ml = reinterpret_cast<float2*>(o + BM * (DP / 4));
    }
};

// Arrival at an item's counter, which is zero before the first and after the last; true for the last.  The summands are 1, and 1 - n for
// the first CTA: their sum is zero whatever comes in between, so calls that overlap on a workspace leave zero behind all the same.
__device__ __forceinline__ bool arrive(unsigned* counter, int i, int n) {
    const unsigned x = i ? 1u : 1u - (unsigned)n;
    return atomicAdd(counter, x) + x == 0u;
}

// Adds the parts of an item, which CTAs c0 .. c1 have written, in order, and writes the result.  NT threads; each has E groups of four columns
// at a time, and B parts of all of them on their way.
template <typename T, int BM, int DP, int NT, int E, int B>
__device__ __forceinline__ void join_groups(const CrossArgs& a, const Item& it, int c0, int c1, int tid) {
    const int all = it.rows * (a.p.D / 4);
    for (int e0 = tid; e0 < all; e0 += E * NT) {
        int r[E], c[E];
        float m[E], l[E];
        float4 o[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {                           // past the last group: that one again, not written
            const int x = min(e0 + e * NT, all - 1);
            c[e] = x / it.rows;
            r[e] = x - c[e] * it.rows;
            m[e] = -INFINITY;
            l[e] = 0.f;
            o[e] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        for (int k0 = c0; k0 <= c1; k0 += B) {
            float4 x[E][B];
            float2 ml[E][B];
#pragma unroll
            for (int k = 0; k < B; ++k)
                if (k0 + k <= c1) {
                    const Part<BM, DP> q(a, k0 + k, k0 + k == c0);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        ml[e][k] = __ldcg(q.ml + r[e]);
                        x[e][k] = __ldcg(q.o + c[e] * BM + r[e]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        ml[e][k] = make_float2(-INFINITY, 0.f);
                        x[e][k] = make_float4(0.f, 0.f, 0.f, 0.f);
                    }
                }
#pragma unroll
            for (int e = 0; e < E; ++e) {
                float top = m[e];
#pragma unroll
                for (int k = 0; k < B; ++k) top = fmaxf(top, ml[e][k].x);
                // o is the mean so far: values near the end of the range stay inside it
                const float base = top == -INFINITY ? 0.f : top, had = l[e] * exp2_fast((m[e] - base) * a.unit);
                m[e] = top;
                l[e] = had;
                float w[B];
#pragma unroll
                for (int k = 0; k < B; ++k) {
                    w[k] = exp2_fast((ml[e][k].x - base) * a.unit);
                    l[e] = fmaf(w[k], ml[e][k].y, l[e]);
                }
                const float inv = l[e] == 0.f ? 0.f : 1.f / l[e], f = had * inv;
                o[e].x *= f; o[e].y *= f; o[e].z *= f; o[e].w *= f;
#pragma unroll
                for (int k = 0; k < B; ++k) {
                    const float by = w[k] * inv;
                    o[e].x = fmaf(by, x[e][k].x, o[e].x); o[e].y = fmaf(by, x[e][k].y, o[e].y);
                    o[e].z = fmaf(by, x[e][k].z, o[e].z); o[e].w = fmaf(by, x[e][k].w, o[e].w);
                }
            }
        }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            if (e0 + e * NT >= all) continue;
            int h;
            const long long row = token_of(a, it, r[e], h) * a.p.q_heads + h;
            put4(static_cast<T*>(a.p.out) + row * a.p.D + 4 * c[e], l[e] == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : o[e]);
            if (c[e] == 0 && a.p.lse) a.p.lse[row] = lse_of(a, m[e], l[e]);
        }
    }
}

template <typename T, int BM, int DP, int NT>
__device__ void join_parts(const CrossArgs& a, const Item& it, int c0, int c1, int tid) {
    if (it.rows * (a.p.D / 4) <= NT) join_groups<T, BM, DP, NT, 1, 16>(a, it, c0, c1, tid);
    else join_groups<T, BM, DP, NT, 4, 4>(a, it, c0, c1, tid);
}

// ---- f32 on the CUDA cores --------------------------------------------------------------------------------------------

// Tiles of BM rows by 64 states, 256 threads: a thread has RT = BM / 16 rows (ty) and every 16th state or group of four columns (tx): eight rows
// take half the reads of shared memory per product of four, but one CTA has an SM then (69 GFLOP, 16 / 4 heads of 128: BM = 128 1547 us, two CTAs of
// 64 2164).  Products are packed pairs; K and V have one buffer each, and the next tile of K is on its way during the products with V, and the other way round.
template <int BM, int DP>
struct Cores {
    static constexpr int BN = 64, NT = 256, RT = BM / 16, LD = DP + 4, LP = BN + 4;
    static constexpr size_t SMEM = (size_t)(BM * LD + BN * LD + BN * DP + BM * LP) * sizeof(float);
    static constexpr int CTAS = BM > 64 || DP > 128 ? 1 : 2;    // of an SM
};

template <int BM, int DP>
__global__ void __launch_bounds__(256, Cores<BM, DP>::CTAS) attn_cross_f32(const __grid_constant__ CrossArgs a) {
    using C = Cores<BM, DP>;
    constexpr int BN = C::BN, NT = C::NT, LD = C::LD, LP = C::LP, CG = DP / 64;
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
    if (a.gate && *a.gate == 0) return;
    Work<BN, 2> work(a);            // (parts, nearly always: eight sequences of 8 tokens, 32 / 8 heads of 128, 1296 states 100 us, whole blocks 152; four of 40,
                                    // 16 / 16 of 64, 2000 states 82 and 271; six of 33 to 257 tokens to 64 to 576 states 103 and 153)
    work.template begin<NT>();
    empty_sequences<float, NT>(a, work);
    for (int e = tid; e < (BM + BN) * (LD / 4); e += NT) reinterpret_cast<float4*>(qs)[e] = make_float4(0.f, 0.f, 0.f, 0.f);   // columns past D
    for (int e = tid; e < BN * (DP / 4); e += NT) reinterpret_cast<float4*>(vs)[e] = make_float4(0.f, 0.f, 0.f, 0.f);
    // An item, with `rt` rows for each thread: no more than it needs, so that the few rows of a ragged end take little.
    auto process = [&](const Item& it, auto rt) {
        constexpr int RT = decltype(rt)::value;
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
            const long long t = token_of(a, it, r, h);
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
                    const float w = exp2_fast((s[x] - base) * a.unit) * a.down;
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
            const long long at = token_of(a, it, row, h) * p.q_heads + h;
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
            const int c0 = it.first / work.per, c1 = (it.first + it.kbs - 1) / work.per;
            __threadfence();
            __syncthreads();
            if (tid == 0) last = arrive(a.counters + c0, blockIdx.x - c0, c1 - c0 + 1);
            __syncthreads();
            if (last) {
                __threadfence();
                join_parts<float, BM, DP, NT>(a, it, c0, c1, tid);
            }
        }
    };
    while (work.more()) {
        // as many rows of a thread as the block needs (six ragged texts of 33 to 257 tokens: always eight 101.8 us, by the block's rows 97.0)
        const Item it = work.next();
        if constexpr (C::RT >= 8) {
            if (it.rows > 64) {
                process(it, std::integral_constant<int, 8>{});
                continue;
            }
        }
        if constexpr (C::RT >= 4) {
            if (it.rows > 32) {
                process(it, std::integral_constant<int, 4>{});
                continue;
            }
            if (it.rows > 16) {
                process(it, std::integral_constant<int, 2>{});
                continue;
            }
        }
        process(it, std::integral_constant<int, 1>{});
    }
}

// ---- bf16 on the tensor cores -----------------------------------------------------------------------------------------

// DP: columns of a row in shared memory (D, rounded up to 64, 128 or 256).  A CTA has TILES tiles of 128 rows, each with four warps that take
// its weights (a thread has a row) and one that issues its products; another one brings K and V by TMA.
//
// S = Q K^T lands in tensor memory, the threads read it, and leave the weights, in bf16, in its place, from where they are the first operand of
// O += P V.  While one tile's weights are worked out, the other tile's products run.  Where there are no more than 128 rows both tiles have
// the same rows and every other tile of states, and their results are added at the end.
//
// What bounds it: the turn from scores to scores of one tile, with 128 columns 3700 cycles: 1700 to take its weights (1024 of them the special
// function unit's, which does a quarter of a warp's powers of two in a cycle; reading and writing tensor memory, sums and rounding do not
// overlap with it in one warp), 1400 for its products (16 instructions at 64 cycles, issued at 80), the rest are barriers.  The tiles' turns
// are kept apart, so the tensor pipe works for 2800 of them.
//
// Roundings.  Scores and sums are fp32; a weight is rounded to bf16 for its product with V, 2^-8 of its size at most: the
// errors of the states' weights are independent, and their mean is below the rounding of the output.  (The pairs of 16-bit floats that the attention
// of one token uses would double the second product, which bounds this one.)
template <int DP_>
struct Tc {
    static constexpr int DP = DP_, TILES = DP <= 128 ? 2 : 1, BN = DP <= 128 ? 128 : 64, ROWS = 128 * TILES;
    static constexpr int Q_BYTES = 128 * DP * 2, STAGE = BN * DP * 2, STAGES = DP == 64 ? 8 : 5;
    // Tiles that a join costs as much as.  28 / 4 heads of 128, four sequences of 33 tokens to 700, 1296, 2600 and 4000 states (whole blocks have 4, 8, 16 and
    // 25 tiles more in a CTA): 17.8, 23.5, 33.5 and 44.5 us, in parts 24.3, 39.9, 42.3 and 45.4; 16 / 16 of 64, 128 tokens to 1024 and 2048 (7
    // and 14 more): 16.4 and 24.1, in parts 18.9 and 20.0; 12 / 1 of 256, four of 100 to 1000, 2000 and 3000 (11, 23, 34 more): 35.7, 60.1 and 81.6, in
    // parts 50.3, 63.5 and 68.6.
    static constexpr int JOIN = DP == 64 ? 10 : 18;
    static constexpr int THREADS = 384, S_COLS = 128, O_COL = 256, O_COLS = DP <= 128 ? 128 : 256;
    static constexpr size_t SMEM = 1024 + TILES * Q_BYTES + STAGES * STAGE;
    // registers of the threads that have weights, and of the others: together what the launch has, 384 times 168
    static constexpr int MANY = 208, FEW = 80;
    static_assert(256 * MANY + 128 * FEW <= THREADS * 168, "more registers than the launch has");
    static_assert(TILES == 1 || 2 * Q_BYTES >= 128 * DP * 4, "a tile's result fits the queries' place");
};

// Largest sum of a tile's weights, but for CrossArgs::down, before their reference follows the maximum.
constexpr int kMostBits = 16;

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
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t (&v)[32]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
                 "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
                 ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
                   "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]),
                   "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]) : "memory");
}
// The same, and whether any of the threads says yes.
__device__ __forceinline__ bool named_barrier_or(int id, int threads, bool yes) {
    int any;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %3, 0;\n\tbar.red.or.pred q, %1, %2, p;\n\tselp.b32 %0, 1, 0, q;\n\t}"
                 : "=r"(any) : "r"(id), "r"(threads), "r"((int)yes) : "memory");
    return any != 0;
}
// Registers of this warpgroup's threads from here on (all four warps call it).
template <int N> __device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void give_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
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

template <int DP, bool BIAS>
__global__ void __launch_bounds__(Tc<DP>::THREADS, 1)
attn_cross_tc(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const __grid_constant__ CrossArgs a) {
    using T = Tc<DP>;
    constexpr int TILES = T::TILES, BN = T::BN, ROWS = T::ROWS, STAGES = T::STAGES, CH = BN / 32;
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t bars[8 + 2 * STAGES + 4];
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
    auto turn = [&](int t) { return drained + 16 + 8 * t; };
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
            mbar_init(kv_free(s), 2);                           // for both tiles of rows
        }
        mbar_init(drained, 1);
        mbar_init(drained + 8, 1);
        mbar_init(turn(0), 1);
        mbar_init(turn(1), 1);
        mbar_fence_init();
        dead_flag = 0;
        asm volatile("prefetch.tensormap [%0];" ::"l"(&kmap) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&vmap) : "memory");
    }
    pdl_trigger();
    pdl_wait();
    if (a.gate && *a.gate == 0) {
        __syncthreads();
        if (warp == 9) tmem_dealloc(tmem_at, 512);
        return;
    }
    Work<BN, T::JOIN> work(a);
    tc_fence_before();
    work.template begin<T::THREADS>();
    __syncthreads();                                            // barriers and tensor memory are there
    tc_fence_after();
    const uint32_t tmem = tmem_at;

    if (warp >= 8) {
        give_registers<T::FEW>();
        if (warp == 11) empty_sequences<__nv_bfloat16, 32>(a, work);
        // ---- K and V, tile after tile, through a ring of stages ----
        if (warp == 8 && lane == 0) {
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
        // ---- products, a warp for each tile of rows ----
        // (One warp for both takes 2450 cycles for the products of a tile of states with a tile of rows, half of them between the
        // instructions; the products themselves take 1250.)
        const int t = warp - 9;
        if (t >= 0 && t < TILES) {
            const uint32_t idesc_s = make_idesc_bf16(128, BN, false, false), idesc_o = make_idesc_bf16(128, 16 * ksteps, false, true);
            const uint64_t q0 = make_desc_layout(qs, 16, 1024, 2), k0 = make_desc_layout(ring, 16, 1024, 2), v0 = make_desc_layout(ring, BN * 128, 1024, 2);
            // What the loops run on is made the same in all lanes where the compiler can tell, so that descriptors stay in uniform registers: their
            // lower halves, which hold the address, are handed out before each group of products.
            auto same = [](int x) { return __shfl_sync(~0u, x, 0); };
            auto desc = [](uint64_t of, uint32_t lower) { return (of >> 32 << 32) | lower; };
            const uint32_t s_of = (uint32_t)same((int)tmem) + t * T::S_COLS, o_of = (uint32_t)same((int)tmem) + T::O_COL + t * T::O_COLS;
            bool ok = true;
            auto wait = [&](uint32_t bar, int parity) {
                if (__all_sync(~0u, mbar_try_wait(bar, parity)) || !ok) return;
                bool there = true;
                if (lane == 0) there = wait_phase(bar, parity, dead, p.status);
                ok = same(there);
            };
            // The next stage of the ring that holds K, or V: every other one.  Each warp waits for all of them in turn and sets all free, also
            // those that only the other one uses, so that neither misses a phase of a barrier.
            struct Cursor {
                int stage, phase;
                __device__ void advance() {
                    stage += 2;
                    if (stage >= STAGES) { stage -= STAGES; phase ^= 1; }
                }
            };
            Cursor kc = {0, 0}, vc = {1, 0};
            auto pass = [&](Cursor& c) {
                wait(kv_full(c.stage), c.phase);
                if (lane == 0) mbar_arrive(kv_free(c.stage));
                c.advance();
            };
            int q_phase = 0, q1_phase = 0, p_phase = 0, turn_phase = 0;
            // The warps take turns, from one product with V and the scores after it to the next: products of both at once would be done
            // together, late, and both tiles' weights then be worked out at once.
            auto take_turn = [&] {
                wait(turn(t), turn_phase);
                turn_phase ^= 1;
            };
            bool first_turn = t == 0;                               // of all
            while (ok && same(work.more())) {
                const Item it = work.next();
                const int count = same(it.count);
                const bool two = TILES == 2 && same(it.rows > 128), both = TILES == 2 && !two;  // two tiles of rows; both take the same rows
                wait(q_full(0), q_phase);
                q_phase ^= 1;
                if (two) {
                    if (t == 1) wait(q_full(1), q1_phase);
                    q1_phase ^= 1;
                }
                const uint32_t q = (uint32_t)same((int)((uint32_t)q0 + ((uint32_t)(both ? 0 : t * T::Q_BYTES) >> 4)));
                // tiles of states: all of them, or every other one
                const int step = both ? 2 : 1, mine = both ? (count - t + 1) / 2 : count;
                const int turns = (both ? (count + 1) / 2 : count) + 1; // of each warp, also where the second one has nothing to do
                if (both && t == 1) { pass(kc); pass(vc); }
                for (int j = -1; j < turns - 1; ++j) {
                    const bool value = j >= 0 && j < mine, score = j < mine - 1;
                    if (score) {                             // (waited for ahead of the turn)
                        if (step == 2 && j >= 0) pass(kc);
                        if (j < 0) wait(kv_full(kc.stage), kc.phase);
                    }
                    if (value) {                                    // O of the tile of states whose weights are next
                        wait(kv_full(vc.stage), vc.phase);
                        wait(p_ready(t), p_phase);
                        p_phase ^= 1;
                    }
                    if (TILES == 2 && !first_turn) take_turn();
                    first_turn = false;
                    if (!ok) break;
                    tc_fence_after();
                    if (value) {
                        const uint32_t v = (uint32_t)same((int)((uint32_t)v0 + ((uint32_t)(vc.stage * T::STAGE) >> 4)));
                        if (elect_one()) {
#pragma unroll
                            for (int x = 0; x < BN / 16; ++x)
                                umma_bf16_ts(o_of, s_of + 8 * x, desc(v0, v + (2048 * x >> 4)), idesc_o, x || j ? 1u : 0u);
                            umma_commit(kv_free(vc.stage));
                            if (TILES == 1) mbar_arrive(kv_free(vc.stage));
                            if (j == mine - 1) umma_commit(o_full(t));
                        }
                        __syncwarp();
                        vc.advance();
                        if (step == 2 && j < mine - 1) pass(vc);
                    }
                    if (score) {                                    // S of the next
                        if (j >= 0) wait(kv_full(kc.stage), kc.phase);
                        if (!ok) break;
                        tc_fence_after();
                        const uint32_t k = (uint32_t)same((int)((uint32_t)k0 + ((uint32_t)(kc.stage * T::STAGE) >> 4)));
                        if (elect_one()) {
#pragma unroll
                            for (int x = 0; x < DP / 16; ++x)
                                if (x < ksteps)
                                    umma_bf16(s_of, desc(q0, q + ((x >> 2) * (128 * 128) + (x & 3) * 32 >> 4)), desc(k0, k + ((x >> 2) * (BN * 128) + (x & 3) * 32 >> 4)), idesc_s, x ? 1u : 0u);
                            umma_commit(s_full(t));
                        }
                        __syncwarp();
                        kc.advance();
                    }
                    if (TILES == 2 && lane == 0) mbar_arrive(turn(1 - t));
                }
                if (both && ((count - t) & 1) == 0 && count > t) { pass(kc); pass(vc); }        // the other one's last
            }
            if (!ok) {                                              // tensor memory is given back below: products in flight end first
                if (elect_one()) umma_commit(drained + 8 * t);
                __syncwarp();
                for (int probes = 0; probes < kLeastProbes && !mbar_try_wait(drained + 8 * t, 0); ++probes) {}
            }
        }
    } else {
        take_registers<T::MANY>();
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
                const long long tok = token_of(a, it, mine_live ? mine : 0, h);
                const unsigned long long src = reinterpret_cast<unsigned long long>(static_cast<const __nv_bfloat16*>(p.q) + tok * p.q_stride + (long long)h * D);
                const unsigned live = __ballot_sync(~0u, mine_live);
                const unsigned flip = a.sign < 0.f ? 0x80008000u : 0u;
                unsigned char* const dst = base + t * T::Q_BYTES + (warp & 3) * (32 * 128);
                // a warp brings its 32 rows together, 16 bytes of a lane next to those of the next one (where there are none, those of another
                // place are read and not used)
                const int pieces = 2 * ksteps;
                const unsigned part = 65536 / pieces + 1;       // piece * part / 65536: exact for 1024 pieces of rows of up to 32
                for (int x0 = 0; x0 < pieces; x0 += 16) {
                    uint4 x[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const unsigned u = (x0 + e) * 32 + lane, row = u * part >> 16, c = u - row * pieces;
                        x[e] = __ldg(reinterpret_cast<const uint4*>(__shfl_sync(~0u, src, row & 31)) + (8 * c < D ? c : 0));
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const unsigned u = (x0 + e) * 32 + lane, row = u * part >> 16, c = u - row * pieces;
                        x[e].x ^= flip; x[e].y ^= flip; x[e].z ^= flip; x[e].w ^= flip;
                        if (8 * c >= D || !((live >> (row & 31)) & 1u)) x[e] = make_uint4(0u, 0u, 0u, 0u);
                        if (row < 32) *reinterpret_cast<uint4*>(dst + (c >> 3) * (128 * 128) + row * 128 + (((c & 7) ^ (row & 7)) << 4)) = x[e];
                    }
                }
                fence_proxy_async();
                mbar_arrive(q_full(t));
            }
            float m = -INFINITY, l = 0.f;
            int blocks = 0;                                     // tiles of states this tile of rows has had
            const int step = both ? 2 : 1;
            for (int j = both ? t : 0; j < it.count && (t == 0 || TILES == 2); j += step, ++blocks) {
                const int kb = it.kb + j, keys = min(BN, it.klen - kb * BN);
                bool gone = r < BN && r >= keys, masked = keys < BN;
                if (BIAS) {
                    if (r < BN) {
                        const float b = gone ? -INFINITY : p.bias[it.k0 + (long long)kb * BN + r];
                        gone = b == -INFINITY;
                        sb[t][r] = b;
                    }
                    masked = named_barrier_or(2 + t, 128, gone);
                }
                wait_phase(s_full(t), s_used++ & 1, dead, p.status);
                tc_fence_after();
                if (r == 0) {                                   // K has been used
                    const uint32_t free = kv_free(2 * (n0 + j) % STAGES);
                    mbar_arrive(free);
                    if (TILES == 1) mbar_arrive(free);
                }
                // the scores; masked ones are -inf whatever the state's rows hold
                auto each_chunk = [&](auto with_masks, auto use) {
                    constexpr bool MASKS = decltype(with_masks)::value;
                    uint32_t s[CH][32];
#pragma unroll
                    for (int c = 0; c < CH; ++c) tmem_ld32(s_at + 32 * c, s[c]);
#pragma unroll
                    for (int c = 0; c < CH; ++c) {
                        tmem_ld_wait32(s[c]);
                        float2 y[16];
#pragma unroll
                        for (int x = 0; x < 16; ++x) y[x] = make_float2(__uint_as_float(s[c][2 * x]), __uint_as_float(s[c][2 * x + 1]));
                        if (BIAS) {
#pragma unroll
                            for (int x = 0; x < 16; x += 2) {
                                const float4 b = *reinterpret_cast<const float4*>(&sb[t][32 * c + 2 * x]);
                                y[x] = fma2(y[x], make_float2(a.c, a.c), make_float2(b.x, b.y));
                                y[x + 1] = fma2(y[x + 1], make_float2(a.c, a.c), make_float2(b.z, b.w));
                                if (MASKS) {
                                    if (b.x == -INFINITY) y[x].x = -INFINITY;
                                    if (b.y == -INFINITY) y[x].y = -INFINITY;
                                    if (b.z == -INFINITY) y[x + 1].x = -INFINITY;
                                    if (b.w == -INFINITY) y[x + 1].y = -INFINITY;
                                }
                            }
                        } else if (MASKS) {
#pragma unroll
                            for (int x = 0; x < 16; ++x) {
                                if (32 * c + 2 * x >= keys) y[x].x = -INFINITY;
                                if (32 * c + 2 * x + 1 >= keys) y[x].y = -INFINITY;
                            }
                        }
                        use(c, y);
                    }
                };
                const float c1 = BIAS ? 1.f : a.c, unit = BIAS ? kLog2e : 1.f;
                // The reference of the weights is the maximum of the first tile.  It follows later ones only where the sum of a tile's weights
                // passes 2^kMostBits: floats, bf16 among them, keep their relative precision up to there, so the maximum need not be known.
                uint32_t w[BN / 2];
                float sum;
                for (bool fresh = __any_sync(~0u, m == -INFINITY);; fresh = true) {
                    if (fresh) {
                        float top = -INFINITY;
                        each_chunk(std::true_type{}, [&](int, const float2 (&y)[16]) {
#pragma unroll
                            for (int x = 0; x < 16; ++x) top = fmaxf(top, fmaxf(y[x].x, y[x].y));
                        });
                        const float now = fmaxf(m, top * c1), from = now == -INFINITY ? 0.f : now, f = exp2_fast((m - from) * unit);
                        m = now;
                        l *= f;
                        if (blocks > 0) {                       // the products of the tiles before are done: the scores came after them
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
                    const float from = BIAS ? (m == -INFINITY ? 0.f : m) : (m == -INFINITY ? 0.f : m) + a.below;
                    float2 sums[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                    auto weigh = [&](auto with_masks) { each_chunk(with_masks, [&](int c, const float2 (&y)[16]) {
#pragma unroll
                        for (int x = 0; x < 16; ++x) {
                            float2 z;
                            if (BIAS) z = fma2(add2(y[x], make_float2(-from, -from)), make_float2(kLog2e, kLog2e), make_float2(-a.below, -a.below));
                            else z = fma2(y[x], make_float2(c1, c1), make_float2(-from, -from));
                            z = make_float2(exp2_fast(z.x), exp2_fast(z.y));
                            sums[x & 1] = add2(sums[x & 1], z);
                            const __nv_bfloat162 two16 = __floats2bfloat162_rn(z.x, z.y);
                            w[16 * c + x] = *reinterpret_cast<const uint32_t*>(&two16);
                        }
                    }); };
                    if (masked) weigh(std::true_type{});
                    else weigh(std::false_type{});
                    const float2 all = add2(sums[0], sums[1]);
                    sum = all.x + all.y;
                    if (fresh || !__any_sync(~0u, sum > a.down * (float)(1 << kMostBits))) break;
                }
                l += sum;
                if (BIAS) named_barrier(2 + t, 128);            // the biases have been read
#pragma unroll
                for (int c = 0; c < BN / 64; ++c) tmem_st32(s_at + 32 * c, *reinterpret_cast<uint32_t(*)[32]>(w + 32 * c));
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
                const long long row = token_of(a, it, mine_live ? mine : 0, h) * p.q_heads + h;
                const unsigned long long to = mine_live ? reinterpret_cast<unsigned long long>(static_cast<__nv_bfloat16*>(p.out) + row * D) : 0ull;
                // 32 columns of the warp's rows go through shared memory, four pieces of 16 bytes of a row each 2 KB apart or less: the place
                // of the warp's own queries, or of what has just been added
                unsigned long long there[4];                    // where a lane's pieces go: of rows lane / 4 + 8 e, the piece lane % 4
#pragma unroll
                for (int e = 0; e < 4; ++e) there[e] = __shfl_sync(~0u, to, 8 * e + (lane >> 2));
                const float inv = l == 0.f ? 0.f : 1.f / l;
                for (int c = 0; c < D; c += 32) {
                    uint32_t o[32];
                    tmem_ld32(o_at + c, o);
                    tmem_ld_wait32(o);
                    unsigned char* const stage = add ? base + ((size_t)(c / 4) * 128 + (warp & 3) * 32) * 16 : base + t * T::Q_BYTES + (warp & 3) * (32 * 128);
                    const int apart = add ? 2048 : 512;
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
                        if (whole) {
                            uint32_t w[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const __nv_bfloat162 two16 = __floats2bfloat162_rn(y[2 * e] * inv, y[2 * e + 1] * inv);
                                w[e] = *reinterpret_cast<const uint32_t*>(&two16);
                            }
                            *reinterpret_cast<uint4*>(stage + x / 8 * apart + lane * 16) = make_uint4(w[0], w[1], w[2], w[3]);
                        } else if (mine_live) {
                            part.o[(c + x) / 4 * ROWS + mine] = make_float4(y[0], y[1], y[2], y[3]);
                            if (c + x + 4 < D) part.o[((c + x) / 4 + 1) * ROWS + mine] = make_float4(y[4], y[5], y[6], y[7]);
                        }
                    }
                    if (whole) {
                        __syncwarp();
                        uint4 out[4];                           // 64 bytes of eight rows at a time
#pragma unroll
                        for (int e = 0; e < 4; ++e) out[e] = *reinterpret_cast<const uint4*>(stage + (lane & 3) * apart + (8 * e + (lane >> 2)) * 16);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (there[e] && c + 8 * (lane & 3) < D) *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(there[e]) + c + 8 * (lane & 3)) = out[e];
                        __syncwarp();
                    }
                }
                if (mine_live) {
                    if (!whole) part.ml[mine] = make_float2(m, l);
                    else if (p.lse) p.lse[row] = lse_of(a, m, l);
                }
            };
            const bool merged = both && it.count > 1;
            float f0 = 1.f, f1 = 0.f;
            if (merged) {
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
                    f0 = exp2_fast((m - from) * a.unit);
                    f1 = exp2_fast((ml.x - from) * a.unit);
                    m = now;
                    l = l * f0 + ml.y * f1;
                }
            }
            if (blocks > 0 && (t == 0 || !merged)) emit(merged, f0, f1);
            if (merged) named_barrier(1, 256);
            tc_fence_before();                                  // O has been read before the next item's weights are announced
            if (!whole) {
                const int c0 = it.first / work.per, c1 = (it.first + it.kbs - 1) / work.per;
                __threadfence();
                named_barrier(1, 256);
                if (tid == 0) last = arrive(a.counters + c0, blockIdx.x - c0, c1 - c0 + 1);
                named_barrier(1, 256);
                if (last) {
                    __threadfence();
                    join_parts<__nv_bfloat16, ROWS, DP, 256>(a, it, c0, c1, tid);
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

// CTAs that there are counters and room for parts of such blocks for.
template <int BM, int DP>
int max_ctas(int ctas) { return std::min(ctas, std::min(kMaxCtas, (int)(kPartsBytes / (2 * Part<BM, DP>::BYTES)))); }

template <int BM, int DP>
int launch_f32(CrossArgs& a) {
    a.block = BM;
    a.shift = BM == 16 ? 4 : BM == 64 ? 6 : 7;
    static std::atomic<unsigned long long> set{0};
    const int ctas = max_ctas<BM, DP>(Cores<BM, DP>::CTAS * sm_count());
    if (!ctas || !allow_smem(attn_cross_f32<BM, DP>, Cores<BM, DP>::SMEM, set)) return LUVC_ERR_CUDA;
    return launch_overlapped(attn_cross_f32<BM, DP>, ctas, Cores<BM, DP>::NT, Cores<BM, DP>::SMEM, a.p.stream, a);
}

template <int BM>
int launch_f32_wide(CrossArgs& a) {
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
int launch_tc(CrossArgs& a) {
    using T = Tc<DP>;
    static std::atomic<unsigned long long> set{0};
    const int sms = max_ctas<T::ROWS, DP>(sm_count());
    // blocks of two tiles of rows where there are enough for all SMs (of one, and both tiles on the same rows, K and V are brought twice as often)
    a.block = T::TILES == 2 && (long long)a.p.q_tokens * a.p.q_heads <= 256ll * 2 * sms ? 128 : T::ROWS;
    a.shift = a.block == 128 ? 7 : 8;
    CUtensorMap kmap, vmap;
    if (!sms || !states_map<T::BN>(&kmap, a.p, a.p.k, a.p.k_stride) || !states_map<T::BN>(&vmap, a.p, a.p.v, a.p.v_stride) ||
        !allow_smem(attn_cross_tc<DP, BIAS>, T::SMEM, set))
        return LUVC_ERR_CUDA;
    return launch_overlapped(attn_cross_tc<DP, BIAS>, sms, T::THREADS, T::SMEM, a.p.stream, kmap, vmap, a);
}

template <int DP>
int launch_tc_bias(CrossArgs& a) {
    return a.p.bias ? launch_tc<DP, true>(a) : launch_tc<DP, false>(a);
}

}  // namespace

// This file's counters and parts, attn_rows' workspace, what it says to the kernel behind it.
size_t attn_cross_workspace_bytes() { return align_up(kCounterBytes + kPartsBytes) + align_up(attn_workspace_bytes()) + 256; }

int attn_cross(const CrossProblem& p) {
    // Few tokens go each on its own, in the form that attends from one token to a cache (tiles of 16 rows where this file's have 128), which reads
    // a sequence's states once for each of its tokens.  Where no sequence has two (a decode step) that is nothing lost: 16 tokens to 1296
    // states each, 28 / 4 heads of 128, 14.6 us, in blocks of 128 rows 24.8; f32, 8 tokens to 576 states, 16 / 16 heads of 64, 8.8 and 34.
    // Beyond that it takes a microsecond for 10 MB read, and blocks take two and one for 150 states more than it does for little (8 sequences of
    // 2, 4, 8 tokens, 1296 states: 15.9, 19.6, 28.0 us, blocks 25; 32 of 4, 300 states: 18.8 and 17.8; one of 4, 16384: 24 and 31); f32 blocks
    // about twice that (8 of 2 and 4: 40 and 68 us, blocks 67 and 72; 32 / 8 heads of 128).
    const double states = (double)p.k_tokens / p.n, state_mb = p.heads * p.D * (p.dtype == LUVC_F32 ? 8e-6 : 4e-6), mb = p.q_tokens * states * state_mb;
    const bool alone = p.q_tokens <= p.n || 0.1 * mb <= (p.dtype == LUVC_F32 ? 2. : 1.) * (2. + std::min(states, 2000.) / 150.);
    CrossArgs a;
    a.gate = nullptr;
    if (alone && p.q_tokens <= kAttnRowsMost && p.k_tokens > 0) {
        AttnProblem r = {};
        r.c.k = const_cast<void*>(p.k); r.c.v = const_cast<void*>(p.v); r.c.heads = p.heads; r.c.D = p.D; r.c.dtype = p.dtype;
        r.c.layers = r.c.pages = r.c.max_pages = r.c.slots = 1; r.c.page_size = kKvBlock;
        r.q = p.q; r.q_stride = p.q_stride; r.bias = p.bias; r.bias_width = p.bias ? p.k_tokens : 0; r.out = p.out; r.lse = p.lse;
        r.n = p.q_tokens; r.q_heads = p.q_heads; r.scale = p.scale; r.status = p.status; r.stream = p.stream;
        r.workspace = static_cast<unsigned char*>(p.workspace) + align_up(kCounterBytes + kPartsBytes);
        r.q_starts = p.q_starts; r.k_starts = p.k_starts; r.n_seqs = p.n; r.k_tokens = p.k_tokens; r.k_stride = p.k_stride; r.v_stride = p.v_stride;
        // That is for lengths near their means, which are all that is known here.  If all tokens can be of one sequence that has all states, and that is
        // much, the lengths decide: attn_rows leaves the call to the blocks where it would read more than three times as much as it was
        // chosen for, and 100 MB; they return at once where it has done it.  (1024 tokens of one of 1024 sequences to 16384 states, 8 / 8 heads of 128:
        // 105 us, each on its own 5746; 60 of one of 64 to 58000, 28 / 4: 124 and 712; the second launch costs 32 sequences of one token
        // and 1296 states 0.9 us of 19.3, 64 of 1000 2.5 of 33.3.)
        const double most = 3. * mb + 100., worst = p.q_starts ? p.q_tokens * (double)p.k_tokens * state_mb : 0.;
        if (worst > 500. && worst > most) {
            r.left = reinterpret_cast<int*>(static_cast<unsigned char*>(p.workspace) + attn_cross_workspace_bytes() - 256);
            r.most_states = (long long)(most / state_mb);
            a.gate = r.left;
        }
        const int status = attn_rows(r);
        if (status != LUVC_OK || !a.gate) return status;
    }
    a.p = p;
    a.group = p.q_heads / p.heads;
    a.c = fabsf(p.scale) * (p.bias ? 1.f : kLog2e);
    a.unit = p.bias ? kLog2e : 1.f;
    a.nat = p.bias ? 1.f : kLn2;
    a.sign = p.scale < 0.f ? -1.f : 1.f;
    // f32: a weight is 1 at most; bf16: those of a tile of 64 states or more sum to 2^kMostBits at most
    int bits = 0;                                               // 2^bits: more than there are states, or tiles of them
    std::frexp((float)(p.dtype == LUVC_F32 ? p.k_tokens : p.k_tokens / 64 + 1), &bits);
    if (p.dtype == LUVC_BF16) bits += kMostBits;
    a.below = (float)bits;
    a.down = std::ldexp(1.f, -bits);
    a.up = std::ldexp(1.f, bits);
    a.counters = static_cast<unsigned*>(p.workspace);
    a.parts = reinterpret_cast<float*>(static_cast<unsigned char*>(p.workspace) + kCounterBytes);
    if (p.dtype == LUVC_BF16) return p.D <= 64 ? launch_tc_bias<64>(a) : p.D <= 128 ? launch_tc_bias<128>(a) : launch_tc_bias<256>(a);
    // few rows of a key head: small blocks
    const bool few = (long long)p.q_tokens * a.group <= 16ll * p.n;
    const bool many = p.D <= 128 && (long long)p.q_tokens * a.group >= 96ll * p.n;
    if (many) return p.D <= 64 ? launch_f32<128, 64>(a) : launch_f32<128, 128>(a);
    return few ? launch_f32_wide<16>(a) : launch_f32_wide<64>(a);
}

}  // namespace luvc
