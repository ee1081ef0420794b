// Attention of one new token per sequence over its paged key-value cache.
//
//   out[i, h] = sum_t p_t V[t] / sum_t p_t,   p_t = exp(s_t - max s),   s_t = scale <q[i, h], K[t]> + bias[i, t]
//
// in one pass: a running maximum m, the sum l of the weights so far and their weighted sum O of value rows; when m grows,
// l and O are scaled by exp(m_old - m_new).  Partial results of parts of a sequence join by the same rule.
//
// Bound.  Every cached row is read once for up to 16 query heads that share it (four, where an f32 row is longer than 512 bytes; each
// further group of so many reads it again): 2 G flops per cached element with G query heads per key head, so HBM bounds long sequences up to the largest G in use, and latency short ones; what matters is to keep enough
// bytes in flight on every SM, whatever the lengths.  Measured: 334 MB (eight sequences of 4173 to 16451 tokens, 8 key heads of 128,
// bf16) in 63.2 us, 5.3 TB/s; while all SMs stream it is 7.2 TB/s, but SMs differ by a tenth in the bandwidth they get, and
// the last 9 us belong to the slow ones.  The smallest call (one sequence of 97 tokens) takes 5.0 us.
//
// Split.  The work is the list of all tiles (KT tokens of one sequence and key head), sequence after sequence.  Each CTA (one per
// SM) takes an equal part of that list, each of its warps an equal part of the CTA's, so no length leaves an SM idle and a
// lone long sequence uses the whole GPU.  A warp works alone: it has a ring of stages in shared memory that TMA fills
// (a lane per box issues; the page numbers of the next 32 pages are held one per lane), and it emits every
// (sequence, head) that lies wholly in its part.  Of the others a warp has at most two, at the ends of its part; their
// partial results stay in the ring stage that was read last (that stage is not filled again) and are joined by the CTA
// when its warps are done, then, where a sequence crosses CTAs, through the workspace by the CTA that comes last (a counter that
// is zero again then; the parts are added in the order of the list, so results do not depend on which that is).
//
// Matrix instructions.  The products are narrow, 8 or 16 columns (the query heads of a key head): mma.sync m16n8k16 with tokens, or
// columns of V, as M and query heads as N.  S^T = K Q^T with K from ldmatrix, then O^T += V^T P^T with V from
// ldmatrix.trans and P^T from the scores' registers by movmatrix.  tcgen05 would want 128 tokens at a time and four warps in
// step for each read of tensor memory; warps that work alone on 16 tokens suit short and ragged sequences, and the tensor
// pipe is not the bound (23 % busy with an e4m3 cache).
// Roundings: Q and K are used as they are (an e4m3 cache goes to f16, which is exact; the query, scaled by a power of two so
// that its largest element is below 2, is rounded to f16's 11 bits, exact unless an element is 2^14 times smaller than the
// largest).  The weights p enter the second product as a pair hi + lo of 16-bit floats, because one 16-bit float would cost as much
// again as the output's own rounding; tensor time is not the bound.  bf16 keeps 16 bits of every weight.  f16, with an e4m3 cache,
// keeps 22, but nothing below 2^-25: there the weights' reference also follows scores that stay far below it, so that a weight is
// off by 2^-16 of the largest one of its 16 tokens at most (see kRise).  f32 caches use
// tf32 products of hi + lo pairs (hi hi + hi lo + lo hi: 23 bits), or, where few heads share a row or it is long, fp32 on the CUDA cores.
// Sums, maxima and O are fp32.

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <math.h>

#include <algorithm>
#include <atomic>

#include "luvc_internal.h"
#include "sm100_ptx.cuh"

namespace luvc {
namespace {

using namespace ptx;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxCtas = 256;                   // CTAs the workspace has room for (one per SM)
constexpr int kMaxPartBytes = 16 * (256 + 2) * 4;   // of a partial result: 16 rows of 256 sums, and their (m, l)
constexpr size_t kCounterBytes = 5 * kMaxCtas * sizeof(unsigned);
constexpr float kSlack = 6.f;                   // the reference of the weights may lag behind the maximum by this much
// With an e4m3 cache weights are f16: below 65504, in steps of 2^-24 of one.  The reference m is set kLead below the maximum of 16
// scores when that is above m + kRise, or below m - kFall (a token far above all others, as at the start of a text, leaves only small
// weights).  So the largest of 16 weights is between e^-kFall and e^kRise, and e^kLead at least where it is the largest so far.  m does
// not follow scores below m - kGone (masks of a lowest value), and only as far as sums of weights stay below 2^kMostGain.
constexpr float kRise = 11.f, kFall = 6.f, kLead = 8.f, kGone = 60.f, kMostGain = 60.f;
constexpr int kWaitProbes = 1 << 20;            // probes before a wait for a copy gives up (seconds)
constexpr int kLeastProbes = 1 << 12;           // and with a limit from the status block (a test's), so that copies which do come are waited for

// ---- the instructions of this file -----------------------------------------------------------------

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const void* tmap, uint32_t bar, int x, int row) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(tmap), "r"(bar), "r"(x), "r"(row) : "memory");
}
// The barrier's phase waits for so many bytes more.
__device__ __forceinline__ void mbar_expect_tx(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_trans(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t movm(uint32_t a) {      // transpose of an 8 x 8 matrix of 16-bit elements
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_tf32(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t two) {
    uint32_t d;
    asm("{\n\t.reg .b16 t;\n\tcvt.u16.u32 t, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, t;\n\t}" : "=r"(d) : "r"(two));
    return d;
}
__device__ __forceinline__ float4 lds4(uint32_t addr) {
    float4 x;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(addr) : "memory");
    return x;
}
__device__ __forceinline__ float2 lds2(uint32_t addr) {
    float2 x;
    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(x.x), "=f"(x.y) : "r"(addr) : "memory");
    return x;
}
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// x as a sum of two tf32 operands: the nearest with 11 bits, and what is left, 12 bits, of which the product's operand keeps 11.  (The
// bit that may be dropped is a tie, so rounding it would not be closer.)  What is not finite shows as a NaN in lo, if not in hi:
// the sum that rounds hi makes 0 of the NaN 0x7fffffff, and infinity of the largest floats.
__device__ __forceinline__ void split_tf32(uint32_t x, uint32_t& hi, uint32_t& lo) {
    hi = (x + 0x1000u) & 0xffffe000u;
    lo = __float_as_uint(__fsub_rn(__uint_as_float(x), __uint_as_float(hi)));
}

// ---- shapes ---------------------------------------------------------------------------------------------

// TC: element of the cache; DPB: bytes of a row in shared memory, 64 or a multiple of 128 (columns past D are filled with zeros by
// TMA); NT: groups of 8 query heads per key head that one tile is multiplied with, or, f32 only, -NT query heads on the CUDA cores.
template <typename TC, int DPB_, int NT_>
struct Shape {
    static constexpr int DPB = DPB_, NT = NT_, ES = sizeof(TC), DP = DPB / ES;
    static constexpr int PITCH = DPB < 128 ? DPB : 128, SEGS = DPB / PITCH, BOX = 16 * PITCH;   // a box: PITCH bytes of 16 rows
    static constexpr int SUBK = 16 * DPB;                       // bytes of 16 rows
    // 16-token parts of a tile: one, or as many as make a stage large enough for a partial result (8 NT rows of DP floats).
    static constexpr int SUB = NT > ES ? 2 : 1;
    static constexpr bool CORES = NT < 0;
    static constexpr int KT = 16 * SUB, STAGE = SUB * 2 * SUBK;
    // Three stages for each warp, 196,608 bytes in all: the more warps the smaller a row is.  Two where an f32 row is long and
    // its products, not HBM, are the bound, for half as many warps again (28 / 4 heads of 128, 158 MB: 46.3 us, with three
    // 47.9; 32 / 8, 317 MB: 70 and 73; 12 / 1 of 256, 79 MB: 64 and 81; 8 / 8 of 256, 77 MB: 23 and 28, but 406 MB: 89 and 87), but
    // not for one head of 128 (32 / 32, 903 MB: 158 with two and 151).
    static constexpr int S = ES == 4 && DPB >= 512 && !(NT == -1 && DPB == 512) ? 2 : 3;
    static constexpr int NW = 196608 / (S * STAGE) < 16 ? 196608 / (S * STAGE) : 16;
    // Tiles by which a part may move its ends to those of a (sequence, head).  A join across CTAs costs about as much as two tiles of
    // every warp: 24 sequences of 886 to 1395 tokens, 28 / 4 heads of 128 in 8 bits (16 warps): 14.5 us, with 12 tiles 16.4; six of
    // 5625 to 6957 in bf16 (8 warps): 18.3 with either; 12 of 600 to 2500, 12 / 1 heads of 256 in f32 (3 warps): 39.7, with 12 tiles
    // 45.9.  (Parts of unequal length can cost more than the joins: 32 / 8 heads, 24 sequences in 8 bits 21.1, with 12 tiles 20.4.)
    static constexpr int SNAP = 2 * NW;
    static constexpr int MT = DP / 16;                          // 16-row groups of O^T
    static constexpr int ROWS = CORES ? 4 : 8 * NT;
    static constexpr int PART = ROWS * (DP + 2);                // floats of a partial result in the workspace: O, then (m, l) of each row
    static constexpr int CAP = NW * S * STAGE / (PART * 4);     // partial results the ring has room for
    static_assert(PART * 4 <= kMaxPartBytes, "the workspace has room for less");
    static_assert(ROWS * DP * 4 <= STAGE, "a partial result must fit a stage");
    static_assert(NW * S * STAGE <= 196608, "ring too large");
};

struct Args {
    AttnProblem p;
    int group, groups;          // query heads per key head; head groups of ROWS
    int page_shift;             // log2 of the page size, -1 if it is no power of two
    int limit;                  // tiles of all sequences up to which the list can be numbered in 32 bits
    float one_grid;             // 1 / CTAs
    int rows_total;             // rows of the layer's pool (a row number beyond it reads as zeros)
    unsigned* counters;         // [5][kMaxCtas]: arrivals of (sequence, head)s, of their first groups, of the other groups; groups that
                                // are done; CTAs that are done with these
    float* parts;               // [2][kMaxCtas][2] of PART floats: of CTAs, of groups of CTAs
};

// Place of float d of row r of O in a stage: rows 2 t and 2 t + 1 of a lane quad start 8 banks apart.
__device__ __forceinline__ int o_index(int r, int d, int dp) { return r * dp + (d ^ (((r >> 1) & 3) << 3)); }

template <typename T> __device__ __forceinline__ void put4(T* p, float4 x);
template <> __device__ __forceinline__ void put4<float>(float* p, float4 x) { *reinterpret_cast<float4*>(p) = x; }
template <> __device__ __forceinline__ void put4<__nv_bfloat16>(__nv_bfloat16* p, float4 x) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(x.x, x.y), b = __floats2bfloat162_rn(x.z, x.w);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

// Arrival number i of n at a counter that is zero before the first and after the last of them; true for the one that completes it.  The
// summands are 1, and 1 - n for i = 0: their sum is zero whatever comes in between, so calls that overlap, and take each other's arrivals
// for their own, leave zero behind all the same.
__device__ __forceinline__ unsigned arrive_count(unsigned* counter, int i, int n) {
    const unsigned x = i ? 1u : 1u - (unsigned)n;
    return atomicAdd(counter, x) + x;
}
__device__ __forceinline__ bool arrive(unsigned* counter, int i, int n) { return arrive_count(counter, i, n) == 0u; }

// One partial result in the workspace: rows of O (o_index) and (m, l) of each row.
struct Part {
    float* o;
    float2* ml;
};

// A join of partial results in one step, where a thread has four columns of one row only: (m, l) are read along with the columns,
// eight parts at a time, and what (m, l, o) hold is joined with them.
template <typename GetMl, typename Columns>
__device__ __forceinline__ void join1(int count, GetMl get_ml, Columns columns, float& m, float& l, float4& o) {
    for (int k0 = 0; k0 < count; k0 += 8) {
        float4 x[8];
        float2 ml[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {                           // past the last part: the last one again, with weight 0
            const int at = min(k0 + k, count - 1);
            ml[k] = get_ml(at);
            x[k] = *columns(at);
        }
        float top = m;
#pragma unroll
        for (int k = 0; k < 8; ++k) top = fmaxf(top, ml[k].x);
        const float base = top == -INFINITY ? 0.f : top, f = exp2_fast((m - base) * kLog2e);
        m = top;
        l *= f; o.x *= f; o.y *= f; o.z *= f; o.w *= f;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (k0 + k >= count) continue;
            const float w = exp2_fast((ml[k].x - base) * kLog2e);
            l = fmaf(w, ml[k].y, l);
            o.x = fmaf(w, x[k].x, o.x); o.y = fmaf(w, x[k].y, o.y);
            o.z = fmaf(w, x[k].z, o.z); o.w = fmaf(w, x[k].w, o.w);
        }
    }
}
// Where a thread has several columns, in two steps.  The first, by one warp for a row: the factor of every part,
// exp(m_k - max m), which put(k, factor) gets, times vscale / l where the result is final; returns (m, l) of the whole.
template <typename GetMl, typename Put>
__device__ __forceinline__ float2 join_factors(int count, GetMl get_ml, Put put, bool final, float vscale, int lane) {
    float2 ml[2] = {make_float2(-INFINITY, 0.f), make_float2(-INFINITY, 0.f)};      // of parts lane and lane + 32
#pragma unroll
    for (int x = 0; x < 2; ++x)
        if (lane + 32 * x < count) ml[x] = get_ml(lane + 32 * x);
    float m = fmaxf(ml[0].x, ml[1].x);
#pragma unroll
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
    const float base = m == -INFINITY ? 0.f : m;
    float f[2], l = 0.f;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        f[x] = exp2_fast((ml[x].x - base) * kLog2e);
        l = fmaf(f[x], ml[x].y, l);
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) l += __shfl_xor_sync(~0u, l, d);
    const float all = !final ? 1.f : l == 0.f ? 0.f : vscale / l;           // no key left: zeros
#pragma unroll
    for (int x = 0; x < 2; ++x)
        if (lane + 32 * x < count) put(lane + 32 * x, f[x] * all);
    return make_float2(m, l);
}
// The second, by a thread for its E times four columns: adds the parts times their factors, part after part, so that the reads of
// all columns are under way together.  factor(k, x) and columns(k, x) are of part k and the thread's columns x; `last`: whether the
// thread has the last of its E (where E times the threads are more than a part's columns, some do not: nothing is read for them).
template <int E, typename Factor, typename Columns>
__device__ __forceinline__ void join4(int count, bool last, Factor factor, Columns columns, float4 (&o)[E]) {
#pragma unroll 2
    for (int k = 0; k < count; ++k) {
        float4 v[E];
        float w[E];
#pragma unroll
        for (int x = 0; x < E; ++x) {
            w[x] = 0.f;
            v[x] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (x < E - 1 || last) { w[x] = factor(k, x); v[x] = *columns(k, x); }
        }
#pragma unroll
        for (int x = 0; x < E; ++x) {
            o[x].x = fmaf(w[x], v[x].x, o[x].x); o[x].y = fmaf(w[x], v[x].y, o[x].y);
            o[x].z = fmaf(w[x], v[x].z, o[x].z); o[x].w = fmaf(w[x], v[x].w, o[x].w);
        }
    }
}
__device__ __forceinline__ float lse_of(float2 ml) { return ml.y == 0.f ? -INFINITY : (ml.x == -INFINITY ? 0.f : ml.x) + logf(ml.y); }

// Final values of four columns of a row of out; no key left: zeros, -inf.
template <typename TQ>
__device__ __forceinline__ void emit4(const AttnProblem& p, long long row, int d, float vscale, float m, float l, float4 o) {
    const float f = vscale / l;
    put4(static_cast<TQ*>(p.out) + row * p.c.D + d,
         l == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o.x * f, o.y * f, o.z * f, o.w * f));
    if (p.lse && d == 0) p.lse[row] = lse_of(make_float2(m, l));
}

// What is joined in a CTA: the parts of warps first_warp .. first_warp + count - 1 of one (sequence, head).
struct Chain {
    int count;                  // 0: none
    int out;                    // 1: begins in this CTA and goes on in the next one
    int from;                   // which of the first warp's two pieces
    int rows, c0, c1, s0;       // c0 < c1: other CTAs have parts of it as well
    float vscale;
    long long row0;             // first row of out
};

// A tile of 16 tokens of an f32 cache on the CUDA cores, for NH query heads: where few heads share a key head, splitting rows for the
// tensor cores costs more than the products (one head of 64: 130 instead of 620 instructions).  Scores: two lanes per token, half a
// row each; weighted values: DP / 32 columns per lane.  qs: [NH][DP], ps: [NH][16] of this warp.  bias: of token lane & 15; gone:
// one bit for each masked token.
template <int DP, int NH>
__device__ __forceinline__ void f32_tile(uint32_t ks, uint32_t vs, const float* qs, float* ps, float scale, float bias, unsigned gone,
                                         float (&m)[NH], float (&l)[NH], float (&o)[NH][DP / 32], int lane) {
    const int key = lane & 15, half = lane >> 4;
    float s[NH][2];
#pragma unroll
    for (int h = 0; h < NH; ++h) s[h][0] = s[h][1] = 0.f;
#pragma unroll
    for (int i = 0; i < DP / 8; ++i) {
        const int c = half * (DP / 8) + i;
        const float4 k = lds4(ks + (c >> 3) * 2048 + key * 128 + (((c & 7) ^ (key & 7)) << 4));
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            const float4 q = *reinterpret_cast<const float4*>(qs + h * DP + c * 4);
            s[h][0] = fmaf(q.x, k.x, s[h][0]); s[h][1] = fmaf(q.y, k.y, s[h][1]);
            s[h][0] = fmaf(q.z, k.z, s[h][0]); s[h][1] = fmaf(q.w, k.w, s[h][1]);
        }
    }
    bool over = false;
#pragma unroll
    for (int h = 0; h < NH; ++h) {
        float x = s[h][0] + s[h][1];
        x += __shfl_xor_sync(~0u, x, 16);
        x = (gone >> key) & 1u ? -INFINITY : fmaf(x, scale, bias);
        s[h][0] = x;
        over = over || x > m[h] + kSlack;
    }
    if (__any_sync(~0u, over)) {
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            float x = s[h][0];
#pragma unroll
            for (int d = 8; d; d >>= 1) x = fmaxf(x, __shfl_xor_sync(~0u, x, d));
            x = fmaxf(x, m[h]);
            const float f = exp2_fast((m[h] - (x == -INFINITY ? 0.f : x)) * kLog2e);
            m[h] = x;
            l[h] *= f;
#pragma unroll
            for (int j = 0; j < DP / 32; ++j) o[h][j] *= f;
        }
    }
#pragma unroll
    for (int h = 0; h < NH; ++h) {
        const float p = exp2_fast((s[h][0] - (m[h] == -INFINITY ? 0.f : m[h])) * kLog2e);
        l[h] += p;
        if (half == 0) ps[h * 16 + key] = p;
    }
    __syncwarp();
#pragma unroll
    for (int k4 = 0; k4 < 4; ++k4) {
        float4 p[NH];
#pragma unroll
        for (int h = 0; h < NH; ++h) p[h] = *reinterpret_cast<const float4*>(ps + h * 16 + 4 * k4);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int row = 4 * k4 + x;
            if ((gone >> row) & 1u) continue;                   // a masked row may hold anything
            float v[DP / 32];
            if constexpr (DP == 64) {
                const float2 y = lds2(vs + (lane >> 4) * 2048 + row * 128 + ((((lane & 15) >> 1) ^ (row & 7)) << 4) + (lane & 1) * 8);
                v[0] = y.x; v[1] = y.y;
            } else {
#pragma unroll
                for (int i = 0; i < DP / 128; ++i) {
                    const float4 y = lds4(vs + (4 * i + (lane >> 3)) * 2048 + row * 128 + (((lane & 7) ^ (row & 7)) << 4));
                    v[4 * i] = y.x; v[4 * i + 1] = y.y; v[4 * i + 2] = y.z; v[4 * i + 3] = y.w;
                }
            }
#pragma unroll
            for (int h = 0; h < NH; ++h) {
                const float w = x == 0 ? p[h].x : x == 1 ? p[h].y : x == 2 ? p[h].z : p[h].w;
#pragma unroll
                for (int j = 0; j < DP / 32; ++j) o[h][j] = fmaf(w, v[j], o[h][j]);
            }
        }
    }
    __syncwarp();                                               // ps is written again
}
// Column of a lane's element j in the form above.
template <int DP>
__device__ __forceinline__ int f32_column(int lane, int j) { return DP == 64 ? 2 * lane + j : 128 * (j >> 2) + 4 * lane + (j & 3); }

__device__ __forceinline__ float as_float(float x) { return x; }
__device__ __forceinline__ float as_float(__nv_bfloat16 x) { return __bfloat162float(x); }

// The partial result of tokens t0 .. t1 - 1 of a (sequence, head group) once more, by a warp, product by product as the formula has
// them, into a stage (O) and ml.  The tensor-core forms split weights, and rows of 32 bits, into parts whose products an infinity or
// a value near the end of the range turns into NaN (inf times the lower part of a weight, which may be 0 or negative; inf - inf), and
// weights above 1, while their reference lags behind, can take values beyond that end.  So a result that is not finite is worked out
// again.  It is rare, and need not be fast.
template <typename T, int DP>
__device__ __noinline__ void plain_piece(const Args& a, int seq, int h, int r0, int rows, int t0, int t1, float scale, float* os, float2* ml) {
    const AttnProblem& p = a.p;
    const int lane = threadIdx.x & 31, ps = p.c.page_size, D = p.c.D;
    const int32_t* const table = p.c.table + (long long)(p.seqs ? p.seqs[seq] : seq) * p.c.max_pages;
    const T* const q0 = static_cast<const T*>(p.q) + seq * p.q_stride + ((long long)h * a.group + r0) * D;
    const size_t layer = (size_t)p.layer * a.rows_total;
    for (int r = 0; r < rows; ++r) {
        float q[DP / 32], o[DP / 32], m = -INFINITY, l = 0.f;
#pragma unroll
        for (int j = 0; j < DP / 32; ++j) {
            q[j] = lane + 32 * j < D ? as_float(q0[r * D + lane + 32 * j]) : 0.f;
            o[j] = 0.f;
        }
        for (int t = t0; t < t1; ++t) {
            const float bias = t < p.bias_width ? p.bias[seq * p.bias_stride + t] : 0.f;
            const int page = table[t / ps];
            if (bias == -INFINITY) continue;
            const bool held = (unsigned)page < (unsigned)p.c.pages;         // as in the tiles: rows of no page are zeros
            const size_t at = (layer + (held ? (page * p.c.heads + h) * ps + t % ps : 0)) * D;
            float s = 0.f, v[DP / 32];
#pragma unroll
            for (int j = 0; j < DP / 32; ++j) {
                const int d = lane + 32 * j;
                v[j] = 0.f;
                if (held && d < D) {
                    s = fmaf(q[j], as_float(static_cast<const T*>(p.c.k)[at + d]), s);
                    v[j] = as_float(static_cast<const T*>(p.c.v)[at + d]);
                }
            }
#pragma unroll
            for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
            s = fmaf(s, scale, bias);
            const float top = fmaxf(m, s), base = top == -INFINITY ? 0.f : top;
            const float f = exp2_fast((m - base) * kLog2e), w = exp2_fast((s - base) * kLog2e);
            m = top;
            l = fmaf(l, f, w);
#pragma unroll
            for (int j = 0; j < DP / 32; ++j) o[j] = lane + 32 * j < D ? fmaf(o[j], f, w * v[j]) : 0.f;
        }
#pragma unroll
        for (int j = 0; j < DP / 32; ++j) os[o_index(r, lane + 32 * j, DP)] = o[j];
        if (lane == 0) ml[r] = make_float2(m, l);
    }
    __syncwarp();
}

template <typename TQ, typename TC, int DPB, int NT>
__global__ void __launch_bounds__(32 * Shape<TC, DPB, NT>::NW, 1)
attn_decode_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const __grid_constant__ Args a) {
    using Sh = Shape<TC, DPB, NT>;
    constexpr int NW = Sh::NW, S = Sh::S, MT = Sh::MT, DP = Sh::DP, ROWS = Sh::ROWS, KT = Sh::KT, NTHR = 32 * NW;
    constexpr bool kF32 = Sh::ES == 4, kF8 = Sh::ES == 1, kCores = Sh::CORES;
    constexpr int NTX = kCores ? 1 : NT, NH = kCores ? -NT : 1; // sizes of arrays that are not used otherwise
    extern __shared__ unsigned char smem_raw[];
    __shared__ __align__(8) uint64_t bars[NW * S];
    __shared__ float2 ml_of[NW][2][ROWS];
    // Results that are not final: of a (sequence, head) that a warp's part of the list begins in (0) or ends in (1).
    __shared__ int piece_off[NW][2];                            // where O is in the ring
    __shared__ Chain chains[NW + 1];                            // that begin with piece 1 of warp w; NW: with piece 0 of warp 0
    __shared__ unsigned scan_warp[NW];
    __shared__ __align__(16) float core_q[kCores ? NW : 1][kCores ? NH * DP : 4], core_p[kCores ? NW : 1][NH * 16];
    __shared__ float factors[ROWS * (DP / 4) > NTHR ? 64 : 1][ROWS];
    __shared__ int last_flag[2], all_flag;
    unsigned char* const ring = smem_raw + ((1024 - (smem_u32(smem_raw) & 1023)) & 1023);
    int* const prefix = reinterpret_cast<int*>(ring + NW * S * Sh::STAGE);      // [n + 1] tiles of the sequences before i

    const AttnProblem& p = a.p;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = p.n, ps = p.c.page_size;
    const int g = lane >> 2, t4 = lane & 3;

    // ---- the list of tiles ----
    if (lane < S) {
        mbar_init(smem_u32(&bars[warp * S + lane]), 1);
        mbar_fence_init();
    }
    if (lane < 2) piece_off[warp][lane] = 0;
    if (lane == 0) {
        chains[warp].count = chains[warp].out = 0;
        if (warp == 0) chains[NW].count = chains[NW].out = 0;
    }
    if (tid < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(tid ? &vmap : &kmap) : "memory");
    pdl_trigger();
    pdl_wait();
    auto out_row = [&](long long row) { return static_cast<TQ*>(p.out) + row * p.c.D; };
    auto slot_of = [&](int i) { return p.seqs ? p.seqs[i] : i; };
    auto length_of = [&](int slot) {
        return slot >= 0 && slot < p.c.slots ? max(0, min(p.c.lengths[slot], p.c.max_pages * ps)) : 0;
    };
    const int segs = p.c.heads * a.groups;
    bool fits;
    int base, lane_tiles = 0, lane_first = 0;                   // tiles of all sequences; up to 32 of them: those of lane, and before it
    auto tiles_of = [&](int i) {
        const int slot = slot_of(i);
        if (slot < 0 || slot >= p.c.slots) *p.status = LUVC_ERR_SHAPE;
        return (int)(((unsigned)length_of(slot) + (KT - 1u)) / (unsigned)KT);       // (up to 2^31 - 1 tokens)
    };
    // at most 2^31 / 16 tiles in a sequence: no warp's sum overflows 32 bits
    auto warp_scan = [&](unsigned x) {
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const unsigned y = __shfl_up_sync(~0u, x, d);
            if (lane >= d) x += y;
        }
        return x;
    };
    if (n <= 32) {                                              // every warp for itself (the same values): no barrier
        lane_tiles = lane < n ? tiles_of(lane) : 0;
        const unsigned x = warp_scan(lane_tiles), all = __shfl_sync(~0u, x, 31);
        lane_first = (int)x - lane_tiles;
        fits = all <= (unsigned)a.limit;
        base = (int)all;
        if (lane == 0) prefix[0] = 0;
        if (lane < n) prefix[lane + 1] = (int)x;
        __syncwarp();
    } else {
        fits = true;
        base = 0;
        if (tid == 0) prefix[0] = 0;
        for (int i0 = 0; i0 < n; i0 += NTHR) {
            const int i = i0 + tid;
            const unsigned x = warp_scan(i < n ? tiles_of(i) : 0u);
            if (lane == 31) scan_warp[warp] = x;
            __syncthreads();
            long long before = base, all = base;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                if (w < warp) before += scan_warp[w];
                all += scan_warp[w];
            }
            fits = fits && all <= a.limit;
            base = fits ? (int)all : 0;
            if (i < n) prefix[i + 1] = fits ? (int)(before + x) : 0;
            __syncthreads();
        }
    }
    if (!fits) {                                                // more than 2^31 tiles, a TB at least
        if (tid == 0) *p.status = LUVC_ERR_SHAPE;
        return;
    }
    const int total = base * segs;

    // sequences without tokens
    for (int i = blockIdx.x; i < n; i += gridDim.x) {
        if (prefix[i + 1] != prefix[i]) continue;
        for (int e = tid; e < p.q_heads * (p.c.D / 4); e += NTHR)
            put4(static_cast<TQ*>(p.out) + (long long)i * p.q_heads * p.c.D + 4 * e, make_float4(0.f, 0.f, 0.f, 0.f));
        if (p.lse)
            for (int e = tid; e < p.q_heads; e += NTHR) p.lse[(long long)i * p.q_heads + e] = -INFINITY;
    }

    // ---- this CTA's part of the list, this warp's part of that ----
    struct Place { int seq, seg, tile, tiles, first; };         // a tile; its (sequence, head) starts at `first` in the list
    auto place_of = [&](int x) {                                // x < total, the same in all lanes
        Place q;
        int first;
        if (n <= 32) {                                          // the last lane that begins at or before x (it has tiles)
            q.seq = 31 - __clz(__ballot_sync(~0u, lane < n && lane_first * segs <= x));
            q.tiles = __shfl_sync(~0u, lane_tiles, q.seq);
            first = __shfl_sync(~0u, lane_first, q.seq);
        } else {
            int lo = 0, hi = n;                                 // prefix[lo] * segs <= x < prefix[hi] * segs
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (prefix[mid] * segs <= x) lo = mid; else hi = mid;
            }
            q.seq = lo;
            first = prefix[lo];
            q.tiles = prefix[lo + 1] - first;
        }
        // quotient below segs <= 2^16: the float one is off by less than one
        const int in = x - first * segs;
        q.seg = (int)__fdividef((float)in, (float)q.tiles);
        q.tile = in - q.seg * q.tiles;
        if (q.tile < 0) { --q.seg; q.tile += q.tiles; }
        if (q.tile >= q.tiles) { ++q.seg; q.tile -= q.tiles; }
        q.first = x - q.tile;
        return q;
    };
    // Equal parts, of a tile for each warp at least (measured at eight sequences of 340 to 463 tokens: 9.0 us, with two tiles
    // 9.6: even then a join across CTAs costs less than a warp's second tile).
    int per = max((int)((float)total * a.one_grid) - 1, 0);     // total / grid, rounded up
    per -= per >> 20;
    while ((long long)per * (int)gridDim.x < total) ++per;
    per = max(per, NW);
    const int tol = min(per / 2, Sh::SNAP);
    auto bound_of = [&](int c) {                                // start of CTA c's part, moved to a near (sequence, head) boundary
        if (c == 0) return 0;
        if ((long long)c * per >= total) return total;
        const int x = c * per;
        const Place q = place_of(x);
        if (q.tile <= tol) return q.first;
        if (q.tiles - q.tile <= tol) return q.first + q.tiles;
        return x;
    };
    const int cta_a = bound_of(blockIdx.x), cta_b = bound_of(blockIdx.x + 1);
    if (cta_a >= cta_b) return;
    const int each = (unsigned)(cta_b - cta_a) / NW, more = (unsigned)(cta_b - cta_a) % NW;     // the first `more` warps take one more
    auto part_of_warp = [&](int w) { return cta_a + w * each + min(w, more); };
    const int wa = part_of_warp(warp), wb = part_of_warp(warp + 1);

    unsigned char* const my_ring = ring + warp * S * Sh::STAGE;
    const uint32_t my_ring_s = smem_u32(my_ring), my_bar = smem_u32(&bars[warp * S]);

    if (wa < wb) {
        // what is to be loaded next
        Place ld = place_of(wa);
        int to_load = wb - wa;
        int ld_left = 0, ld_page = 0, ld_off = 0, ld_len = 0, ld_h = 0, pg_first = 0, pg = -1;
        const int32_t* ld_row = nullptr;
        auto fetch_pages = [&] {
            pg_first = ld_page;
            pg = ld_page + lane < p.c.max_pages ? ld_row[ld_page + lane] : -1;
        };
        auto load_start = [&](bool new_seq) {                   // at a new (sequence, head), or at the warp's first tile
            if (new_seq) {
                const int slot = slot_of(ld.seq);
                ld_len = length_of(slot);
                ld_row = p.c.table + (long long)slot * p.c.max_pages;
            }
            const int token = ld.tile * KT;
            ld_left = ld_len - token;
            ld_page = a.page_shift >= 0 ? token >> a.page_shift : token / ps;
            ld_off = token - ld_page * ps;
            if (new_seq || ld_page < pg_first || ld_page >= pg_first + 32) fetch_pages();
            ld_h = a.groups == 1 ? ld.seg : ld.seg / a.groups;
            // its queries are wanted soon
            const int r0 = (ld.seg - ld_h * a.groups) * ROWS;
            const char* const q0 = reinterpret_cast<const char*>(static_cast<const TQ*>(p.q) + ld.seq * p.q_stride +
                                                                 ((long long)ld_h * a.group + r0) * p.c.D);
            const int bytes = min(ROWS, a.group - r0) * p.c.D * (int)sizeof(TQ);
            for (int b = lane * 128; b < bytes; b += 32 * 128) asm volatile("prefetch.global.L1 [%0];" ::"l"(q0 + b));
        };
        const bool is_v = lane & 1;                             // one lane per box: PITCH bytes of 16 rows of K (even lanes) or V
        const CUtensorMap* const my_map = is_v ? &vmap : &kmap;
        const uint32_t my_dst = my_ring_s + (is_v ? Sh::SUBK : 0) + (lane >> 1) * Sh::BOX;
        auto load = [&](int stage) {
            const uint32_t bar = my_bar + 8 * stage;
            if (lane == 0) mbar_arrive_expect_tx(bar, Sh::SUB == 1 || ld_left > 16 ? Sh::STAGE : 2 * Sh::SUBK);
            __syncwarp();
#pragma unroll
            for (int j = 0; j < Sh::SUB; ++j) {
                if (j == 0 || 16 * j < ld_left) {
                    if (ld_page >= pg_first + 32) fetch_pages();
                    const int page = __shfl_sync(~0u, pg, ld_page - pg_first);
                    const int row = (unsigned)page < (unsigned)p.c.pages ? (page * p.c.heads + ld_h) * ps + ld_off : a.rows_total;
                    if (lane < 2 * Sh::SEGS)
                        tma_load_2d(my_dst + stage * Sh::STAGE + j * 2 * Sh::SUBK, my_map, bar, (lane >> 1) * (Sh::PITCH / Sh::ES), row);
                    ld_off += 16;
                    if (ld_off == ps) { ld_off = 0; ++ld_page; }
                }
            }
            ld_left -= KT;
            if (--to_load > 0 && ++ld.tile == ld.tiles) {       // the next (sequence, head)
                ld.tile = 0;
                bool new_seq = false;
                if (++ld.seg == segs) {
                    ld.seg = 0;
                    new_seq = true;
                    do { ++ld.seq; } while (prefix[ld.seq + 1] == prefix[ld.seq]);
                    ld.tiles = prefix[ld.seq + 1] - prefix[ld.seq];
                }
                load_start(new_seq);
            }
        };
        Place at = ld;
        load_start(true);
        // a test's knob: the first wait of the first warp cannot end
        if (blockIdx.x == 0 && tid == 0 && p.status[kStatusHoldBack] > 0) mbar_expect_tx(my_bar, 16);
        __syncwarp();
        unsigned order = 0, phases = 0;                         // stages in the order they were filled (4 bits each); their phases
        int filled = 0;
        for (; filled < S && to_load > 0; ++filled) {
            load(filled);
            order |= (unsigned)filled << (4 * filled);
        }

        // A lane's row address for ldmatrix: chunk c of row r of a box lies at r * 128 + 16 * (c ^ (r & 7)), where rows are of 64
        // bytes at r * 64 + 16 * (c ^ (r / 2 & 3)) (TMA's swizzles; eight rows meet no bank twice).  Matrices 0 .. 3 of
        // K are (rows 0-7, c), (rows 8-15, c), (rows 0-7, c + 1), (rows 8-15, c + 1); of a 16-bit V the middle two change places.
        // The next two chunks are at the address with 32 flipped in.
        const int k_row = lane & 15, v_row = (lane & 7) + ((lane >> 4) << 3);
        auto chunk_at = [](int r, int c) { return Sh::PITCH == 64 ? r * 64 + ((c ^ ((r >> 1) & 3)) << 4) : r * 128 + ((c ^ (r & 7)) << 4); };
        const uint32_t k_lane = chunk_at(k_row, lane >> 4), v_lane = chunk_at(v_row, (lane >> 3) & 1);
        int left = wb - wa;
        bool dead = false;                                      // a wait gave up: what is left is passed over, so that joins and counters go on
        while (left > 0) {
            const int h = a.groups == 1 ? at.seg : at.seg / a.groups, r0 = (at.seg - h * a.groups) * ROWS;
            const int rows = min(ROWS, a.group - r0);
            const int len = length_of(slot_of(at.seq));
            const float vscale = p.c.v_scale ? p.c.v_scale[p.layer * p.c.heads + h] : 1.f;
            const float scale = p.scale * (p.c.k_scale ? p.c.k_scale[p.layer * p.c.heads + h] : 1.f);
            // queries: B operand of S^T = K Q^T, head g of each group of 8
            const TQ* const qrow = static_cast<const TQ*>(p.q) + at.seq * p.q_stride + ((long long)h * a.group + r0) * p.c.D;
            constexpr int KS = DPB / 32;                        // steps of 32 bytes of a row
            uint32_t q[NTX][KS][kF8 ? 4 : 2];
            float qmul[NTX][2];
            if constexpr (kCores) {
                __syncwarp();                                   // the queries before have been used
                for (int x = lane; x < NH * DP; x += 32) {
                    const int r = x / DP, d = x % DP;
                    core_q[warp][x] = r < rows && d < p.c.D ? reinterpret_cast<const float*>(qrow)[r * p.c.D + d] : 0.f;
                }
                __syncwarp();
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const TQ* const qh = qrow + (long long)(nt * 8 + g) * p.c.D;
                const bool live = nt * 8 + g < rows;
                if constexpr (kF32) {
#pragma unroll
                    for (int k = 0; k < KS; ++k)
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            const int d = 8 * k + 4 * b + t4;
                            q[nt][k][b] = live && d < p.c.D ? reinterpret_cast<const uint32_t*>(qh)[d] : 0u;
                        }
                    qmul[nt][0] = qmul[nt][1] = scale;
                } else if constexpr (!kF8) {
#pragma unroll
                    for (int k = 0; k < KS; ++k)
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            const int d = 16 * k + 8 * b + 2 * t4;
                            q[nt][k][b] = live && d < p.c.D ? *reinterpret_cast<const uint32_t*>(qh + d) : 0u;
                        }
                    qmul[nt][0] = qmul[nt][1] = scale;
                } else {
                    // a 16-byte piece of a row is one k step; lane t4 holds its bytes 4 t4 .. 4 t4 + 3
                    uint2 raw[2 * KS];
                    float big = 0.f;
#pragma unroll
                    for (int k = 0; k < 2 * KS; ++k) {
                        const int d = 16 * k + 4 * t4;
                        raw[k] = live && d < p.c.D ? *reinterpret_cast<const uint2*>(qh + d) : make_uint2(0u, 0u);
                        big = fmaxf(big, fmaxf(fmaxf(fabsf(__uint_as_float(raw[k].x << 16)), fabsf(__uint_as_float(raw[k].x & 0xffff0000u))),
                                               fmaxf(fabsf(__uint_as_float(raw[k].y << 16)), fabsf(__uint_as_float(raw[k].y & 0xffff0000u)))));
                    }
                    big = fmaxf(big, __shfl_xor_sync(~0u, big, 1));
                    big = fmaxf(big, __shfl_xor_sync(~0u, big, 2));
                    // 2^e <= big < 2^(e+1), kept where 2^e and 2^-e are normal floats
                    const int e = big == 0.f ? 0 : max(-125, min(125, (int)(__float_as_uint(big) >> 23) - 127));
                    const float down = __uint_as_float((unsigned)(127 - e) << 23), up = __uint_as_float((unsigned)(127 + e) << 23);
#pragma unroll
                    for (int k = 0; k < 2 * KS; ++k) {
                        const __half2 x = __floats2half2_rn(__uint_as_float(raw[k].x << 16) * down, __uint_as_float(raw[k].x & 0xffff0000u) * down);
                        const __half2 y = __floats2half2_rn(__uint_as_float(raw[k].y << 16) * down, __uint_as_float(raw[k].y & 0xffff0000u) * down);
                        q[nt][k >> 1][2 * (k & 1)] = *reinterpret_cast<const uint32_t*>(&x);
                        q[nt][k >> 1][2 * (k & 1) + 1] = *reinterpret_cast<const uint32_t*>(&y);
                    }
                    qmul[nt][0] = scale * __shfl_sync(~0u, up, 8 * t4);         // of heads 2 t4 and 2 t4 + 1
                    qmul[nt][1] = scale * __shfl_sync(~0u, up, 8 * t4 + 4);
                }
            }

            float core_m[NH], core_l[NH], core_o[NH][DP / 32];
            if constexpr (kCores)
#pragma unroll
                for (int h2 = 0; h2 < NH; ++h2) {
                    core_m[h2] = -INFINITY;
                    core_l[h2] = 0.f;
#pragma unroll
                    for (int j = 0; j < DP / 32; ++j) core_o[h2][j] = 0.f;
                }
            float m[NTX][2], l[NTX][2], o[MT][NTX][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) m[nt][0] = m[nt][1] = -INFINITY, l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 4; ++c) o[mt][nt][c] = 0.f;

            const int count = min(at.tiles - at.tile, left);
            const bool whole = at.tile == 0 && count == at.tiles;
            int stage = 0;
            for (int k = 0; k < count; ++k, ++at.tile) {
                stage = order & 15;
                order >>= 4;
                --filled;
                // a tile with biases, or past the end (which is a bias of -inf)
                const bool masked = p.bias_width > 0 || len - at.tile * KT < KT;
                float bias[Sh::SUB][2];
#pragma unroll
                for (int j = 0; j < Sh::SUB; ++j)
#pragma unroll
                    for (int x = 0; x < 2; ++x) bias[j][x] = 0.f;
                if (masked)
#pragma unroll
                    for (int j = 0; j < Sh::SUB; ++j)
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const int token = at.tile * KT + 16 * j + (kCores ? lane & 15 : 8 * x + g);
                            if (token >= len) bias[j][x] = -INFINITY;
                            else if (token < p.bias_width) bias[j][x] = p.bias[at.seq * p.bias_stride + token];
                        }
                if (!dead) {
                    const uint32_t bar = my_bar + 8 * stage;
                    int probes = 0, limit = kWaitProbes;
                    while (!mbar_try_wait(bar, (phases >> stage) & 1) && ++probes < limit)
                        if (probes == kLeastProbes - 1) {
                            const int knob = *reinterpret_cast<volatile int*>(p.status + kStatusProbeLimit);
                            if (knob > 0) limit = max(kLeastProbes, knob);
                        }
                    phases ^= 1u << stage;
                    if (__any_sync(~0u, probes >= limit)) {
                        dead = true;
                        to_load = 0;
                        for (; filled > 0; --filled, order >>= 4)   // let the copies in flight land
                            for (probes = 0; !mbar_try_wait(my_bar + 8 * (order & 15), (phases >> (order & 15)) & 1) && ++probes < kWaitProbes;) {}
                        if (lane == 0) *p.status = LUVC_ERR_TIMEOUT;
                    }
                }
                if (dead) continue;
#pragma unroll
                for (int j = 0; j < Sh::SUB; ++j) {
                    if (j > 0 && at.tile * KT + 16 * j >= len) break;
                    const uint32_t ks = my_ring_s + stage * Sh::STAGE + j * 2 * Sh::SUBK, vs = ks + Sh::SUBK;
                    if constexpr (kCores) {
                        const unsigned gone = masked ? __ballot_sync(~0u, bias[j][0] == -INFINITY) & 0xffffu : 0u;
                        f32_tile<DP, NH>(ks, vs, core_q[warp], core_p[warp], scale, bias[j][0], gone, core_m, core_l, core_o, lane);
                    } else {
                        // ---- S^T: rows are the 16 tokens, columns the query heads ----
                        float s[NTX][4], s2[NTX][4], s3[NTX][4];    // sums that do not wait for one another
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int c = 0; c < 4; ++c) s[nt][c] = s2[nt][c] = s3[nt][c] = 0.f;
                        float done[NTX][4];                         // f32: finished sums of S
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int c = 0; c < 4; ++c) done[nt][c] = 0.f;
#pragma unroll
                        for (int k2 = 0; k2 < KS; ++k2) {           // 32 bytes of each of the 16 rows
                            uint32_t r[4];
                            ldsm4(((ks + k_lane) ^ (32 * (k2 & 3))) + (k2 >> 2) * 2048, r);
                            if constexpr (kF32) {
                                uint32_t hi[4], lo[4];
#pragma unroll
                                for (int c = 0; c < 4; ++c) split_tf32(r[c], hi[c], lo[c]);
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) {
                                    uint32_t qh[2], ql[2];
                                    split_tf32(q[nt][k2][0], qh[0], ql[0]);
                                    split_tf32(q[nt][k2][1], qh[1], ql[1]);
                                    mma_tf32(s2[nt], lo, qh[0], qh[1]);
                                    mma_tf32(NT == 1 ? s3[nt] : s2[nt], hi, ql[0], ql[1]);
                                    // tensor-core sums truncate: four steps at most in one, the rest rounded
                                    float part[4] = {0.f, 0.f, 0.f, 0.f};
                                    mma_tf32(k2 % 4 ? s[nt] : part, hi, qh[0], qh[1]);
                                    if (k2 % 4 == 0)
#pragma unroll
                                        for (int c = 0; c < 4; ++c) { done[nt][c] += s[nt][c]; s[nt][c] = part[c]; }
                                }
                            } else if constexpr (!kF8) {
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) mma_bf16(k2 & 1 ? s2[nt] : s[nt], r, q[nt][k2][0], q[nt][k2][1]);
                            } else {
                                const uint32_t x[4] = {e4m3x2_to_f16x2(r[0]), e4m3x2_to_f16x2(r[1]), e4m3x2_to_f16x2(r[0] >> 16), e4m3x2_to_f16x2(r[1] >> 16)};
                                const uint32_t y[4] = {e4m3x2_to_f16x2(r[2]), e4m3x2_to_f16x2(r[3]), e4m3x2_to_f16x2(r[2] >> 16), e4m3x2_to_f16x2(r[3] >> 16)};
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) {
                                    mma_f16(s[nt], x, q[nt][k2][0], q[nt][k2][1]);
                                    mma_f16(s2[nt], y, q[nt][k2][2], q[nt][k2][3]);
                                }
                            }
                        }
                        // ---- weights ----
                        // Their reference m follows the maximum only when a score passes it by kSlack (e4m3: kRise): weights stay
                        // below e^kSlack, sums lose nothing, and most tiles need no maximum across the warp.
                        bool over = false;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                const float x = kF32 ? done[nt][c] + s[nt][c] + (s2[nt][c] + s3[nt][c]) : s[nt][c] + s2[nt][c];
                                s[nt][c] = fmaf(x, qmul[nt][c & 1], bias[j][c >> 1]);
                            }
                        unsigned gone = 0;
                        if (masked) {                               // whatever a masked row holds
                            const bool gone0 = bias[j][0] == -INFINITY, gone1 = bias[j][1] == -INFINITY;
                            gone = __ballot_sync(~0u, gone0 || gone1);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int c = 0; c < 4; ++c)
                                    if (c >> 1 ? gone1 : gone0) s[nt][c] = -INFINITY;
                        }
                        if constexpr (kF8) {
                            unsigned seen = 0;                      // a bit per head whose largest score is not too small; bit 16: one is too large
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int b = 0; b < 2; ++b) {
                                    const float x = fmaxf(s[nt][b], s[nt][b + 2]);
                                    if (x >= m[nt][b] - kFall) seen |= 1u << (8 * nt + b);
                                    over = over || x > m[nt][b] + kRise;
                                }
                            if (__reduce_or_sync(~0u, seen << (2 * t4) | (over ? 1u << 16 : 0u)) != (1u << (8 * NTX)) - 1u) {
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                    for (int b = 0; b < 2; ++b) {
                                        float x = fmaxf(s[nt][b], s[nt][b + 2]), most = l[nt][b];
#pragma unroll
                                        for (int d = 4; d <= 16; d *= 2) {
                                            x = fmaxf(x, __shfl_xor_sync(~0u, x, d));
                                            most = fmaxf(most, __shfl_xor_sync(~0u, most, d));
                                        }
                                        float to = m[nt][b];
                                        if (x > to + kRise) to = x - kLead;
                                        else if (x < to - kFall && x > to - kGone)
                                            to -= fminf(to - (x - kLead), fmaxf(kMostGain - __log2f(most), 0.f) / kLog2e);
                                        const float f = exp2_fast((m[nt][b] - (to == -INFINITY ? 0.f : to)) * kLog2e);
                                        m[nt][b] = to;
                                        l[nt][b] *= f;
#pragma unroll
                                        for (int mt = 0; mt < MT; ++mt) { o[mt][nt][b] *= f; o[mt][nt][b + 2] *= f; }
                                    }
                            }
                        } else
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int c = 0; c < 4; ++c) over = over || s[nt][c] > m[nt][c & 1] + kSlack;
                        if (!kF8 && __any_sync(~0u, over)) {
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int b = 0; b < 2; ++b) {
                                    float x = fmaxf(s[nt][b], s[nt][b + 2]);
                                    x = fmaxf(x, __shfl_xor_sync(~0u, x, 4));
                                    x = fmaxf(x, __shfl_xor_sync(~0u, x, 8));
                                    x = fmaxf(x, __shfl_xor_sync(~0u, x, 16));
                                    x = fmaxf(x, m[nt][b]);
                                    const float f = exp2_fast((m[nt][b] - (x == -INFINITY ? 0.f : x)) * kLog2e);
                                    m[nt][b] = x;
                                    l[nt][b] *= f;
#pragma unroll
                                    for (int mt = 0; mt < MT; ++mt) { o[mt][nt][b] *= f; o[mt][nt][b + 2] *= f; }
                                }
                        }
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                const float mb = m[nt][c & 1] == -INFINITY ? 0.f : m[nt][c & 1];
                                s[nt][c] = exp2_fast((s[nt][c] - mb) * kLog2e);
                            }
                        uint32_t ph[NTX][2], pl[NTX][2];            // P^T, B operand: tokens 2 t4, 2 t4 + 1 (and + 8) of head g
                        float pf[NTX][4];
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            l[nt][0] += s[nt][0] + s[nt][2];
                            l[nt][1] += s[nt][1] + s[nt][3];
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                const float p0 = s[nt][2 * x], p1 = s[nt][2 * x + 1];
                                if constexpr (kF32) {
                                    const uint32_t u0 = __float_as_uint(p0), u1 = __float_as_uint(p1);
                                    const uint32_t up = movm(__byte_perm(u0, u1, 0x7632)), down = movm(__byte_perm(u0, u1, 0x5410));
                                    pf[nt][2 * x] = __uint_as_float(__byte_perm(down, up, 0x5410));
                                    pf[nt][2 * x + 1] = __uint_as_float(__byte_perm(down, up, 0x7632));
                                } else if constexpr (!kF8) {
                                    const __nv_bfloat162 hi = __floats2bfloat162_rn(p0, p1);
                                    const __nv_bfloat162 lo = __floats2bfloat162_rn(p0 - __low2float(hi), p1 - __high2float(hi));
                                    ph[nt][x] = movm(*reinterpret_cast<const uint32_t*>(&hi));
                                    pl[nt][x] = movm(*reinterpret_cast<const uint32_t*>(&lo));
                                } else {
                                    const __half2 hi = __floats2half2_rn(p0, p1);
                                    const __half2 lo = __floats2half2_rn(p0 - __low2float(hi), p1 - __high2float(hi));
                                    ph[nt][x] = movm(*reinterpret_cast<const uint32_t*>(&hi));
                                    pl[nt][x] = movm(*reinterpret_cast<const uint32_t*>(&lo));
                                }
                            }
                        }
                        // ---- O^T += V^T P^T; rows of V that are masked may hold anything and are replaced by zeros ----
                        uint32_t keep0 = ~0u, keep1 = ~0u;          // 16-bit halves of a register: tokens 2 t4, 2 t4 + 1 (+ 8)
                        if (gone) {                                 // token g (+ 8) is that of lanes 4 g ..
                            const unsigned g0 = __ballot_sync(~0u, bias[j][0] == -INFINITY), g1 = __ballot_sync(~0u, bias[j][1] == -INFINITY);
                            keep0 = ((g0 >> (8 * t4)) & 1u ? 0u : 0xffffu) | ((g0 >> (8 * t4 + 4)) & 1u ? 0u : 0xffff0000u);
                            keep1 = ((g1 >> (8 * t4)) & 1u ? 0u : 0xffffu) | ((g1 >> (8 * t4 + 4)) & 1u ? 0u : 0xffff0000u);
                        }
                        if constexpr (kF32) {
                            // step x: tokens 8 x .. 8 x + 7; k = t4 is token 2 t4, k = t4 + 4 is token 2 t4 + 1 (bank-conflict free)
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                const uint32_t keep = x ? keep1 : keep0;
                                const bool drop0 = !(keep & 0xffffu), drop1 = !(keep >> 16);
                                uint32_t bh[NTX][2], bl[NTX][2];
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) {
                                    split_tf32(__float_as_uint(pf[nt][2 * x]), bh[nt][0], bl[nt][0]);
                                    split_tf32(__float_as_uint(pf[nt][2 * x + 1]), bh[nt][1], bl[nt][1]);
                                }
                                const int row0 = 8 * x + 2 * t4, row1 = row0 + 1;
                                constexpr int MB = NT == 1 ? 4 : 1;             // 16-column groups at a time: products that do not wait for one another
#pragma unroll
                                for (int m0 = 0; m0 < MT; m0 += MB) {
                                    uint32_t hi[MB][4], lo[MB][4];
#pragma unroll
                                    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                                        for (int c = 0; c < 4; ++c) {
                                            const int d = 16 * (m0 + mb) + 8 * (c & 1) + g, row = c >> 1 ? row1 : row0;
                                            uint32_t u;
                                            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(u)
                                                         : "r"(vs + (d >> 5) * 2048 + row * 128 + ((((d & 31) >> 2) ^ (row & 7)) << 4) + (d & 3) * 4) : "memory");
                                            if (c >> 1 ? drop1 : drop0) u = 0u;
                                            split_tf32(u, hi[mb][c], lo[mb][c]);
                                        }
                                    float add[MB][NTX][4];                      // a long sum is kept with rounded additions
#pragma unroll
                                    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                                        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                                            for (int c = 0; c < 4; ++c) add[mb][nt][c] = 0.f;
                                            mma_tf32(add[mb][nt], lo[mb], bh[nt][0], bh[nt][1]);
                                        }
#pragma unroll
                                    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                                        for (int nt = 0; nt < NT; ++nt) mma_tf32(add[mb][nt], hi[mb], bl[nt][0], bl[nt][1]);
#pragma unroll
                                    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                                        for (int nt = 0; nt < NT; ++nt) mma_tf32(add[mb][nt], hi[mb], bh[nt][0], bh[nt][1]);
#pragma unroll
                                    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                            for (int c = 0; c < 4; ++c) o[m0 + mb][nt][c] += add[mb][nt][c];
                                }
                            }
                        } else if constexpr (!kF8) {
#pragma unroll
                            for (int mt = 0; mt < MT; ++mt) {
                                uint32_t r[4];
                                ldsm4_trans(((vs + v_lane) ^ (32 * (mt & 3))) + (mt >> 2) * 2048, r);
                                if (gone) { r[0] &= keep0; r[1] &= keep0; r[2] &= keep1; r[3] &= keep1; }
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) {
                                    mma_bf16(o[mt][nt], r, pl[nt][0], pl[nt][1]);
                                    mma_bf16(o[mt][nt], r, ph[nt][0], ph[nt][1]);
                                }
                            }
                        } else {
                            // a transposed 8 x 8 matrix of byte pairs: tokens 2 t4 and 2 t4 + 1 of columns 2 g and 2 g + 1
#pragma unroll
                            for (int m2 = 0; m2 < MT / 2; ++m2) {   // two 16-byte pieces
                                uint32_t r[4];
                                ldsm4_trans(((vs + k_lane) ^ (32 * (m2 & 3))) + (m2 >> 2) * 2048, r);
                                if (gone) { r[0] &= keep0; r[2] &= keep0; r[1] &= keep1; r[3] &= keep1; }
#pragma unroll
                                for (int x = 0; x < 2; ++x) {
                                    const uint32_t u = __byte_perm(r[2 * x], 0u, 0x3120), w = __byte_perm(r[2 * x + 1], 0u, 0x3120);
                                    const uint32_t v[4] = {e4m3x2_to_f16x2(u), e4m3x2_to_f16x2(u >> 16), e4m3x2_to_f16x2(w), e4m3x2_to_f16x2(w >> 16)};
#pragma unroll
                                    for (int nt = 0; nt < NT; ++nt) {
                                        mma_f16(o[2 * m2 + x][nt], v, pl[nt][0], pl[nt][1]);
                                        mma_f16(o[2 * m2 + x][nt], v, ph[nt][0], ph[nt][1]);
                                    }
                                }
                            }
                        }
                    }
                }
                __syncwarp();
                if (k < count - 1 && to_load > 0) {             // the stage has been read
                    load(stage);
                    order |= (unsigned)stage << (4 * filled);
                    ++filled;
                }
            }
            left -= count;

            // ---- the result, through the stage that was read last ----
            float* const os = reinterpret_cast<float*>(my_ring + stage * Sh::STAGE);
            const int which = at.tile > count ? 0 : 1;          // 0: it began in the part of the warp before
            if constexpr (kCores) {
#pragma unroll
                for (int r = 0; r < NH; ++r) {
                    float x = core_l[r];
#pragma unroll
                    for (int d = 8; d; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
                    if (lane == 0) ml_of[warp][which][r] = make_float2(core_m[r], x);
#pragma unroll
                    for (int j = 0; j < DP / 32; ++j) os[o_index(r, f32_column<DP>(lane, j), DP)] = core_o[r][j];
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    float x = l[nt][b];
                    x += __shfl_xor_sync(~0u, x, 4);
                    x += __shfl_xor_sync(~0u, x, 8);
                    x += __shfl_xor_sync(~0u, x, 16);
                    if (g == 0) ml_of[warp][which][nt * 8 + 2 * t4 + b] = make_float2(m[nt][b], x);
                }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int d = 16 * mt + (kF8 ? 2 * g + (c >> 1) : g + 8 * (c >> 1));
                        os[o_index(nt * 8 + 2 * t4 + (c & 1), d, DP)] = o[mt][nt][c];
                    }
            __syncwarp();
            if constexpr (!kF8) {                               // (an e4m3 cache has no infinities, and its rows are not split)
                float z[4] = {0.f, 0.f, 0.f, 0.f};              // 0, or NaN
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        z[c] = fmaf(l[nt][c & 1], 0.f, z[c]);
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt) z[c] = fmaf(o[mt][nt][c], 0.f, z[c]);
                    }
                if constexpr (kCores)
#pragma unroll
                    for (int r = 0; r < NH; ++r)
#pragma unroll
                        for (int j = 0; j < DP / 32; ++j) z[j & 3] = fmaf(core_o[r][j], 0.f, z[j & 3]);
                if (__any_sync(~0u, z[0] + z[1] + (z[2] + z[3]) != 0.f) && !dead)
                    plain_piece<TC, DP>(a, at.seq, h, r0, rows, (at.tile - count) * KT, min(at.tile * KT, len), scale, os, ml_of[warp][which]);
            }
            const long long row0 = (long long)at.seq * p.q_heads + h * a.group + r0;
            if (whole) {
                if (lane < rows) {                              // the factor takes the maximum's place
                    const float2 ml = ml_of[warp][1][lane];
                    if (p.lse) p.lse[row0 + lane] = lse_of(ml);
                    ml_of[warp][1][lane].x = ml.y == 0.f ? 0.f : vscale / ml.y;
                }
                __syncwarp();
                for (int e = lane; e < ROWS * (DP / 4); e += 32) {
                    const int r = e / (DP / 4), d = e % (DP / 4) * 4;
                    if (r >= rows || d >= p.c.D) continue;
                    const float4 x = *reinterpret_cast<const float4*>(os + o_index(r, d, DP));
                    const float f = ml_of[warp][1][r].x;
                    put4(out_row(row0 + r) + d, f == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(x.x * f, x.y * f, x.z * f, x.w * f));
                }
                fence_proxy_async();                            // the stage was written by this warp; TMA writes it next
                __syncwarp();
                if (to_load > 0) {
                    load(stage);
                    order |= (unsigned)stage << (4 * filled);
                    ++filled;
                }
            } else if (lane == 0) {
                piece_off[warp][which] = (warp * S + stage) * Sh::STAGE;
                if (which == 1 || warp == 0) {                  // a chain begins here
                    Chain& c = chains[which ? warp : NW];
                    const int s0 = prefix[at.seq] * segs + at.seg * at.tiles, s1 = s0 + at.tiles;
                    const int x = min(s1, cta_b) - 1 - cta_a, y = x - more * (each + 1);    // its last tile here, and whose that is
                    const int last = y < 0 ? x / (each + 1) : more + y / each;
                    c.count = last - warp + 1;
                    c.from = which;
                    c.rows = rows;
                    c.vscale = vscale;
                    c.row0 = row0;
                    c.s0 = s0;
                    c.c0 = c.c1 = c.out = 0;
                    if (s0 < cta_a || s1 > cta_b) {
                        c.c0 = (s0 + tol) / per;
                        c.c1 = (s1 - tol - 1) / per;
                        c.out = s0 >= cta_a;
                    }
                }
            }
            if (left > 0) {                                     // the next (sequence, head)
                at.tile = 0;
                if (++at.seg == segs) {
                    at.seg = 0;
                    do { ++at.seq; } while (prefix[at.seq + 1] == prefix[at.seq]);
                    at.tiles = prefix[at.seq + 1] - prefix[at.seq];
                }
            }
        }
    }
    __syncthreads();

    // ---- joins: the parts of this CTA's warps; then, of a (sequence, head) that other CTAs share, theirs, by the one that
    //      arrives last ----
    auto global_part = [&](int cta, int slot) {
        float* const o = a.parts + ((size_t)cta * 2 + slot) * Sh::PART;
        return Part{o, reinterpret_cast<float2*>(o + ROWS * DP)};
    };
    const unsigned some = __ballot_sync(~0u, lane <= NW && chains[min(lane, NW)].count);
    const int out_chain = __ffs(__ballot_sync(~0u, lane <= NW && chains[min(lane, NW)].out)) - 1;    // at most one: its last tile is this CTA's
    constexpr int E = (ROWS * (DP / 4) + NTHR - 1) / NTHR;      // four columns each, of a thread
    const bool all_columns = E * NTHR == ROWS * (DP / 4) || tid + (E - 1) * NTHR < ROWS * (DP / 4);     // the last E included
    if constexpr (E == 1) {
        const int r = tid / (DP / 4), d = tid % (DP / 4) * 4, at = o_index(r, d, DP);
#pragma unroll 1
        for (unsigned left = some; left; left &= left - 1) {
            const int c = __ffs(left) - 1, w0 = c == NW ? 0 : c;
            const Chain& ch = chains[c];
            if (r >= ch.rows || d >= p.c.D) continue;
            float m = -INFINITY, l = 0.f;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
            join1(ch.count, [&](int k) { return ml_of[w0 + k][k ? 0 : ch.from][r]; },
                  [&](int k) { return reinterpret_cast<const float4*>(reinterpret_cast<const float*>(ring + piece_off[w0 + k][k ? 0 : ch.from]) + at); },
                  m, l, o);
            if (ch.c0 == ch.c1) {
                emit4<TQ>(p, ch.row0 + r, d, ch.vscale, m, l, o);
            } else {
                const Part q = global_part(blockIdx.x, ch.s0 >= cta_a);
                *reinterpret_cast<float4*>(q.o + at) = o;
                if (d == 0) q.ml[r] = make_float2(m, l);
            }
        }
    } else {
        for (unsigned left = some; left; left &= left - 1) {
            const int c = __ffs(left) - 1, w0 = c == NW ? 0 : c;
            const Chain& ch = chains[c];
            const bool final = ch.c0 == ch.c1;
            for (int r = warp; r < ch.rows; r += NW) {              // the factors take the places of the maxima
                auto ml = [&](int k) -> float2& { return ml_of[w0 + k][k ? 0 : ch.from][r]; };
                const float2 all = join_factors(ch.count, ml, [&](int k, float f) { ml(k).x = f; }, final, ch.vscale, lane);
                if (lane == 0) {
                    if (!final) global_part(blockIdx.x, ch.s0 >= cta_a).ml[r] = all;
                    else if (p.lse) p.lse[ch.row0 + r] = lse_of(all);
                }
            }
        }
        __syncthreads();
#pragma unroll 1
        for (unsigned left = some; left; left &= left - 1) {
            const int c = __ffs(left) - 1, w0 = c == NW ? 0 : c;
            const Chain& ch = chains[c];
            float4 o[E];
#pragma unroll
            for (int x = 0; x < E; ++x) o[x] = make_float4(0.f, 0.f, 0.f, 0.f);
            // (rows of a part past the last head's hold sums of nothing: they are read, and not written)
            join4<E>(ch.count, all_columns, [&](int k, int x) { return ml_of[w0 + k][k ? 0 : ch.from][(tid + x * NTHR) / (DP / 4)].x; },
                     [&](int k, int x) {
                         const int e = tid + x * NTHR;
                         return reinterpret_cast<const float4*>(reinterpret_cast<const float*>(ring + piece_off[w0 + k][k ? 0 : ch.from]) +
                                                                o_index(e / (DP / 4), e % (DP / 4) * 4, DP));
                     }, o);
#pragma unroll
            for (int x = 0; x < E; ++x) {
                const int e = tid + x * NTHR, r = e / (DP / 4), d = e % (DP / 4) * 4;
                if (r >= ch.rows || d >= p.c.D) continue;
                if (ch.c0 == ch.c1) put4(out_row(ch.row0 + r) + d, o[x]);
                else *reinterpret_cast<float4*>(global_part(blockIdx.x, ch.s0 >= cta_a).o + o_index(r, d, DP)) = o[x];
            }
        }
    }
    const bool in = chains[NW].count && chains[NW].c0 != chains[NW].c1;   // shared with the CTA before / with the next one only
    if (!in && out_chain < 0) return;
    // Up to kDirect parts are joined at once.  More (few long sequences with few heads) are joined in groups of kGroup, by the last
    // to arrive of each group, and the groups by the last of these: 148 parts take two short joins instead of one long one.
    constexpr int kDirect = Sh::CAP < 48 ? Sh::CAP : 48, kGroup = 12;
    // How often the groups' counter is counted up depends on who is last of each, and goes wrong where calls overlap: so the CTA that is
    // the last of all to pass it sets it to zero (which it is, in calls that do not).
    auto pass_groups = [&](const Chain& ch) { return arrive_count(a.counters + 4 * kMaxCtas + ch.c0, blockIdx.x - ch.c0, ch.c1 - ch.c0 + 1); };
    auto groups_passed = [&](const Chain& ch, unsigned count) {
        if (count == 0u) a.counters[3 * kMaxCtas + ch.c0] = 0u;
    };
    __threadfence();
    __syncthreads();
    if (tid < 64 && lane == 0) {
        bool last = false;
        if (warp == 0 ? in : out_chain >= 0) {
            const Chain& ch = chains[warp == 0 ? NW : out_chain];
            const int count = ch.c1 - ch.c0 + 1, i = blockIdx.x - ch.c0, first = i / kGroup * kGroup;       // of this CTA's group
            if (count <= kDirect) {
                last = arrive(a.counters + ch.c0, i, count);
            } else {
                // a CTA can be the first of a group of the (sequence, head) it begins in, and the beginning of another one
                last = arrive(a.counters + (first == 0 ? kMaxCtas + ch.c0 : 2 * kMaxCtas + ch.c0 + first), i - first, min(kGroup, count - first));
                if (!last) groups_passed(ch, pass_groups(ch));
            }
        }
        last_flag[warp] = last;
    }
    __syncthreads();

    // Joins `count` parts (at most 64), copied to shared memory as many as fit at a time.
    auto gather = [&](const Chain& ch, int count, auto part_of, bool final, Part to) {
        float m = -INFINITY, l = 0.f;
        float4 o[E];
#pragma unroll
        for (int x = 0; x < E; ++x) o[x] = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k0 = 0; k0 < count; k0 += Sh::CAP) {
            const int now = min(Sh::CAP, count - k0);
            __syncthreads();                                    // the ring has been read
            for (int k = warp; k < now; k += NW) {
                const float* const src = part_of(k0 + k).o;
                const uint32_t dst = smem_u32(ring) + k * (Sh::PART * 4);
#pragma unroll
                for (int x = lane; x < Sh::PART / 4; x += 32) cp_async16(dst + x * 16, src + x * 4, true);
            }
            cp_async_commit();
            if (E > 1 && k0 == 0)                               // meanwhile the factors of all parts
                for (int r = warp; r < ch.rows; r += NW) {
                    const float2 all = join_factors(count, [&](int k) { return __ldcg(&part_of(k).ml[r]); },
                                                    [&](int k, float f) { factors[k][r] = f; }, final, ch.vscale, lane);
                    if (lane == 0) {
                        if (!final) to.ml[r] = all;
                        else if (p.lse) p.lse[ch.row0 + r] = lse_of(all);
                    }
                }
            cp_async_wait<0>();
            __syncthreads();
            const float* const parts = reinterpret_cast<const float*>(ring);
            auto columns = [&](int k, int x) {
                const int e = tid + x * NTHR;
                return reinterpret_cast<const float4*>(parts + k * Sh::PART + o_index(e / (DP / 4), e % (DP / 4) * 4, DP));
            };
            if constexpr (E == 1) {
                const int r = tid / (DP / 4);
                if (r < ch.rows)
                    join1(now, [&](int k) { return reinterpret_cast<const float2*>(parts + k * Sh::PART + ROWS * DP)[r]; },
                          [&](int k) { return columns(k, 0); }, m, l, o[0]);
            } else {
                join4<E>(now, all_columns, [&](int k, int x) { return factors[k0 + k][(tid + x * NTHR) / (DP / 4)]; }, columns, o);
            }
        }
#pragma unroll
        for (int x = 0; x < E; ++x) {
            const int e = tid + x * NTHR, r = e / (DP / 4), d = e % (DP / 4) * 4;
            if (r >= ch.rows || d >= p.c.D) continue;
            if (final) {
                if constexpr (E == 1) emit4<TQ>(p, ch.row0 + r, d, ch.vscale, m, l, o[x]);
                else put4(out_row(ch.row0 + r) + d, o[x]);
            } else {
                *reinterpret_cast<float4*>(to.o + o_index(r, d, DP)) = o[x];
                if (E == 1 && d == 0) to.ml[r] = make_float2(m, l);
            }
        }
    };
#pragma unroll 1
    for (int x = 0; x < 2; ++x) {
        if (!last_flag[x]) continue;
        __threadfence();
        const Chain& ch = chains[x == 0 ? NW : out_chain];
        const int c0 = ch.c0, count = ch.c1 - c0 + 1;
        const bool grouped = count > kDirect;
        const int first = grouped ? (blockIdx.x - c0) / kGroup * kGroup : 0, members = grouped ? min(kGroup, count - first) : count;
        // a group's result lies as far behind its first part as there are parts
        auto group_part = [&](int k) { return global_part(kMaxCtas + c0 + k * kGroup, k == 0); };
        gather(ch, members, [&](int k) { return global_part(c0 + first + k, first + k == 0); }, !grouped, group_part(first / kGroup));
        if (!grouped) continue;
        const int groups = (count + kGroup - 1) / kGroup;
        __threadfence();
        __syncthreads();
        if (tid == 0) all_flag = arrive(a.counters + 3 * kMaxCtas + c0, first / kGroup, groups);
        __syncthreads();
        __threadfence();
        const unsigned passed = tid == 0 ? pass_groups(ch) : 1u;     // the answer is looked at after the join
        if (all_flag) gather(ch, groups, group_part, true, Part{});
        groups_passed(ch, passed);
    }
}

// ---- launch -----------------------------------------------------------------------------------------------

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

// The rows of one layer as a matrix [rows_total][D], fetched in boxes of 16 rows by PITCH bytes.
template <typename TC, int PITCH>
bool layer_map(CUtensorMap* map, const luvc_kv_cache& c, void* pool, int layer, int rows_total) {
    EncodeTiledFn encode = encode_tiled_fn();
    if (!encode) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)c.D, (cuuint64_t)rows_total}, strides[1] = {(cuuint64_t)c.D * sizeof(TC)};
    const cuuint32_t box[2] = {PITCH / (cuuint32_t)sizeof(TC), 16u}, ones[2] = {1u, 1u};
    void* base = static_cast<unsigned char*>(pool) + (size_t)layer * rows_total * c.D * sizeof(TC);
    const CUtensorMapDataType type = sizeof(TC) == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : sizeof(TC) == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_UINT8;
    return encode(map, type, 2, base, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, PITCH == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename TQ, typename TC, int DPB, int NT>
int launch(const AttnProblem& p) {
    using Sh = Shape<TC, DPB, NT>;
    Args a;
    a.p = p;
    a.group = p.q_heads / p.c.heads;
    a.groups = (a.group + Sh::ROWS - 1) / Sh::ROWS;
    const int sms = std::min(sm_count(), kMaxCtas);
    if (!sms) return LUVC_ERR_CUDA;
    a.limit = (2147483647 - Sh::SNAP) / (p.c.heads * a.groups);
    a.one_grid = 1.f / sms;
    a.page_shift = (p.c.page_size & (p.c.page_size - 1)) ? -1 : __builtin_ctz(p.c.page_size);
    a.rows_total = p.c.pages * p.c.heads * p.c.page_size;
    a.counters = static_cast<unsigned*>(p.workspace);
    a.parts = reinterpret_cast<float*>(static_cast<unsigned char*>(p.workspace) + kCounterBytes);
    CUtensorMap kmap, vmap;
    if (!layer_map<TC, Sh::PITCH>(&kmap, p.c, p.c.k, p.layer, a.rows_total) ||
        !layer_map<TC, Sh::PITCH>(&vmap, p.c, p.c.v, p.layer, a.rows_total))
        return LUVC_ERR_CUDA;
    const size_t smem = 1024 + (size_t)Sh::NW * Sh::S * Sh::STAGE + (size_t)(p.n + 1) * sizeof(int);
    static std::atomic<unsigned long long> set{0};              // devices on which the kernel may use this much
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return LUVC_ERR_CUDA;
    if (dev > 63 || !((set.load(std::memory_order_relaxed) >> dev) & 1)) {
        if (cudaFuncSetAttribute(attn_decode_kernel<TQ, TC, DPB, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 1024 + Sh::NW * Sh::S * Sh::STAGE + (kKvMaxSeqs + 1) * (int)sizeof(int)) != cudaSuccess) {
            cudaGetLastError();
            return LUVC_ERR_CUDA;
        }
        if (dev <= 63) set.fetch_or(1ull << dev, std::memory_order_relaxed);
    }
    return launch_overlapped(attn_decode_kernel<TQ, TC, DPB, NT>, sms, 32 * Sh::NW, smem, p.stream, kmap, vmap, a);
}

template <typename TQ, typename TC, int DPB>
int launch_heads(const AttnProblem& p) {
    return p.q_heads / p.c.heads <= 8 ? launch<TQ, TC, DPB, 1>(p) : launch<TQ, TC, DPB, 2>(p);
}

// f32 caches with up to four query heads per key head run on the CUDA cores (measured, against the tensor cores: 32 / 32 heads of
// 128, 812 MB, 141 and 168 us; 16 / 16 of 64, 203 MB, 42.7 and 42.4, 38 MB 12.3 and 15.3; 32 / 8 of 128, 203 MB, 49 and 52; 8 / 8 of
// 256, 406 MB, 89 and 141), and all with rows longer than 512 bytes, four heads at a time (79 MB: 12 / 1 heads of 256 64 and 68 us, 8 / 1
// 50 and 53).  The others do not: 28 / 4 of 128, 158 MB, 63 us in this form, 46 on the tensor cores; 16 / 2 of 64, 40 MB, 24 and 16.
template <int DPB>
int launch_cores(const AttnProblem& p) {
    return p.q_heads == p.c.heads ? launch<float, float, DPB, -1>(p) : launch<float, float, DPB, -4>(p);
}

}  // namespace

size_t attn_workspace_bytes() { return kCounterBytes + (size_t)2 * kMaxCtas * 2 * kMaxPartBytes; }

int attn_decode(const AttnProblem& p) {
    const int bytes = p.c.D * (int)kv_elem_size(p.c.dtype);
    if (p.c.dtype == LUVC_F32 && (p.q_heads <= 4 * p.c.heads || bytes > 512))
        return bytes <= 256 ? launch_cores<256>(p) : bytes <= 512 ? launch_cores<512>(p) : launch_cores<1024>(p);
    if (p.c.dtype == LUVC_F32)
        return bytes <= 256 ? launch_heads<float, float, 256>(p) : launch_heads<float, float, 512>(p);
    if (p.c.dtype == LUVC_BF16)
        return bytes <= 128 ? launch_heads<__nv_bfloat16, __nv_bfloat16, 128>(p) : bytes <= 256 ? launch_heads<__nv_bfloat16, __nv_bfloat16, 256>(p)
                                                                                               : launch_heads<__nv_bfloat16, __nv_bfloat16, 512>(p);
    // rows of 64 bytes halve the conversions and products (16 / 16 heads of 64, 79 MB: 28.0 us, as rows of 128 bytes 35.1)
    return bytes <= 64 ? launch_heads<__nv_bfloat16, __nv_fp8_e4m3, 64>(p) : bytes <= 128 ? launch_heads<__nv_bfloat16, __nv_fp8_e4m3, 128>(p) : launch_heads<__nv_bfloat16, __nv_fp8_e4m3, 256>(p);
}

}  // namespace luvc
