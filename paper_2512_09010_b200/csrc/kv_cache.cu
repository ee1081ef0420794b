// Paged key-value cache: pages for new tokens, rows written, sequences forked, freed and compacted.
//
// Books.  A sequence is a slot: lengths[slot] tokens in the pages table[slot][0 ..].  refs[page] counts the
// sequences that hold a page, 0 is free, and a call takes the free pages with the lowest numbers, in the order
// of its sequences; so the books after a call follow from those before it, whatever the timing.  A call that
// takes pages first runs one CTA over the books (kv_plan_kernel): it works out what each sequence needs, finds
// the free pages by an ordered scan of refs, and either commits everything or leaves the books as they were and
// reports in the status word.  Rows are then copied by a second, wide kernel (kv_move_kernel).  Nothing is ever
// copied in place: a compacted sequence gets new pages, so no row is overwritten while it is still to be read,
// every row can move at the same time, and a page that other sequences share is never written.
//
// Layout.  A page holds, per layer and head, page_size consecutive rows of D elements ([layer][page][head][slot][D]):
// the attention kernel reads a head's part of a page as one contiguous piece.

#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include "luvc_internal.h"

namespace luvc {
namespace {

constexpr int kPlanThreads = 1024, kPlanWarps = kPlanThreads / 32;
constexpr int kPerThread = 16;                              // pages a thread looks at per sweep over refs
constexpr int kSweep = kPlanThreads * kPerThread;
constexpr int kCounts = kPerThread * kPlanWarps;            // one count of free pages per ballot
constexpr int kClaimed = -1;                                // lengths[] of a slot that the running call has claimed

__device__ __forceinline__ bool stopped(const int* status) { return *reinterpret_cast<const volatile int*>(status) != 0; }

__device__ __forceinline__ int ceil_div(int a, int b) { return (int)(((long long)a + b - 1) / b); }

// The plan's result for kv_move_kernel, in the call's workspace.
struct MoveList {
    int* total;      // pages to fill
    int2* items;     // [total] (sequence of the call, page index within it)
    int* old;        // [n, max_pages] compact: the sequences' pages before the call
};

MoveList move_list(void* ws, const luvc_kv_cache& c, int n) {
    unsigned char* p = static_cast<unsigned char*>(ws);
    MoveList m;
    m.total = reinterpret_cast<int*>(p);
    m.items = reinterpret_cast<int2*>(p + 256);
    m.old = reinterpret_cast<int*>(p + 256 + align_up((size_t)n * c.max_pages * sizeof(int2)));
    return m;
}

enum PlanKind { kReserve, kFork, kCompact };

struct PlanArgs {
    luvc_kv_cache c;
    const int32_t* seqs;     // fork: the destinations
    const int32_t* src;      // fork
    const int32_t* counts;   // reserve: tokens to add; compact: kept tokens of the block (may be null)
    const int32_t *first, *span, *idx;
    int n, keep;
    MoveList move;
    int* status;
};

// Shared memory of the plan; start / from / len have n + 1, n and n entries.
struct PlanShared {
    int error;               // highest luvc_status found
    int total;               // pages to take
    unsigned long long wide_total;
    int warp_sum[kPlanWarps];
    int count[kCounts];
    int* start;              // exclusive sums of the pages the sequences need
    int* from;               // first page index of each sequence that is to be taken
    int* len;                // length before the call; kClaimed where the slot was not obtained
};

// Exclusive scan over the block of one value per thread; the total goes to every thread.
__device__ int block_scan(int v, int* warp_sum, int* total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int x = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(~0u, x, d);
        if (lane >= d) x += y;
    }
    __syncthreads();                                        // warp_sum of an earlier scan has been read
    if (lane == 31) warp_sum[warp] = x;
    __syncthreads();
    if (warp == 0) {
        int s = warp_sum[lane];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int y = __shfl_up_sync(~0u, s, d);
            if (lane >= d) s += y;
        }
        warp_sum[lane] = s;
    }
    __syncthreads();
    *total = warp_sum[kPlanWarps - 1];
    return x - v + (warp ? warp_sum[warp - 1] : 0);
}

// start[i] holds the pages sequence i needs; afterwards start[] is their exclusive sum, start[n] the total.
// More than the pool has is an error; the sum is checked in 64 bits first, so that the scan cannot overflow.
__device__ void scan_needs(PlanShared& s, int n, int pages) {
    unsigned long long mine = 0;
    for (int i = threadIdx.x; i < n; i += kPlanThreads) mine += (unsigned)s.start[i];
    if (mine) atomicAdd(&s.wide_total, mine);
    __syncthreads();
    const bool fits = s.wide_total <= (unsigned long long)pages;
    int base = 0;
    for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
        const int i = i0 + threadIdx.x;
        int sum;
        const int before = block_scan(fits && i < n ? s.start[i] : 0, s.warp_sum, &sum);
        if (i < n) s.start[i] = base + before;
        base += sum;
    }
    if (threadIdx.x == 0) {
        s.start[n] = base; s.total = base;
        if (!fits) atomicMax(&s.error, (int)LUVC_ERR_PAGES);
    }
    __syncthreads();
}

// Hands the `total` lowest free pages to the sequences: give(i, page index, page).  False (nothing given) if
// there are too few.  All threads call it.
template <typename F>
__device__ bool take_pages(PlanShared& s, int* refs, int pages, int n, F give) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, total = s.total;
    unsigned free_mask[kPerThread];                         // ballot of this warp, per sweep row
    int sum = 0;
    auto sweep = [&](int c0) {                              // count[] = exclusive sums in page order
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) {
            const int page = c0 + k * kPlanThreads + threadIdx.x;
            const bool is_free = page < pages && refs[page] == 0;
            free_mask[k] = __ballot_sync(~0u, is_free);
        }
        __syncthreads();                                    // count[] of the sweep before has been used
        if (lane == 0)
#pragma unroll
            for (int k = 0; k < kPerThread; ++k) s.count[k * kPlanWarps + warp] = __popc(free_mask[k]);
        __syncthreads();
        const int mine = threadIdx.x < kCounts ? s.count[threadIdx.x] : 0;
        const int before = block_scan(mine, s.warp_sum, &sum);
        if (threadIdx.x < kCounts) s.count[threadIdx.x] = before;
        __syncthreads();
    };
    auto hand_out = [&](int c0, int base) {
#pragma unroll
        for (int k = 0; k < kPerThread; ++k) {
            if (!((free_mask[k] >> lane) & 1u)) continue;
            const int rank = base + s.count[k * kPlanWarps + warp] + __popc(free_mask[k] & ((1u << lane) - 1u));
            if (rank >= total) continue;
            int lo = 0, hi = n;                             // start[lo] <= rank < start[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s.start[mid] <= rank) lo = mid; else hi = mid;
            }
            const int page = c0 + k * kPlanThreads + threadIdx.x;
            refs[page] = 1;
            give(lo, s.from[lo] + rank - s.start[lo], rank, page);
        }
    };
    if (total == 0) return true;
    int found = 0, c0 = 0;
    for (; c0 < pages; c0 += kSweep) {
        sweep(c0);
        found += sum;
        if (found >= total) break;
    }
    if (found < total) return false;
    if (c0 == 0) {
        hand_out(0, 0);                                     // one sweep saw them all
    } else {
        int base = 0;
        for (int c = 0; c <= c0; c += kSweep) {
            sweep(c);
            hand_out(c, base);
            base += sum;
        }
    }
    return true;
}

// Number of leading entries with idx[j] == j of a strictly ascending list (one warp; the predicate is monotone).
__device__ int identity_prefix(const int32_t* idx, int count, int lane) {
    int lo = 0, hi = count;                                 // the answer is in [lo, hi]
    bool gallop = true;                                     // a prune seldom keeps a long run at the start of its block
    while (lo < hi) {
        int probe;                                          // entry whose truth extends the prefix to probe + 1
        if (gallop) {
            probe = lo + (lane < 30 ? (1 << lane) - 1 : 0x3fffffff);
        } else {
            const int step = (hi - lo + 31) / 32;
            probe = lo + (lane + 1) * step - 1;
        }
        gallop = false;
        const bool yes = probe >= lo && probe < hi && idx[probe] == probe;
        const unsigned m = __ballot_sync(~0u, yes);
        const int good = __popc(m);                         // probes ascend: the true ones are the first `good`
        const int last = good ? __shfl_sync(~0u, probe, good - 1) : lo - 1;
        const int next = __shfl_sync(~0u, probe, good < 32 ? good : 31);
        if (good < 32 && next < hi && next >= lo) hi = next;
        lo = last + 1;
    }
    return lo;
}

template <PlanKind KIND>
__global__ void __launch_bounds__(kPlanThreads) kv_plan_kernel(const __grid_constant__ PlanArgs a) {
    extern __shared__ int dyn[];
    __shared__ PlanShared s;
    const luvc_kv_cache& c = a.c;
    const int n = a.n, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        s.error = 0; s.wide_total = 0;
        s.start = dyn; s.from = dyn + n + 1; s.len = dyn + 2 * n + 1;
        if (KIND != kReserve) *a.move.total = 0;
    }
    if (__syncthreads_or(stopped(a.status))) return;
    const long long most = (long long)c.max_pages * c.page_size;
    auto slot_of = [&](int i) { return a.seqs ? a.seqs[i] : i; };

    // what each sequence needs; its slot is claimed, so that one named twice is noticed
    if (KIND == kFork) {
        for (int i = tid; i < n; i += kPlanThreads) {
            const int src = a.src[i];
            int len = -1;
            if (src >= 0 && src < c.slots) len = c.lengths[src];
            if (len < 0 || len > most) { atomicMax(&s.error, (int)LUVC_ERR_SHAPE); len = 0; }
            s.from[i] = len / c.page_size;
            s.start[i] = len % c.page_size ? 1 : 0;
            s.len[i] = len;
        }
        __syncthreads();                                    // a source that is also a destination has been read
        for (int i = tid; i < n; i += kPlanThreads) {
            const int dst = slot_of(i);
            const int was = dst >= 0 && dst < c.slots ? atomicCAS(&c.lengths[dst], 0, kClaimed) : kClaimed;
            if (was != 0) {
                atomicMax(&s.error, was == kClaimed ? (int)LUVC_ERR_SHAPE : (int)LUVC_ERR_TARGET);
                s.len[i] = kClaimed;
            }
        }
    } else if (KIND == kReserve) {
        for (int i = tid; i < n; i += kPlanThreads) {
            const int slot = slot_of(i), add = a.counts[i];
            int len = kClaimed;
            if (slot >= 0 && slot < c.slots) len = a.seqs ? atomicExch(&c.lengths[slot], kClaimed) : c.lengths[slot];
            s.len[i] = len;
            int need = 0, have = 0;
            if (len < 0 || add < 0) {
                atomicMax(&s.error, (int)LUVC_ERR_SHAPE);
            } else if ((long long)len + add > most) {
                atomicMax(&s.error, (int)LUVC_ERR_PAGES);
            } else {
                have = ceil_div(len, c.page_size);
                need = ceil_div(len + add, c.page_size) - have;
            }
            s.from[i] = have;
            s.start[i] = need;
        }
    } else {
        for (int i = warp; i < n; i += kPlanWarps) {
            const int slot = slot_of(i);
            int len = kClaimed;
            if (lane == 0 && slot >= 0 && slot < c.slots)
                len = a.seqs ? atomicExch(&c.lengths[slot], kClaimed) : c.lengths[slot];
            const int first = a.first[i], span = a.span[i], count = a.counts ? a.counts[i] : a.keep;
            len = __shfl_sync(~0u, len, 0);
            int still = 0, need = 0, bad = 0;
            if (len < 0 || len > most) bad = LUVC_ERR_SHAPE;
            else if (first < 0 || span < 0 || (long long)first + span > len || count < 0 || count > span || count > a.keep)
                bad = LUVC_ERR_KEEP;
            if (!bad) {
                const int now = len - span + count;
                const int same = count == span ? now : first + identity_prefix(a.idx + (long long)i * a.keep, count, lane);
                still = same / c.page_size;
                need = ceil_div(now, c.page_size) - still;
                for (int p = still + lane; p < ceil_div(len, c.page_size); p += 32)
                    a.move.old[(long long)i * c.max_pages + p] = c.table[(long long)slot * c.max_pages + p];
            }
            if (lane == 0) {
                if (bad) atomicMax(&s.error, bad);
                s.len[i] = len; s.from[i] = still; s.start[i] = need;
            }
        }
    }
    __syncthreads();
    scan_needs(s, n, c.pages);
    bool ok = s.error == 0;
    if (ok) {
        ok = take_pages(s, c.refs, c.pages, n, [&](int i, int index, int rank, int page) {
            c.table[(long long)slot_of(i) * c.max_pages + index] = page;
            if (KIND != kReserve) a.move.items[rank] = make_int2(i, index);
        });
        if (!ok && tid == 0) s.error = LUVC_ERR_PAGES;
        __syncthreads();
    }
    if (!ok) {                                              // give the claimed slots back
        for (int i = tid; i < n; i += kPlanThreads) {
            if (s.len[i] == kClaimed) continue;
            if (KIND == kFork) c.lengths[slot_of(i)] = 0;
            else if (a.seqs) c.lengths[slot_of(i)] = s.len[i];
        }
        if (tid == 0) *a.status = s.error;
        return;
    }
    // commit: lengths, and the pages that were shared or given up (several warps per sequence when there are few)
    for (int i = tid; i < n; i += kPlanThreads) {
        int now = s.len[i];
        if (KIND == kReserve) now += a.counts[i];
        if (KIND == kCompact) now += (a.counts ? a.counts[i] : a.keep) - a.span[i];
        c.lengths[slot_of(i)] = now;
    }
    if (KIND == kReserve) return;
    if (tid == 0) *a.move.total = s.total;
    int team = 1;
    while (team < kPlanWarps && 2 * team * n <= kPlanWarps) team *= 2;
    for (int i = warp / team; i < n; i += kPlanWarps / team) {
        int32_t* row = c.table + (long long)slot_of(i) * c.max_pages;
        const int lane0 = (warp % team) * 32 + lane;
        if (KIND == kFork) {
            const int32_t* from = c.table + (long long)a.src[i] * c.max_pages;
            for (int p = lane0; p < s.from[i]; p += team * 32) {
                const int page = from[p];
                row[p] = page;
                if (page >= 0 && page < c.pages) atomicAdd(&c.refs[page], 1);
            }
        } else {
            const int before = ceil_div(s.len[i], c.page_size);
            const int now = s.from[i] + s.start[i + 1] - s.start[i];
            for (int p = s.from[i] + lane0; p < before; p += team * 32) {
                const int page = a.move.old[(long long)i * c.max_pages + p];
                if (page >= 0 && page < c.pages) atomicSub(&c.refs[page], 1);
                if (p >= now) row[p] = -1;
            }
        }
    }
}

struct MoveArgs {
    luvc_kv_cache c;
    const int32_t* seqs;     // fork: the destinations
    const int32_t* src;      // fork: the sources; null: compact
    const int32_t *first, *span, *idx, *counts;
    int keep;
    int es;                  // bytes of an element
    MoveList move;
    int* status;
};

// Fills the pages of the plan's list.  A work item is one page for up to kLanes (layer, K or V, head) triples; a thread
// copies 16 bytes of a row for all of them, so a row's place is looked up once for kLanes copies and as many loads
// are in flight per thread.
constexpr int kMoveLanes = 8, kMoveThreads = 256;

template <bool FORK>
__global__ void __launch_bounds__(kMoveThreads) kv_move_kernel(const __grid_constant__ MoveArgs a) {
    const luvc_kv_cache& c = a.c;
    const int triples = c.layers * 2 * c.heads, groups = (triples + kMoveLanes - 1) / kMoveLanes;
    const long long work = (long long)*a.move.total * groups;
    const int ps = c.page_size, units = c.D * a.es / 16;
    const size_t head_bytes = (size_t)ps * c.D * a.es, layer_bytes = (size_t)c.pages * c.heads * head_bytes;
    for (long long w = blockIdx.x; w < work; w += gridDim.x) {
        const int2 item = a.move.items[w / groups];
        const int g = (int)(w % groups) * kMoveLanes;
        const int i = item.x, p = item.y;
        const int slot = a.seqs ? a.seqs[i] : i;
        const int rows = min(ps, c.lengths[slot] - p * ps);
        const int to_page = c.table[(long long)slot * c.max_pages + p];
        unsigned char* base[kMoveLanes];
#pragma unroll
        for (int k = 0; k < kMoveLanes; ++k) {
            const int t = min(g + k, triples - 1), layer = t / (2 * c.heads), rest = t % (2 * c.heads);
            base[k] = static_cast<unsigned char*>(rest >= c.heads ? c.v : c.k) + layer * layer_bytes +
                      (rest % c.heads) * head_bytes;
        }
        for (int u = threadIdx.x; u < rows * units; u += kMoveThreads) {
            const int r = u / units, off = (u - r * units) * 16;
            int from = p * ps + r;                          // token of the old sequence that becomes row r of this page
            int from_page;
            if (FORK) {
                from_page = c.table[(long long)a.src[i] * c.max_pages + p];
            } else {
                const int first = a.first[i], span = a.span[i], count = a.counts ? a.counts[i] : a.keep;
                if (from >= first + count) {
                    from += span - count;
                } else if (from >= first) {
                    const int e = a.idx[(long long)i * a.keep + from - first];
                    const int in = min(max(e, 0), span - 1);
                    if (in != e) *a.status = LUVC_ERR_KEEP;
                    from = first + in;
                }
                from_page = a.move.old[(long long)i * c.max_pages + from / ps];
            }
            if (from_page < 0 || from_page >= c.pages || to_page < 0 || to_page >= c.pages) continue;
            const size_t src = (size_t)from_page * c.heads * head_bytes + (size_t)(from % ps) * c.D * a.es + off;
            const size_t dst = (size_t)to_page * c.heads * head_bytes + (size_t)r * c.D * a.es + off;
            uint4 v[kMoveLanes];
#pragma unroll
            for (int k = 0; k < kMoveLanes; ++k) v[k] = __ldg(reinterpret_cast<const uint4*>(base[k] + src));
#pragma unroll
            for (int k = 0; k < kMoveLanes; ++k)
                if (g + k < triples) *reinterpret_cast<uint4*>(base[k] + dst) = v[k];
        }
    }
}

__global__ void __launch_bounds__(128) kv_free_kernel(luvc_kv_cache c, const int32_t* seqs, int* status) {
    __shared__ int len;
    if (__syncthreads_or(stopped(status))) return;
    const int slot = seqs ? seqs[blockIdx.x] : (int)blockIdx.x;
    if (slot < 0 || slot >= c.slots) {
        if (threadIdx.x == 0) *status = LUVC_ERR_SHAPE;
        return;
    }
    if (threadIdx.x == 0) len = atomicExch(&c.lengths[slot], 0);
    __syncthreads();
    const int pages = min(ceil_div(max(len, 0), c.page_size), c.max_pages);
    for (int p = threadIdx.x; p < pages; p += blockDim.x) {
        int32_t* entry = c.table + (long long)slot * c.max_pages + p;
        const int page = *entry;
        *entry = -1;
        if (page >= 0 && page < c.pages) atomicSub(&c.refs[page], 1);
    }
}

struct WriteArgs {
    luvc_kv_cache c;
    int layer, n, tokens;
    const int32_t *seqs, *starts, *sizes;
    const void *k, *v;
    long long k_stride, v_stride;
    int* status;
};

template <typename T> struct Vec;                           // the elements of 16 input bytes, as floats
template <> struct Vec<float> {
    static constexpr int N = 4;
    static __device__ void load(const float* p, float (&f)[8]) {
        const float4 x = *reinterpret_cast<const float4*>(p);
        f[0] = x.x; f[1] = x.y; f[2] = x.z; f[3] = x.w;
    }
};
template <> struct Vec<__nv_bfloat16> {
    static constexpr int N = 8;
    static __device__ void load(const __nv_bfloat16* p, float (&f)[8]) {
        const uint4 x = *reinterpret_cast<const uint4*>(p);
        const unsigned w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            f[2 * q] = __uint_as_float(w[q] << 16);
            f[2 * q + 1] = __uint_as_float(w[q] & 0xffff0000u);
        }
    }
};

__device__ __forceinline__ void store_row(float* p, const float (&f)[8], float) {
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
}
__device__ __forceinline__ void store_row(__nv_bfloat16* p, const float (&f)[8], float) {
    unsigned r[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const __nv_bfloat162 pr = __floats2bfloat162_rn(f[2 * q], f[2 * q + 1]);
        r[q] = *reinterpret_cast<const unsigned*>(&pr);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(r[0], r[1], r[2], r[3]);
}
// x / scale, saturated, to nearest even: a true division, so that the stored value is the nearest one to the quotient
__device__ __forceinline__ void store_row(__nv_fp8_e4m3* p, const float (&f)[8], float scale) {
    unsigned r[2] = {0, 0};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float2 x = make_float2(f[2 * q] / scale, f[2 * q + 1] / scale);
        r[q >> 1] |= (unsigned)__nv_cvt_float2_to_fp8x2(x, __NV_SATFINITE, __NV_E4M3) << (16 * (q & 1));
    }
    *reinterpret_cast<uint2*>(p) = make_uint2(r[0], r[1]);
}

constexpr int kWriteTokens = 16, kWriteThreads = 256;

template <typename TI, typename TC>
__global__ void __launch_bounds__(kWriteThreads) kv_write_kernel(const __grid_constant__ WriteArgs a) {
    constexpr int V = Vec<TI>::N;
    __shared__ long long row_of[kWriteTokens];              // row of head 0 in the layer's pool, -1: not written
    __shared__ float bias_of[kWriteTokens];
    const luvc_kv_cache& c = a.c;
    if (__syncthreads_or(stopped(a.status))) return;
    const int t0 = blockIdx.x * kWriteTokens, ps = c.page_size;
    if (threadIdx.x < kWriteTokens) {
        const int t = t0 + threadIdx.x;
        long long row = -1;
        if (t < a.tokens) {
            int i = t, behind = 1;                          // tokens of the sequence from this one to its end
            if (a.starts) {
                int lo = 0, hi = a.n;                       // starts[lo] <= t < starts[hi]
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (a.starts[mid] <= t) lo = mid; else hi = mid;
                }
                i = lo;
                behind = a.starts[lo + 1] - t;
            }
            const int slot = a.seqs ? a.seqs[i] : i;
            const int pos = slot >= 0 && slot < c.slots ? c.lengths[slot] - behind : -1;
            if (behind >= 1 && pos >= 0 && pos / ps < c.max_pages) {
                const int page = c.table[(long long)slot * c.max_pages + pos / ps];
                if (page >= 0 && page < c.pages) row = (long long)page * c.heads * ps + pos % ps;
            }
            if (row < 0) *a.status = LUVC_ERR_SHAPE;
            bias_of[threadIdx.x] = a.sizes ? logf((float)a.sizes[t]) : 0.f;
        }
        row_of[threadIdx.x] = row;
    }
    __syncthreads();
    const int per_row = c.D / V, per_token = c.heads * per_row;
    const long long layer_row = (long long)a.layer * c.pages * c.heads * ps;
    TC* const kd = static_cast<TC*>(c.k);
    TC* const vd = static_cast<TC*>(c.v);
    for (int e = threadIdx.x; e < kWriteTokens * per_token; e += kWriteThreads) {
        const int t = e / per_token, in = e - t * per_token, h = in / per_row;
        const long long row = row_of[t];
        if (row < 0) continue;
        const long long dst = (layer_row + row + (long long)h * ps) * c.D + (long long)(in - h * per_row) * V;
        float k[8], v[8];
        Vec<TI>::load(static_cast<const TI*>(a.k) + (t0 + t) * a.k_stride + (long long)in * V, k);
        Vec<TI>::load(static_cast<const TI*>(a.v) + (t0 + t) * a.v_stride + (long long)in * V, v);
        const float b = bias_of[t];
        if (a.sizes)
#pragma unroll
            for (int q = 0; q < V; ++q) v[q] += b;
        const float ks = c.k_scale ? c.k_scale[a.layer * c.heads + h] : 1.f;
        const float vs = c.v_scale ? c.v_scale[a.layer * c.heads + h] : 1.f;
        store_row(kd + dst, k, ks);
        store_row(vd + dst, v, vs);
    }
}

int sm_count() {
    static int sms = 0;
    if (!sms) {
        int dev = 0;
        cudaGetDevice(&dev);
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    }
    return sms;
}

template <PlanKind KIND>
int launch_plan(const PlanArgs& a, cudaStream_t stream) {
    const size_t smem = (size_t)(3 * a.n + 1) * sizeof(int);
    if (smem > 40 * 1024) cudaFuncSetAttribute(kv_plan_kernel<KIND>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    kv_plan_kernel<KIND><<<1, kPlanThreads, smem, stream>>>(a);
    count_launch();
    return cudaGetLastError() == cudaSuccess ? LUVC_OK : LUVC_ERR_CUDA;
}

template <bool FORK>
int launch_move(const MoveArgs& a, cudaStream_t stream) {
    kv_move_kernel<FORK><<<4 * sm_count(), kMoveThreads, 0, stream>>>(a);
    count_launch();
    return cudaGetLastError() == cudaSuccess ? LUVC_OK : LUVC_ERR_CUDA;
}

}  // namespace

size_t kv_elem_size(int dtype) { return dtype == LUVC_F32 ? 4 : dtype == LUVC_BF16 ? 2 : 1; }

size_t kv_workspace_bytes(const luvc_kv_cache& c, int n) {
    return 256 + align_up((size_t)n * c.max_pages * sizeof(int2)) + align_up((size_t)n * c.max_pages * sizeof(int));
}

int kv_reserve(const luvc_kv_cache& c, const int32_t* seqs, int n, const int32_t* counts, int* status, cudaStream_t stream) {
    PlanArgs a = {};
    a.c = c; a.seqs = seqs; a.n = n; a.counts = counts; a.status = status;
    return launch_plan<kReserve>(a, stream);
}

int kv_fork(const luvc_kv_cache& c, const int32_t* src, const int32_t* dst, int n, void* ws, int* status, cudaStream_t stream) {
    PlanArgs a = {};
    a.c = c; a.seqs = dst; a.src = src; a.n = n; a.move = move_list(ws, c, n); a.status = status;
    const int rc = launch_plan<kFork>(a, stream);
    if (rc) return rc;
    MoveArgs m = {};
    m.c = c; m.seqs = dst; m.src = src; m.es = (int)kv_elem_size(c.dtype); m.move = a.move; m.status = status;
    return launch_move<true>(m, stream);
}

int kv_compact(const luvc_kv_cache& c, const int32_t* seqs, int n, const int32_t* first, const int32_t* span, const int32_t* idx,
               int keep, const int32_t* counts, void* ws, int* status, cudaStream_t stream) {
    PlanArgs a = {};
    a.c = c; a.seqs = seqs; a.n = n; a.first = first; a.span = span; a.idx = idx; a.keep = keep; a.counts = counts;
    a.move = move_list(ws, c, n); a.status = status;
    const int rc = launch_plan<kCompact>(a, stream);
    if (rc) return rc;
    MoveArgs m = {};
    m.c = c; m.seqs = seqs; m.first = first; m.span = span; m.idx = idx; m.counts = counts; m.keep = keep;
    m.es = (int)kv_elem_size(c.dtype); m.move = a.move; m.status = status;
    return launch_move<false>(m, stream);
}

int kv_free(const luvc_kv_cache& c, const int32_t* seqs, int n, int* status, cudaStream_t stream) {
    kv_free_kernel<<<n, 128, 0, stream>>>(c, seqs, status);
    count_launch();
    return cudaGetLastError() == cudaSuccess ? LUVC_OK : LUVC_ERR_CUDA;
}

int kv_write(const luvc_kv_cache& c, int layer, const int32_t* seqs, int n, const void* k, const void* v, long long k_stride,
             long long v_stride, int tokens, const int32_t* starts, const int32_t* sizes, int* status, cudaStream_t stream) {
    WriteArgs a;
    a.c = c; a.layer = layer; a.n = n; a.tokens = tokens; a.seqs = seqs; a.starts = starts; a.sizes = sizes;
    a.k = k; a.v = v; a.k_stride = k_stride; a.v_stride = v_stride; a.status = status;
    const int grid = (tokens + kWriteTokens - 1) / kWriteTokens;
    if (c.dtype == LUVC_F32) kv_write_kernel<float, float><<<grid, kWriteThreads, 0, stream>>>(a);
    else if (c.dtype == LUVC_BF16) kv_write_kernel<__nv_bfloat16, __nv_bfloat16><<<grid, kWriteThreads, 0, stream>>>(a);
    else kv_write_kernel<__nv_bfloat16, __nv_fp8_e4m3><<<grid, kWriteThreads, 0, stream>>>(a);
    count_launch();
    return cudaGetLastError() == cudaSuccess ? LUVC_OK : LUVC_ERR_CUDA;
}

}  // namespace luvc
