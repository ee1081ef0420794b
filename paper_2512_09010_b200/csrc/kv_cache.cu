// Paged key-value cache: pages for new tokens, rows written, sequences forked, freed and compacted.
//
// Books.  A sequence is a slot: lengths[slot] tokens in the pages table[slot][0 ..].  refs[page] counts the
// sequences that hold a page, 0 is free, and a call takes the free pages with the lowest numbers, in the order
// of its sequences; so the books after a call follow from those before it, whatever the timing.  A call that
// takes pages first runs one CTA over the books (kv_plan_kernel): it works out what each sequence needs, finds
// the free pages by an ordered scan of refs, and either commits or leaves the books as they were and reports in
// the status word.  What is left then is wide and has no order (kv_move_kernel): rows to copy, pages to share
// or to give back.  Nothing is ever copied in place: a compacted sequence gets new pages, so no row is
// overwritten while it is still to be read, every row can move at the same time, and a page that other sequences share is
// never written.  The kernels are launched with overlap (programmatic dependent launch): the books are so little
// work that the gaps between launches would be as long as the kernels.
//
// Layout.  A page holds, per layer and head, page_size consecutive rows of D elements ([layer][page][head][slot][D]):
// the attention kernel reads a head's part of a page as one contiguous piece.

#include <cuda_bf16.h>
#include <cuda_fp8.h>

#include <atomic>

#include "luvc_internal.h"
#include "sm100_ptx.cuh"

namespace luvc {
namespace {

using namespace ptx;

constexpr int kPerLane = 8;                                 // pages a lane looks at per sweep over refs
constexpr int kWarpPages = 32 * kPerLane;
constexpr int kMaxNeed = 1 << 26;                           // pages one call takes for one sequence (2^30 tokens at least)
constexpr int kClaimed = -1;                                // lengths[] of a slot that the running call has claimed

__device__ __forceinline__ int status_of(int* status) { return *reinterpret_cast<volatile int*>(status); }

// For a call that has found the status word set and does nothing: rows that a write has skipped become a plain status, at which further
// writes stop too.
__device__ __forceinline__ void stop_writes(int* status, int word) {
    if (word == kRowsSkipped && threadIdx.x == 0) *status = word & kStatusMask;
}

__device__ __forceinline__ int ceil_div(int a, int b) { return (int)(((unsigned)a + (unsigned)b - 1u) / (unsigned)b); }

// The plan's result for kv_move_kernel, in the call's workspace.
struct MoveList {
    int* head;       // [0]: pages to fill; [1]: 1 if the plan was committed
    int2* items;     // [pages to fill] (sequence of the call, page index within it)
    int* len;        // [n] tokens before the call
    int* from;       // [n] first page that is not as before
    int* old;        // [n, max_pages] compact: the sequences' pages before the call, from `from` on
};

MoveList move_list(void* ws, const luvc_kv_cache& c, int n) {
    unsigned char* p = static_cast<unsigned char*>(ws);
    MoveList m;
    m.head = reinterpret_cast<int*>(p);
    m.len = reinterpret_cast<int*>(p += 256);
    m.from = reinterpret_cast<int*>(p += align_up((size_t)n * sizeof(int)));
    m.items = reinterpret_cast<int2*>(p += align_up((size_t)n * sizeof(int)));
    m.old = reinterpret_cast<int*>(p + align_up((size_t)n * c.max_pages * sizeof(int2)));
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

// Shared memory of the plan, run by THREADS threads; the arrays have n + 1, n, n and n entries.
template <int THREADS>
struct PlanShared {
    static constexpr int WARPS = THREADS / 32, SWEEP = WARPS * kWarpPages;
    int error;                              // highest luvc_status found
    int page_count[2][WARPS];               // free pages each warp saw in a sweep (two sweeps alternate)
    unsigned need_sum[WARPS];
    int list[SWEEP];                        // free pages of a sweep, in order
    int* start;                             // pages the sequences need; then their exclusive sums
    int* from;                              // first page index of each sequence that is to be taken
    int* len;                               // length before the call; kClaimed where the slot was not obtained
    int* slot;
};

template <typename T>
__device__ __forceinline__ T warp_inclusive(T x, int lane) {
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const T y = __shfl_up_sync(~0u, x, d);
        if (lane >= d) x += y;
    }
    return x;
}

// start[i] holds the pages sequence i needs (at most kMaxNeed each); afterwards start[] is their exclusive sum, start[n] the
// total, which is returned (-1: more than the pool has; the sum over warps is formed in 64 bits, and only one that fits is
// used).  take_pages has a barrier before it reads start[].
template <int THREADS>
__device__ int scan_needs(PlanShared<THREADS>& s, int n, int pages) {
    constexpr int WARPS = THREADS / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (n <= 32) {                                          // every warp for itself; the first one writes
        const unsigned v = lane < n ? s.start[lane] : 0, x = warp_inclusive(v, lane), all = __shfl_sync(~0u, x, 31);
        __syncthreads();                                    // all have read the needs
        if (warp == 0 && lane < n) s.start[lane] = (int)(x - v);
        if (threadIdx.x == 0) s.start[n] = (int)all;
        return all > (unsigned)pages ? -1 : (int)all;
    }
    unsigned long long base = 0;
    for (int i0 = 0; i0 < n; i0 += THREADS) {
        const int i = i0 + threadIdx.x;
        const unsigned v = i < n ? s.start[i] : 0, x = warp_inclusive(v, lane);
        if (lane == 31) s.need_sum[warp] = x;
        __syncthreads();
        const unsigned long long all = warp_inclusive(lane < WARPS ? (unsigned long long)s.need_sum[lane] : 0ull, lane);
        const unsigned long long before = __shfl_sync(~0u, all, (warp + 31) & 31);
        if (i < n) s.start[i] = (int)(base + (warp ? before : 0) + x - v);
        base += __shfl_sync(~0u, all, 31);
        if (n > THREADS) __syncthreads();              // need_sum is written again
    }
    if (threadIdx.x == 0) s.start[n] = (int)base;
    return base > (unsigned long long)pages ? -1 : (int)base;
}

// One sweep over SWEEP pages from c0 on: every warp looks at kWarpPages consecutive ones.
struct Sweep {
    unsigned mask[kPerLane];                // free pages, one ballot per 32
    int first;                              // free pages of the sweep before this warp's
    int sum;
};

__device__ __forceinline__ void sweep_load(const int32_t* refs, int pages, int c0, int (&r)[kPerLane]) {
    const int at = c0 + (threadIdx.x >> 5) * kWarpPages + (threadIdx.x & 31);
#pragma unroll
    for (int k = 0; k < kPerLane; ++k) r[k] = at + 32 * k < pages ? refs[at + 32 * k] : 1;
}

template <int THREADS>
__device__ __forceinline__ void sweep_count(PlanShared<THREADS>& s, const int (&r)[kPerLane], int turn, Sweep& w) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int mine = 0;
#pragma unroll
    for (int k = 0; k < kPerLane; ++k) {
        w.mask[k] = __ballot_sync(~0u, r[k] == 0);
        mine += __popc(w.mask[k]);
    }
    if (lane == 0) s.page_count[turn & 1][warp] = mine;
    __syncthreads();
    const int all = warp_inclusive(lane < THREADS / 32 ? s.page_count[turn & 1][lane] : 0, lane);
    w.sum = __shfl_sync(~0u, all, 31);
    w.first = __shfl_sync(~0u, all, warp) - mine;
}

// Hands the `total` lowest free pages to the sequences: give(i, page index, rank, page).  False (nothing given) if there are too
// few.  r: the first sweep's counts, loaded ahead.  All threads call it.
template <int THREADS, typename F>
__device__ __forceinline__ bool take_pages(PlanShared<THREADS>& s, int32_t* refs, int pages, int n, int total, int (&r)[kPerLane], F give) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // first the sweep's free pages in order, then a page per thread: which sequence it goes to is searched for once, not per ballot
    auto hand_out = [&](const Sweep& w, int c0, int base) {
        int rank0 = w.first;
#pragma unroll
        for (int k = 0; k < kPerLane; ++k) {
            if ((w.mask[k] >> lane) & 1u) s.list[rank0 + __popc(w.mask[k] & ((1u << lane) - 1u))] = c0 + warp * kWarpPages + 32 * k + lane;
            rank0 += __popc(w.mask[k]);
        }
        __syncthreads();
        for (int j = threadIdx.x; j < min(w.sum, total - base); j += THREADS) {
            const int page = s.list[j], rank = base + j;
            int lo = 0, hi = n;                             // start[lo] <= rank < start[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (s.start[mid] <= rank) lo = mid; else hi = mid;
            }
            refs[page] = 1;
            give(lo, s.from[lo] + rank - s.start[lo], rank, page);
        }
    };
    if (total == 0) return true;
    Sweep w;
    sweep_count(s, r, 0, w);
    if (w.sum >= total) {                                   // one sweep saw them all
        hand_out(w, 0, 0);
        return true;
    }
    int found = w.sum, end = PlanShared<THREADS>::SWEEP, turn = 1;
    for (; found < total && end < pages; end += PlanShared<THREADS>::SWEEP, ++turn) {
        sweep_load(refs, pages, end, r);
        sweep_count(s, r, turn, w);
        found += w.sum;
    }
    if (found < total) return false;
    for (int c0 = 0, base = 0; c0 < end; c0 += PlanShared<THREADS>::SWEEP, ++turn) {
        sweep_load(refs, pages, c0, r);
        sweep_count(s, r, turn, w);
        hand_out(w, c0, base);
        base += w.sum;
        __syncthreads();                                    // the list has been read
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

template <PlanKind KIND, int THREADS>
__global__ void __launch_bounds__(THREADS) kv_plan_kernel(const __grid_constant__ PlanArgs a) {
    extern __shared__ int dyn[];
    __shared__ PlanShared<THREADS> s;
    const luvc_kv_cache& c = a.c;
    const int n = a.n, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) {
        s.error = 0;
        s.start = dyn; s.from = dyn + n + 1; s.len = dyn + 2 * n + 1; s.slot = dyn + 3 * n + 1;
    }
    pdl_trigger();
    pdl_wait();
    int r[kPerLane];                                        // looked at last, but independent of everything before
    sweep_load(c.refs, c.pages, 0, r);
    if (KIND != kReserve && tid == 0) a.move.head[1] = 0;
    const int word = status_of(a.status);
    if (__syncthreads_or(word)) {
        stop_writes(a.status, word);
        return;
    }
    const long long most = (long long)c.max_pages * c.page_size;

    // what each sequence needs; its slot is claimed, so that one named twice is noticed
    if (KIND == kFork) {
        for (int i = tid; i < n; i += THREADS) {
            const int src = a.src[i], dst = a.seqs[i];
            int len = -1;
            if (src >= 0 && src < c.slots) len = c.lengths[src];
            if (len < 0 || len > most) { atomicMax(&s.error, (int)LUVC_ERR_SHAPE); len = 0; }
            s.from[i] = len / c.page_size;
            s.start[i] = len % c.page_size ? 1 : 0;
            s.len[i] = len;
            s.slot[i] = dst;
        }
        __syncthreads();                                    // a source that is also a destination has been read
        for (int i = tid; i < n; i += THREADS) {
            const int dst = s.slot[i];
            const int was = dst >= 0 && dst < c.slots ? atomicCAS(&c.lengths[dst], 0, kClaimed) : kClaimed;
            if (was != 0) {
                atomicMax(&s.error, was == kClaimed ? (int)LUVC_ERR_SHAPE : (int)LUVC_ERR_TARGET);
                s.len[i] = kClaimed;
            }
        }
    } else if (KIND == kReserve) {
        for (int i = tid; i < n; i += THREADS) {
            const int slot = a.seqs ? a.seqs[i] : i, add = a.counts[i];
            int len = kClaimed;
            if (slot >= 0 && slot < c.slots) len = a.seqs ? atomicExch(&c.lengths[slot], kClaimed) : c.lengths[slot];
            int need = 0, have = 0;
            if (len < 0 || add < 0) {
                atomicMax(&s.error, (int)LUVC_ERR_SHAPE);
            } else if ((long long)len + add > most) {
                atomicMax(&s.error, (int)LUVC_ERR_PAGES);
            } else {
                have = ceil_div(len, c.page_size);
                need = ceil_div(len + add, c.page_size) - have;
            }
            if (need > kMaxNeed) atomicMax(&s.error, (int)LUVC_ERR_PAGES), need = 0;
            s.len[i] = len; s.from[i] = have; s.start[i] = need; s.slot[i] = slot;
        }
    } else {
        for (int i = warp; i < n; i += (THREADS / 32)) {
            const int slot = a.seqs ? a.seqs[i] : i;
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
                if (need > kMaxNeed) bad = LUVC_ERR_PAGES, need = 0;
                for (int p = still + lane; p < ceil_div(len, c.page_size); p += 32)
                    a.move.old[(long long)i * c.max_pages + p] = c.table[(long long)slot * c.max_pages + p];
            }
            if (lane == 0) {
                if (bad) atomicMax(&s.error, bad);
                s.len[i] = len; s.from[i] = still; s.start[i] = need; s.slot[i] = slot;
                a.move.len[i] = len; a.move.from[i] = still;
            }
        }
    }
    __syncthreads();
    const int total = scan_needs(s, n, c.pages);
    int error = s.error;
    if (total < 0 && error < LUVC_ERR_PAGES) error = LUVC_ERR_PAGES;
    if (!error && !take_pages(s, c.refs, c.pages, n, total, r, [&](int i, int index, int rank, int page) {
            c.table[(long long)s.slot[i] * c.max_pages + index] = page;
            if (KIND != kReserve) a.move.items[rank] = make_int2(i, index);
        }))
        error = LUVC_ERR_PAGES;
    for (int i = tid; i < n; i += THREADS) {           // lengths: committed, or the claimed slots given back
        int now = s.len[i];
        if (error) {
            if (now == kClaimed || !a.seqs) continue;
            if (KIND == kFork) now = 0;
        } else {
            if (KIND == kReserve) now += a.counts[i];
            if (KIND == kCompact) now += (a.counts ? a.counts[i] : a.keep) - a.span[i];
        }
        c.lengths[s.slot[i]] = now;
    }
    if (tid == 0) {
        if (error) *a.status = error;
        else if (KIND != kReserve) { a.move.head[0] = total; a.move.head[1] = 1; }
    }
}

struct MoveArgs {
    luvc_kv_cache c;
    const int32_t* seqs;     // fork: the destinations
    const int32_t* src;      // fork: the sources; null: compact
    const int32_t *first, *span, *idx, *counts;
    int n, keep;
    int es;                  // bytes of an element
    MoveList move;
    int* status;
    // of the launch: (layer, K or V, head) triples and groups of them; rows of a piece at most, pieces of a page, pieces looked up at a
    // time; 16-byte parts of a row; teams, and threads of one
    int triples, groups, cap, chunks, batch, units, teams, size;
};

// Fills the pages of the plan's list, and settles the pages that change hands.  The work is the list of all (page, up to
// kMoveRows of its rows, group of kMoveLanes (layer, K or V, head) triples); a CTA takes an equal, contiguous part of it.  Where rows
// come from is looked up first, a row per thread, once for all the groups of the part; a thread then copies 16 bytes of a row for
// all triples of a group, with as many loads in flight.  (Four triples and 64 registers let four CTAs share an SM: 190 us for
// the 1.09 GB of a prune of eight videos, 10.0 for one image; with eight triples and two CTAs 193 and 10.5.)  Where a piece of
// a page has no more 16-byte parts than half the threads, the CTA works in TEAMS, each on a group of its own (16 heads of 64 in
// 8 bits, pages of 16, 620 MB: 140 us, without 211; a fork of 16 such sequences 15.1 and 21.5).
constexpr int kMoveLanes = 4, kMoveRows = 64, kMoveThreads = 256;

template <bool FORK, bool TEAMS>
__global__ void __launch_bounds__(kMoveThreads, 4) kv_move_kernel(const __grid_constant__ MoveArgs a) {
    __shared__ long long src_row[kMoveThreads];             // row of head 0 of a layer's pool; -1: none
    __shared__ long long dst_row[kMoveThreads / 16];        // first row of a piece (a page's rows, at most kMoveRows)
    __shared__ int rows_of[kMoveThreads / 16];
    const luvc_kv_cache& c = a.c;
    const int tid = threadIdx.x, lane = tid & 31, ps = c.page_size;
    pdl_trigger();
    pdl_wait();
    if (!a.move.head[1]) return;

    // pages that change hands, a sequence per warp
    for (int i = blockIdx.x * (kMoveThreads / 32) + (tid >> 5); i < a.n; i += gridDim.x * (kMoveThreads / 32)) {
        const int slot = a.seqs ? a.seqs[i] : i;
        int32_t* const row = c.table + (long long)slot * c.max_pages;
        if (FORK) {
            const int32_t* const from = c.table + (long long)a.src[i] * c.max_pages;
            const int full = c.lengths[slot] / ps;
            for (int p = lane; p < full; p += 32) {
                const int page = from[p];
                row[p] = page;
                if (page >= 0 && page < c.pages) atomicAdd(&c.refs[page], 1);
            }
        } else {
            const int before = ceil_div(a.move.len[i], ps), now = ceil_div(c.lengths[slot], ps);
            for (int p = a.move.from[i] + lane; p < before; p += 32) {
                const int page = a.move.old[(long long)i * c.max_pages + p];
                if (page >= 0 && page < c.pages) atomicSub(&c.refs[page], 1);
                if (p >= now) row[p] = -1;
            }
        }
    }

    const int triples = a.triples, groups = a.groups, cap = a.cap, chunks = a.chunks, batch = a.batch, units = a.units, teams = TEAMS ? a.teams : 1;
    // below 2^31: each item is 256 bytes of a pool at least
    const unsigned work = (unsigned)(a.move.head[0] * chunks * groups), share = work / gridDim.x, more = work % gridDim.x;
    const unsigned w0 = share * blockIdx.x + min(blockIdx.x, more), w1 = w0 + share + (blockIdx.x < more);
    if (w0 >= w1) return;
    const size_t row_bytes = (size_t)c.D * a.es, head_bytes = ps * row_bytes, layer_bytes = (size_t)c.pages * c.heads * head_bytes;
    const int size = TEAMS ? a.size : kMoveThreads, team = TEAMS ? tid / size : 0, unit0 = tid - team * size, row0 = unit0 / units, off0 = (unit0 - row0 * units) * 16;      // a thread's first 16 bytes of a piece
    const unsigned first_piece = w0 / groups, last_piece = (w1 - 1) / groups;

    for (unsigned piece0 = first_piece; piece0 <= last_piece; piece0 += batch) {
        __syncthreads();                                    // the pieces before have been copied
        const int k = tid / cap, r = tid - k * cap;
        const unsigned piece = piece0 + k;
        if (k < batch && piece <= last_piece) {
            const int2 it = a.move.items[piece / chunks];
            const int i = it.x, p = it.y, skip = (int)(piece % (unsigned)chunks) * kMoveRows, slot = a.seqs ? a.seqs[i] : i;
            const int to = c.table[(long long)slot * c.max_pages + p];
            const int rows = to >= 0 && to < c.pages ? min(cap, min(ps, c.lengths[slot] - p * ps) - skip) : 0;
            if (r == 0) {
                dst_row[k] = (long long)to * c.heads * ps + skip;
                rows_of[k] = rows;
            }
            if (r < rows) {
                int from = p * ps + skip + r, page;         // token of the old sequence that becomes this row
                if (FORK) {
                    page = c.table[(long long)a.src[i] * c.max_pages + p];
                } else {
                    const int first = a.first[i], span = a.span[i], count = a.counts ? a.counts[i] : a.keep;
                    if (from >= first + count) {
                        from += span - count;
                    } else if (from >= first) {
                        const int e = a.idx[(long long)i * a.keep + from - first], in = min(max(e, 0), span - 1);
                        if (in != e) *a.status = LUVC_ERR_KEEP;
                        from = first + in;
                    }
                    // a token moves towards the start, so it comes from a page that is not as before; only an entry that was replaced
                    // (or is out of order) can stand for one on a page that stays
                    if (from < p * ps && from / ps < a.move.from[i]) page = c.table[(long long)slot * c.max_pages + from / ps];
                    else page = a.move.old[(long long)i * c.max_pages + from / ps];
                }
                src_row[tid] = page >= 0 && page < c.pages ? (long long)page * c.heads * ps + from % ps : -1;
            }
        }
        __syncthreads();
        const unsigned wa = max(w0, piece0 * groups), wb = min(w1, (piece0 + batch) * groups);
        int at = 0, group = wa - piece0 * groups;           // (only the first piece of the part may begin inside)
        int layer = group * kMoveLanes / (2 * c.heads), rest = group * kMoveLanes - layer * 2 * c.heads;   // of the group's first triple
        for (unsigned w = team < teams ? wa + team : wb; w < wb; w += teams) {
            if (TEAMS) {
                at = w / groups - piece0;
                group = w % groups;
                layer = group * kMoveLanes / (2 * c.heads);
                rest = group * kMoveLanes - layer * 2 * c.heads;
            }
            const int live = min(kMoveLanes, triples - group * kMoveLanes);
            unsigned char* base[kMoveLanes];
#pragma unroll
            for (int x = 0; x < kMoveLanes; ++x) {
                if (x < live) {
                    base[x] = static_cast<unsigned char*>(rest >= c.heads ? c.v : c.k) + layer * layer_bytes +
                              (rest >= c.heads ? rest - c.heads : rest) * head_bytes;
                    if (++rest == 2 * c.heads) { rest = 0; ++layer; }
                } else {
                    base[x] = base[0];
                }
            }
            int row = row0, off = off0;
            for (int u = unit0; u < rows_of[at] * units; u += size) {
                if (u != unit0) { row = u / units; off = (u - row * units) * 16; }
                const long long from = src_row[at * cap + row];
                if (from < 0) continue;
                const size_t src = from * row_bytes + off, dst = (dst_row[at] + row) * row_bytes + off;
                uint4 v[kMoveLanes];
#pragma unroll
                for (int x = 0; x < kMoveLanes; ++x) v[x] = __ldcs(reinterpret_cast<const uint4*>(base[x] + src));
#pragma unroll
                for (int x = 0; x < kMoveLanes; ++x)
                    if (x < live) __stcs(reinterpret_cast<uint4*>(base[x] + dst), v[x]);
            }
            if (++group == groups) { group = 0; layer = rest = 0; ++at; }
        }
    }
}

// A CTA per sequence.  Each looks at all slots of the call first: whether any of them is out of range, and then none is freed, must not
// depend on which CTA comes first (the status word that one sets is read by the others).
__global__ void __launch_bounds__(128) kv_free_kernel(const __grid_constant__ luvc_kv_cache c, const int32_t* seqs, int* status) {
    __shared__ int len;
    pdl_trigger();
    pdl_wait();
    const int slot = seqs ? seqs[blockIdx.x] : (int)blockIdx.x;
    const int word = status_of(status);
    bool bad = false;
    if (seqs)                                               // else slots 0 .. n - 1, which the host has checked
        for (int i = threadIdx.x; i < (int)gridDim.x; i += blockDim.x) bad = bad || (unsigned)seqs[i] >= (unsigned)c.slots;
    if (__syncthreads_or(word || bad)) {
        if (!word && threadIdx.x == 0 && blockIdx.x == 0) *status = LUVC_ERR_SHAPE;
        stop_writes(status, word);
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
    int layer, n, tokens, per;                              // per: tokens of a CTA
    const int32_t *seqs, *starts, *sizes;
    const void *k, *v;
    long long k_stride, v_stride;
    int* status;
};

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

__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    unsigned long long d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d)
        : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)), "l"(*reinterpret_cast<unsigned long long*>(&c)));
    return *reinterpret_cast<float2*>(&d);
}
// What an e4m3 row is divided by: the scale, its reciprocal, and the largest quotient the short way is taken for.
struct Scale {
    float s, r, most;
    __device__ explicit Scale(float scale) : s(scale), r(1.f / scale), most(isinf(1.f / scale) ? -1.f : 1024.f) {}
};
__device__ __forceinline__ void store_row(float* p, const float (&f)[8], const Scale&) {
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
}
__device__ __forceinline__ void store_row(__nv_bfloat16* p, const float (&f)[8], const Scale&) {
    unsigned r[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const __nv_bfloat162 pr = __floats2bfloat162_rn(f[2 * q], f[2 * q + 1]);
        r[q] = *reinterpret_cast<const unsigned*>(&pr);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(r[0], r[1], r[2], r[3]);
}
// x / scale, saturated, to nearest even.  The quotient is the correctly rounded one, so that the stored value is what a
// division gives, at a third of its instructions: Markstein's method (q = x r, then q + r (x - q scale), fused), with r the
// correctly rounded reciprocal.  Quotients far beyond 448, which include infinities, and scales below 2^-128 are divided.
__device__ __forceinline__ void store_row(__nv_fp8_e4m3* p, const float (&f)[8], const Scale& scale) {
    float q[8], big = 0.f;
#pragma unroll
    for (int x = 0; x < 8; ++x) {
        q[x] = f[x] * scale.r;
        big = fmaxf(big, fabsf(q[x]));
    }
    if (big < scale.most) {
#pragma unroll
        for (int x = 0; x < 8; x += 2) {                    // two at a time
            float2 a = make_float2(q[x], q[x + 1]);
            const float2 rest = fma2(make_float2(-a.x, -a.y), make_float2(scale.s, scale.s), make_float2(f[x], f[x + 1]));
            a = fma2(rest, make_float2(scale.r, scale.r), a);
            q[x] = a.x; q[x + 1] = a.y;
        }
    } else {
#pragma unroll
        for (int x = 0; x < 8; ++x) q[x] = f[x] / scale.s;
    }
    unsigned w[2];
#pragma unroll
    for (int x = 0; x < 2; ++x)
        w[x] = (unsigned)__nv_cvt_float2_to_fp8x2(make_float2(q[4 * x], q[4 * x + 1]), __NV_SATFINITE, __NV_E4M3) |
               (unsigned)__nv_cvt_float2_to_fp8x2(make_float2(q[4 * x + 2], q[4 * x + 3]), __NV_SATFINITE, __NV_E4M3) << 16;
    *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
}

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

// A CTA writes up to kWriteTokens tokens.  A thread keeps its place in a token's row (16 bytes of K and of V) and takes every
// `step`-th token; the first rows are on their way while the warps find out where the tokens go.
constexpr int kWriteTokens = 32, kWriteThreads = 256, kWriteBatch = 4;

template <typename TI, typename TC>
__global__ void __launch_bounds__(kWriteThreads, 4) kv_write_kernel(const __grid_constant__ WriteArgs a) {
    constexpr int V = Vec<TI>::N;
    __shared__ long long row_of[kWriteTokens];              // row of head 0 in the layer's pool, -1: not written
    __shared__ float bias_of[kWriteTokens];
    const luvc_kv_cache& c = a.c;
    const int t0 = blockIdx.x * a.per, ps = c.page_size, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int per_row = c.D / V, per_token = c.heads * per_row, cols = min(per_token, kWriteThreads), step = kWriteThreads / cols;
    const int mine = threadIdx.x / cols, tokens = min(a.per, a.tokens - t0);
    pdl_trigger();
    pdl_wait();
    const int word = status_of(a.status);                   // this launch sets no other value than the one that does not stop it
    if (__syncthreads_or(word != 0 && word != kRowsSkipped)) return;
    uint4 kx[kWriteBatch], vx[kWriteBatch];
    auto fetch = [&](int col, int t) {
#pragma unroll
        for (int b = 0; b < kWriteBatch; ++b)
            if (t + b * step < tokens) {
                const long long at = t0 + t + b * step;
                kx[b] = __ldcs(reinterpret_cast<const uint4*>(static_cast<const TI*>(a.k) + at * a.k_stride + col * V));
                vx[b] = __ldcs(reinterpret_cast<const uint4*>(static_cast<const TI*>(a.v) + at * a.v_stride + col * V));
            }
    };
    const int col0 = threadIdx.x - mine * cols;
    if (mine < step) fetch(col0, mine);
    if (warp == 0) {                                        // a token per lane, from the owner of the first one on
        int i = a.starts ? owner_of(a.starts, a.n, t0, lane) : t0 + lane;
        if (lane < tokens) {
            const int t = t0 + lane;
            int behind = 1;                                 // tokens of the sequence from this one to its end
            if (a.starts) {
                int end = a.starts[i + 1];
                while (end <= t && i + 1 < a.n) end = a.starts[++i + 1];
                behind = end - t;
            }
            long long row = -1;
            const int slot = a.seqs ? a.seqs[i] : i;
            const int pos = slot >= 0 && slot < c.slots ? c.lengths[slot] - behind : -1;
            if (behind >= 1 && pos >= 0 && pos / ps < c.max_pages) {
                const int page = c.table[(long long)slot * c.max_pages + pos / ps];
                if (page >= 0 && page < c.pages) row = (long long)page * c.heads * ps + pos % ps;
            }
            if (row < 0) *a.status = kRowsSkipped;
            bias_of[lane] = a.sizes ? logf((float)a.sizes[t]) : 0.f;
            row_of[lane] = row;
        }
    }
    __syncthreads();
    if (mine >= step) return;
    const long long layer_row = (long long)a.layer * c.pages * c.heads * ps;
    for (int col = col0; col < per_token; col += cols) {
        const int h = col / per_row;
        const long long in = (long long)h * ps * c.D + (long long)(col - h * per_row) * V;
        TC* const kd = static_cast<TC*>(c.k) + in;
        TC* const vd = static_cast<TC*>(c.v) + in;
        const Scale ks(c.k_scale ? c.k_scale[a.layer * c.heads + h] : 1.f), vs(c.v_scale ? c.v_scale[a.layer * c.heads + h] : 1.f);
        for (int t = mine; t < tokens; t += kWriteBatch * step) {
            if (col != col0 || t != mine) fetch(col, t);
#pragma unroll
            for (int b = 0; b < kWriteBatch; ++b) {
                const int j = t + b * step;
                if (j >= tokens || row_of[j] < 0) continue;
                const long long dst = (layer_row + row_of[j]) * c.D;
                float f[8];
                Vec<TI>::unpack(kx[b], f);
                store_row(kd + dst, f, ks);
                Vec<TI>::unpack(vx[b], f);
                if (a.sizes)
#pragma unroll
                    for (int x = 0; x < V; ++x) f[x] += bias_of[j];
                store_row(vd + dst, f, vs);
            }
        }
    }
}

template <PlanKind KIND, int THREADS>
int launch_plan_as(const PlanArgs& a, cudaStream_t stream) {
    // The attribute belongs to the kernel, not to the call, and other threads launch it too: the most that any call needs, once per device.
    static std::atomic<unsigned long long> set{0};
    const size_t smem = (size_t)(4 * a.n + 1) * sizeof(int);
    if (sizeof(PlanShared<THREADS>) + smem > 48 * 1024) {
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess) {
            cudaGetLastError();
            return LUVC_ERR_CUDA;
        }
        if (dev > 63 || !((set.load(std::memory_order_relaxed) >> dev) & 1)) {
            if (cudaFuncSetAttribute(kv_plan_kernel<KIND, THREADS>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                     (4 * kKvMaxSeqs + 1) * (int)sizeof(int)) != cudaSuccess) {
                cudaGetLastError();
                return LUVC_ERR_CUDA;
            }
            if (dev <= 63) set.fetch_or(1ull << dev, std::memory_order_relaxed);
        }
    }
    return launch_overlapped(kv_plan_kernel<KIND, THREADS>, 1, THREADS, smem, stream, a);
}

// A small CTA has shorter barriers (one token for 32 sequences: 3.8 us, with 1024 threads 4.9; 256 forks in all: 21.4, with 1024 22.4),
// a large one gets through a large pool in fewer sweeps (about 0.6 us each).
template <PlanKind KIND>
int launch_plan(const PlanArgs& a, cudaStream_t stream) {
    return a.n <= 256 && a.c.pages <= 4 * PlanShared<256>::SWEEP ? launch_plan_as<KIND, 256>(a, stream) : launch_plan_as<KIND, 1024>(a, stream);
}

// `pages`: about how many are filled.  Four CTAs per SM run at a time; up to six times as many are launched for long copies, so
// that SMs that get less bandwidth take fewer of them, as long as each has 128 KB to copy (1.09 GB: 189 us, with one wave of CTAs
// 201, with four 191; last pages of 256 forks, 59 MB at most: one wave 20.8, two 21.7).
template <bool FORK>
int launch_move(MoveArgs& a, long long pages, cudaStream_t stream) {
    const luvc_kv_cache& c = a.c;
    a.triples = c.layers * 2 * c.heads;
    a.groups = (a.triples + kMoveLanes - 1) / kMoveLanes;
    a.cap = c.page_size < kMoveRows ? c.page_size : kMoveRows;          // page sizes: 16 and up
    a.chunks = (c.page_size + kMoveRows - 1) / kMoveRows;
    a.batch = kMoveThreads / a.cap;
    a.units = c.D * a.es / 16;
    a.teams = 2 * a.cap * a.units <= kMoveThreads ? kMoveThreads / (a.cap * a.units) : 1;
    a.size = a.teams > 1 ? a.cap * a.units : kMoveThreads;
    const int sms = sm_count();
    if (!sms) return LUVC_ERR_CUDA;
    const long long one = 4ll * sms, bytes = pages * c.page_size * c.layers * 2 * c.heads * c.D * a.es;
    const long long waves = bytes / (one * (128 << 10)), grid = one * (waves < 1 ? 1 : waves > 6 ? 6 : waves);
    return a.teams > 1 ? launch_overlapped(kv_move_kernel<FORK, true>, (unsigned)grid, kMoveThreads, 0, stream, a)
                       : launch_overlapped(kv_move_kernel<FORK, false>, (unsigned)grid, kMoveThreads, 0, stream, a);
}

}  // namespace

size_t kv_elem_size(int dtype) { return dtype == LUVC_F32 ? 4 : dtype == LUVC_BF16 ? 2 : 1; }

size_t kv_workspace_bytes(const luvc_kv_cache& c, int n) {
    return 256 + 2 * align_up((size_t)n * sizeof(int)) + align_up((size_t)n * c.max_pages * sizeof(int2)) +
           align_up((size_t)n * c.max_pages * sizeof(int));
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
    m.c = c; m.seqs = dst; m.src = src; m.n = n; m.es = (int)kv_elem_size(c.dtype); m.move = a.move; m.status = status;
    return launch_move<true>(m, n, stream);
}

int kv_compact(const luvc_kv_cache& c, const int32_t* seqs, int n, const int32_t* first, const int32_t* span, const int32_t* idx,
               int keep, const int32_t* counts, void* ws, int* status, cudaStream_t stream) {
    PlanArgs a = {};
    a.c = c; a.seqs = seqs; a.n = n; a.first = first; a.span = span; a.idx = idx; a.keep = keep; a.counts = counts;
    a.move = move_list(ws, c, n); a.status = status;
    const int rc = launch_plan<kCompact>(a, stream);
    if (rc) return rc;
    MoveArgs m = {};
    m.c = c; m.seqs = seqs; m.first = first; m.span = span; m.idx = idx; m.counts = counts; m.n = n; m.keep = keep;
    m.es = (int)kv_elem_size(c.dtype); m.move = a.move; m.status = status;
    return launch_move<false>(m, (long long)n * ((keep + c.page_size - 1) / c.page_size), stream);
}

int kv_free(const luvc_kv_cache& c, const int32_t* seqs, int n, int* status, cudaStream_t stream) {
    return launch_overlapped(kv_free_kernel, n, 128, 0, stream, c, seqs, status);
}

int kv_write(const luvc_kv_cache& c, int layer, const int32_t* seqs, int n, const void* k, const void* v, long long k_stride,
             long long v_stride, int tokens, const int32_t* starts, const int32_t* sizes, int* status, cudaStream_t stream) {
    WriteArgs a;
    a.c = c; a.layer = layer; a.n = n; a.tokens = tokens; a.seqs = seqs; a.starts = starts; a.sizes = sizes;
    a.k = k; a.v = v; a.k_stride = k_stride; a.v_stride = v_stride; a.status = status;
    // four CTAs per SM while there are few tokens (what counts then is the time of one), at least 4 tokens each
    const int sms = sm_count();
    if (!sms) return LUVC_ERR_CUDA;
    const int even = (int)(((long long)tokens + 4 * sms - 1) / (4 * sms));
    a.per = even < 4 ? 4 : even > kWriteTokens ? kWriteTokens : even;
    const int grid = (tokens - 1) / a.per + 1;             // tokens: 1 .. 2^31 - 1
    if (c.dtype == LUVC_F32) return launch_overlapped(kv_write_kernel<float, float>, grid, kWriteThreads, 0, stream, a);
    if (c.dtype == LUVC_BF16) return launch_overlapped(kv_write_kernel<__nv_bfloat16, __nv_bfloat16>, grid, kWriteThreads, 0, stream, a);
    return launch_overlapped(kv_write_kernel<__nv_bfloat16, __nv_fp8_e4m3>, grid, kWriteThreads, 0, stream, a);
}

}  // namespace luvc
