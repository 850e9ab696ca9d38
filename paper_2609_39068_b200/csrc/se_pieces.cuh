// How the persistent prompt kernels share out a packed batch.  The batch is a list of items in the order (request, kv-head,
// index in the request), each a run of units (KV tiles that a query tile sees, or query tiles that see a KV tile).
// The list is cut into pieces at unit borders, so a piece may begin and end inside an item; such an item's pieces leave partial
// results, and whoever completes its count of units merges them in piece order.
//
// Pieces of equal cost do not take equal time: SMs differ in their distance to the data, and no cost model knows every short
// item.  With one piece per CTA the slowest CTA took 9 % (one long prompt) to 29 % (mixed batches) longer than the mean.
// So a large batch can be cut twice: 148 pieces with 9/10 of the cost, 148 with the rest; a CTA begins with the piece of its
// number and then takes the next one that nobody has.  Attention with it, and with one piece each: eight packed prompts 366-372
// and 371-375 us, mixed batch 1252 and 1265 us, prompt of 32768 8.37 and 8.43 ms; 2048 tokens over 65536 take 2.0 ms either way.
// (Three sizes, 7/10, 2/10 and 1/10, were slower than one on an earlier build: 428 us where two took 403 and one 410.)
//
// A border is found by a search, because an item's cost has a closed form: every CTA makes one prefix sum over the
// requests, and looks up the borders of the pieces that it takes or merges.  There is no planning kernel, and no table that
// CTAs share (148 of them writing the same one took 10 us).
//
// A `Work` describes the list:
//   TokenRange tokens(r)               the request, n = 0 if it takes no part
//   int items(t)                       items of one kv-head
//   long long cost(t, i)               cost of the first i items of one kv-head (0 <= i <= items)
//   int units(t, i)                    units of item i
//   int unit_at(t, i, z)               unit that cost z into the item falls in
//   long long min_cost()               least cost of a piece
//   kCrumb                             least units of a part of a split item
//   kGrain, long long coarse()         pieces of less cost than coarse() begin and end at multiples of kGrain units
//   kShares                            whether a large batch is cut into pieces of two sizes;
//   kShareCost                         then: least cost of the small ones
//   long long longest(t)               then: a bound on the cost of the request's items
#pragma once

#include <stddef.h>

#include "se_tc.cuh"

namespace se {

constexpr int kPromptCtas = 148;       // one per SM
constexpr int kMaxPieces = 2 * kPromptCtas;
constexpr int kSmemRequests = 88;      // batches up to here keep their prefix sums in shared memory

// Head of the workspace of the prompt calls.  The counters are zero when no call is running, unless a call gave up a wait: then
// needs_init is set, and the kernels that count do nothing but report SE_DEV_WAIT_TIMEOUT until the workspace is initialised
// again (reading the status word does not clear it).
struct PromptControl {
    uint32_t status, needs_init, next_piece, ended, pad[60];
    uint32_t tickets[2 * kMaxPieces];
};
static_assert(offsetof(PromptControl, needs_init) == kNeedsInitWord * sizeof(uint32_t), "the word that warp_wait sets");
constexpr size_t kPromptControlBytes = (sizeof(PromptControl) + 255) / 256 * 256;

// Prefix sums over the requests: cost and number of items before each, [B + 1].
constexpr size_t prefix_bytes(int B) { return ((size_t)(B + 1) * 12 + 15) / 16 * 16; }
// workspace for the prefix sums of all CTAs (each has its own)
inline size_t prefix_workspace_bytes(int B) { return B > kSmemRequests ? prefix_bytes(B) * kPromptCtas : 0; }

// The partial results, from a border of 32 bytes (the workspace begins on one of 16): up to two per piece and stream, each of
// 128 rows of D channels and two statistics.  The prefix sums lie behind them.
inline float *partials_of(uint8_t *workspace) {
    return reinterpret_cast<float *>(((uintptr_t)workspace + kPromptControlBytes + 31) & ~(uintptr_t)31);
}
inline size_t prefix_workspace_offset(int D) {
    return kPromptControlBytes + 256 + (size_t)kMaxPieces * 4 * ((size_t)128 * D + 256) * sizeof(float);
}

// Where a piece begins: number of the item in the list, unit in it; request (B: the end of the list), kv-head, index.
struct Border {
    int item, unit, r, h, i;
};

template <class Work>
struct List {
    Work w;
    int B, H_kv;
    const long long *cost;
    const int *first;
    int pieces;
    long long total, size;             // size: cost of a piece where all are equal

    __device__ __forceinline__ Border border(int p) const {
        const long long large = total / 10 * 9;
        const long long at = pieces == kPromptCtas ? size * p
                             : p < kPromptCtas     ? large * p / kPromptCtas
                                                   : large + (total - large) * (p - kPromptCtas) / kPromptCtas;
        Border b = {first[B], 0, B, 0, 0};
        if (at >= total) return b;
        int lo = 0, hi = B;                // last request whose cost begins at or before `at`
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (cost[mid] <= at) lo = mid; else hi = mid;
        }
        b.r = lo;
        const TokenRange t = w.tokens(b.r);
        const int items = w.items(t);
        const long long each = w.cost(t, items), x = at - cost[b.r];
        // (a division of 64 bits is a hundred instructions)
        b.h = (x | each) >> 32 ? (int)(x / each) : (int)((uint32_t)x / (uint32_t)each);
        const long long y = x - b.h * each;
        int i0 = 0, i1 = items;
        while (i1 - i0 > 1) {
            const int mid = (i0 + i1) >> 1;
            if (w.cost(t, mid) <= y) i0 = mid; else i1 = mid;
        }
        b.i = i0;
        const int units = w.units(t, b.i);
        b.unit = w.unit_at(t, b.i, y - w.cost(t, b.i));
        if (size < w.coarse()) b.unit -= b.unit % Work::kGrain;
        b.item = first[b.r] + b.h * items + b.i;
        // no crumbs: a part of an item that is split has a few units at least
        if (b.unit < Work::kCrumb) {
            b.unit = 0;
        } else if (b.unit > units - Work::kCrumb) {
            b.unit = 0, ++b.item;
            if (++b.i == items) {
                b.i = 0;
                if (++b.h == H_kv) {
                    b.h = 0, ++b.r;
                    while (b.r < B && first[b.r + 1] == first[b.r]) ++b.r;
                }
            }
        }
        return b;
    }
};

// The list of a batch; all threads of the CTA.  `own` holds the prefix sums for good: shared memory, or the CTA's part of the
// workspace; sums: 20 bytes of shared memory a warp, free afterwards.  Ends with a barrier.
template <int kThreads, class Work>
__device__ __forceinline__ List<Work> make_list(const Work &w, int B, int H_kv, PromptControl *ctl, void *own, void *sums) {
    constexpr int kWarps = kThreads / 32;
    long long *cost = reinterpret_cast<long long *>(own);
    int *first = reinterpret_cast<int *>(cost + B + 1);
    long long *s_cost = reinterpret_cast<long long *>(sums);
    long long *s_long = s_cost + kWarps;
    int *s_items = reinterpret_cast<int *>(s_long + kWarps);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (B + kThreads - 1) / kThreads;
    long long sum = 0, longest = 0;
    int n = 0;
    for (int k = 0; k < per; ++k) {
        const int r = tid * per + k;
        if (r >= B) break;
        const TokenRange t = w.tokens(r);
        if (!t.valid && blockIdx.x == 0) atomicOr(&ctl->status, SE_DEV_BAD_LENGTH);
        const int items = t.n ? w.items(t) : 0;
        const long long c = t.n ? w.cost(t, items) : 0;
        cost[r] = c, first[r] = items;
        sum += c * H_kv, n += items * H_kv;
        if constexpr (Work::kShares) longest = max(longest, t.n ? w.longest(t) : 0ll);
    }
    long long si = sum;
    int ni = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(kFull, si, o);
        const int y = __shfl_up_sync(kFull, ni, o);
        if (lane >= o) si += x, ni += y;
        longest = max(longest, __shfl_xor_sync(kFull, longest, o));
    }
    if (lane == 31) s_cost[warp] = si, s_items[warp] = ni, s_long[warp] = longest;
    __syncthreads();
    long long sb = si - sum;
    int nb = ni - n;
    for (int k = 0; k < warp; ++k) sb += s_cost[k], nb += s_items[k];
    for (int k = 0; k < kWarps; ++k) longest = max(longest, s_long[k]);
    for (int k = 0; k < per; ++k) {
        const int r = tid * per + k;
        if (r >= B) break;
        const long long c = cost[r];
        const int items = first[r];
        cost[r] = sb, first[r] = nb;
        sb += c * H_kv, nb += items * H_kv;
    }
    if (tid == kThreads - 1) cost[B] = sb, first[B] = nb;
    __syncthreads();
    List<Work> l = {w, B, H_kv, cost, first, kMaxPieces, cost[B], 0};
    // the small pieces have to be worth their partial results, and no item may fall into more than 148 of them and a few others
    if constexpr (Work::kShares) {
        if (l.total / 10 < kPromptCtas * Work::kShareCost || l.total / 10 < longest) l.pieces = kPromptCtas;
    } else {
        l.pieces = kPromptCtas;
    }
    l.size = (l.total + kPromptCtas - 1) / kPromptCtas;
    if (l.size < w.min_cost()) l.size = w.min_cost();
    return l;
}

// The parts of items that a CTA works on (a `Segment` of the kernel), on their way from the warp that walks the CTA's pieces to
// the other roles, a few at a time: the roles read what they need where they need it, and keep their registers.
template <class Segment>
struct SegmentQueue {
    static constexpr uint32_t kDepth = 4;
    uint64_t full[kDepth], empty[kDepth];
    Segment entry[kDepth];
    int more[kDepth];                  // 0: the list has ended

    __device__ __forceinline__ void init(int listeners) {
        for (uint32_t k = 0; k < kDepth; ++k) {
            mbar_init(smem_u32(&full[k]), 1);
            mbar_init(smem_u32(&empty[k]), listeners);
        }
    }
    // by the warp that walks, the n-th entry; false: a wait gave up
    __device__ __forceinline__ bool put(uint32_t n, const Segment *s, volatile int *gave_up, uint32_t *status, int lane) {
        const uint32_t k = n % kDepth;
        if (!warp_wait(smem_u32(&empty[k]), (n / kDepth & 1) ^ 1, gave_up, status)) return false;
        if (lane == 0) {
            if (s) entry[k] = *s;
            more[k] = s != nullptr;
            mbar_arrive(smem_u32(&full[k]));
        }
        __syncwarp();
        return true;
    }
    // by the other warps, one entry after the other; nullptr: no more, or a wait gave up
    __device__ __forceinline__ const Segment *get(uint32_t n, volatile int *gave_up, uint32_t *status, int lane) {
        if (n > 0) {                   // done with the one before
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&empty[(n - 1) % kDepth]));
            __syncwarp();
        }
        const uint32_t k = n % kDepth;
        if (!warp_wait(smem_u32(&full[k]), n / kDepth & 1, gave_up, status) || !*(volatile int *)&more[k]) return nullptr;
        return &entry[k];
    }
};

// One warp's way through the items of its CTA's pieces.  An item that an earlier piece began comes last: whole items and the
// item that a later piece ends are walked from their first unit, and what is left of the first item then falls on the units
// that the neighbours are at, so CTAs that share a head read the same tiles at about the same time and all but one of them
// find the tile in L2.
template <class Work>
struct Walk {
    const List<Work> &l;
    PromptControl *ctl;
    int lane;
    bool begun = false;
    Border first;                      // of the piece
    int end_item, end_unit_;
    // the item that the walk has come to
    int r, h, i, unit, item, piece;
    TokenRange t;
    int late = 2;                      // 0 no item to come back to, 1 still to come, 2 being done

    __device__ __forceinline__ Walk(const List<Work> &l, PromptControl *ctl, int lane) : l(l), ctl(ctl), lane(lane) {}

    __device__ __forceinline__ void to_begin() {
        item = first.item, unit = first.unit, r = first.r, h = first.h, i = first.i;
        t = TokenRange{0, 0, 0, false};
        if (r < l.B) t = l.w.tokens(r);
    }
    __device__ __forceinline__ bool take() {
        piece = blockIdx.x;
        if (begun) {
            if (l.pieces == (int)gridDim.x) return false;
            if (lane == 0) piece = (int)(gridDim.x + atomicAdd(&ctl->next_piece, 1u));
            piece = __shfl_sync(kFull, piece, 0);
            if (piece >= l.pieces) {
                // the last CTA to see the end leaves the counters as it found them
                if (lane == 0 && atomicInc(&ctl->ended, gridDim.x - 1) == gridDim.x - 1) atomicExch(&ctl->next_piece, 0u);
                __syncwarp();
                return false;
            }
        }
        begun = true;
        Border b = {};
        if (lane < 2) b = l.border(piece + lane);
        __syncwarp();
        first = Border{__shfl_sync(kFull, b.item, 0), __shfl_sync(kFull, b.unit, 0), __shfl_sync(kFull, b.r, 0), __shfl_sync(kFull, b.h, 0),
                       __shfl_sync(kFull, b.i, 0)};
        end_item = __shfl_sync(kFull, b.item, 1), end_unit_ = __shfl_sync(kFull, b.unit, 1);
        return true;
    }
    // Units of the item that belong to the piece end here.
    __device__ __forceinline__ int end_unit(int units) const { return item == end_item ? min(end_unit_, units) : units; }
    __device__ __forceinline__ void next() {
        unit = 0;
        ++item;
        if (++i < l.w.items(t)) return;
        i = 0;
        if (++h < l.H_kv) return;
        h = 0;
        do {
            if (++r < l.B) t = l.w.tokens(r);
        } while (r < l.B && t.n == 0);
    }
    // On an item (or a part of one) to work on; false: no more.
    __device__ __forceinline__ bool find() {
        for (;;) {
            if (begun) {
                if (late < 2 && r < l.B && (item < end_item || (item == end_item && unit < end_unit_))) return true;
                if (late == 1) {
                    to_begin();
                    late = 2;
                    return true;
                }
            }
            if (!take()) return false;
            to_begin();
            late = r < l.B && unit > 0 && item < end_item;
            if (late) next();
        }
    }
};

// The pieces that share an item, for a whole warp: the first one, and for each its units.
template <class Work>
__device__ __forceinline__ int first_piece_of(const List<Work> &l, int item, int piece, int lane) {
    for (;; piece -= 32) {
        const int p = max(piece - lane, 0);
        const Border b = l.border(p);
        const unsigned begins = __ballot_sync(kFull, !(b.item == item && b.unit > 0));
        if (begins) return max(piece - (__ffs(begins) - 1), 0);
    }
}
template <class Work, typename F>
__device__ __forceinline__ void each_piece_of(const List<Work> &l, int item, int units, int from, int lane, F f) {
    int start = 0;
    for (int y = from;; y += 32) {
        const Border e = l.border(min(y + lane + 1, l.pieces));
        const unsigned ends = __ballot_sync(kFull, !(e.item == item && e.unit > 0));
        const int n = ends ? __ffs(ends) : 32;
        const int b = ends && lane == n - 1 ? units : e.unit;
        int a = __shfl_up_sync(kFull, b, 1);
        if (lane == 0) a = start;
        for (int q = 0; q < n; ++q) {
            const int aq = __shfl_sync(kFull, a, q), bq = __shfl_sync(kFull, b, q);
            if (bq > aq) f(y + q, aq, bq);
        }
        if (ends) return;
        start = __shfl_sync(kFull, b, 31);
    }
}

}  // namespace se
