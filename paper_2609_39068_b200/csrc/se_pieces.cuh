// How the persistent prompt kernels share out a packed batch.  The batch is a list of items in the order (request, kv-head,
// index in the request), each a run of units (KV tiles that a query tile sees, or query tiles that see a KV tile).
// The list is cut into pieces at unit borders, so a piece may begin and end inside an item; such an item's pieces leave partial
// results, and whoever completes its count of units merges them in piece order.
//
// Pieces of equal cost do not take equal time: SMs differ in their distance to the data, and no cost model knows every short
// item.  With one piece per CTA the slowest CTA took 9 % (one long prompt) to 29 % (mixed batches) longer than the mean.
// So a large batch is cut three times: 148 pieces with 7/10 of the cost, 148 with 2/10, 148 with 1/10; a CTA begins with
// the piece of its number and then takes the next one that nobody has.
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
#pragma once

#include "se_tc.cuh"

namespace se {

constexpr int kPromptCtas = 148;       // one per SM
constexpr int kPromptThreads = 384;
constexpr int kMaxPieces = 3 * kPromptCtas;
constexpr int kSmemRequests = 96;      // batches up to here keep their prefix sums in shared memory

// Head of the workspace of the prompt calls (zero when no call is running).
struct PromptControl {
    uint32_t status, next_piece, ended, pad[61];
    uint32_t tickets[2 * kMaxPieces];
};
constexpr size_t kPromptControlBytes = (sizeof(PromptControl) + 255) / 256 * 256;

// Prefix sums over the requests: cost and number of items before each, [B + 1].
constexpr size_t prefix_bytes(int B) { return ((size_t)(B + 1) * 12 + 15) / 16 * 16; }
// workspace for the prefix sums of all CTAs (each has its own)
inline size_t prefix_workspace_bytes(int B) { return B > kSmemRequests ? prefix_bytes(B) * kPromptCtas : 0; }

// Behind the partial results: up to two per piece and stream, each of 128 rows of D channels and two statistics.
inline size_t prefix_workspace_offset(int D) {
    return kPromptControlBytes + (size_t)kMaxPieces * 4 * ((size_t)128 * D + 256) * sizeof(float);
}

// Where a piece begins: number of the item in the list, unit in it; request (B: the end of the list), kv-head, index.
struct Border {
    int item, unit, r, h, i;
};

template <class Work>
struct List {
    const Work &w;
    int B, H_kv;
    const long long *cost;
    const int *first;
    int pieces;
    long long total, size;             // size: cost of a piece where all are equal

    __device__ __forceinline__ Border border(int p) const {
        const int level = p / kPromptCtas, k = p - level * kPromptCtas;
        const long long tenth = total / 10;
        const long long at = pieces == kPromptCtas ? size * p
                             : level == 0          ? tenth * 7 * k / kPromptCtas
                             : level == 1          ? tenth * 7 + tenth * 2 * k / kPromptCtas
                             : level == 2          ? tenth * 9 + (total - tenth * 9) * k / kPromptCtas
                                                   : total;
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
        b.h = (int)(x / each);
        const long long y = x - b.h * each;
        int i0 = 0, i1 = items;
        while (i1 - i0 > 1) {
            const int mid = (i0 + i1) >> 1;
            if (w.cost(t, mid) <= y) i0 = mid; else i1 = mid;
        }
        b.i = i0;
        const int units = w.units(t, b.i);
        b.unit = w.unit_at(t, b.i, y - w.cost(t, b.i));
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
// workspace; sums: 144 bytes of shared memory, free afterwards.  Ends with a barrier.
template <class Work>
__device__ __forceinline__ List<Work> make_list(const Work &w, int B, int H_kv, PromptControl *ctl, void *own, void *sums) {
    constexpr int kWarps = kPromptThreads / 32;
    long long *cost = reinterpret_cast<long long *>(own);
    int *first = reinterpret_cast<int *>(cost + B + 1);
    long long *s_cost = reinterpret_cast<long long *>(sums);
    int *s_items = reinterpret_cast<int *>(s_cost + kWarps);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (B + kPromptThreads - 1) / kPromptThreads;
    long long sum = 0;
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
    }
    long long si = sum;
    int ni = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long x = __shfl_up_sync(kFull, si, o);
        const int y = __shfl_up_sync(kFull, ni, o);
        if (lane >= o) si += x, ni += y;
    }
    if (lane == 31) s_cost[warp] = si, s_items[warp] = ni;
    __syncthreads();
    long long sb = si - sum;
    int nb = ni - n;
    for (int k = 0; k < warp; ++k) sb += s_cost[k], nb += s_items[k];
    for (int k = 0; k < per; ++k) {
        const int r = tid * per + k;
        if (r >= B) break;
        const long long c = cost[r];
        const int items = first[r];
        cost[r] = sb, first[r] = nb;
        sb += c * H_kv, nb += items * H_kv;
    }
    if (tid == kPromptThreads - 1) cost[B] = sb, first[B] = nb;
    __syncthreads();
    List<Work> l = {w, B, H_kv, cost, first, kMaxPieces, cost[B], 0};
    // the small pieces have to be worth their partial results
    if (l.total / 10 < (long long)kPromptCtas * 5 * w.min_cost()) l.pieces = kPromptCtas;
    l.size = (l.total + kPromptCtas - 1) / kPromptCtas;
    if (l.size < w.min_cost()) l.size = w.min_cost();
    return l;
}

// Pieces on their way through the roles of a CTA: one warp takes them, the others (listeners) hear of them through shared
// memory, two at a time.
struct PieceQueue {
    uint64_t full[2], empty[2];
    struct {
        int piece;         // -1: no more
        Border begin;
        int e_item, e_unit;
    } entry[2];

    __device__ __forceinline__ void init(int listeners) {
        for (int k = 0; k < 2; ++k) {
            mbar_init(smem_u32(&full[k]), 1);
            mbar_init(smem_u32(&empty[k]), listeners);
        }
    }
};

// A role's way through the items of its CTA's pieces; every role does it for itself.  An item that an earlier piece began comes
// last: whole items and the item that a later piece ends are walked from their first unit, and what is left of the first item
// then falls on the units that the neighbours are at, so CTAs that share a head read the same tiles at about the same time
// and all but one of them find the tile in L2.
template <class Work>
struct Walk {
    const List<Work> &l;
    PromptControl *ctl;
    PieceQueue *queue;
    volatile int *gave_up;
    int lane;
    bool taker;
    uint32_t turn = 0;                 // pieces so far
    // the item that the walk has come to
    int r, h, i, unit, item, piece;
    TokenRange t;
    int late = 2;                      // 0 no item to come back to, 1 still to come, 2 being done

    __device__ __forceinline__ Walk(const List<Work> &l, PromptControl *ctl, PieceQueue *queue, volatile int *gave_up, int lane, bool taker)
        : l(l), ctl(ctl), queue(queue), gave_up(gave_up), lane(lane), taker(taker) {}

    __device__ __forceinline__ volatile int *entry() const {
        return reinterpret_cast<volatile int *>(&queue->entry[(turn - 1) & 1]);
    }
    __device__ __forceinline__ void to_begin() {
        const volatile int *e = entry();
        item = e[1], unit = e[2], r = e[3], h = e[4], i = e[5];
        t = TokenRange{0, 0, 0, false};
        if (r < l.B) t = l.w.tokens(r);
    }
    // One piece taken and announced; false: no more, or a wait gave up.
    __device__ __forceinline__ bool take() {
        int p = blockIdx.x;
        if (turn > 0) {
            p = -1;
            if (l.pieces > (int)gridDim.x) {
                if (lane == 0) p = (int)(gridDim.x + atomicAdd(&ctl->next_piece, 1u));
                p = __shfl_sync(kFull, p, 0);
                if (p >= l.pieces) p = -1;
            }
        }
        Border b = {};
        if (p >= 0 && lane < 2) b = l.border(p + lane);
        __syncwarp();
        const uint32_t k = turn & 1;
        if (!warp_wait(smem_u32(&queue->empty[k]), (turn >> 1 & 1) ^ 1, gave_up, &ctl->status)) return false;
        volatile int *e = reinterpret_cast<volatile int *>(&queue->entry[k]);
        if (lane == 0) e[0] = p, e[1] = b.item, e[2] = b.unit, e[3] = b.r, e[4] = b.h, e[5] = b.i;
        if (lane == 1) e[6] = b.item, e[7] = b.unit;
        __syncwarp();
        if (lane == 0) {
            mbar_arrive(smem_u32(&queue->full[k]));
            // the last CTA to see the end leaves the counters as it found them
            if (p < 0 && l.pieces > (int)gridDim.x && atomicInc(&ctl->ended, gridDim.x - 1) == gridDim.x - 1) atomicExch(&ctl->next_piece, 0u);
        }
        __syncwarp();
        ++turn;
        piece = p;
        return p >= 0;
    }
    __device__ __forceinline__ bool hear() {
        if (turn > 0) {                // done with the last one
            if (lane == 0) mbar_arrive(smem_u32(&queue->empty[(turn - 1) & 1]));
            __syncwarp();
        }
        if (!warp_wait(smem_u32(&queue->full[turn & 1]), turn >> 1 & 1, gave_up, &ctl->status)) return false;
        ++turn;
        piece = entry()[0];
        return piece >= 0;
    }
    // Units of the item that belong to the piece end here.
    __device__ __forceinline__ int end_unit(int units) const {
        const volatile int *e = entry();
        return item == e[6] ? min(e[7], units) : units;
    }
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
    // On an item (or a part of one) to work on; false: no more, or a wait gave up.
    __device__ __forceinline__ bool find() {
        for (;;) {
            if (turn > 0) {
                const volatile int *e = entry();
                if (late < 2 && r < l.B && (item < e[6] || (item == e[6] && unit < e[7]))) return true;
                if (late == 1) {
                    to_begin();
                    late = 2;
                    return true;
                }
            }
            if (!(taker ? take() : hear())) return false;
            to_begin();
            late = r < l.B && unit > 0 && item < entry()[6];
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
