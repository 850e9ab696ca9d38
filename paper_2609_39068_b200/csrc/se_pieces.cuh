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
// Every CTA computes all borders for itself: one prefix sum over the requests, then a search per border, because an
// item's cost has a closed form.  That spares a planning kernel and its launch.  All CTAs write the same table into the
// workspace; each reads what it has written.
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
constexpr int kPieceScratch = 131072 + 12 * 16;

// Border p: where piece p begins (and piece p - 1 ends).
struct Border {
    int item, unit;        // number of the item in the list, unit in it
    int r, h, i;           // the item: request (B: the end of the list), kv-head, index
    int pad[3];
};

// Head of the workspace of the prompt calls (zero when no call is running, but for the table).
struct PromptControl {
    uint32_t status, next_piece, ended, pad[61];
    uint32_t tickets[2 * kMaxPieces];
    uint32_t pad2[8];
    Border borders[kMaxPieces + 1];
};
constexpr size_t kPromptControlBytes = (sizeof(PromptControl) + 255) / 256 * 256;

// scratch: kPieceScratch bytes of shared memory (up to 8193 x 12 of prefix sums); all threads; ends without a barrier.
// Returns the number of pieces.
template <class Work>
__device__ __forceinline__ int cut_work(const Work &w, int B, int H_kv, PromptControl *ctl, uint8_t *scratch) {
    constexpr int kWarps = kPromptThreads / 32;
    long long *cost = reinterpret_cast<long long *>(scratch);              // [B + 1]
    int *first = reinterpret_cast<int *>(cost + B + 1);                    // [B + 1]
    long long *s_cost = reinterpret_cast<long long *>(scratch + 131072);   // per-warp sums
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
    const long long total = cost[B];
    // the small pieces have to be worth their partial results
    const bool one = total / 10 < (long long)kPromptCtas * 8 * w.min_cost();
    const int pieces = one ? kPromptCtas : kMaxPieces;
    long long size = (total + kPromptCtas - 1) / kPromptCtas;
    if (size < w.min_cost()) size = w.min_cost();
    for (int p = tid; p <= pieces; p += kPromptThreads) {
        const int level = p / kPromptCtas, k = p - level * kPromptCtas;
        const long long tenth = total / 10;
        const long long at = one          ? size * p
                             : level == 0 ? tenth * 7 * k / kPromptCtas
                             : level == 1 ? tenth * 7 + tenth * 2 * k / kPromptCtas
                             : level == 2 ? tenth * 9 + (total - tenth * 9) * k / kPromptCtas
                                          : total;
        Border b = {first[B], 0, B, 0, 0, {0, 0, 0}};
        if (at < total) {
            int lo = 0, hi = B;            // last request whose cost begins at or before `at`
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
        }
        ctl->borders[p] = b;
    }
    return pieces;
}

// A walk over a piece's items; every role of the CTA does it for itself.  An item that an earlier piece began comes last:
// whole items and the item that a later piece ends are walked from their first unit, and what is left of the first item then
// falls on the units that the neighbours are at, so CTAs that share a head read the same tiles at about the same time
// and all but one of them find the tile in L2.
struct Cursor {
    int r, h, i, unit, item, e_item, e_unit;
    TokenRange t;
    int piece, late;       // late: 0 no item to come back to, 1 still to come, 2 being done
};

__device__ __forceinline__ int2 border_at(const PromptControl *ctl, int p) {
    return __ldcg(reinterpret_cast<const int2 *>(&ctl->borders[p]));
}
// Where this piece's part of the cursor's item ends.
__device__ __forceinline__ int piece_end(const Cursor &c, int units) { return c.item == c.e_item ? min(c.e_unit, units) : units; }

template <class Work>
__device__ __forceinline__ void piece_begin(const Work &w, int B, const PromptControl *ctl, Cursor &c) {
    const int4 b = __ldcg(reinterpret_cast<const int4 *>(&ctl->borders[c.piece]));
    c.item = b.x, c.unit = b.y, c.r = b.z, c.h = b.w;
    c.i = __ldcg(&ctl->borders[c.piece].i);
    c.t = TokenRange{0, 0, 0, false};
    if (c.r < B) c.t = w.tokens(c.r);
}
template <class Work>
__device__ __forceinline__ void next_item(const Work &w, int B, int H_kv, Cursor &c) {
    c.unit = 0;
    ++c.item;
    if (++c.i < w.items(c.t)) return;
    c.i = 0;
    if (++c.h < H_kv) return;
    c.h = 0;
    do {
        if (++c.r < B) c.t = w.tokens(c.r);
    } while (c.r < B && c.t.n == 0);
}
template <class Work>
__device__ __forceinline__ Cursor first_item(const Work &w, int B, int H_kv, const PromptControl *ctl, int piece) {
    Cursor c;
    c.piece = piece;
    const int2 e = border_at(ctl, piece + 1);
    c.e_item = e.x, c.e_unit = e.y;
    piece_begin(w, B, ctl, c);
    c.late = c.r < B && c.unit > 0 && c.item < c.e_item;
    if (c.late) next_item(w, B, H_kv, c);
    return c;
}
// Nothing left; moves on to the item that was left for the end.
template <class Work>
__device__ __forceinline__ bool piece_done(const Work &w, int B, const PromptControl *ctl, Cursor &c) {
    if (c.late < 2 && c.r < B && (c.item < c.e_item || (c.item == c.e_item && c.unit < c.e_unit))) return false;
    if (c.late != 1) return true;
    piece_begin(w, B, ctl, c);
    c.late = 2;
    return false;
}

// The pieces that share an item: the first one, and for each its units.
__device__ __forceinline__ int first_piece_of(const PromptControl *ctl, int item, int piece) {
    for (;; --piece) {
        const int2 b = border_at(ctl, piece);
        if (!(b.x == item && b.y > 0)) return piece;
    }
}
// A whole warp; the borders of 32 pieces are fetched at once.
template <typename F>
__device__ __forceinline__ void each_piece_of(const PromptControl *ctl, int item, int units, int from, int lane, F f) {
    int start = 0;
    for (int y = from;; y += 32) {
        const int2 e = border_at(ctl, min(y + lane + 1, kMaxPieces));
        const unsigned ends = __ballot_sync(kFull, !(e.x == item && e.y > 0));
        const int n = ends ? __ffs(ends) : 32;
        const int b = ends && lane == n - 1 ? units : e.y;
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

// Pieces on their way through the roles of a CTA: one warp takes them, the others (kListeners warps) hear of them
// through shared memory, two at a time.
struct PieceQueue {
    uint64_t full[2], empty[2];
    int piece[2];          // -1: no more

    __device__ __forceinline__ void init(int listeners) {
        for (int k = 0; k < 2; ++k) {
            mbar_init(smem_u32(&full[k]), 1);
            mbar_init(smem_u32(&empty[k]), listeners);
        }
    }
    // The taking warp; `turn` counts its calls.  -1: no more, or a wait gave up.
    __device__ __forceinline__ int take(uint32_t turn, int pieces, PromptControl *ctl, volatile int *gave_up, int lane) {
        int p = blockIdx.x;
        if (turn > 0) {
            p = -1;
            if (pieces > (int)gridDim.x) {
                if (lane == 0) p = (int)(gridDim.x + atomicAdd(&ctl->next_piece, 1u));
                p = __shfl_sync(kFull, p, 0);
                if (p >= pieces) p = -1;
            }
        }
        const uint32_t k = turn & 1;
        if (!warp_wait(smem_u32(&empty[k]), (turn >> 1 & 1) ^ 1, gave_up, &ctl->status)) return -1;
        if (lane == 0) {
            piece[k] = p;
            mbar_arrive(smem_u32(&full[k]));
            // the last CTA to see the end leaves the counters as it found them
            if (p < 0 && pieces > (int)gridDim.x && atomicInc(&ctl->ended, gridDim.x - 1) == gridDim.x - 1) atomicExch(&ctl->next_piece, 0u);
        }
        __syncwarp();
        return p;
    }
    __device__ __forceinline__ int hear(uint32_t turn, PromptControl *ctl, volatile int *gave_up, int lane) {
        const uint32_t k = turn & 1;
        if (!warp_wait(smem_u32(&full[k]), turn >> 1 & 1, gave_up, &ctl->status)) return -1;
        const int p = *const_cast<volatile int *>(&piece[k]);
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&empty[k]));
        return p;
    }
};

// A role's way through all the items of its CTA.
template <class Work>
struct Walk {
    const Work &w;
    int B, H_kv, lane, n_pieces;       // n_pieces: the taking warp; 0: a listener
    PromptControl *ctl;
    PieceQueue *queue;
    volatile int *gave_up;
    uint32_t turn = 0;
    bool have = false;
    Cursor c = {};

    __device__ __forceinline__ Walk(const Work &w, int B, int H_kv, PromptControl *ctl, PieceQueue *queue, volatile int *gave_up, int lane,
                                    int n_pieces = 0)
        : w(w), B(B), H_kv(H_kv), lane(lane), n_pieces(n_pieces), ctl(ctl), queue(queue), gave_up(gave_up) {}
    // c is an item (or the part of one) to work on; false: no more, or a wait gave up
    __device__ __forceinline__ bool item() {
        while (!have || piece_done(w, B, ctl, c)) {
            const int p = n_pieces ? queue->take(turn, n_pieces, ctl, gave_up, lane) : queue->hear(turn, ctl, gave_up, lane);
            if (p < 0) return false;
            ++turn;
            have = true;
            c = first_item(w, B, H_kv, ctl, p);
        }
        return true;
    }
    __device__ __forceinline__ void next() { next_item(w, B, H_kv, c); }
};

}  // namespace se
