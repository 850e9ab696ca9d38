// How the persistent prompt kernels share out a packed batch.  The batch is a list of items in the order (request, kv-head,
// index in the request), each a run of units (KV tiles that a query tile sees, or query tiles that see a KV tile).
// The list is cut into one piece per CTA of equal cost at unit borders, so a piece may begin and end inside an item; such
// an item's CTAs leave partial results, and the CTA that completes its count of units merges them in CTA order.
//
// Every CTA computes all borders for itself: one prefix sum over the requests, then a search per border, because an
// item's cost has a closed form.  That costs about a microsecond and spares a planning kernel and its launch.
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

#include "se_device.cuh"

namespace se {

constexpr int kPromptCtas = 148;       // one per SM
constexpr int kPromptThreads = 384;
constexpr int kPieceScratch = 131072 + 12 * 16;

struct Pieces {
    int item[kPromptCtas + 2], unit[kPromptCtas + 2];   // border c: where CTA c begins
    int begin[3];                                       // request, kv-head, index of this CTA's first item (request B: none)
};

// A walk over this CTA's items; every role of the CTA does it for itself.  An item that an earlier CTA began comes last:
// whole items and the item that a later CTA ends are walked from their first unit, and what is left of the first item then
// falls on the units that the neighbours are at, so CTAs that share a head read the same tiles at about the same time
// and all but one of them find the tile in L2.
struct Cursor {
    int r, h, i, unit, item;
    TokenRange t;
    int late;              // 0: no item to come back to, 1: still to come, 2: being done
};

// scratch: kPieceScratch bytes of shared memory (up to 8193 x 12 of prefix sums); all threads; ends without a barrier.
template <class Work>
__device__ __forceinline__ void cut_work(const Work &w, int B, int H_kv, uint32_t *status, Pieces *out, uint8_t *scratch) {
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
        if (!t.valid && blockIdx.x == 0) atomicOr(status, SE_DEV_BAD_LENGTH);
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
    long long piece = (total + gridDim.x - 1) / gridDim.x;
    if (piece < w.min_cost()) piece = w.min_cost();
    if (tid > (int)gridDim.x) return;
    const long long at = piece * tid;
    int item = first[B], unit = 0;
    int r = B, h = 0, i = 0;
    if (at < total) {
        int lo = 0, hi = B;                // last request whose cost begins at or before `at`
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (cost[mid] <= at) lo = mid; else hi = mid;
        }
        r = lo;
        const TokenRange t = w.tokens(r);
        const int items = w.items(t);
        const long long each = w.cost(t, items), x = at - cost[r];
        h = (int)(x / each);
        const long long y = x - h * each;
        int i0 = 0, i1 = items;
        while (i1 - i0 > 1) {
            const int mid = (i0 + i1) >> 1;
            if (w.cost(t, mid) <= y) i0 = mid; else i1 = mid;
        }
        i = i0;
        const int units = w.units(t, i);
        unit = w.unit_at(t, i, y - w.cost(t, i));
        item = first[r] + h * items + i;
        // no crumbs: a part of an item that is split has a few units at least
        if (unit < Work::kCrumb) {
            unit = 0;
        } else if (unit > units - Work::kCrumb) {
            unit = 0, ++item;
            if (++i == items) {
                i = 0;
                if (++h == H_kv) {
                    h = 0, ++r;
                    while (r < B && first[r + 1] == first[r]) ++r;
                }
            }
        }
    }
    out->item[tid] = item, out->unit[tid] = unit;
    if (tid == (int)blockIdx.x) out->begin[0] = r, out->begin[1] = h, out->begin[2] = i;
}

// Where this CTA's part of the cursor's item ends.
__device__ __forceinline__ int piece_end(const Cursor &c, const Pieces &p, int units) {
    return c.item == p.item[blockIdx.x + 1] ? min(p.unit[blockIdx.x + 1], units) : units;
}
template <class Work>
__device__ __forceinline__ Cursor piece_begin(const Work &w, int B, const Pieces &p) {
    Cursor c;
    c.r = p.begin[0], c.h = p.begin[1], c.i = p.begin[2];
    c.item = p.item[blockIdx.x], c.unit = p.unit[blockIdx.x];
    c.t = TokenRange{0, 0, 0, false};
    if (c.r < B) c.t = w.tokens(c.r);
    return c;
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
__device__ __forceinline__ Cursor first_piece(const Work &w, int B, int H_kv, const Pieces &p) {
    Cursor c = piece_begin(w, B, p);
    c.late = c.r < B && c.unit > 0 && c.item < p.item[blockIdx.x + 1];
    if (c.late) next_item(w, B, H_kv, c);
    return c;
}
// Nothing left; moves on to the item that was left for the end.
template <class Work>
__device__ __forceinline__ bool piece_done(const Work &w, int B, const Pieces &p, Cursor &c) {
    const int e_item = p.item[blockIdx.x + 1], e_unit = p.unit[blockIdx.x + 1];
    if (c.late < 2 && c.r < B && (c.item < e_item || (c.item == e_item && c.unit < e_unit))) return false;
    if (c.late != 1) return true;
    c = piece_begin(w, B, p);
    c.late = 2;
    return false;
}

// The CTAs that share an item: the first one, and for each its units.
__device__ __forceinline__ int first_cta(const Pieces &p, int item) {
    int y = blockIdx.x;
    while (p.item[y] == item && p.unit[y] > 0) --y;
    return y;
}
template <typename F>
__device__ __forceinline__ void each_cta(const Pieces &p, int item, int units, int from, F f) {
    for (int y = from;; ++y) {
        const bool ends = !(p.item[y + 1] == item && p.unit[y + 1] > 0);
        const int a = y == from ? 0 : p.unit[y], b = ends ? units : p.unit[y + 1];
        if (b > a) f(y, a, b);
        if (ends) return;
    }
}

}  // namespace se
