// Attention of a packed batch of new tokens (Appendix A, attention equations of "MHA, MQA, and GQA"), over the paged
// cache or over contiguous K and V.
//
// Mathematics.  A query tile is 128 rows = 128/G tokens x the G query heads of one kv-head, so the heads of a group share
// every K and V tile.  Over the KV tiles j of 64 tokens:  S = Q K_j^T,  p = 2^(S sl - m)  with sl = sm_scale log2 e,
// O += P V_j, l += rowsum p;  out = O / l,  lse = (m + log2 l) ln 2.  m is a row maximum that is moved (and O, l
// rescaled) only when the scores exceed it by more than 40, so nearly all steps leave O alone.
//
// What bounds it.  Per (128 rows x 128 tokens) at D = 128 the two products take 1024 cycles of the tensor cores and
// the 16384 exponentials 1024 cycles of the special-function units: both have to run all the time.  So a CTA (one per
// SM, persistent) works on two streams of tiles: two warpgroups do the softmax of one stream each, two warps issue a
// stream's products each, two warps copy.  S (fp32), P (bf16, in S's columns) and O (fp32) live in tensor memory: 2 x (128 + D)
// of 512 columns.
//   pair   more than 128 query rows left: the streams are two neighbouring query tiles, K and V tiles are shared
//   alt    up to 128 rows (decode tokens, short chunks, ends of prompts): both streams are the same query tile, one
//          takes the even and one the odd KV tiles; their results are merged at the end
//
// Split.  The CTAs cut the whole batch's work - query tile pairs in the order (request, kv-head, tile), each as long as
// the tokens it sees - into equal pieces at KV-tile borders.  A piece that begins or ends inside a query tile leaves
// fp32 partial results (O, m, l) in the workspace; whichever CTA completes the tile's count of KV tiles merges them, in
// CTA order, so the result does not depend on who is last.  Long contexts with few rows and long prompts take the same
// path, and there is no second kernel.
#include <math.h>

#include "se_internal.h"
#include "se_pieces.cuh"
#include "se_tc.cuh"

namespace se {

namespace {

constexpr int kThreads = kPromptThreads;   // 2 softmax warpgroups, K warp, 2 product warps, V warp
constexpr int kKWarp = 8, kMmaWarp = 9, kVWarp = 11;
constexpr int kTile = 128;             // query rows of a tile
constexpr int kKv = 64;                // tokens of a KV tile
constexpr int kMaxParts = 320;         // partial results of a query tile: two per piece, 148 pieces of it at most
constexpr int kItemCost = 128;         // cost of starting a query tile, in tokens
constexpr int kMinCost = 512;          // a CTA takes at least 256 tokens of a pair, 512 of a single tile
// The running maximum may lag: weights up to 2^40 lose nothing (bf16 and fp32 keep their exponents, and 2^40 * 131072
// tokens is far from the end of the range).
constexpr float kSlack = 40.f;

template <int D>
struct Cfg {
    static constexpr int kHalves = D / 64;
    static constexpr int kTileBytes = kTile * D * 2;              // query tile
    static constexpr int kKvBytes = kKv * D * 2;                  // K or V tile
    static constexpr int kSlots = 10 * 128 / D;                   // ring of K and V tiles, 160 KB
    static constexpr int kMasks = 16;
    static constexpr int kSlotFloats = kTile * D + 2 * kTile;     // a partial result: O, m, l
    static constexpr int kTmemO = 256;                            // S0, S1 at columns 0, 128; O0, O1 behind
};

struct AttendArgs {
    const int32_t *cu, *seq_lens, *page_table;
    const uint16_t *v;                 // rows of the last, partly filled 16-token group are copied by hand
    long long v_stride;                // contiguous V: elements between tokens
    uint16_t *out;
    float *lse;
    float *partials;
    PromptControl *ctl;
    uint8_t *prefixes;                 // prefix sums of batches too large for shared memory
    int B, H_q, H_kv, G, T, max_pages, P_phys;
    float scale_log2;
};

enum Bar { kQFull, kQEmpty, kSFull, kPReady = kSFull + 4, kODone = kPReady + 4, kOLast = kODone + 2, kOFree = kOLast + 2, kAll = kOFree + 2, kVerdict = kAll + 2, kSwap = kVerdict + 2,
           kDrain, kRing = kDrain + 2 };

template <int D>
struct Control {
    uint64_t bars[kRing + 2 * Cfg<D>::kSlots];
    PieceQueue queue;
    alignas(8) uint8_t prefix[prefix_bytes(kSmemRequests)];
    uint32_t mask[Cfg<D>::kMasks];     // present 16-token groups of the tiles in flight
    int parts[2];                      // partial results to merge, 0: another CTA does
    uint16_t part[2][kMaxParts];
    int gave_up;
    uint32_t tmem;
};

// ---- the work list -----------------------------------------------------------------
// item = two query tiles (the last one of a request may be a single tile), unit = KV tile.  Cost in tokens seen, twice
// for two tiles.
struct AttendWork {
    const int32_t *cu, *seq_lens;
    int T, max_tokens, tpt;            // tpt: new tokens of a query tile

    __device__ __forceinline__ explicit AttendWork(const AttendArgs &a)
        : cu(a.cu), seq_lens(a.seq_lens), T(a.T), max_tokens(a.page_table ? a.max_pages * kPage : a.T), tpt(kTile / a.G) {}
    __device__ __forceinline__ TokenRange tokens(int r) const { return token_range(cu, seq_lens, r, T, max_tokens); }
    __device__ __forceinline__ int items(const TokenRange &t) const { return (t.n + 2 * tpt - 1) / (2 * tpt); }
    __device__ __forceinline__ int new_tokens(const TokenRange &t, int i) const { return min(2 * tpt, t.n - i * 2 * tpt); }
    __device__ __forceinline__ long long cost(const TokenRange &t, long long i) const {
        const int full = t.n / (2 * tpt);
        const long long m = min(i, (long long)full);
        long long c = 2 * (m * (t.past + kItemCost) + 2 * tpt * (m * (m + 1) / 2));
        if (i > full) c += (long long)(t.n - full * 2 * tpt > tpt ? 2 : 1) * (t.past + t.n + kItemCost);
        return c;
    }
    __device__ __forceinline__ int units(const TokenRange &t, int i) const {
        return (t.past + i * 2 * tpt + new_tokens(t, i) + kKv - 1) / kKv;
    }
    __device__ __forceinline__ int unit_at(const TokenRange &t, int i, long long z) const {
        return (int)(z / (kKv * (new_tokens(t, i) > tpt ? 2 : 1)));
    }
    __device__ __forceinline__ long long min_cost() const { return kMinCost; }
    static constexpr int kCrumb = 4;   // least units of a part of an item
};

struct Segment {
    int r, h, item;
    TokenRange t;
    int tok0, ntok;        // new tokens of the item, relative to the request
    bool alt;
    int piece, a, b, nkv;  // piece, its KV tiles of the item, the item's
    int steps0, steps1;    // KV tiles per stream
    __device__ __forceinline__ int steps(int st) const { return st ? steps1 : steps0; }
};

// The next part of an item in the piece; every role walks the same list.
__device__ __forceinline__ bool next_segment(Walk<AttendWork> &walk, Segment &s) {
    if (!walk.find()) return false;
    const AttendWork &w = walk.l.w;
    s.r = walk.r, s.h = walk.h, s.item = walk.item, s.t = walk.t;
    s.tok0 = walk.i * 2 * w.tpt;
    s.ntok = w.new_tokens(walk.t, walk.i);
    s.alt = s.ntok <= w.tpt;
    s.nkv = w.units(walk.t, walk.i);
    s.a = walk.unit, s.piece = walk.piece;
    s.b = walk.end_unit(s.nkv);
    if (s.alt) {
        s.steps0 = (s.b - s.a + 1) / 2;
        s.steps1 = (s.b - s.a) / 2;
    } else {
        const int n0 = (walk.t.past + s.tok0 + w.tpt + kKv - 1) / kKv;        // the first tile's tokens see no more than this
        s.steps0 = max(min(s.b, n0) - s.a, 0);
        s.steps1 = s.b - s.a;
    }
    walk.next();
    return true;
}

// ---- copies ------------------------------------------------------------------------
// One warp brings K (and Q), one V: each has every second slot of the ring.  A tile is 64 tokens of one head.  K lies as
// [D/64][64 tokens][64 channels]: a page is D/64 copies (one for all where K is contiguous).  V lies as
// [4][D/64][16 tokens][64 channels], because a product takes 16 tokens at a time: a page is one copy.
// Groups that are absent or past the end come from behind the tensor's last row, which reads as zeros.

// Pages of 32 groups of 16 tokens at a time, a lane each, and of the next 32 ahead.  Contiguous K and V: 0 for "present".
struct Pages {
    int ids, next, block;

    __device__ __forceinline__ int fetch(const AttendArgs &a, const Segment &s, int g, bool report) const {
        if (g * kPage >= s.t.past + s.t.n) return -1;
        if (!a.page_table) return 0;
        const int pid = a.page_table[(size_t)s.r * a.max_pages + g];
        if (pid >= a.P_phys) {
            if (report) atomicOr(&a.ctl->status, SE_DEV_BAD_PAGE_ID);
            return -1;
        }
        return pid < 0 ? -1 : pid;
    }
    __device__ __forceinline__ void begin(const AttendArgs &a, const Segment &s, int tile, bool report, int lane) {
        block = tile / 8;
        ids = fetch(a, s, block * 32 + lane, report);
        next = fetch(a, s, block * 32 + 32 + lane, report);
    }
    // tiles come in ascending order
    __device__ __forceinline__ void reach(const AttendArgs &a, const Segment &s, int tile, bool report, int lane) {
        if (tile / 8 == block) return;
        ++block;
        ids = next;
        next = fetch(a, s, block * 32 + 32 + lane, report);
    }
    __device__ __forceinline__ int of(int tile, int pg) const { return __shfl_sync(kFull, ids, (tile & 7) * 4 + pg); }
};

// The end of a copying warp, whose next position would be `pos`: nothing may still be on its way to the CTA's shared memory
// when the CTA ends - copies, and the products' arrivals on the barriers of the slots they have let go.
template <int D>
__device__ __forceinline__ void leave_ring(bool ok, uint32_t pos, uint32_t first, uint32_t bars, volatile int *gave_up,
                                           const AttendArgs &a) {
    constexpr uint32_t kSlots = Cfg<D>::kSlots;
    for (uint32_t p = pos >= kSlots + first ? pos - kSlots : first; p < pos; p += 2) {
        const uint32_t bar = bars + 8 * (kRing + p % kSlots), parity = p / kSlots & 1;
        if (ok) ok = warp_wait(bar + 8 * kSlots, parity, gave_up, &a.ctl->status);
        else mbar_wait(bar, parity);
    }
}

template <int D>
__device__ __forceinline__ void k_role(const AttendArgs &a, const List<AttendWork> &list, const CUtensorMap *q_map, const CUtensorMap *k_map, const CUtensorMap *k_wide,
                                       Control<D> *ctl, uint32_t q_smem, uint32_t ring, uint32_t bars, int lane) {
    using C = Cfg<D>;
    volatile int *gave_up = &ctl->gave_up;
    const int tpt = kTile / a.G;
    Segment s;
    Pages pages;
    uint32_t pos = 0, tiles = 0, queries = 0;
    const bool chosen = elect_one();
    bool ok = true;
    Walk<AttendWork> walk(list, a.ctl, &ctl->queue, gave_up, lane, true);
    while (ok && next_segment(walk, s)) {
        const int stop = s.t.past + s.t.n;                                 // tokens of the request
        pages.begin(a, s, s.a, true, lane);
        ok = warp_wait(bars + 8 * kQEmpty, (queries & 1) ^ 1, gave_up, &a.ctl->status);
        if (!ok) break;
        if (chosen) {
            mbar_expect_tx(bars + 8 * kQFull, (s.alt ? 1 : 2) * tpt * a.G * D * 2);
            for (int st = 0; st < (s.alt ? 1 : 2); ++st)
                for (int half = 0; half < C::kHalves; ++half)
                    tma_load_3d(q_smem + st * C::kTileBytes + half * (kTile * 128), q_map, half * 64, s.h * a.G,
                                s.t.start + s.tok0 + st * tpt, bars + 8 * kQFull);
        }
        __syncwarp();
        ++queries;
        for (int t = s.a; t < s.b; ++t, ++tiles, pos += 2) {
            const uint32_t slot = pos % C::kSlots, bar = bars + 8 * (kRing + slot), dst = ring + slot * C::kKvBytes;
            pages.reach(a, s, t, true, lane);
            const unsigned mask = __ballot_sync(kFull, pages.ids >= 0) >> (t & 7) * 4 & 0xfu;
            int pid[4];
#pragma unroll
            for (int pg = 0; pg < 4; ++pg) pid[pg] = pages.of(t, pg);
            ok = warp_wait(bar + 8 * C::kSlots, (pos / C::kSlots & 1) ^ 1, gave_up, &a.ctl->status);
            if (!ok) break;
            if (chosen) {
                ctl->mask[tiles % C::kMasks] = mask;
                mbar_expect_tx(bar, C::kKvBytes);
                if (!a.page_table && (t + 1) * kKv <= stop) {
                    tma_load_4d(dst, k_wide, 0, s.h, s.t.start + t * kKv, 0, bar);
                } else {
#pragma unroll
                    for (int pg = 0; pg < 4; ++pg) {
                        const int y = a.page_table ? 0 : s.h;
                        const int z = pid[pg] < 0 ? (a.page_table ? a.P_phys * a.H_kv * kPage : a.T)
                                                  : a.page_table ? (pid[pg] * a.H_kv + s.h) * kPage : s.t.start + t * kKv + pg * kPage;
#pragma unroll
                        for (int half = 0; half < C::kHalves; ++half)
                            tma_load_3d(dst + half * (kKv * 128) + pg * (kPage * 128), k_map, half * 64, y, z, bar);
                    }
                }
            }
            __syncwarp();
        }
    }
    leave_ring<D>(ok, pos, 0, bars, gave_up, a);
    if (queries) {
        if (ok) warp_wait(bars + 8 * kQEmpty, (queries - 1) & 1, gave_up, &a.ctl->status);
        else mbar_wait(bars + 8 * kQFull, (queries - 1) & 1);
    }
}

template <int D>
__device__ __forceinline__ void v_role(const AttendArgs &a, const List<AttendWork> &list, const CUtensorMap *v_map, Control<D> *ctl, uint32_t ring, uint32_t bars, int lane) {
    using C = Cfg<D>;
    volatile int *gave_up = &ctl->gave_up;
    Segment s;
    Pages pages;
    uint32_t pos = 1;
    const bool chosen = elect_one();
    bool ok = true;
    Walk<AttendWork> walk(list, a.ctl, &ctl->queue, gave_up, lane, false);
    while (ok && next_segment(walk, s)) {
        const int stop = s.t.past + s.t.n;                                 // tokens of the request
        pages.begin(a, s, s.a, false, lane);
        for (int t = s.a; t < s.b; ++t, pos += 2) {
            const uint32_t slot = pos % C::kSlots, bar = bars + 8 * (kRing + slot), dst = ring + slot * C::kKvBytes;
            pages.reach(a, s, t, false, lane);
            int pid[4];
#pragma unroll
            for (int pg = 0; pg < 4; ++pg) pid[pg] = pages.of(t, pg);
            ok = warp_wait(bar + 8 * C::kSlots, (pos / C::kSlots & 1) ^ 1, gave_up, &a.ctl->status);
            if (!ok) break;
            // The group that holds the end of the request is copied row by row: what lies behind the end may be anything, and
            // a weight of zero would not hide a NaN.
            const int part = stop % kPage && stop / kKv == t ? stop % kKv / kPage : -1;
            bool by_hand = false;
#pragma unroll
            for (int pg = 0; pg < 4; ++pg) {
                if (pg != part || pid[pg] < 0) continue;
                by_hand = true;
                const int tok = t * kKv + pg * kPage;
                const uint16_t *base = a.page_table ? a.v + ((size_t)pid[pg] * a.H_kv + s.h) * (kPage * D)
                                                    : a.v + (long long)(s.t.start + tok) * a.v_stride + s.h * D;
                const long long pitch = a.page_table ? D : a.v_stride;
                constexpr int kPieces = D / 8;
#pragma unroll
                for (int i = 0; i < kPage * kPieces / 32; ++i) {
                    const int e = i * 32 + lane, row = e / kPieces, ch = e % kPieces;
                    uint4 x = make_uint4(0, 0, 0, 0);
                    if (row < stop - tok) x = *reinterpret_cast<const uint4 *>(base + row * pitch + ch * 8);
                    const uint32_t at = dst + pg * (kPage * D * 2) + (ch >> 3) * (kPage * 128) + row * 128 + (((ch & 7) ^ (row & 7)) << 4);
                    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
                }
                fence_async_proxy();
                __syncwarp();
            }
            if (chosen) {
                mbar_expect_tx(bar, C::kKvBytes - (by_hand ? kPage * D * 2 : 0));
#pragma unroll
                for (int pg = 0; pg < 4; ++pg) {
                    if (pg == part && by_hand) continue;
                    const int y = a.page_table ? 0 : s.h;
                    const int z = pid[pg] < 0 ? (a.page_table ? a.P_phys * a.H_kv * kPage : a.T)
                                              : a.page_table ? (pid[pg] * a.H_kv + s.h) * kPage : s.t.start + t * kKv + pg * kPage;
                    tma_load_4d(dst + pg * (kPage * D * 2), v_map, 0, y, z, 0, bar);
                }
            }
            __syncwarp();
        }
    }
    leave_ring<D>(ok, pos, 1, bars, gave_up, a);
}

// ---- products ----------------------------------------------------------------------
// The scores of a KV tile of 64 tokens take 64 columns, so every stream has two score buffers, and the next scores are there
// when the softmax gets to them.  (Tiles of 128 tokens leave room for one buffer: products and softmax of a stream then
// wait for one another, and the tensor cores stood idle for 40 % of the time.  A score product of 64 columns is bound by
// shared memory, 49 cycles instead of 32: 20 % of both products, the smaller loss.)
// One warp per stream issues its products: a wait queues up behind the products that its own warp has issued, so a single
// warp for both streams let the tensor cores run dry at every wait.  The whole warp walks the list, so that addresses stay in
// uniform registers; one elected lane issues.
template <int D, int ST>
__device__ __forceinline__ void mma_role(const AttendArgs &a, const List<AttendWork> &list, Control<D> *ctl, uint32_t q_smem, uint32_t ring, uint32_t bars, int lane) {
    using C = Cfg<D>;
    volatile int *gave_up = &ctl->gave_up;
    const uint32_t tmem_s = ctl->tmem + ST * kTile, tmem_o = ctl->tmem + C::kTmemO + ST * D;
    Segment s = {};
    uint32_t pos = 0, queries = 0, o_used = 0, n = 0;                      // n: steps so far
    bool any = false;
    const bool chosen = elect_one();
    auto wait = [&](int bar, uint32_t parity) { return warp_wait(bars + 8 * bar, parity & 1, gave_up, &a.ctl->status); };
    auto slot = [&](uint32_t at) { return ring + at % C::kSlots * C::kKvBytes; };
    // a ring slot is free when both streams have let it go
    auto let_go = [&](uint32_t at) { mma_commit(bars + 8 * (kRing + C::kSlots + at % C::kSlots)); };
    // S = Q K^T of the n-th step
    auto scores = [&](uint32_t at, uint32_t n) {
        const uint64_t qd = smem_operand(q_smem + (s.alt ? 0 : ST * C::kTileBytes), 16, 1024), kd = smem_operand(slot(at), 16, 1024);
        const uint32_t d = tmem_s + (n & 1) * kKv;
        tc_fence_after();
        if (chosen) {
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
                mma_ss(d, qd + (k / 4) * (kTile * 128 >> 4) + (k % 4) * 2, kd + (k / 4) * (kKv * 128 >> 4) + (k % 4) * 2, mma_instr(kKv, false),
                       k > 0);
            mma_commit(bars + 8 * (kSFull + 2 * ST + (n & 1)));
            let_go(at);
        }
        __syncwarp();
    };
    // O += P V
    auto values = [&](uint32_t at, uint32_t n, bool accumulate, bool last) {
        const uint64_t vd = smem_operand(slot(at), kPage * 128, 1024);
        const uint32_t p = tmem_s + (n & 1) * kKv;
        tc_fence_after();
        if (chosen) {
#pragma unroll
            for (int k = 0; k < kKv / 16; ++k) mma_ts(tmem_o, p + k * 8, vd + k * (kPage * D * 2 >> 4), mma_instr(D, true), accumulate || k > 0);
            mma_commit(bars + 8 * ((last ? kOLast : kODone) + ST));
            let_go(at);
        }
        __syncwarp();
    };
    bool ok = true;
    Walk<AttendWork> walk(list, a.ctl, &ctl->queue, gave_up, lane, false);
    while (ok && next_segment(walk, s)) {
        const int steps = ST ? s.steps1 : s.steps0;
        const int tiles = s.b - s.a, stride = s.alt ? 2 : 1, first = s.alt ? ST : 0;   // this stream's tiles: first, first + stride, ...
        // Every tile's barriers are waited for, in order, and the tiles of the other stream let go at once: a barrier tells its
        // phases apart by parity alone, so a warp that left one out could take the phase before for the one it waits for.
        auto reach = [&](int &next, int last, uint32_t v) {
            for (; next <= last; ++next) {
                const uint32_t at = pos + 2 * next + v;
                if (!wait(kRing + at % C::kSlots, at / C::kSlots)) return false;
                const bool mine = s.alt ? (next & 1) == ST : next < steps;
                if (!mine && chosen) mbar_arrive(bars + 8 * (kRing + C::kSlots + at % C::kSlots));
                __syncwarp();
            }
            return true;
        };
        int k_next = 0, v_next = 0;
        ok = wait(kQFull, queries);
        ++queries;
        for (int u = 0; u < 2 && u < steps && ok; ++u)
            if ((ok = reach(k_next, first + u * stride, 0))) scores(pos + 2 * (first + u * stride), n + u);
        any = any || steps > 0;
        if (!ok) break;
        if (chosen && steps <= 2) {
            if (steps > 0) mma_commit(bars + 8 * kQEmpty);
            else mbar_arrive(bars + 8 * kQEmpty);
        }
        __syncwarp();
        for (int u = 0, t = first; u < steps && ok; ++u, ++n, t += stride) {
            // everything that can be waited for early comes before the wait for the weights
            const bool more = u + 2 < steps;
            ok = reach(v_next, t, 1) && (!more || reach(k_next, t + 2 * stride, 0));
            if (ok && u == 0) {          // the epilogue of the stream's last piece has read O
                ok = wait(kOFree + ST, o_used ^ 1);
                o_used ^= 1;
            }
            ok = ok && wait(kPReady + 2 * ST + (n & 1), n >> 1);
            if (!ok) break;
            values(pos + 2 * t + 1, n, u > 0, u + 1 == steps);
            if (more) scores(pos + 2 * (t + 2 * stride), n);
            if (chosen && u + 3 == steps) mma_commit(bars + 8 * kQEmpty);   // the last product with Q is on its way
            __syncwarp();
        }
        while (ok && v_next < tiles) ok = reach(k_next, v_next, 0) && reach(v_next, v_next, 1);
        __syncwarp();
        pos += 2u * tiles;
    }
    if (any) {                           // nothing may be running when tensor memory goes away
        if (chosen) mma_commit(bars + 8 * (kDrain + ST));
        __syncwarp();
        mbar_wait(bars + 8 * (kDrain + ST), 0);
    }
}

// ---- softmax and epilogue ----------------------------------------------------------
__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }

// Partial results: two kinds per piece (of the item that it ends, of the item that it begins) and stream.
__device__ __forceinline__ int partial_index(int piece, int kind, int st) { return (piece * 2 + kind) * 2 + st; }
template <int D>
__device__ __forceinline__ float *partial_slot(const AttendArgs &a, int index) {
    return a.partials + (size_t)index * Cfg<D>::kSlotFloats;
}

// Merges `parts` partial results of one query tile, at(k) their indexes, and writes its output.  A warp takes rows row_from,
// row_from + row_step, ...
template <int D, typename At>
__device__ __forceinline__ void merge_rows(const AttendArgs &a, const Segment &s, int st, int row_from, int row_step, int parts, At at,
                                           int lane) {
    constexpr int V = D / 32, R = 8;   // channels of a lane, rows at a time
    const int tpt = kTile / a.G;
    const int tok = s.tok0 + (s.alt ? 0 : st * tpt);
    const int rows = min(tpt, s.tok0 + s.ntok - tok) * a.G;
    const long long out0 = ((long long)(s.t.start + tok) * a.H_q + s.h * a.G);
    const int my = row_from + row_step * lane;                             // statistics: a lane per row
    const bool have = my < rows;
    float M = -INFINITY, L = 0.f;
#pragma unroll 4
    for (int k = 0; k < parts; ++k) {
        const float *p = partial_slot<D>(a, at(k)) + kTile * D;
        const float m = have ? __ldcg(p + my) : -INFINITY, l = have ? __ldcg(p + kTile + my) : 0.f;
        const float top = fmaxf(M, m), ref = top == -INFINITY ? 0.f : top;
        L = L * ex2(M - ref) + l * ex2(m - ref);
        M = top;
    }
    const float inv = L > 0.f ? 1.f / L : 0.f, ref = M == -INFINITY ? 0.f : M;
    if (have && a.lse) a.lse[out0 + (long long)(my / a.G) * a.H_q + my % a.G] = L > 0.f ? (M + log2f(L)) * kLn2 : -INFINITY;
    const int mine = rows > row_from ? (rows - row_from + row_step - 1) / row_step : 0;
    for (int k0 = 0; k0 < mine; k0 += R) {
        float acc[R][V] = {};
#pragma unroll 2
        for (int q = 0; q < parts; ++q) {
            const float *p = partial_slot<D>(a, at(q));
            const float w = have ? ex2(__ldcg(p + kTile * D + my) - ref) * inv : 0.f;
            float x[R][V];
#pragma unroll
            for (int k = 0; k < R; ++k) {
                // a row beyond the last is read as the last
                const float *src = p + (size_t)(row_from + row_step * min(k0 + k, mine - 1)) * D + lane * V;
                if constexpr (V == 4) {
                    const float4 f = __ldcg(reinterpret_cast<const float4 *>(src));
                    x[k][0] = f.x, x[k][1] = f.y, x[k][2] = f.z, x[k][3] = f.w;
                } else {
                    const float2 f = __ldcg(reinterpret_cast<const float2 *>(src));
                    x[k][0] = f.x, x[k][1] = f.y;
                }
            }
#pragma unroll
            for (int k = 0; k < R; ++k) {
                const float wk = __shfl_sync(kFull, w, min(k0 + k, 31));
#pragma unroll
                for (int v = 0; v < V; ++v) acc[k][v] += wk > 0.f ? wk * x[k][v] : 0.f;   // a result without weight may be anything
            }
        }
#pragma unroll
        for (int k = 0; k < R; ++k) {
            if (k0 + k >= mine) break;
            const int row = row_from + row_step * (k0 + k);
            uint32_t w[V / 2];
#pragma unroll
            for (int v = 0; v < V / 2; ++v) {
                const __nv_bfloat162 b = __float22bfloat162_rn(make_float2(acc[k][2 * v], acc[k][2 * v + 1]));
                w[v] = *reinterpret_cast<const uint32_t *>(&b);
            }
            uint16_t *dst = a.out + (out0 + (long long)(row / a.G) * a.H_q + row % a.G) * D + lane * V;
            if constexpr (V == 4) *reinterpret_cast<uint2 *>(dst) = make_uint2(w[0], w[1]);
            else *reinterpret_cast<uint32_t *>(dst) = w[0];
        }
    }
}

template <int D>
__device__ __forceinline__ void softmax_role(const AttendArgs &a, const List<AttendWork> &list, Control<D> *ctl, uint32_t bars, int st) {
    using C = Cfg<D>;
    volatile int *gave_up = &ctl->gave_up;
    const int row = threadIdx.x & 127, lane = threadIdx.x & 31, warp = row >> 5;
    const int tpt = kTile / a.G;
    const uint32_t lanes = (uint32_t)(warp * 32) << 16;
    const uint32_t t_s = ctl->tmem + lanes + st * kTile, t_o = ctl->tmem + lanes + C::kTmemO + st * D;
    const float sl = a.scale_log2;
    Segment s;
    uint32_t step = 0, tiles = 0, verdicts = 0, swaps = 0, ends = 0;
    uint32_t inner = 0;                                                    // steps so far that were not a piece's last of an item
    // both warpgroups have come here
    auto swap_sync = [&] {
        __syncwarp();
        if (lane == 0) mbar_arrive(bars + 8 * kSwap);
        return warp_wait(bars + 8 * kSwap, swaps++ & 1, gave_up, &a.ctl->status);
    };
    Walk<AttendWork> walk(list, a.ctl, &ctl->queue, gave_up, lane, false);
    while (next_segment(walk, s)) {
        const int tok = s.tok0 + (s.alt ? 0 : st * tpt);                   // the tile's first new token
        const int ntok = min(tpt, s.tok0 + s.ntok - tok);
        const int q = min(row / a.G, ntok - 1);
        const int sees = s.t.past + tok + q + 1;                           // tokens the row sees
        const int least = __reduce_min_sync(kFull, sees);
        const int steps = s.steps(st);
        float m = -INFINITY;                                               // in units of the raw scores
        float2 l2 = make_float2(0.f, 0.f);
        for (int u = 0; u < steps; ++u, ++step) {
            const int rel = s.alt ? 2 * u + st : u, first = (s.a + rel) * kKv;
            const uint32_t buf = 2 * st + (step & 1), t_p = t_s + (step & 1) * kKv;
            if (!warp_wait(bars + 8 * (kSFull + buf), step >> 1 & 1, gave_up, &a.ctl->status)) return;
            tc_fence_after();
            float x[kKv];
            tmem_ld32(t_p, x);
            tmem_ld32(t_p + 32, x + 32);
            const unsigned mask = ctl->mask[(tiles + rel) % C::kMasks];
            tmem_wait_ld();
            settle<kKv>(x);
            if (first + kKv > least || mask != 0xfu) {
                const int limit = sees - first;
#pragma unroll
                for (int k = 0; k < kKv; ++k)
                    if (k >= limit || !(mask >> (k / kPage) & 1)) x[k] = -INFINITY;
            }
            float top[4] = {m, m, m, m};
#pragma unroll
            for (int k = 0; k < kKv; k += 8)
#pragma unroll
                for (int e = 0; e < 4; ++e) top[e] = max3(top[e], x[k + e], x[k + 4 + e]);
            const float mn = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
            if (__any_sync(kFull, (mn - m) * sl > kSlack)) {
                const float f = m == -INFINITY ? 0.f : ex2((m - mn) * sl);
                m = mn;
                l2.x *= f, l2.y *= f;
                if (u > 0) {
                    // O + P V of the last step; the one before is complete (these scores were issued behind it), so the barrier's
                    // parity says which of two phases it is in
                    if (!warp_wait(bars + 8 * (kODone + st), (inner + u - 1) & 1, gave_up, &a.ctl->status)) return;
                    tc_fence_after();
#pragma unroll 1
                    for (int k = 0; k < D; k += 32) {
                        float o[32];
                        tmem_ld32(t_o + k, o);
                        tmem_wait_ld();
                        settle<32>(o);
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] *= f;
                        tmem_st32(t_o + k, reinterpret_cast<const uint32_t *>(o));
                    }
                }
            }
            const float off = m == -INFINITY ? 0.f : -m * sl;
            uint32_t p[kKv / 2];
#pragma unroll
            for (int e = 0; e < kKv / 2; ++e) {
                const float2 y = ffma2(make_float2(x[2 * e], x[2 * e + 1]), make_float2(sl, sl), make_float2(off, off));
                const float2 w = make_float2(ex2(y.x), ex2(y.y));
                l2 = __fadd2_rn(l2, w);
                // the weights enter the product with V as bf16 (8 significant bits), their sum keeps fp32
                const __nv_bfloat162 b = __float22bfloat162_rn(w);
                p[e] = *reinterpret_cast<const uint32_t *>(&b);
            }
            tmem_st32(t_p, p);
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bars + 8 * (kPReady + buf));
            __syncwarp();
        }
        tiles += s.b - s.a;
        inner += max(steps - 1, 0);
        if (steps > 0) {
            if (!warp_wait(bars + 8 * (kOLast + st), ends++ & 1, gave_up, &a.ctl->status)) return;
            tc_fence_after();
        }

        // ---- epilogue ----
        const float l = l2.x + l2.y, m2 = m == -INFINITY ? m : m * sl;
        const bool live = row < ntok * a.G;
        const bool whole = s.a == 0 && s.b == s.nkv;
        const bool direct = whole && (!s.alt || s.nkv == 1);
        const long long orow = (long long)(s.t.start + tok + q) * a.H_q + s.h * a.G + row % a.G;
        if (direct) {
            if (s.alt && st == 1) continue;                                // a single KV tile: stream 0 has it all
            const float inv = l > 0.f ? 1.f / l : 0.f;
            uint4 *dst = reinterpret_cast<uint4 *>(a.out + orow * D);
#pragma unroll
            for (int k = 0; k < D; k += 32) {
                float o[32];
                tmem_ld32(t_o + k, o);
                tmem_wait_ld();
                settle<32>(o);
                uint32_t w[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const __nv_bfloat162 b = __float22bfloat162_rn(make_float2(o[2 * e] * inv, o[2 * e + 1] * inv));
                    w[e] = *reinterpret_cast<const uint32_t *>(&b);
                }
                if (live) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) dst[k / 8 + e] = make_uint4(w[4 * e], w[4 * e + 1], w[4 * e + 2], w[4 * e + 3]);
                }
            }
            if (live && a.lse) a.lse[orow] = l > 0.f ? (m2 + log2f(l)) * kLn2 : -INFINITY;
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bars + 8 * (kOFree + st));
            __syncwarp();
            continue;
        }
        const int kind = s.a == 0;
        if (steps > 0 || !s.alt) {
            float *slot = partial_slot<D>(a, partial_index(s.piece, kind, st));
            if (steps > 0) {
#pragma unroll
                for (int k = 0; k < D; k += 32) {
                    float o[32];
                    tmem_ld32(t_o + k, o);
                    tmem_wait_ld();
                    settle<32>(o);
                    if (live) {
                        float4 *dst = reinterpret_cast<float4 *>(slot + (size_t)row * D + k);
#pragma unroll
                        for (int e = 0; e < 8; ++e) __stcg(dst + e, make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]));
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bars + 8 * (kOFree + st));
                __syncwarp();
            }
            __stcg(slot + kTile * D + row, m2);
            __stcg(slot + kTile * D + kTile + row, l);
        }
        if (whole) {
            // alt, all KV tiles in this CTA: the two warpgroups exchange their results and merge half of the rows each
            if (!swap_sync()) return;
            const int slot = partial_index(s.piece, kind, 0);
            merge_rows<D>(a, s, st, st * 4 + warp, 8, 2, [&](int k) { return slot + k; }, lane);
            if (!swap_sync()) return;                                      // the slots may be written again
            continue;
        }
        if (steps == 0 && s.alt) continue;
        __threadfence();
        __syncwarp();
        if (lane == 0) mbar_arrive(bars + 8 * (kAll + st));
        __syncwarp();
        if (warp == 0) {
            const int from = first_piece_of(list, s.item, s.piece, lane);
            if (!warp_wait(bars + 8 * (kAll + st), verdicts & 1, gave_up, &a.ctl->status)) return;
            int last = 0;
            if (lane == 0) {
                __threadfence();
                uint32_t *ticket = a.ctl->tickets + 2 * from + (s.alt ? 0 : st);
                const uint32_t add = s.alt ? steps : s.b - s.a;
                last = atomicAdd(ticket, add) + add == (uint32_t)s.nkv;
                if (last) atomicExch(ticket, 0u);
            }
            int parts = 0;
            if (__shfl_sync(kFull, last, 0)) {
                auto add = [&](int index) {
                    if (lane == 0 && parts < kMaxParts) ctl->part[st][parts] = (uint16_t)index;
                    ++parts;
                };
                each_piece_of(list, s.item, s.nkv, from, lane, [&](int y, int ya, int yb) {
                    add(partial_index(y, ya == 0, s.alt ? 0 : st));
                    if (s.alt && yb - ya > 1) add(partial_index(y, ya == 0, 1));
                });
            }
            if (lane == 0) {
                ctl->parts[st] = min(parts, kMaxParts);
                mbar_arrive(bars + 8 * (kVerdict + st));
            }
            __syncwarp();
        }
        if (!warp_wait(bars + 8 * (kVerdict + st), verdicts & 1, gave_up, &a.ctl->status)) return;
        ++verdicts;
        const int parts = ctl->parts[st];
        if (parts) {
            __threadfence();
            merge_rows<D>(a, s, st, warp, 4, parts, [&](int k) { return (int)ctl->part[st][k]; }, lane);
        }
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
attend_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
              const __grid_constant__ CUtensorMap k_wide, const __grid_constant__ CUtensorMap v_map,
              const __grid_constant__ AttendArgs a) {
    using C = Cfg<D>;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    Control<D> *ctl = reinterpret_cast<Control<D> *>(smem + 2 * C::kTileBytes + C::kSlots * C::kKvBytes);
    const uint32_t bars = smem_u32(ctl->bars);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (base & 1023u) {                  // the swizzle pattern hangs on the address
        if (threadIdx.x == 0) atomicOr(&a.ctl->status, SE_DEV_WAIT_TIMEOUT);
        return;
    }

    if (threadIdx.x == 0) {
        mbar_init(bars + 8 * kQFull, 1);
        mbar_init(bars + 8 * kQEmpty, 2);
        for (int st = 0; st < 2; ++st) {
            for (int buf = 2 * st; buf < 2 * st + 2; ++buf) {
                mbar_init(bars + 8 * (kSFull + buf), 1);
                mbar_init(bars + 8 * (kPReady + buf), 4);
            }
            mbar_init(bars + 8 * (kODone + st), 1);
            mbar_init(bars + 8 * (kOLast + st), 1);
            mbar_init(bars + 8 * (kOFree + st), 4);
            mbar_init(bars + 8 * (kAll + st), 4);
            mbar_init(bars + 8 * (kVerdict + st), 1);
            mbar_init(bars + 8 * (kDrain + st), 1);
        }
        mbar_init(bars + 8 * kSwap, 8);
        for (int i = 0; i < C::kSlots; ++i) {
            mbar_init(bars + 8 * (kRing + i), 1);
            mbar_init(bars + 8 * (kRing + C::kSlots + i), 2);
        }
        ctl->queue.init(11);
        mbar_fence_init();
        ctl->gave_up = 0;
    }
    if (warp == kMmaWarp) tmem_alloc(smem_u32(&ctl->tmem), 512);
    const AttendWork work(a);
    const List<AttendWork> list = make_list(work, a.B, a.H_kv, a.ctl,
                                            a.B > kSmemRequests ? a.prefixes + prefix_bytes(a.B) * blockIdx.x : ctl->prefix, smem);
    // query rows that no tensor copy fills (G does not divide 128) stay zero
    for (int i = threadIdx.x; i < 2 * C::kTileBytes / 16; i += kThreads)
        reinterpret_cast<uint4 *>(smem)[i] = make_uint4(0, 0, 0, 0);
    fence_async_proxy();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();

    if (warp < 8) {
        softmax_role<D>(a, list, ctl, bars, warp >> 2);
    } else {
        if (warp == kKWarp) k_role<D>(a, list, &q_map, &k_map, &k_wide, ctl, base, base + 2 * C::kTileBytes, bars, lane);
        else if (warp == kVWarp) v_role<D>(a, list, &v_map, ctl, base + 2 * C::kTileBytes, bars, lane);
        else if (warp == kMmaWarp) mma_role<D, 0>(a, list, ctl, base, base + 2 * C::kTileBytes, bars, lane);
        else if (warp == kMmaWarp + 1) mma_role<D, 1>(a, list, ctl, base, base + 2 * C::kTileBytes, bars, lane);
        __syncwarp();
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_free(ctl->tmem, 512);
    }
}

// ---- host side ---------------------------------------------------------------------
template <int D>
cudaError_t launch_attend(const se_params &p, const AttendCall &c, cudaStream_t stream) {
    using C = Cfg<D>;
    const int G = p.H_q / p.H_kv;
    CUtensorMap q_map, k_map, k_wide, v_map;
    bool ok = make_rows_map(&q_map, c.q, D, p.H_q, c.total_tokens, c.q_stride, G, kTile / G);
    if (c.page_table) {
        const long long rows = (long long)p.num_phys_pages * p.H_kv * kPage;
        ok = ok && make_rows_map(&k_map, c.k, D, 1, rows, D, 1, kPage) && make_split_map(&v_map, c.v, D, 1, rows, D, kPage);
        k_wide = k_map;                                          // not used
    } else {
        ok = ok && make_rows_map(&k_map, c.k, D, p.H_kv, c.total_tokens, c.k_stride, 1, kPage) &&
             make_split_map(&k_wide, c.k, D, p.H_kv, c.total_tokens, c.k_stride, kKv) &&
             make_split_map(&v_map, c.v, D, p.H_kv, c.total_tokens, c.v_stride, kPage);
    }
    if (!ok) return cudaErrorInvalidValue;
    AttendArgs a = {};
    a.cu = c.cu_seqlens, a.seq_lens = c.seq_lens, a.page_table = c.page_table;
    a.v = static_cast<const uint16_t *>(c.v), a.v_stride = c.v_stride;
    a.out = static_cast<uint16_t *>(c.out), a.lse = c.lse;
    a.ctl = reinterpret_cast<PromptControl *>(c.workspace);
    a.partials = reinterpret_cast<float *>(c.workspace + kPromptControlBytes);
    a.prefixes = c.workspace + prefix_workspace_offset(p.D);
    a.B = p.B, a.H_q = p.H_q, a.H_kv = p.H_kv, a.G = G, a.T = c.total_tokens, a.max_pages = p.max_pages;
    a.P_phys = p.num_phys_pages, a.scale_log2 = effective_scale(p) * kLog2e;
    auto kern = attend_kernel<D>;
    cudaError_t e;
    const size_t smem = 2 * C::kTileBytes + C::kSlots * C::kKvBytes + sizeof(Control<D>);
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    kern<<<kPromptCtas, kThreads, smem, stream>>>(q_map, k_map, k_wide, v_map, a);
    return cudaGetLastError();
}

}  // namespace

size_t prompt_workspace_control_bytes() { return kPromptControlBytes; }
size_t prompt_workspace_bytes(const se_params &p) {
    return prefix_workspace_offset(p.D) + (prefix_workspace_bytes(p.B) + 255) / 256 * 256;
}

cudaError_t launch_prompt_attend(const se_params &p, const AttendCall &c, cudaStream_t stream) {
    return p.D == 128 ? launch_attend<128>(p, c, stream) : launch_attend<64>(p, c, stream);
}

}  // namespace se
