// Attention of a packed batch of new tokens (Appendix A, attention equations of "MHA, MQA, and GQA"), over the paged
// cache or over contiguous K and V.
//
// Mathematics.  A query tile is 128 rows = 128/G tokens x the G query heads of one kv-head, so the heads of a group share
// every K and V tile.  Over the KV tiles j of 128 tokens:  S = Q K_j^T,  p = 2^(S sl - m)  with sl = sm_scale log2 e,
// O += P V_j, l += rowsum p (with compensation);  out = O / l,  lse = (m + log2 l) ln 2.  m is a row maximum that is moved (and O, l
// rescaled) only when the scores exceed it by more than 40, so nearly all steps leave O alone.
//
// What bounds it.  Per (128 rows x 128 tokens) at D = 128 the two products take 1024 cycles of the tensor cores and
// the 16384 exponentials 1024 cycles of the special-function units: both have to run all the time.  So a CTA (one per
// SM, persistent) works on two streams of tiles: two warpgroups do the softmax of one stream each, one warp issues all
// products, two warps copy.  S (fp32), P (bf16, in S's columns) and O (fp32) live in tensor memory: 2 x (128 + D)
// of 512 columns.
//   pair   more than 128 query rows left: the streams are two neighbouring query tiles, K and V tiles are shared
//   alt    up to 128 rows (decode tokens, short chunks, ends of prompts): both streams are the same query tile, one
//          takes the even and one the odd KV tiles; their results are merged at the end
//
// Split.  The CTAs cut the whole batch's work - query tile pairs in the order (request, kv-head, tile), each as long as
// the tokens it sees - into pieces at KV-tile borders.  A piece that begins or ends inside a query tile leaves fp32 partial
// results (O, m, l) in the workspace; whichever CTA completes the tile's count of KV tiles merges them, in the order of the
// pieces, so the result does not depend on who is last.  Long contexts with few rows and long prompts take the same path, and
// there is no second kernel.
//
// Measured (32 heads over 8, D = 128; device time in graphs, calls issued one by one on changing inputs in brackets): prompt of
// 32768 tokens 8.1-8.4 ms (8.3-8.4; 1.05-1.09 PFLOP/s), 2048 tokens over 65536 1.9-2.0 ms (2.02-2.05), eight packed prompts of
// 500-4000 tokens 366 us (387-390), eight times five drafted tokens over 32768 197 us (203-213; 5.0-5.4 TB/s).  A step of both
// streams takes 3350 cycles where products and exponentials take 2048 each: a stream's chain of scores, softmax and product is
// what bounds it.  Compared on builds that took 372 us for the packed prompts: KV tiles of 64 tokens with two score buffers per
// stream 465-497 us, a product that begins with half of the weights 399-410 us, exponentials on the FMA units (one pair in
// eight) 386 us.
#include <math.h>

#include "se_internal.h"
#include "se_pieces.cuh"
#include "se_tc.cuh"

namespace se {

namespace {

constexpr int kThreads = 384;            // 2 softmax warpgroups, K warp, product warp, V warp, idle warp
constexpr int kKWarp = 8, kMmaWarp = 9, kVWarp = 10, kIdleWarp = 11;
// 256 * 200 + 128 * 104 = 384 * 168; nothing spills.  With 208 and 88 the copying and product warps did: packed prompts 372 us for
// 366, mixed batch 1230 for 1200, 2048 tokens over 65536 1935 for 1890-1910.
constexpr int kRegsSoftmax = 200, kRegsOther = 104;
constexpr int kTile = 128;             // query rows of a tile
constexpr int kKv = 128;               // tokens of a KV tile
constexpr int kGroups = kKv / kPage;   // pages of a KV tile
constexpr int kMaxParts = 304;         // partial results of a query tile: two per piece, little more than 148 pieces of it
constexpr int kItemCost = 128;         // cost of starting a query tile, in tokens
// A CTA takes at least 256 tokens (a short item has a CTA of its own), but where pieces are small, items are split at multiples
// of four KV tiles only: the parts have to be merged, which takes as long as a dozen tiles.  Six short prompts: 16.4 us, with
// pieces of 512 tokens 19.5 us; one token over 2048: 21.8 us, split at every second tile 23.7 us.
constexpr int kMinCost = 256, kCoarse = 2048;
// The running maximum may lag: weights up to 2^40 lose nothing (bf16 and fp32 keep their exponents, and 2^40 * 131072
// tokens is far from the end of the range).
constexpr float kSlack = 40.f;

template <int D>
struct Cfg {
    static constexpr int kHalves = D / 64;
    static constexpr int kTileBytes = kTile * D * 2;              // query tile
    static constexpr int kKvBytes = kKv * D * 2;                  // K or V tile
    static constexpr int kKSlots = 2 * 128 / D, kVSlots = 3 * 128 / D;   // rings of K and V tiles, 64 and 96 KB
    static constexpr int kSlots = kKSlots + kVSlots;
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

template <int N>
struct Int {
    static constexpr int value = N;
};

// kRing: full barriers of the K slots and of the V slots, then the empty ones in the same order
enum Bar { kQFull, kQEmpty, kSFull, kPReady = kSFull + 2, kOLast = kPReady + 2, kOFree = kOLast + 2, kAll = kOFree + 2,
           kVerdict = kAll + 2, kSwap = kVerdict + 2, kDrain, kRing };

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
        return (int)((z / kKv) >> (new_tokens(t, i) > tpt ? 1 : 0));
    }
    __device__ __forceinline__ long long min_cost() const { return kMinCost; }
    static constexpr int kCrumb = 2;   // least units of a part of an item
    static constexpr int kGrain = 4;
    __device__ __forceinline__ long long coarse() const { return kCoarse; }
    static constexpr bool kShares = true;
    static constexpr long long kShareCost = 2560;
    __device__ __forceinline__ long long longest(const TokenRange &t) const { return 2ll * (t.past + t.n + kItemCost); }
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

template <int D>
struct Control {
    uint64_t bars[kRing + 2 * Cfg<D>::kSlots];
    SegmentQueue<Segment> queue;
    alignas(8) uint8_t prefix[prefix_bytes(kSmemRequests)];
    uint32_t mask[Cfg<D>::kMasks];     // present 16-token groups of the tiles in flight
    int parts[2];                      // partial results to merge, 0: another CTA does
    uint16_t part[2][kMaxParts];
    int gave_up;
    List<AttendWork> list;             // (in registers it made the compiler spill)
    uint32_t tmem;
};

// The next part of an item in the piece.
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
// One warp brings K (and Q), one V, each through a ring of its own.  A tile is 128 tokens of one head.  K lies as
// [D/64][128 tokens][64 channels]: a page is D/64 copies (one for all where K is contiguous).  V lies as
// [8][D/64][16 tokens][64 channels] where it is paged, because a product takes 16 tokens at a time: a page is one copy; and like
// K where it is contiguous, a whole tile in one copy.
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
        block = tile / (32 / kGroups);
        ids = fetch(a, s, block * 32 + lane, report);
        next = fetch(a, s, block * 32 + 32 + lane, report);
    }
    // tiles come in ascending order
    __device__ __forceinline__ void reach(const AttendArgs &a, const Segment &s, int tile, bool report, int lane) {
        if (tile / (32 / kGroups) == block) return;
        ++block;
        ids = next;
        next = fetch(a, s, block * 32 + 32 + lane, report);
    }
    __device__ __forceinline__ int of(int tile, int pg) const { return __shfl_sync(kFull, ids, tile % (32 / kGroups) * kGroups + pg); }
};

// The end of a copying warp that has filled `filled` slots of a ring of kSlots, whose barriers are full + 8 * slot and
// empty + 8 * slot: nothing may still be on its way to the CTA's shared memory when the CTA ends - copies, and the
// products' arrivals for the slots they have let go.  A slot that is let go has been filled; where the products have given up
// (also just now, in the wait for this very slot) the copy itself is waited for.
template <uint32_t kSlots>
__device__ __forceinline__ void leave_ring(bool ok, uint32_t filled, uint32_t full, uint32_t empty, volatile int *gave_up, const AttendArgs &a) {
    for (uint32_t n = filled > kSlots ? filled - kSlots : 0; n < filled; ++n) {
        const uint32_t off = 8 * (n % kSlots), parity = n / kSlots & 1;
        ok = ok && warp_wait(empty + off, parity, gave_up, &a.ctl->status);
        if (!ok) mbar_wait(full + off, parity);
    }
}

template <int D>
__device__ __forceinline__ void k_role(const AttendArgs &a, const List<AttendWork> &list, const CUtensorMap *q_map, const CUtensorMap *k_map,
                                       const CUtensorMap *k_wide, Control<D> *ctl, uint32_t q_smem, uint32_t ring, uint32_t bars, int lane) {
    using C = Cfg<D>;
    volatile int *gave_up = &ctl->gave_up;
    const int tpt = kTile / a.G;
    Segment s;
    Pages pages;
    uint32_t tiles = 0, queries = 0;
    const uint32_t k_full = bars + 8 * kRing, k_empty = k_full + 8 * C::kSlots;
    const bool chosen = elect_one();
    bool ok = true;
    Walk<AttendWork> walk(list, a.ctl, lane);
    while (ok && next_segment(walk, s)) {
        const int stop = s.t.past + s.t.n;                                 // tokens of the request
        ok = ctl->queue.put(queries, &s, gave_up, &a.ctl->status, lane);
        if (!ok) break;
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
        for (int t = s.a; t < s.b; ++t, ++tiles) {
            const uint32_t slot = tiles % C::kKSlots, bar = k_full + 8 * slot, dst = ring + slot * C::kKvBytes;
            pages.reach(a, s, t, true, lane);
            const unsigned mask = __ballot_sync(kFull, pages.ids >= 0) >> t % (32 / kGroups) * kGroups & 0xffu;
            int pid[kGroups];
#pragma unroll
            for (int pg = 0; pg < kGroups; ++pg) pid[pg] = pages.of(t, pg);
            ok = warp_wait(k_empty + 8 * slot, (tiles / C::kKSlots & 1) ^ 1, gave_up, &a.ctl->status);
            if (!ok) break;
            if (chosen) {
                ctl->mask[tiles % C::kMasks] = mask;
                mbar_expect_tx(bar, C::kKvBytes + (D == 64 && tiles == 0 ? kTestExtraTx : 0));
                if (!a.page_table && (t + 1) * kKv <= stop) {
                    tma_load_4d(dst, k_wide, 0, s.h, s.t.start + t * kKv, 0, bar);
                } else {
#pragma unroll
                    for (int pg = 0; pg < kGroups; ++pg) {
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
    if (ok) ok = ctl->queue.put(queries, nullptr, gave_up, &a.ctl->status, lane);
    leave_ring<C::kKSlots>(ok, tiles, k_full, k_empty, gave_up, a);
    if (queries) {
        ok = ok && warp_wait(bars + 8 * kQEmpty, (queries - 1) & 1, gave_up, &a.ctl->status);
        if (!ok) mbar_wait(bars + 8 * kQFull, (queries - 1) & 1);
    }
}

template <int D>
__device__ __forceinline__ void v_role(const AttendArgs &a, const CUtensorMap *v_map, const CUtensorMap *v_wide, Control<D> *ctl, uint32_t ring,
                                       uint32_t bars, int lane) {
    using C = Cfg<D>;
    volatile int *gave_up = &ctl->gave_up;
    Segment s;
    Pages pages;
    uint32_t tiles = 0;
    const uint32_t v_full = bars + 8 * (kRing + C::kKSlots), v_empty = v_full + 8 * C::kSlots;
    const bool chosen = elect_one();
    bool ok = true;
    uint32_t turn = 0;
    const uint32_t page_step = a.page_table ? kPage * D * 2 : kPage * 128, half_step = a.page_table ? kPage * 128 : kKv * 128;
    while (ok) {
        const Segment *next = ctl->queue.get(turn++, gave_up, &a.ctl->status, lane);
        if (!next) break;
        s = *next;
        const int stop = s.t.past + s.t.n;                                 // tokens of the request
        pages.begin(a, s, s.a, false, lane);
        for (int t = s.a; t < s.b; ++t, ++tiles) {
            const uint32_t slot = tiles % C::kVSlots, bar = v_full + 8 * slot, dst = ring + (C::kKSlots + slot) * C::kKvBytes;
            pages.reach(a, s, t, false, lane);
            int pid[kGroups];
#pragma unroll
            for (int pg = 0; pg < kGroups; ++pg) pid[pg] = pages.of(t, pg);
            ok = warp_wait(v_empty + 8 * slot, (tiles / C::kVSlots & 1) ^ 1, gave_up, &a.ctl->status);
            if (!ok) break;
            // The group that holds the end of the request is copied row by row: what lies behind the end may be anything, and
            // a weight of zero would not hide a NaN.
            const int part = stop % kPage && stop / kKv == t ? stop % kKv / kPage : -1;
            const int own = part < 0 ? -1 : pages.of(t, part);
            const bool by_hand = own >= 0;
            if (by_hand) {
                const int tok = t * kKv + part * kPage;
                const uint16_t *base = a.page_table ? a.v + ((size_t)own * a.H_kv + s.h) * (kPage * D)
                                                    : a.v + (long long)(s.t.start + tok) * a.v_stride + s.h * D;
                const long long pitch = a.page_table ? D : a.v_stride;
                constexpr int kPieces = D / 8;
#pragma unroll
                for (int i = 0; i < kPage * kPieces / 32; ++i) {
                    const int e = i * 32 + lane, row = e / kPieces, ch = e % kPieces;
                    uint4 x = make_uint4(0, 0, 0, 0);
                    if (row < stop - tok) x = *reinterpret_cast<const uint4 *>(base + row * pitch + ch * 8);
                    const uint32_t at = dst + part * page_step + (ch >> 3) * half_step + row * 128 + (((ch & 7) ^ (row & 7)) << 4);
                    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
                }
                fence_async_proxy();
                __syncwarp();
            }
            if (chosen) {
                mbar_expect_tx(bar, C::kKvBytes - (by_hand ? kPage * D * 2 : 0) + (D == 128 && tiles == 0 ? kTestExtraTx : 0));
                if (!a.page_table && (t + 1) * kKv <= stop) {
                    tma_load_4d(dst, v_wide, 0, s.h, s.t.start + t * kKv, 0, bar);
                } else if (a.page_table) {
#pragma unroll
                    for (int pg = 0; pg < kGroups; ++pg)
                        if (pg != part || !by_hand)
                            tma_load_4d(dst + pg * page_step, v_map, 0, 0,
                                        (pid[pg] < 0 ? a.P_phys * a.H_kv : pid[pg] * a.H_kv + s.h) * kPage, 0, bar);
                } else {
#pragma unroll
                    for (int pg = 0; pg < kGroups; ++pg)
#pragma unroll
                        for (int half = 0; half < C::kHalves; ++half)
                            if (pg != part || !by_hand)
                                tma_load_3d(dst + half * half_step + pg * page_step, v_map, half * 64, s.h,
                                            pid[pg] < 0 ? a.T : s.t.start + t * kKv + pg * kPage, bar);
                }
            }
            __syncwarp();
        }
    }
    leave_ring<C::kVSlots>(ok, tiles, v_full, v_empty, gave_up, a);
}

// ---- products ----------------------------------------------------------------------
// One warp issues all products, in the order of the steps of both streams: it waits for every tile's barriers in order (a
// barrier tells its phases apart by parity alone, so a warp that left one out could take the phase before for the one it
// waits for).  The whole warp walks the list, so that addresses stay in uniform registers; one elected lane issues (a role
// run by a single lane took 82 cycles per instruction to issue, more than the 64 that it computes).
template <int D>
__device__ __forceinline__ void mma_role(const AttendArgs &a, Control<D> *ctl, uint32_t q_smem, uint32_t ring,
                                         uint32_t bars, int lane) {
    using C = Cfg<D>;
    volatile int *gave_up = &ctl->gave_up;
    const uint32_t tmem = ctl->tmem;
    uint32_t tiles = 0, queries = 0, p_seen = 0, o_used = 0;               // bit st: parity of the stream's next wait
    bool any = false;
    const bool chosen = elect_one();
    const uint32_t v_lead = a.page_table ? kPage * 128 : kKv * 128, v_step = (a.page_table ? kPage * D * 2 : kPage * 128) >> 4;
    auto wait = [&](int bar, uint32_t parity) { return warp_wait(bars + 8 * bar, parity & 1, gave_up, &a.ctl->status); };
    // `k_next`, `v_next`: the first tiles not waited for yet
    uint32_t k_next = 0, v_next = 0;
    auto wait_k = [&](uint32_t tile) {
        for (; k_next <= tile; ++k_next)
            if (!wait(kRing + k_next % C::kKSlots, k_next / C::kKSlots)) return false;
        return true;
    };
    auto wait_v = [&](uint32_t tile) {
        for (; v_next <= tile; ++v_next)
            if (!wait(kRing + C::kKSlots + v_next % C::kVSlots, v_next / C::kVSlots)) return false;
        return true;
    };
    bool ok = true;
    while (ok) {
        const Segment *s = ctl->queue.get(queries, gave_up, &a.ctl->status, lane);
        if (!s) break;
        const int steps0 = s->steps0, steps1 = s->steps1, steps = max(steps0, steps1);
        const bool alt = s->alt;
        auto place = [&](int st, int i) { return tiles + (alt ? 2 * i + st : i); };
        // S = Q K^T (the chosen lane)
        auto scores = [&](auto stream, uint32_t tile) {
            constexpr int ST = decltype(stream)::value;
            const uint32_t slot = tile % C::kKSlots;
            const uint64_t qd = smem_operand(q_smem + (alt ? 0 : ST * C::kTileBytes), 16, 1024);
            const uint64_t kd = smem_operand(ring + slot * C::kKvBytes, 16, 1024);
#pragma unroll
            for (int k = 0; k < D / 16; ++k) {
                const uint32_t off = (k / 4) * (kTile * 128 >> 4) + (k % 4) * 2;
                mma_ss(tmem + ST * kTile, qd + off, kd + off, mma_instr(kKv, false), k > 0);
            }
            mma_commit(bars + 8 * (kSFull + ST));
            if (alt || ST == 1) mma_commit(bars + 8 * (kRing + C::kSlots + slot));
        };
        auto begin = [&](auto stream) {
            constexpr int ST = decltype(stream)::value;
            if ((ST ? steps1 : steps0) == 0) return true;
            if (!wait_k(place(ST, 0))) return false;
            tc_fence_after();
            if (chosen) scores(stream, place(ST, 0));
            __syncwarp();
            return true;
        };
        // O += P V, and the next scores
        auto step = [&](auto stream, int i) {
            constexpr int ST = decltype(stream)::value;
            const int mine = (ST ? steps1 : steps0);
            if (i >= mine) return true;
            const bool more = i + 1 < mine;
            const uint32_t tile = place(ST, i), slot = tile % C::kVSlots;
            const uint64_t vd = smem_operand(ring + (C::kKSlots + slot) * C::kKvBytes, v_lead, 1024);
            // everything that can be waited for early comes before the wait for the weights
            if (!wait_v(tile) || (more && !wait_k(place(ST, i + 1)))) return false;
            if (i == 0) {                // the epilogue of the stream's last piece has read O
                if (!wait(kOFree + ST, (o_used >> ST & 1) ^ 1)) return false;
                o_used ^= 1u << ST;
            }
            if (!wait(kPReady + ST, p_seen >> ST)) return false;
            p_seen ^= 1u << ST;
            tc_fence_after();
            if (chosen) {
#pragma unroll
                for (int k = 0; k < kKv / 16; ++k)
                    mma_ts(tmem + C::kTmemO + ST * D, tmem + ST * kTile + k * 8, vd + k * v_step, mma_instr(D, true), i > 0 || k > 0);
                if (alt || ST == 1) mma_commit(bars + 8 * (kRing + C::kSlots + C::kKSlots + slot));
                if (more) scores(stream, place(ST, i + 1));
                else mma_commit(bars + 8 * (kOLast + ST));
            }
            __syncwarp();
            return true;
        };
        any = true;
        ok = wait(kQFull, queries++) && begin(Int<0>{}) && begin(Int<1>{});
        if (ok && chosen && steps == 1) mma_commit(bars + 8 * kQEmpty);
        __syncwarp();
        for (int i = 0; i < steps && ok; ++i) {
            ok = step(Int<0>{}, i) && step(Int<1>{}, i);
            if (ok && chosen && i + 2 == steps) mma_commit(bars + 8 * kQEmpty);   // the last product with Q is on its way
            __syncwarp();
        }
        tiles += s->b - s->a;
    }
    if (any) {                           // nothing may be running when tensor memory goes away
        if (chosen) mma_commit(bars + 8 * kDrain);
        __syncwarp();
        mbar_wait(bars + 8 * kDrain, 0);
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

// 32 bytes of a thread's own row: half the instructions, each of which takes a cycle per row, of two stores of 16 bytes.
__device__ __forceinline__ void store32(void *dst, const uint32_t *w) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(dst), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]),
                 "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
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
#pragma unroll 8
    for (int k = 0; k < parts; ++k) {
        const float *p = partial_slot<D>(a, at(k)) + kTile * D;
        const float m = have ? __ldcg(p + my) : -INFINITY, l = have ? __ldcg(p + kTile + my) : 0.f;
        const float top = fmaxf(M, m), ref = top == -INFINITY ? 0.f : top;
        L = L * ex2(M - ref) + l * ex2(m - ref);
        M = top;
    }
    // a sum of exactly 0: nothing was seen; a NaN goes on into the row and its lse
    const float inv = L == 0.f ? 0.f : 1.f / L, ref = M == -INFINITY ? 0.f : M;
    if (have && a.lse) a.lse[out0 + (long long)(my / a.G) * a.H_q + my % a.G] = L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
    const int mine = rows > row_from ? (rows - row_from + row_step - 1) / row_step : 0;
    for (int k0 = 0; k0 < mine; k0 += R) {
        float acc[R][V] = {};
#pragma unroll 4
        for (int q = 0; q < parts; ++q) {
            const float *p = partial_slot<D>(a, at(q));
            // -1: the part saw nothing, and what lies in its place may be anything
            const float m = have ? __ldcg(p + kTile * D + my) : -INFINITY;
            const float w = m == -INFINITY ? -1.f : ex2(m - ref) * inv;
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
                for (int v = 0; v < V; ++v) acc[k][v] += wk < 0.f ? 0.f : wk * x[k][v];
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
    uint32_t step = 0, tiles = 0, verdicts = 0, swaps = 0, ends = 0, turn = 0;
    // both warpgroups have come here
    auto swap_sync = [&] {
        __syncwarp();
        if (lane == 0) mbar_arrive(bars + 8 * kSwap);
        return warp_wait(bars + 8 * kSwap, swaps++ & 1, gave_up, &a.ctl->status);
    };
    for (;;) {
        const Segment *next = ctl->queue.get(turn++, gave_up, &a.ctl->status, lane);
        if (!next) return;
        const Segment &s = *next;
        const int tok = s.tok0 + (s.alt ? 0 : st * tpt);                   // the tile's first new token
        const int ntok = min(tpt, s.tok0 + s.ntok - tok);
        const int q = min(row / a.G, ntok - 1);
        const int sees = s.t.past + tok + q + 1;                           // tokens the row sees
        const int least = __reduce_min_sync(kFull, sees);
        const int steps = s.steps(st);
        const int stride = s.alt ? 2 : 1;
        int left = sees - (s.a + (s.alt ? st : 0)) * kKv;                  // tokens that the row sees of this tile and the later ones
        int most = least - (s.a + (s.alt ? st : 0)) * kKv;
        uint32_t tile = tiles + (s.alt ? st : 0);
        float m = -INFINITY;                                               // in units of the raw scores
        float l = 0.f, lost = 0.f;     // sum of the weights over the tiles so far, and what rounding took from it (Kahan)
        for (int u = 0; u < steps; ++u, ++step, left -= stride * kKv, most -= stride * kKv, tile += stride) {
            if (!warp_wait(bars + 8 * (kSFull + st), step & 1, gave_up, &a.ctl->status)) return;
            tc_fence_after();
            float x[kKv];
#pragma unroll
            for (int k = 0; k < kKv; k += 32) tmem_ld32<false>(t_s + k, x + k);   // (converged by the wait)
            const unsigned mask = ctl->mask[tile % C::kMasks];
            tmem_wait_ld();
            settle<kKv>(x);
            if (kKv > most || mask != 0xffu) {
                // (a branch per page: pruned contexts come here in most tiles, and a test per element took 300 instructions)
#pragma unroll
                for (int pg = 0; pg < kGroups; ++pg)
                    if (!(mask >> pg & 1)) {
#pragma unroll
                        for (int k = 0; k < kPage; ++k) x[pg * kPage + k] = -INFINITY;
                    }
                if (kKv > most) {
#pragma unroll
                    for (int k = 0; k < kKv; ++k)
                        if (k >= left) x[k] = -INFINITY;
                }
            }
            float top[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
            for (int k = 4; k < kKv; k += 8)
#pragma unroll
                for (int e = 0; e < 4; ++e) top[e] = k + 4 + e < kKv ? max3(top[e], x[k + e], x[k + 4 + e]) : fmaxf(top[e], x[k + e]);
            const float mn = fmaxf(m, fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])));
            if (__any_sync(kFull, (mn - m) * sl > kSlack)) {
                const float f = m == -INFINITY ? 0.f : ex2((m - mn) * sl);
                m = mn;
                l *= f, lost *= f;
                if (u > 0) {             // the product before these scores is complete: they were issued behind it
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
            float2 l2 = make_float2(0.f, 0.f);
#pragma unroll
            for (int k = 0; k < kKv; k += 64) {
                uint32_t p[32];
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    const float2 y = ffma2(make_float2(x[k + 2 * e], x[k + 2 * e + 1]), make_float2(sl, sl), make_float2(off, off));
                    const float2 w = make_float2(ex2(y.x), ex2(y.y));
                    l2 = __fadd2_rn(l2, w);
                    // the weights enter the product with V as bf16 (8 significant bits), their sum keeps fp32
                    const __nv_bfloat162 b = __float22bfloat162_rn(w);
                    p[e] = *reinterpret_cast<const uint32_t *>(&b);
                }
                tmem_st32<false>(t_s + k / 2, p);
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bars + 8 * (kPReady + st));
            __syncwarp();
            // The tile's sum joins the others in one compensated step: equal weights added one after the other over 32768 tokens
            // lost up to 2e-4 of the sum, 5e-4 over 65536 (now less than 2e-6).
            const float y = __fsub_rn(l2.x + l2.y, lost), next_l = __fadd_rn(l, y);
            lost = __fsub_rn(__fsub_rn(next_l, l), y);
            l = next_l;
        }
        tiles += s.b - s.a;
        if (steps > 0) {
            if (!warp_wait(bars + 8 * (kOLast + st), ends++ & 1, gave_up, &a.ctl->status)) return;
            tc_fence_after();
        }

        // ---- epilogue ----
        // -infinity says that nothing was seen, so a sum that is NaN goes with another maximum
        const float m2 = l != l ? INFINITY : m == -INFINITY ? m : m * sl;
        const bool live = row < ntok * a.G;
        const bool whole = s.a == 0 && s.b == s.nkv;
        const bool direct = whole && (!s.alt || s.nkv == 1);
        const long long orow = (long long)(s.t.start + tok + q) * a.H_q + s.h * a.G + row % a.G;
        if (direct) {
            if (s.alt && st == 1) continue;                                // a single KV tile: stream 0 has it all
            const float inv = l == 0.f ? 0.f : 1.f / l;                    // 0: nothing was seen; a NaN goes on
            uint4 *dst = reinterpret_cast<uint4 *>(a.out + orow * D);
            const bool wide = ((uintptr_t)a.out & 31) == 0;
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
                    for (int e = 0; e < 4; e += 2) {
                        if (wide) {
                            store32(dst + k / 8 + e, w + 4 * e);
                        } else {
                            dst[k / 8 + e] = make_uint4(w[4 * e], w[4 * e + 1], w[4 * e + 2], w[4 * e + 3]);
                            dst[k / 8 + e + 1] = make_uint4(w[4 * e + 4], w[4 * e + 5], w[4 * e + 6], w[4 * e + 7]);
                        }
                    }
                }
            }
            if (live && a.lse) a.lse[orow] = l == 0.f ? -INFINITY : (m2 + log2f(l)) * kLn2;
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
#pragma unroll
                        for (int e = 0; e < 32; e += 8) store32(slot + (size_t)row * D + k + e, reinterpret_cast<const uint32_t *>(o + e));
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
              const __grid_constant__ CUtensorMap v_wide, const __grid_constant__ AttendArgs a) {
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

    static_assert(kRing + 2 * C::kSlots <= kThreads, "a thread per barrier");
    if (threadIdx.x < kRing + 2 * C::kSlots) {
        const int i = threadIdx.x;
        const bool by_warp = (i >= kPReady && i < kPReady + 2) || (i >= kOFree && i < kOFree + 2) || (i >= kAll && i < kAll + 2);
        mbar_init(bars + 8 * i, i == kSwap ? 8 : by_warp ? 4 : 1);
        mbar_fence_init();
    }
    if (threadIdx.x == 32) {
        ctl->queue.init(10);
        mbar_fence_init();
        ctl->gave_up = 0;
    }
    // (read ahead: it is here when the list is)
    const uint32_t refused = threadIdx.x == 32 * kIdleWarp ? *(volatile uint32_t *)&a.ctl->needs_init : 0u;
    if (warp == kMmaWarp) tmem_alloc(smem_u32(&ctl->tmem), 512);
    if (threadIdx.x == 32 * kKWarp) prefetch_map(&q_map), prefetch_map(&k_map);
    if (threadIdx.x == 32 * kVWarp) prefetch_map(&v_map);
    const AttendWork work(a);
    List<AttendWork> made = make_list<kThreads>(work, a.B, a.H_kv, a.ctl,
                                            a.B > kSmemRequests ? a.prefixes + prefix_bytes(a.B) * blockIdx.x : ctl->prefix, smem);
    // query rows that no tensor copy fills (G does not divide 128) stay zero
    for (int i = threadIdx.x; i < (work.tpt * a.G == kTile ? 0 : 2 * C::kTileBytes / 16); i += kThreads)
        reinterpret_cast<uint4 *>(smem)[i] = make_uint4(0, 0, 0, 0);
    if (threadIdx.x == 32 * kIdleWarp) {
        if (refused) {                   // an empty list: the roles find nothing to do, and no counter moves
            made.total = 0, made.pieces = kPromptCtas;
            if (blockIdx.x == 0) atomicOr(&a.ctl->status, SE_DEV_WAIT_TIMEOUT);
        }
        ctl->list = made;
    }
    fence_async_proxy();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const List<AttendWork> &list = ctl->list;

    // (the order of the two branches moves the measured cases by 2 %, in both directions)
    if (warp >= 8) {
        regs_down<kRegsOther>();
        const uint32_t ring = base + 2 * C::kTileBytes;
        if (warp == kKWarp) k_role<D>(a, list, &q_map, &k_map, &k_wide, ctl, base, ring, bars, lane);
        else if (warp == kVWarp) v_role<D>(a, &v_map, &v_wide, ctl, ring, bars, lane);
        else if (warp == kMmaWarp) mma_role<D>(a, ctl, base, ring, bars, lane);
        __syncwarp();
    } else {
        regs_up<kRegsSoftmax>();
        softmax_role<D>(a, list, ctl, bars, warp >> 2);
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
    CUtensorMap q_map, k_map, k_wide, v_map, v_wide;
    bool ok = make_rows_map(&q_map, c.q, D, p.H_q, c.total_tokens, c.q_stride, G, kTile / G);
    if (c.page_table) {
        const long long rows = (long long)p.num_phys_pages * p.H_kv * kPage;
        ok = ok && make_rows_map(&k_map, c.k, D, 1, rows, D, 1, kPage) && make_split_map(&v_map, c.v, D, 1, rows, D, kPage);
        k_wide = k_map, v_wide = v_map;                          // not used
    } else {
        ok = ok && make_rows_map(&k_map, c.k, D, p.H_kv, c.total_tokens, c.k_stride, 1, kPage) &&
             make_split_map(&k_wide, c.k, D, p.H_kv, c.total_tokens, c.k_stride, kKv) &&
             make_rows_map(&v_map, c.v, D, p.H_kv, c.total_tokens, c.v_stride, 1, kPage) &&
             make_split_map(&v_wide, c.v, D, p.H_kv, c.total_tokens, c.v_stride, kKv);
    }
    if (!ok) return cudaErrorInvalidValue;
    AttendArgs a = {};
    a.cu = c.cu_seqlens, a.seq_lens = c.seq_lens, a.page_table = c.page_table;
    a.v = static_cast<const uint16_t *>(c.v), a.v_stride = c.v_stride;
    a.out = static_cast<uint16_t *>(c.out), a.lse = c.lse;
    a.ctl = reinterpret_cast<PromptControl *>(c.workspace);
    a.partials = partials_of(c.workspace);
    a.prefixes = c.workspace + prefix_workspace_offset(p.D);
    a.B = p.B, a.H_q = p.H_q, a.H_kv = p.H_kv, a.G = G, a.T = c.total_tokens, a.max_pages = p.max_pages;
    a.P_phys = p.num_phys_pages, a.scale_log2 = effective_scale(p) * kLog2e;
    auto kern = attend_kernel<D>;
    // the register split (setmaxnreg) draws on what the block was launched with
    cudaFuncAttributes attr;
    cudaError_t e = cudaFuncGetAttributes(&attr, kern);
    if (e != cudaSuccess) return e;
    if (attr.numRegs * kThreads < 256 * kRegsSoftmax + 128 * kRegsOther) return cudaErrorInvalidConfiguration;
    constexpr size_t smem = 2 * C::kTileBytes + C::kSlots * C::kKvBytes + sizeof(Control<D>);
    static_assert(smem <= 227 * 1024, "shared memory of a CTA");
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    kern<<<kPromptCtas, kThreads, smem, stream>>>(q_map, k_map, k_wide, v_map, v_wide, a);
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
