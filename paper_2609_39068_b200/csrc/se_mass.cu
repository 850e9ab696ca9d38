// Accumulated attention weights of a chunk (Appendix A, H2O accumulated score equation, summed over the queries of a chunk):
//     u[j,h] += sum over the new tokens i >= j and the heads a of group h of exp(z_ij^a - lse_i^a).
//
// The sum runs over queries, so the tile is laid the other way round than in the attention kernel: a tile of 128 cached
// tokens is the M side (tensor-memory lanes), a query tile of 128/G tokens x G heads the N side (columns), S^T = K Q^T.
// A thread owns one cached token and adds up 2^(S sl - lse log2 e) along half of its columns in a register: no reduction
// between threads but the one addition of the halves, no atomics, no second pass, and the result does not depend on timing.
//
// What bounds it: per 128 x 128 tile one product of 512 tensor cycles (D = 128) and 16384 exponentials, seven in eight of them
// on the special-function units, which takes those 896 cycles; K is read once per item, the queries come from L2.  A CTA works
// on two tiles of cached tokens (two warpgroups each) that share every query tile.  Scores are double-buffered in tensor memory
// (4 x 128 columns), so the products of the next query tile run under the exponentials of this one.
// Prompt of 16384 tokens (32 heads over 8, D = 128): 1320-1430 us in graphs, 1460-1475 as calls on changing inputs (750 TFLOP/s of
// products counted below the diagonal); chunks of four requests over 32768 cached tokens: 571-576 and 597-605 us.  Of the latter's
// cycles the special-function units are busy for 59 %, the tensor cores for 33 %, and an instruction is issued in 52 %.  With one
// warpgroup per tile (all columns in a thread) 1412 and 599 us in graphs, on a build that took 1320 and 566.
//
// Item = 256 cached tokens of one (request, kv-head), unit = query tile; pieces and merging as in se_pieces.cuh (a partial
// result is one number per cached token).
#include <math.h>

#include "se_internal.h"
#include "se_pieces.cuh"
#include "se_tc.cuh"

namespace se {

namespace {

// One pair of weights in eight is computed without the special-function units (side by side, prompt of 16384: none 1350 us, one
// in eight 1320 us, one in four 1408 us, where the issue of instructions becomes the bound).
// 2^x of a pair: x = j + f with |f| <= 1/2 (j by adding and taking off 1.5 * 2^23), 2^f by a
// minimax polynomial of degree 5 with 2^0 = 1 (own fit; relative error 1.6e-7, fp32 rounding included), j added to the exponent
// field.  x is held to [-127, 128], where the exponent field comes out as 0 and as that of infinity; below -126 the result is
// less than 2^-126.  The integer arithmetic loses a NaN, so `nan` collects them: 0, or NaN once x has been one.
__device__ __forceinline__ float2 ex2_fma(float2 x, float2 &nan) {
    constexpr float kMagic = 12582912.f;
    auto hold = [](float v) {
        asm("max.NaN.f32 %0, %0, 0fC2FE0000;\n\tmin.NaN.f32 %0, %0, 0f43000000;" : "+f"(v));
        return v;
    };
    x = make_float2(hold(x.x), hold(x.y));
    nan = ffma2(x, make_float2(0.f, 0.f), nan);
    const float2 t = __fadd2_rn(x, make_float2(kMagic, kMagic));
    const float2 f = __fadd2_rn(x, ffma2(t, make_float2(-1.f, -1.f), make_float2(kMagic, kMagic)));
    float2 p = make_float2(0.0013274633092805743f, 0.0013274633092805743f);
    auto step = [&](float k) { p = ffma2(p, f, make_float2(k, k)); };
    step(0.009671961888670921f), step(0.055506784468889236f), step(0.24022234976291656f), step(0.6931470632553101f), step(1.f);
    return make_float2(__int_as_float(__float_as_int(p.x) + (__float_as_int(t.x) << 23)),
                       __int_as_float(__float_as_int(p.y) + (__float_as_int(t.y) << 23)));
}

constexpr int kThreads = 640;          // 4 summing warpgroups, copy warp, product warp, lse warp, idle warp
constexpr int kCopyWarp = 16, kMmaWarp = 17, kLseWarp = 18;
constexpr int kRegsSum = 104, kRegsOther = 64;   // 512 * 104 + 128 * 64 = 640 * 96
constexpr int kTile = 128;             // cached tokens of a tile, query rows of a tile
constexpr int kLseSlots = 2;

template <int D>
struct Cfg {
    static constexpr int kHalves = D / 64;
    static constexpr int kTileBytes = kTile * D * 2;
    static constexpr int kPairs = 2;                              // K tile pairs in shared memory
    static constexpr int kSlots = 3 * 128 / D;                    // ring of query tiles, 96 KB
};

struct MassArgs {
    const int32_t *cu, *seq_lens, *page_table;
    const float *lse;
    float *accum, *partials;
    PromptControl *ctl;
    uint8_t *prefixes;                 // prefix sums of batches too large for shared memory
    int B, H_q, H_kv, G, T, max_pages, P_phys;
    float scale_log2;
};

enum Bar { kSFull, kSFree = kSFull + 4, kLseFull = kSFree + 4, kLseEmpty = kLseFull + kLseSlots, kKFull = kLseEmpty + kLseSlots,
           kKEmpty = kKFull + 2, kAll = kKEmpty + 2, kVerdict = kAll + 2, kHalfFull = kVerdict + 2,
           kHalfFree = kHalfFull + 2, kDrain = kHalfFree + 2, kRing };

struct MassWork {
    const int32_t *cu, *seq_lens;
    int T, max_tokens, tpt;            // tpt: new tokens of a query tile

    __device__ __forceinline__ explicit MassWork(const MassArgs &a)
        : cu(a.cu), seq_lens(a.seq_lens), T(a.T), max_tokens(a.max_pages * kPage), tpt(kTile / a.G) {}
    __device__ __forceinline__ TokenRange tokens(int r) const { return token_range(cu, seq_lens, r, T, max_tokens); }
    __device__ __forceinline__ int items(const TokenRange &t) const { return (t.past + t.n + 2 * kTile - 1) / (2 * kTile); }
    // new tokens that see nothing of a tile of cached tokens beginning at `pos`
    __device__ __forceinline__ int blind(const TokenRange &t, int pos) const { return max(pos - t.past, 0); }
    // cost: new tokens that see the item, and the start of an item as much as two query tiles
    __device__ __forceinline__ long long cost(const TokenRange &t, long long i) const {
        const long long all = t.past / (2 * kTile) + 1;           // items that every new token sees
        long long c = i * (t.n + 2 * tpt);
        if (i > all) c -= 2 * kTile * (i * (i - 1) / 2 - all * (all - 1) / 2) - (i - all) * t.past;
        return c;
    }
    __device__ __forceinline__ int query_tiles(const TokenRange &t) const { return (t.n + tpt - 1) / tpt; }
    __device__ __forceinline__ int units(const TokenRange &t, int i) const {
        return query_tiles(t) - blind(t, i * 2 * kTile) / tpt;
    }
    __device__ __forceinline__ int unit_at(const TokenRange &, int, long long z) const { return (int)(z / tpt); }
    __device__ __forceinline__ long long min_cost() const { return 4 * tpt; }
    static constexpr int kCrumb = 2;   // least units of a part of an item
    static constexpr int kGrain = 1;
    __device__ __forceinline__ long long coarse() const { return 0; }
    static constexpr bool kShares = false;
};

struct Segment {
    int r, h, item;
    TokenRange t;
    int pos0;              // first cached token of the item
    int piece, units, a, b;   // piece, query tiles: all of the item's, the piece's
    int q0;                // the item's first query tile within the request
    int skip1;             // units before the second tile of cached tokens is seen
};

template <int D>
struct Control {
    uint64_t bars[kRing + 2 * Cfg<D>::kSlots];
    alignas(16) float lse[kLseSlots][kTile];   // -lse log2 e of the query tiles' rows, -inf for rows that count for nothing
    SegmentQueue<Segment> queue;
    alignas(8) uint8_t prefix[prefix_bytes(kSmemRequests)];
    int last[2];
    int gave_up;
    uint32_t refused;                  // the workspace has to be initialised first
    uint32_t tmem;
};

__device__ __forceinline__ bool next_segment(Walk<MassWork> &walk, Segment &s) {
    if (!walk.find()) return false;
    const MassWork &w = walk.l.w;
    s.r = walk.r, s.h = walk.h, s.item = walk.item, s.t = walk.t;
    s.pos0 = walk.i * 2 * kTile;
    s.units = w.units(walk.t, walk.i);
    s.a = walk.unit, s.b = walk.end_unit(s.units), s.piece = walk.piece;
    s.q0 = w.blind(walk.t, s.pos0) / w.tpt;
    s.skip1 = s.pos0 + kTile >= walk.t.past + walk.t.n ? s.units : w.blind(walk.t, s.pos0 + kTile) / w.tpt - s.q0;
    walk.next();
    return true;
}

// Page of 16-token group g of the request, -1 if absent, past the end or out of range.
__device__ __forceinline__ int group_page(const MassArgs &a, const Segment &s, int g, bool report) {
    if (g * kPage >= s.t.past + s.t.n) return -1;
    const int pid = a.page_table[(size_t)s.r * a.max_pages + g];
    if (pid >= a.P_phys) {
        if (report) atomicOr(&a.ctl->status, SE_DEV_BAD_PAGE_ID);
        return -1;
    }
    return pid < 0 ? -1 : pid;
}

template <int D>
__device__ __forceinline__ void copy_role(const MassArgs &a, const List<MassWork> &list, const CUtensorMap *q_map, const CUtensorMap *k_map,
                                          Control<D> *ctl, uint32_t k_smem, uint32_t ring, uint32_t bars, int lane) {
    using C = Cfg<D>;
    volatile int *gave_up = &ctl->gave_up;
    Walk<MassWork> walk(list, a.ctl, lane);
    Segment s;
    uint32_t pos = 0, pairs = 0;
    const bool chosen = elect_one();
    bool ok = true;
    while (ok && next_segment(walk, s)) {
        ok = ctl->queue.put(pairs, &s, gave_up, &a.ctl->status, lane);
        if (!ok) break;
        // K: 16 groups of 16 tokens.  Absent groups come from behind the tensor's last row, which reads as zeros.
        const int pid = group_page(a, s, s.pos0 / kPage + (lane & 15), lane < 16);
        const int z = pid >= 0 ? (pid * a.H_kv + s.h) * kPage : a.P_phys * a.H_kv * kPage;
        const uint32_t kb = pairs & 1, kbar = bars + 8 * (kKFull + kb);
        ok = warp_wait(bars + 8 * (kKEmpty + kb), (pairs >> 1 & 1) ^ 1, gave_up, &a.ctl->status);
        if (!ok) break;
        if (chosen) mbar_expect_tx(kbar, 2 * C::kTileBytes + (D == 64 && pairs == 0 ? kTestExtraTx : 0));
#pragma unroll
        for (int g = 0; g < 16; ++g) {
            const int row = __shfl_sync(kFull, z, g);
            if (chosen) {
#pragma unroll
                for (int half = 0; half < C::kHalves; ++half)
                    tma_load_3d(k_smem + (2 * kb + (g >> 3)) * C::kTileBytes + half * (kTile * 128) + (g & 7) * (kPage * 128), k_map,
                                half * 64, 0, row, kbar);
            }
            __syncwarp();
        }
        ++pairs;
        for (int u = s.a; u < s.b; ++u, ++pos) {
            const uint32_t slot = pos % C::kSlots, bar = bars + 8 * (kRing + slot);
            ok = warp_wait(bar + 8 * C::kSlots, (pos / C::kSlots & 1) ^ 1, gave_up, &a.ctl->status);
            if (!ok) break;
            if (chosen) {
                mbar_expect_tx(bar, list.w.tpt * a.G * D * 2 + (D == 128 && pos == 0 ? kTestExtraTx : 0));
#pragma unroll
                for (int half = 0; half < C::kHalves; ++half)
                    tma_load_3d(ring + slot * C::kTileBytes + half * (kTile * 128), q_map, half * 64, s.h * a.G,
                                s.t.start + (s.q0 + u) * list.w.tpt, bar);
            }
            __syncwarp();
        }
    }
    if (ok) ok = ctl->queue.put(pairs, nullptr, gave_up, &a.ctl->status, lane);
    // nothing may still be on its way to the CTA's shared memory when the CTA ends: copies, and the products' arrivals on the
    // barriers of the tiles they have let go.  A tile that is let go has been filled; where the products have given up (also
    // just now, in the wait for this very tile) the copy itself is waited for.
    for (uint32_t p = pos > C::kSlots ? pos - C::kSlots : 0; p < pos; ++p) {
        const uint32_t bar = bars + 8 * (kRing + p % C::kSlots), parity = p / C::kSlots & 1;
        ok = ok && warp_wait(bar + 8 * C::kSlots, parity, gave_up, &a.ctl->status);
        if (!ok) mbar_wait(bar, parity);
    }
    for (uint32_t p = pairs > 2 ? pairs - 2 : 0; p < pairs; ++p) {
        ok = ok && warp_wait(bars + 8 * (kKEmpty + (p & 1)), p >> 1 & 1, gave_up, &a.ctl->status);
        if (!ok) mbar_wait(bars + 8 * (kKFull + (p & 1)), p >> 1 & 1);
    }
}

// The query tiles' log-sum-exps, a tile ahead in registers.
template <int D>
__device__ __forceinline__ void lse_role(const MassArgs &a, const List<MassWork> &list, Control<D> *ctl, uint32_t bars, int lane) {
    volatile int *gave_up = &ctl->gave_up;
    uint32_t tiles = 0, turn = 0;
    const int live = list.w.tpt * a.G;
    for (;;) {
        const Segment *next = ctl->queue.get(turn++, gave_up, &a.ctl->status, lane);
        if (!next) break;
        const Segment s = *next;
        float x[4];
        auto fetch = [&](int u) {
            const int tok = (s.q0 + u) * list.w.tpt;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int row = lane + 32 * k, q = tok + row / a.G;
                x[k] = row < live && q < s.t.n ? a.lse[(size_t)(s.t.start + q) * a.H_q + s.h * a.G + row % a.G] : INFINITY;
            }
        };
        fetch(s.a);
        for (int u = s.a; u < s.b; ++u, ++tiles) {
            const uint32_t slot = tiles % kLseSlots;
            if (!warp_wait(bars + 8 * (kLseEmpty + slot), (tiles / kLseSlots & 1) ^ 1, gave_up, &a.ctl->status)) return;
#pragma unroll
            for (int k = 0; k < 4; ++k) ctl->lse[slot][lane + 32 * k] = x[k] == -INFINITY ? -INFINITY : -x[k] * kLog2e;
            __syncwarp();
            if (lane == 0) mbar_arrive(bars + 8 * (kLseFull + slot));
            if (u + 1 < s.b) fetch(u + 1);
        }
    }
}

template <int D>
__device__ __forceinline__ void mma_role(const MassArgs &a, Control<D> *ctl, uint32_t k_smem, uint32_t ring, uint32_t bars, int lane) {
    using C = Cfg<D>;
    volatile int *gave_up = &ctl->gave_up;
    constexpr uint32_t kInstr = mma_instr(kTile, false);
    const uint32_t tmem = ctl->tmem;
    uint32_t pos = 0, pairs = 0, step0 = 0, step1 = 0;
    const bool chosen = elect_one();
    bool ok = true, any = false;
    while (ok) {
        const Segment *next = ctl->queue.get(pairs, gave_up, &a.ctl->status, lane);
        if (!next) break;
        const Segment s = *next;
        const uint32_t kb = pairs & 1;
        ok = warp_wait(bars + 8 * (kKFull + kb), pairs >> 1 & 1, gave_up, &a.ctl->status);
        ++pairs;
        for (int u = s.a; u < s.b && ok; ++u, ++pos) {
            const uint32_t slot = pos % C::kSlots;
            ok = warp_wait(bars + 8 * (kRing + slot), pos / C::kSlots & 1, gave_up, &a.ctl->status);
            const uint64_t qd = smem_operand(ring + slot * C::kTileBytes, 16, 1024);
            for (int st = 0; st < 2 && ok; ++st) {
                if (st == 1 && u < s.skip1) continue;
                const uint32_t step = st ? step1++ : step0++, buf = 2 * st + (step & 1);
                ok = warp_wait(bars + 8 * (kSFree + buf), (step >> 1 & 1) ^ 1, gave_up, &a.ctl->status);
                if (!ok) break;
                tc_fence_after();
                const uint64_t kd = smem_operand(k_smem + (2 * kb + st) * C::kTileBytes, 16, 1024);
                if (chosen) {
#pragma unroll
                    for (int k = 0; k < D / 16; ++k) {
                        const uint32_t off = (k / 4) * (kTile * 128 >> 4) + (k % 4) * 2;
                        mma_ss(tmem + buf * kTile, kd + off, qd + off, kInstr, k > 0);
                    }
                    mma_commit(bars + 8 * (kSFull + buf));
                }
                __syncwarp();
                any = true;
            }
            if (ok && chosen) mma_commit(bars + 8 * (kRing + C::kSlots + slot));
            __syncwarp();
        }
        if (ok && chosen) mma_commit(bars + 8 * (kKEmpty + kb));
        __syncwarp();
    }
    if (any) {                           // nothing may be running when tensor memory goes away
        if (chosen) mma_commit(bars + 8 * kDrain);
        __syncwarp();
        mbar_wait(bars + 8 * kDrain, 0);
    }
}

template <int D>
__device__ __forceinline__ void sum_role(const MassArgs &a, const List<MassWork> &list, Control<D> *ctl, uint32_t bars, int st, int half) {
    volatile int *gave_up = &ctl->gave_up;
    const int row = threadIdx.x & 127, lane = threadIdx.x & 31, warp = row >> 5;
    const int col = half * (kTile / 2);                                    // the warpgroup's first column
    const uint32_t t_s = ctl->tmem + ((uint32_t)(warp * 32) << 16) + 2 * st * kTile + col;
    const float2 sl = make_float2(a.scale_log2, a.scale_log2);
    uint32_t step = 0, tiles = 0, verdicts = 0, halves = 0, turn = 0;
    // the second half's sum on its way to the first half (behind the partial results; shared memory is full)
    volatile float *other = a.partials + (size_t)kMaxPieces * 4 * kTile + (blockIdx.x * 2 + st) * kTile + row;
    for (;;) {
        const Segment *next = ctl->queue.get(turn++, gave_up, &a.ctl->status, lane);
        if (!next) break;
        const Segment s = *next;
        const int pos = s.pos0 + st * kTile + row;                         // the thread's cached token
        const int pid = group_page(a, s, pos / kPage, false);
        float sum = 0.f, lost = 0.f;   // of the query tiles so far, and what rounding took from it (Kahan)
        for (int u = s.a; u < s.b; ++u, ++tiles) {
            const uint32_t slot = tiles % kLseSlots;
            if (!warp_wait(bars + 8 * (kLseFull + slot), tiles / kLseSlots & 1, gave_up, &a.ctl->status)) return;
            if (st == 0 || u >= s.skip1) {
                const int tok = (s.q0 + u) * list.w.tpt;                     // the tile's first new token
                // columns [from, to) count: the queries at or behind the cached token, and of this request
                const int from = min(max(pos - s.t.past - tok, 0), kTile) * a.G - col, to = (s.t.n - tok) * a.G - col;
                const bool masked = __any_sync(kFull, from > 0) || to < min(list.w.tpt * a.G - col, kTile / 2);
                const uint32_t buf = step & 1;
                if (!warp_wait(bars + 8 * (kSFull + 2 * st + buf), step >> 1 & 1, gave_up, &a.ctl->status)) return;
                ++step;
                tc_fence_after();
                const float4 *nl = reinterpret_cast<const float4 *>(ctl->lse[slot] + col);
                float2 s0 = make_float2(0.f, 0.f), s1 = s0, nan = s0;
                float x[2][32];
                tmem_ld32(t_s + buf * kTile, x[0]);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    tmem_wait_ld();
                    settle<32>(x[k & 1]);
                    if (k == 0) tmem_ld32(t_s + buf * kTile + 32, x[1]);
                    if (k == 1) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(bars + 8 * (kSFree + 2 * st + buf));
                        __syncwarp();
                    }
                    float *y = x[k & 1];
                    if (masked) {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (32 * k + e < from || 32 * k + e >= to) y[e] = -INFINITY;
                    }
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        const float4 n = nl[8 * k + e / 4];
                        const float2 z0 = ffma2(make_float2(y[e], y[e + 1]), sl, make_float2(n.x, n.y));
                        const float2 z1 = ffma2(make_float2(y[e + 2], y[e + 3]), sl, make_float2(n.z, n.w));
                        s0 = __fadd2_rn(s0, make_float2(ex2(z0.x), ex2(z0.y)));
                        s1 = __fadd2_rn(s1, e % 16 == 0 ? ex2_fma(z1, nan) : make_float2(ex2(z1.x), ex2(z1.y)));
                    }
                }
                // 65536 weights added one after the other would lose 5e-6 of the sum
                const float y = __fsub_rn((s0.x + s0.y) + (s1.x + s1.y) + (nan.x + nan.y), lost), next = __fadd_rn(sum, y);
                lost = __fsub_rn(__fsub_rn(next, sum), y);
                sum = next;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(bars + 8 * (kLseEmpty + slot));
            __syncwarp();
        }
        // the two halves of the columns
        if (half == 1) {
            if (!warp_wait(bars + 8 * (kHalfFree + st), (halves++ & 1) ^ 1, gave_up, &a.ctl->status)) return;
            *other = sum;
            __syncwarp();
            if (lane == 0) mbar_arrive(bars + 8 * (kHalfFull + st));
            __syncwarp();
            continue;
        }
        if (!warp_wait(bars + 8 * (kHalfFull + st), halves++ & 1, gave_up, &a.ctl->status)) return;
        sum += *other;
        __syncwarp();
        if (lane == 0) mbar_arrive(bars + 8 * (kHalfFree + st));
        __syncwarp();
        const size_t at = ((size_t)max(pid, 0) * a.H_kv + s.h) * kPage + pos % kPage;
        if (s.a == 0 && s.b == s.units) {
            // the only addition to this token in this call
            if (pid >= 0 && pos < s.t.past + s.t.n) a.accum[at] += sum;
            continue;
        }
        auto part = [&](int piece, int kind) { return a.partials + (size_t)((piece * 2 + kind) * 2 + st) * kTile + row; };
        __stcg(part(s.piece, s.a == 0), sum);
        const int from = first_piece_of(list, s.item, s.piece, lane);
        __threadfence();
        __syncwarp();
        if (lane == 0) mbar_arrive(bars + 8 * (kAll + st));
        __syncwarp();
        if (warp == 0) {
            if (!warp_wait(bars + 8 * (kAll + st), verdicts & 1, gave_up, &a.ctl->status)) return;
            if (lane == 0) {
                __threadfence();
                uint32_t *ticket = a.ctl->tickets + 2 * from + st;
                const uint32_t add = s.b - s.a;
                const bool last = atomicAdd(ticket, add) + add == (uint32_t)s.units;
                if (last) atomicExch(ticket, 0u);
                ctl->last[st] = last;
                mbar_arrive(bars + 8 * (kVerdict + st));
            }
            __syncwarp();
        }
        if (!warp_wait(bars + 8 * (kVerdict + st), verdicts & 1, gave_up, &a.ctl->status)) return;
        ++verdicts;
        if (ctl->last[st]) {
            __threadfence();
            float all = 0.f;
            each_piece_of(list, s.item, s.units, from, lane, [&](int y, int ya, int) { all += __ldcg(part(y, ya == 0)); });
            if (pid >= 0 && pos < s.t.past + s.t.n) a.accum[at] += all;
        }
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
mass_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ MassArgs a) {
    using C = Cfg<D>;
    constexpr int kTiles = 2 * C::kPairs + C::kSlots;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    Control<D> *ctl = reinterpret_cast<Control<D> *>(smem + kTiles * C::kTileBytes);
    const uint32_t bars = smem_u32(ctl->bars), ring = base + 2 * C::kPairs * C::kTileBytes;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (base & 1023u) {                  // the swizzle pattern hangs on the address
        if (threadIdx.x == 0) atomicOr(&a.ctl->status, SE_DEV_WAIT_TIMEOUT);
        return;
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < 4; ++i) {
            mbar_init(bars + 8 * (kSFull + i), 1);
            mbar_init(bars + 8 * (kSFree + i), 8);
        }
        for (int i = 0; i < kLseSlots; ++i) {
            mbar_init(bars + 8 * (kLseFull + i), 1);
            mbar_init(bars + 8 * (kLseEmpty + i), 16);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bars + 8 * (kKFull + i), 1);
            mbar_init(bars + 8 * (kKEmpty + i), 1);
            mbar_init(bars + 8 * (kAll + i), 4);
            mbar_init(bars + 8 * (kVerdict + i), 1);
            mbar_init(bars + 8 * (kHalfFull + i), 4);
            mbar_init(bars + 8 * (kHalfFree + i), 4);
        }
        mbar_init(bars + 8 * kDrain, 1);
        for (int i = 0; i < 2 * C::kSlots; ++i) mbar_init(bars + 8 * (kRing + i), 1);
        ctl->queue.init(18);
        mbar_fence_init();
        ctl->gave_up = 0;
    }
    // (read ahead: it is here when the list is)
    const uint32_t refused = threadIdx.x == 32 ? *(volatile uint32_t *)&a.ctl->needs_init : 0u;
    if (warp == kMmaWarp) tmem_alloc(smem_u32(&ctl->tmem), 512);
    const MassWork work(a);
    const List<MassWork> list = make_list<kThreads>(work, a.B, a.H_kv, a.ctl,
                                          a.B > kSmemRequests ? a.prefixes + prefix_bytes(a.B) * blockIdx.x : ctl->prefix, smem);
    // query rows that no tensor copy fills (G does not divide 128) stay zero
    for (int i = threadIdx.x; i < (work.tpt * a.G == kTile ? 0 : C::kSlots * C::kTileBytes / 16); i += kThreads)
        reinterpret_cast<uint4 *>(smem + 2 * C::kPairs * C::kTileBytes)[i] = make_uint4(0, 0, 0, 0);
    if (threadIdx.x == 32) ctl->refused = refused;
    fence_async_proxy();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();

    if (ctl->refused) {
        if (threadIdx.x == 0 && blockIdx.x == 0) atomicOr(&a.ctl->status, SE_DEV_WAIT_TIMEOUT);
    } else if (warp < 16) {
        regs_up<kRegsSum>();
        sum_role<D>(a, list, ctl, bars, warp >> 2 & 1, warp >> 3);
    } else {
        regs_down<kRegsOther>();
        if (warp == kCopyWarp) copy_role<D>(a, list, &q_map, &k_map, ctl, base, ring, bars, lane);
        else if (warp == kLseWarp) lse_role<D>(a, list, ctl, bars, lane);
        else if (warp == kMmaWarp) mma_role<D>(a, ctl, base, ring, bars, lane);
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_free(ctl->tmem, 512);
    }
}

template <int D>
cudaError_t launch_mass(const se_params &p, const AttendCall &c, float *score_accum, cudaStream_t stream) {
    using C = Cfg<D>;
    const int G = p.H_q / p.H_kv;
    CUtensorMap q_map, k_map;
    if (!make_rows_map(&q_map, c.q, D, p.H_q, c.total_tokens, c.q_stride, G, kTile / G) ||
        !make_rows_map(&k_map, c.k, D, 1, (long long)p.num_phys_pages * p.H_kv * kPage, D, 1, kPage))
        return cudaErrorInvalidValue;
    MassArgs a = {};
    a.cu = c.cu_seqlens, a.seq_lens = c.seq_lens, a.page_table = c.page_table;
    a.lse = c.lse, a.accum = score_accum;
    a.ctl = reinterpret_cast<PromptControl *>(c.workspace);
    a.partials = partials_of(c.workspace);
    a.prefixes = c.workspace + prefix_workspace_offset(p.D);
    a.B = p.B, a.H_q = p.H_q, a.H_kv = p.H_kv, a.G = G, a.T = c.total_tokens, a.max_pages = p.max_pages;
    a.P_phys = p.num_phys_pages, a.scale_log2 = effective_scale(p) * kLog2e;
    constexpr size_t smem = (2 * C::kPairs + C::kSlots) * C::kTileBytes + sizeof(Control<D>);
    static_assert(smem <= 227 * 1024, "shared memory of a CTA");
    auto kern = mass_kernel<D>;
    // the register split (setmaxnreg) draws on what the block was launched with
    cudaFuncAttributes attr;
    cudaError_t e = cudaFuncGetAttributes(&attr, kern);
    if (e != cudaSuccess) return e;
    if (attr.numRegs * kThreads < 512 * kRegsSum + 128 * kRegsOther) return cudaErrorInvalidConfiguration;
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    kern<<<kPromptCtas, kThreads, smem, stream>>>(q_map, k_map, a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_h2o_accumulate(const se_params &p, const AttendCall &c, float *score_accum, cudaStream_t stream) {
    return p.D == 128 ? launch_mass<128>(p, c, score_accum, stream) : launch_mass<64>(p, c, score_accum, stream);
}

}  // namespace se
