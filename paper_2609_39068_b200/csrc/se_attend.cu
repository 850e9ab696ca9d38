// Attention of a packed batch of new tokens (Appendix A, attention equations of "MHA, MQA, and GQA"), over the paged
// cache or over contiguous K and V.
//
// Mathematics.  A query tile is 128 rows = 128/G tokens x the G query heads of one kv-head, so the heads of a group share
// every K and V tile.  Over the KV tiles j of 128 tokens:  S = Q K_j^T,  p = 2^(S sl - m)  with sl = sm_scale log2 e,
// O += P V_j, l += rowsum p;  out = O / l,  lse = (m + log2 l) ln 2.  m is a row maximum that is moved (and O, l
// rescaled) only when the tile's maximum exceeds it by more than 8, so p <= 2^8 and most tiles leave O alone.
//
// What bounds it.  Per (128 rows x 128 tokens) at D = 128 the two products take 1024 cycles of the tensor cores and
// the 16384 exponentials 1024 cycles of the special-function units: both have to run all the time.  So a CTA (one per
// SM, persistent) works on two streams of tiles: two warpgroups do the softmax of one stream each, one thread issues all
// products, one warp all copies.  S (fp32), P (bf16, in S's columns) and O (fp32) live in tensor memory: 2 x (128 + D)
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

constexpr int kThreads = kPromptThreads;   // 2 softmax warpgroups, copy warp, product warp, 2 idle warps
constexpr int kCopyWarp = 8, kMmaWarp = 9;
constexpr int kRegsSoftmax = 208, kRegsOther = 88;   // 256 * 208 + 128 * 88 = 384 * 168
constexpr int kTile = 128;             // query rows of a tile, tokens of a KV tile
constexpr int kControlBytes = 2048;    // status word, tickets
constexpr int kItemCost = 128;         // cost of starting a query tile, in tokens
constexpr int kMinCost = 4 * kTile;    // a CTA takes at least two shared KV tiles
constexpr float kSlack = 8.f;          // the running maximum may lag by 2^8

template <int D>
struct Cfg {
    static constexpr int kHalves = D / 64;
    static constexpr int kTileBytes = kTile * D * 2;
    static constexpr int kSlots = 5 * 128 / D;                    // ring of K and V tiles, 160 KB
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
    uint32_t *status, *tickets;
    int B, H_q, H_kv, G, T, max_pages, P_phys;
    float scale_log2;
};

template <int ST>
struct Stream {
    static constexpr int value = ST;
};

enum Bar { kQFull, kQEmpty, kSFull, kPReady = kSFull + 2, kODone = kPReady + 2, kOFree = kODone + 2, kAll = kOFree + 2, kVerdict = kAll + 2, kSwap = kVerdict + 2,
           kDrain, kRing };

template <int D>
struct Control {
    uint64_t bars[kRing + 2 * Cfg<D>::kSlots];
    Pieces pieces;
    uint32_t mask[Cfg<D>::kMasks];     // present 16-token groups of the tiles in flight
    int last[2];
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
        return (t.past + i * 2 * tpt + new_tokens(t, i) + kTile - 1) / kTile;
    }
    __device__ __forceinline__ int unit_at(const TokenRange &t, int i, long long z) const {
        return (int)(z / (kTile * (new_tokens(t, i) > tpt ? 2 : 1)));
    }
    __device__ __forceinline__ long long min_cost() const { return kMinCost; }
};

struct Segment {
    int r, h, item;
    TokenRange t;
    int tok0, ntok;        // new tokens of the item, relative to the request
    bool alt;
    int a, b, nkv;         // KV tiles of this piece, of the item
    int steps0, steps1;    // per stream
    __device__ __forceinline__ int steps(int st) const { return st ? steps1 : steps0; }
};

// This CTA's next piece; every role walks the same list.
__device__ __forceinline__ bool next_segment(const AttendArgs &a, const AttendWork &w, const Pieces &p, Cursor &c, Segment &s) {
    if (piece_done(w, a.B, p, c)) return false;
    s.r = c.r, s.h = c.h, s.item = c.item, s.t = c.t;
    s.tok0 = c.i * 2 * w.tpt;
    s.ntok = w.new_tokens(c.t, c.i);
    s.alt = s.ntok <= w.tpt;
    s.nkv = w.units(c.t, c.i);
    s.a = c.unit;
    s.b = piece_end(c, p, s.nkv);
    if (s.alt) {
        s.steps0 = (s.b - s.a + 1) / 2;
        s.steps1 = (s.b - s.a) / 2;
    } else {
        const int n0 = (c.t.past + s.tok0 + w.tpt + kTile - 1) / kTile;    // the first tile's tokens see no more than this
        s.steps0 = max(min(s.b, n0) - s.a, 0);
        s.steps1 = s.b - s.a;
    }
    next_item(w, a.B, a.H_kv, c);
    return true;
}

// ---- copies ------------------------------------------------------------------------
// One K or V tile (128 tokens of one head) into a ring slot, by a warp.  A lane brings 16 tokens x 64 channels; groups that
// are absent or past the end come from behind the tensor's last row, which reads as zeros.  With `by_hand` (V) the group
// that holds the end of the request is copied row by row, so that what lies behind the end, which may be anything, is zero.
template <int D>
__device__ __forceinline__ void load_tile(const AttendArgs &a, const CUtensorMap *map, const CUtensorMap *wide, const Segment &s, int tile, int pid, int end,
                                          bool by_hand, uint32_t slot, uint32_t bar, int lane) {
    using C = Cfg<D>;
    if (!a.page_table && (tile + 1) * kTile <= end) {
        if (lane == 0) mbar_expect_tx(bar, C::kTileBytes);
        __syncwarp();
        if (lane < C::kHalves)
            tma_load_3d(slot + lane * (kTile * 128), wide, lane * 64, s.h, s.t.start + tile * kTile, bar);
        return;
    }
    const int pg = lane & 7, half = lane >> 3;
    const int tok = tile * kTile + pg * kPage;                             // the group's first token
    const bool part = by_hand && pid >= 0 && tok < end && end - tok < kPage;
    const unsigned parts = __ballot_sync(kFull, part && half == 0);
    if (parts) {
        const int src = __ffs(parts) - 1;
        const int ppid = __shfl_sync(kFull, pid, src), ptok = __shfl_sync(kFull, tok, src), rows = end - ptok;
        const uint16_t *base = a.page_table ? a.v + ((size_t)ppid * a.H_kv + s.h) * (kPage * D)
                                            : a.v + (long long)(s.t.start + ptok) * a.v_stride + s.h * D;
        const long long pitch = a.page_table ? D : a.v_stride;
        constexpr int kPieces = D / 8;
#pragma unroll
        for (int i = 0; i < kPage * kPieces / 32; ++i) {
            const int e = i * 32 + lane, row = e / kPieces, c = e % kPieces, at = src * kPage + row;
            uint4 x = make_uint4(0, 0, 0, 0);
            if (row < rows) x = *reinterpret_cast<const uint4 *>(base + row * pitch + c * 8);
            const uint32_t dst = slot + (c >> 3) * (kTile * 128) + at * 128 + (((c & 7) ^ (at & 7)) << 4);
            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(dst), "r"(x.x), "r"(x.y), "r"(x.z), "r"(x.w) : "memory");
        }
        fence_async_proxy();
        __syncwarp();
    }
    const int groups = parts ? 7 : 8;
    if (lane == 0) mbar_expect_tx(bar, groups * kPage * D * 2);
    __syncwarp();
    if (half < Cfg<D>::kHalves && !part) {
        int y = 0, z;
        if (a.page_table) {
            z = pid >= 0 ? (pid * a.H_kv + s.h) * kPage : a.P_phys * a.H_kv * kPage;
        } else {
            y = s.h;
            z = pid >= 0 ? s.t.start + tok : a.T;
        }
        tma_load_3d(slot + half * (kTile * 128) + pg * (kPage * 128), map, half * 64, y, z, bar);
    }
}

// Page of the lane's 16-token group of a tile: >= 0 present (contiguous K and V: 0), -1 absent or past the end.
__device__ __forceinline__ int group_page(const AttendArgs &a, const Segment &s, int tile, int end, int lane) {
    const int g = tile * (kTile / kPage) + (lane & 7);
    if (g * kPage >= end) return -1;
    if (!a.page_table) return 0;
    const int pid = a.page_table[(size_t)s.r * a.max_pages + g];
    if (pid >= a.P_phys) {
        if (lane < 8) atomicOr(a.status, SE_DEV_BAD_PAGE_ID);
        return -1;
    }
    return pid < 0 ? -1 : pid;
}

template <int D>
__device__ __forceinline__ void copy_role(const AttendArgs &a, const CUtensorMap *q_map, const CUtensorMap *k_map,
                                          const CUtensorMap *v_map, const CUtensorMap *k_wide, const CUtensorMap *v_wide,
                                          Control<D> *ctl, uint32_t q_smem, uint32_t ring, uint32_t bars,
                                          int lane) {
    using C = Cfg<D>;
    volatile int *gave_up = &ctl->gave_up;
    const int tpt = kTile / a.G;
    const AttendWork work(a);
    Cursor c = first_piece(work, a.B, a.H_kv, ctl->pieces);
    Segment s;
    uint32_t pos = 0, tiles = 0, pieces = 0;
    bool ok = true;
    while (ok && next_segment(a, work, ctl->pieces, c, s)) {
        const int stop = s.t.past + s.t.n;                                 // tokens the request has
        int pid = group_page(a, s, s.a, stop, lane);
        ok = warp_wait(bars + 8 * kQEmpty, (pieces & 1) ^ 1, gave_up, a.status);
        if (!ok) break;
        if (lane == 0) mbar_expect_tx(bars + 8 * kQFull, (s.alt ? 1 : 2) * tpt * a.G * D * 2);
        __syncwarp();
        if (lane < 2 * C::kHalves) {
            const int st = lane / C::kHalves, half = lane % C::kHalves;
            if (st == 0 || !s.alt)
                tma_load_3d(q_smem + st * C::kTileBytes + half * (kTile * 128), q_map, half * 64, s.h * a.G,
                            s.t.start + s.tok0 + st * tpt, bars + 8 * kQFull);
        }
        ++pieces;
        for (int t = s.a; t < s.b; ++t) {
            const int next_pid = t + 1 < s.b ? group_page(a, s, t + 1, stop, lane) : -1;
            const unsigned mask = __ballot_sync(kFull, pid >= 0) & 0xffu;
            if (lane == 0) ctl->mask[tiles % C::kMasks] = mask;
            ++tiles;
            for (int kv = 0; kv < 2 && ok; ++kv, ++pos) {
                const uint32_t slot = pos % C::kSlots, bar = bars + 8 * (kRing + slot);
                ok = warp_wait(bar + 8 * C::kSlots, (pos / C::kSlots & 1) ^ 1, gave_up, a.status);
                if (!ok) break;
                load_tile<D>(a, kv ? v_map : k_map, kv ? v_wide : k_wide, s, t, pid, stop, kv == 1, ring + slot * C::kTileBytes, bar, lane);
            }
            if (!ok) break;
            pid = next_pid;
        }
    }
    // no copy may be in flight when the CTA's shared memory goes away
    if (!ok) {
        const uint32_t first = pos > C::kSlots ? pos - C::kSlots : 0;
        for (uint32_t p = first; p < pos; ++p) mbar_wait(bars + 8 * (kRing + p % C::kSlots), p / C::kSlots & 1);
        if (pieces) mbar_wait(bars + 8 * kQFull, (pieces - 1) & 1);
    }
}

// ---- products ----------------------------------------------------------------------
// The whole warp walks the list, so that addresses stay in uniform registers; one elected lane issues (a role run by a
// single lane took 82 cycles per instruction to issue, more than the 64 that it computes).
template <int D, int ST>
struct Products {
    using C = Cfg<D>;
    // S[ST] = Q K^T
    static __device__ __forceinline__ void scores(uint32_t tmem, uint32_t q, uint32_t k, uint32_t bars, int release) {
        const uint64_t qd = smem_operand(q, 16, 1024), kd = smem_operand(k, 16, 1024);
        if (elect_one()) {
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                const uint32_t off = (i / 4) * (kTile * 128 >> 4) + (i % 4) * 2;
                mma_ss(tmem + ST * kTile, qd + off, kd + off, mma_instr(kTile, false), i > 0);
            }
            mma_commit(bars + 8 * (kSFull + ST));
            if (release >= 0) mma_commit(bars + 8 * release);
        }
    }
    // O[ST] += P V
    static __device__ __forceinline__ void values(uint32_t tmem, uint32_t v, bool accumulate, uint32_t bars, int release) {
        const uint64_t vd = smem_operand(v, kTile * 128, 1024);
        if (elect_one()) {
#pragma unroll
            for (int i = 0; i < kTile / 16; ++i)
                mma_ts(tmem + C::kTmemO + ST * D, tmem + ST * kTile + i * 8, vd + i * (16 * 128 >> 4), mma_instr(D, true),
                       accumulate || i > 0);
            mma_commit(bars + 8 * (kODone + ST));
            if (release >= 0) mma_commit(bars + 8 * release);
        }
    }
};

template <int D>
__device__ __forceinline__ void mma_role(const AttendArgs &a, Control<D> *ctl, uint32_t q_smem, uint32_t ring, uint32_t bars) {
    using C = Cfg<D>;
    volatile int *gave_up = &ctl->gave_up;
    const uint32_t tmem = ctl->tmem;
    const AttendWork work(a);
    Cursor c = first_piece(work, a.B, a.H_kv, ctl->pieces);
    Segment s;
    uint32_t pos = 0, pieces = 0, p_seen = 0, o_used = 0;                  // bit st: parity of the stream's next wait
    bool any = false;
    auto wait = [&](int bar, uint32_t parity) { return warp_wait(bars + 8 * bar, parity & 1, gave_up, a.status); };
    // K and V tiles are waited for in order: `k_next`, `v_next` are the first ring positions not waited for yet
    uint32_t k_next = 0, v_next = 1;
    auto wait_k = [&](uint32_t at) {
        for (; k_next <= at; k_next += 2)
            if (!wait(kRing + k_next % C::kSlots, k_next / C::kSlots)) return false;
        return true;
    };
    auto wait_v = [&](uint32_t at) {
        for (; v_next <= at; v_next += 2)
            if (!wait(kRing + v_next % C::kSlots, v_next / C::kSlots)) return false;
        return true;
    };
    while (next_segment(a, work, ctl->pieces, c, s)) {
        const int steps = max(s.steps0, s.steps1);
        const uint32_t q1 = q_smem + (s.alt ? 0 : C::kTileBytes);
        // ring position of the K tile of step i of stream st; its V tile follows
        auto place = [&](int st, int i) { return pos + 2u * (s.alt ? 2 * i + st : i); };
        auto slot = [&](uint32_t at) { return ring + at % C::kSlots * C::kTileBytes; };
        auto release = [&](int st, uint32_t at) { return s.alt || st == 1 ? (int)(kRing + C::kSlots + at % C::kSlots) : -1; };
        // a step: everything that can be waited for early comes before the wait for the weights
        auto step = [&](auto stream, int i) {
            constexpr int ST = decltype(stream)::value;
            const int mine = ST ? s.steps1 : s.steps0;
            if (i >= mine) return true;
            const bool more = i + 1 < mine;
            const uint32_t at = place(ST, i), next = place(ST, i + 1);
            if (!wait_v(at + 1) || (more && !wait_k(next))) return false;
            if (i == 0) {                // the epilogue of the stream's last piece has read O
                if (!wait(kOFree + ST, (o_used >> ST & 1) ^ 1)) return false;
                o_used ^= 1u << ST;
            }
            if (!wait(kPReady + ST, p_seen >> ST)) return false;
            p_seen ^= 1u << ST;
            tc_fence_after();
            Products<D, ST>::values(tmem, slot(at + 1), i > 0, bars, release(ST, at + 1));
            if (more) Products<D, ST>::scores(tmem, ST ? q1 : q_smem, slot(next), bars, release(ST, next));
            return true;
        };
        if (!wait(kQFull, pieces)) break;
        ++pieces;
        any = true;
        if (s.steps0 > 0) {
            if (!wait_k(place(0, 0))) break;
            tc_fence_after();
            Products<D, 0>::scores(tmem, q_smem, slot(place(0, 0)), bars, release(0, place(0, 0)));
        }
        if (s.steps1 > 0) {
            if (!wait_k(place(1, 0))) break;
            tc_fence_after();
            Products<D, 1>::scores(tmem, q1, slot(place(1, 0)), bars, release(1, place(1, 0)));
        }
        if (steps == 1 && elect_one()) mma_commit(bars + 8 * kQEmpty);
        bool ok = true;
        for (int i = 0; i < steps && ok; ++i) {
            ok = step(Stream<0>{}, i) && step(Stream<1>{}, i);
            if (i + 2 == steps && elect_one()) mma_commit(bars + 8 * kQEmpty);   // the last product with Q is on its way
        }
        if (!ok) break;
        pos += 2u * (s.b - s.a);
    }
    if (any) {                           // nothing may be running when tensor memory goes away
        if (elect_one()) mma_commit(bars + 8 * kDrain);
        __syncwarp();
        mbar_wait(bars + 8 * kDrain, 0);
    }
}

// ---- softmax and epilogue ----------------------------------------------------------
__device__ __forceinline__ float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }

template <int D>
__device__ __forceinline__ float *partial_slot(const AttendArgs &a, int cta, int kind, int st) {
    return a.partials + (size_t)((cta * 2 + kind) * 2 + st) * Cfg<D>::kSlotFloats;
}

// Merges the partial results of one query tile and writes its output.  128 threads; warp w takes rows w, w + 4, ...
// `slots`: calls f(pointer) for every contribution, in CTA order.
template <int D, typename Each>
__device__ __forceinline__ void merge_rows(const AttendArgs &a, const Segment &s, int st, int row_from, int row_step, Each each,
                                           int lane) {
    constexpr int V = D / 32;
    const int tpt = kTile / a.G;
    const int tok = s.tok0 + (s.alt ? 0 : st * tpt);
    const int rows = min(tpt, s.tok0 + s.ntok - tok) * a.G;
    const long long out0 = ((long long)(s.t.start + tok) * a.H_q + s.h * a.G);
    const int my = row_from + row_step * lane;                             // statistics: a lane per row
    const bool have = my < rows;
    float M = -INFINITY, L = 0.f;
    each([&](const float *p) {
        const float m = have ? __ldcg(p + kTile * D + my) : -INFINITY, l = have ? __ldcg(p + kTile * D + kTile + my) : 0.f;
        if (m == -INFINITY) return;
        const float top = fmaxf(M, m);
        L = L * ex2(M - top) + l * ex2(m - top);
        M = top;
    });
    const float inv = L > 0.f ? 1.f / L : 0.f;
    if (have && a.lse) a.lse[out0 + (long long)(my / a.G) * a.H_q + my % a.G] = L > 0.f ? (M + log2f(L)) * kLn2 : -INFINITY;
    const int mine = rows > row_from ? (rows - row_from + row_step - 1) / row_step : 0;
    for (int k0 = 0; k0 < mine; k0 += 8) {
        float acc[8][V] = {};
        each([&](const float *p) {
            const float m = have ? __ldcg(p + kTile * D + my) : -INFINITY;
            const float w = m == -INFINITY ? 0.f : ex2(m - M) * inv;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const float wk = __shfl_sync(kFull, w, k0 + k);
                if (k0 + k < mine && wk > 0.f) {
                    const float *src = p + (size_t)(row_from + row_step * (k0 + k)) * D + lane * V;
                    float x[V];
                    if constexpr (V == 4) {
                        const float4 f = __ldcg(reinterpret_cast<const float4 *>(src));
                        x[0] = f.x, x[1] = f.y, x[2] = f.z, x[3] = f.w;
                    } else {
                        const float2 f = __ldcg(reinterpret_cast<const float2 *>(src));
                        x[0] = f.x, x[1] = f.y;
                    }
#pragma unroll
                    for (int v = 0; v < V; ++v) acc[k][v] += wk * x[v];
                }
            }
        });
#pragma unroll
        for (int k = 0; k < 8; ++k) {
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
__device__ __forceinline__ void softmax_role(const AttendArgs &a, Control<D> *ctl, uint32_t bars, int st) {
    using C = Cfg<D>;
    volatile int *gave_up = &ctl->gave_up;
    const int row = threadIdx.x & 127, lane = threadIdx.x & 31, warp = row >> 5;
    const int tpt = kTile / a.G;
    const uint32_t lanes = (uint32_t)(warp * 32) << 16;
    const uint32_t t_s = ctl->tmem + lanes + st * kTile, t_o = ctl->tmem + lanes + C::kTmemO + st * D;
    const float sl = a.scale_log2;
    const AttendWork work(a);
    Cursor c = first_piece(work, a.B, a.H_kv, ctl->pieces);
    Segment s;
    uint32_t step = 0, tiles = 0, verdicts = 0, swaps = 0;
    // both warpgroups have come here
    auto swap_sync = [&] {
        __syncwarp();
        if (lane == 0) mbar_arrive(bars + 8 * kSwap);
        return warp_wait(bars + 8 * kSwap, swaps++ & 1, gave_up, a.status);
    };
    while (next_segment(a, work, ctl->pieces, c, s)) {
        const int tok = s.tok0 + (s.alt ? 0 : st * tpt);                   // the tile's first new token
        const int ntok = min(tpt, s.tok0 + s.ntok - tok);
        const int q = min(row / a.G, ntok - 1);
        const int sees = s.t.past + tok + q + 1;                           // tokens the row sees
        const int least = __reduce_min_sync(kFull, sees);
        const int steps = s.steps(st);
        float m = -INFINITY;                                               // in units of the raw scores
        float2 l2 = make_float2(0.f, 0.f);
        for (int i = 0; i < steps; ++i, ++step) {
            const int rel = s.alt ? 2 * i + st : i, tile = s.a + rel;
            if (!warp_wait(bars + 8 * (kSFull + st), step & 1, gave_up, a.status)) return;
            tc_fence_after();
            float x[kTile];
#pragma unroll
            for (int k = 0; k < kTile; k += 32) tmem_ld32(t_s + k, x + k);
            const unsigned mask = ctl->mask[(tiles + rel) % C::kMasks];
            tmem_wait_ld();
            settle<kTile>(x);
            if (tile * kTile + kTile > least || mask != 0xffu) {
                const int limit = sees - tile * kTile;
#pragma unroll
                for (int k = 0; k < kTile; ++k)
                    if (k >= limit || !(mask >> (k / kPage) & 1)) x[k] = -INFINITY;
            }
            float top[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
            for (int k = 4; k < kTile; k += 8)
#pragma unroll
                for (int e = 0; e < 4; ++e) top[e] = k + 4 + e < kTile ? max3(top[e], x[k + e], x[k + 4 + e]) : fmaxf(top[e], x[k + e]);
            const float tm = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
            const float mn = fmaxf(m, tm);
            if (__any_sync(kFull, (mn - m) * sl > kSlack)) {
                const float f = m == -INFINITY ? 0.f : ex2((m - mn) * sl);
                m = mn;
                l2.x *= f, l2.y *= f;
                if (i > 0) {
                    if (!warp_wait(bars + 8 * (kODone + st), (step - 1) & 1, gave_up, a.status)) return;
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
#pragma unroll
            for (int k = 0; k < kTile; k += 64) {
                uint32_t p[32];
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    const float2 y = ffma2(make_float2(x[k + 2 * e], x[k + 2 * e + 1]), make_float2(sl, sl), make_float2(off, off));
                    const float2 w = make_float2(ex2(y.x), ex2(y.y));
                    l2 = __fadd2_rn(l2, w);
                    // the weights enter the product with V as bf16 (8 significant bits), the sum l keeps fp32
                    const __nv_bfloat162 b = __float22bfloat162_rn(w);
                    p[e] = *reinterpret_cast<const uint32_t *>(&b);
                }
                tmem_st32(t_s + k / 2, p);
            }
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bars + 8 * (kPReady + st));
        }
        tiles += s.b - s.a;
        if (steps > 0) {
            if (!warp_wait(bars + 8 * (kODone + st), (step - 1) & 1, gave_up, a.status)) return;
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
            continue;
        }
        const int kind = s.a == 0;
        if (steps > 0 || !s.alt) {
            float *slot = partial_slot<D>(a, blockIdx.x, kind, st);
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
            }
            __stcg(slot + kTile * D + row, m2);
            __stcg(slot + kTile * D + kTile + row, l);
        }
        if (whole) {
            // alt, all KV tiles in this CTA: the two warpgroups exchange their results and merge half of the rows each
            if (!swap_sync()) return;
            const float *s0 = partial_slot<D>(a, blockIdx.x, kind, 0), *s1 = partial_slot<D>(a, blockIdx.x, kind, 1);
            merge_rows<D>(a, s, st, st * 4 + warp, 8, [&](auto f) { f(s0); f(s1); }, lane);
            if (!swap_sync()) return;                                      // the slots may be written again
            continue;
        }
        if (steps == 0 && s.alt) continue;
        // the CTAs of the item: from the one that begins it to the one that ends it
        const int from = first_cta(ctl->pieces, s.item);
        uint32_t *ticket = a.tickets + 2 * from + (s.alt ? 0 : st);
        __threadfence();
        __syncwarp();
        if (lane == 0) mbar_arrive(bars + 8 * (kAll + st));
        if (warp == 0) {
            if (!warp_wait(bars + 8 * (kAll + st), verdicts & 1, gave_up, a.status)) return;
            if (lane == 0) {
                __threadfence();
                const uint32_t add = s.alt ? steps : s.b - s.a;
                const bool last = atomicAdd(ticket, add) + add == (uint32_t)s.nkv;
                if (last) atomicExch(ticket, 0u);
                ctl->last[st] = last;
                mbar_arrive(bars + 8 * (kVerdict + st));
            }
            __syncwarp();
        }
        if (!warp_wait(bars + 8 * (kVerdict + st), verdicts & 1, gave_up, a.status)) return;
        ++verdicts;
        if (ctl->last[st]) {
            __threadfence();
            auto each = [&](auto f) {
                each_cta(ctl->pieces, s.item, s.nkv, from, [&](int y, int ya, int yb) {
                    f((const float *)partial_slot<D>(a, y, ya == 0, s.alt ? 0 : st));
                    if (s.alt && yb - ya > 1) f((const float *)partial_slot<D>(a, y, ya == 0, 1));
                });
            };
            merge_rows<D>(a, s, st, warp, 4, each, lane);
        }
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
attend_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
              const __grid_constant__ CUtensorMap v_map, const __grid_constant__ CUtensorMap k_wide,
              const __grid_constant__ CUtensorMap v_wide, const __grid_constant__ AttendArgs a) {
    using C = Cfg<D>;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    Control<D> *ctl = reinterpret_cast<Control<D> *>(smem + 2 * C::kTileBytes + C::kSlots * C::kTileBytes);
    const uint32_t bars = smem_u32(ctl->bars);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (base & 1023u) {                  // the swizzle pattern hangs on the address
        if (threadIdx.x == 0) atomicOr(a.status, SE_DEV_WAIT_TIMEOUT);
        return;
    }

    if (threadIdx.x == 0) {
        mbar_init(bars + 8 * kQFull, 1);
        mbar_init(bars + 8 * kQEmpty, 1);
        for (int st = 0; st < 2; ++st) {
            mbar_init(bars + 8 * (kSFull + st), 1);
            mbar_init(bars + 8 * (kPReady + st), 4);
            mbar_init(bars + 8 * (kODone + st), 1);
            mbar_init(bars + 8 * (kOFree + st), 4);
            mbar_init(bars + 8 * (kAll + st), 4);
            mbar_init(bars + 8 * (kVerdict + st), 1);
        }
        mbar_init(bars + 8 * kSwap, 8);
        mbar_init(bars + 8 * kDrain, 1);
        for (int i = 0; i < 2 * C::kSlots; ++i) mbar_init(bars + 8 * (kRing + i), 1);
        mbar_fence_init();
        ctl->gave_up = 0;
    }
    if (warp == kMmaWarp) tmem_alloc(smem_u32(&ctl->tmem), 512);
    cut_work(AttendWork(a), a.B, a.H_kv, a.status, &ctl->pieces, smem + 2 * C::kTileBytes);
    // query rows that no tensor copy fills (G does not divide 128) stay zero
    for (int i = threadIdx.x; i < 2 * C::kTileBytes / 16; i += kThreads)
        reinterpret_cast<uint4 *>(smem)[i] = make_uint4(0, 0, 0, 0);
    fence_async_proxy();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();

    if (warp < 8) {
        regs_up<kRegsSoftmax>();
        softmax_role<D>(a, ctl, bars, warp >> 2);
    } else {
        regs_down<kRegsOther>();
        if (warp == kCopyWarp) copy_role<D>(a, &q_map, &k_map, &v_map, &k_wide, &v_wide, ctl, base, base + 2 * C::kTileBytes, bars, lane);
        else if (warp == kMmaWarp) mma_role<D>(a, ctl, base, base + 2 * C::kTileBytes, bars);
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
    CUtensorMap q_map, k_map, v_map, k_wide, v_wide;
    bool ok = make_rows_map(&q_map, c.q, D, p.H_q, c.total_tokens, c.q_stride, G, kTile / G);
    if (c.page_table) {
        const long long rows = (long long)p.num_phys_pages * p.H_kv * kPage;
        ok = ok && make_rows_map(&k_map, c.k, D, 1, rows, D, 1, kPage) && make_rows_map(&v_map, c.v, D, 1, rows, D, 1, kPage);
        k_wide = k_map, v_wide = v_map;                      // not used
    } else {
        ok = ok && make_rows_map(&k_map, c.k, D, p.H_kv, c.total_tokens, c.k_stride, 1, kPage) &&
             make_rows_map(&v_map, c.v, D, p.H_kv, c.total_tokens, c.v_stride, 1, kPage) &&
             make_rows_map(&k_wide, c.k, D, p.H_kv, c.total_tokens, c.k_stride, 1, kTile) &&
             make_rows_map(&v_wide, c.v, D, p.H_kv, c.total_tokens, c.v_stride, 1, kTile);
    }
    if (!ok) return cudaErrorInvalidValue;
    AttendArgs a = {};
    a.cu = c.cu_seqlens, a.seq_lens = c.seq_lens, a.page_table = c.page_table;
    a.v = static_cast<const uint16_t *>(c.v), a.v_stride = c.v_stride;
    a.out = static_cast<uint16_t *>(c.out), a.lse = c.lse;
    a.status = reinterpret_cast<uint32_t *>(c.workspace), a.tickets = reinterpret_cast<uint32_t *>(c.workspace + 256);
    a.partials = reinterpret_cast<float *>(c.workspace + kControlBytes);
    a.B = p.B, a.H_q = p.H_q, a.H_kv = p.H_kv, a.G = G, a.T = c.total_tokens, a.max_pages = p.max_pages;
    a.P_phys = p.num_phys_pages, a.scale_log2 = effective_scale(p) * kLog2e;
    auto kern = attend_kernel<D>;
    // the register split (setmaxnreg) draws on what the block was launched with
    cudaFuncAttributes attr;
    cudaError_t e = cudaFuncGetAttributes(&attr, kern);
    if (e != cudaSuccess) return e;
    if (attr.numRegs * kThreads < 256 * kRegsSoftmax + 128 * kRegsOther) return cudaErrorInvalidConfiguration;
    const size_t smem = (2 + C::kSlots) * C::kTileBytes + sizeof(Control<D>);
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    kern<<<kPromptCtas, kThreads, smem, stream>>>(q_map, k_map, v_map, k_wide, v_wide, a);
    return cudaGetLastError();
}

}  // namespace

size_t prompt_workspace_control_bytes() { return kControlBytes; }
size_t prompt_workspace_bytes(const se_params &p) {
    const size_t slot = ((size_t)kTile * p.D + 2 * kTile) * sizeof(float);
    return kControlBytes + (size_t)kPromptCtas * 4 * slot;
}

cudaError_t launch_prompt_attend(const se_params &p, const AttendCall &c, cudaStream_t stream) {
    return p.D == 128 ? launch_attend<128>(p, c, stream) : launch_attend<64>(p, c, stream);
}

}  // namespace se
