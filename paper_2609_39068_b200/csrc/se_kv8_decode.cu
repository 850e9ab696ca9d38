// Attention of one token per request over an 8-bit paged cache (Appendix A, "Attention over Selected Positions", with K and V
// held as e4m3 codes with a power-of-two scale per page and kv-head): over the pages of a selection, or over all present pages.
//
// Mathematics.  For a page with scales s_K, s_V and codes c:  z_j = sm_scale s_K (q . c_j),  out = sum_j p_j s_V c_j / sum_j p_j,
// p_j = 2^(z_j log2 e - m).  Both products run on codes, as they lie in the cache, on the fifth-generation tensor cores; what is not
// a code is split into several:
//   q          2^-e q = hi + lo, two rows of codes per head (largest magnitude at most 448; exact for everything above 2^-10 of it)
//   p_j s_V    = 2^(w_j - M) with w = z log2 e + log2 s_V and M the running maximum of w, so that the largest weights are near 1
//              whatever the scales; as five codes, r_0 = p, c_i = code(r_i), r_(i+1) = 16 (r_i - c_i): 20 bits below the weight's
//              first, which the fp32 output needs.  Each of the five has a column of its own in the product.
// Tokens are the M side: S (128 tokens x heads) = K (128 x D) q^T, a thread per token; then O (D x 5 heads) = V^T (D x 128) p.
//
// What bounds it: HBM, 2 * 2 * D bytes per token and kv-head.  A tile of 128 tokens is 32 KB at D = 128, 1400 cycles of an SM's
// share of the bandwidth; the products take a few hundred, a thread's exponentials and codes about as many instructions.  (The same
// on mma.sync with codes turned into halves needed 330 instructions per warp and page, and could not go faster than half of the
// bandwidth: 64 requests x 2048 tokens 63 us.)
//
// Split.  A tile is eight pages of a (request, kv-head) pair's list.  The tiles of all pairs are cut into 148 runs of equal
// length, one per CTA.  Four warps look the pages up (selection, page and scale a block of 32 apart) and fetch K and V, one splits q
// a pair ahead, two issue the products, two warpgroups take every second tile each.  At the end of a pair each puts its
// sums aside and goes on; they take turns in merging them.  A pair that several CTAs share leaves partial results in the
// workspace, and the CTA that arrives last merges them in order: equal inputs give equal bits.
#include <math.h>

#include "se_internal.h"
#include "se_kv8.cuh"
#include "se_pieces.cuh"

namespace se {

namespace {

constexpr int kThreads = 480;          // two warpgroups, then a warp each
constexpr int kScoreWarp = 8, kOutWarp = 9, kQueryWarp = 10, kFetchWarp = 11, kFetchers = 2;   // (and two each for K and V)
constexpr int kTile = 128, kGroups = kTile / kPage;
constexpr int kChunks = 1024;          // prefix sums that a CTA keeps: of every pair, or of runs of pairs
constexpr int kParts = 5;              // codes of a weight
constexpr float kSlack = 8.f;          // the running maximum may lag: weights up to 2^8 are below the largest code
constexpr int kQueries = 4;            // pairs whose q is kept

template <int D>
struct Cfg {
    static constexpr int kPageBytes = kPage * D, kTileBytes = kTile * D;      // of K or of V, one head
    static constexpr int kKStages = D == 128 ? 4 : 6, kVStages = D == 128 ? 6 : 10;
    static constexpr int kWeightBytes = kTile * 64;                           // a token's codes: up to 48 of 64 bytes
    static constexpr int kQueryBytes = 16 * D;                                // eight rows of hi, eight of lo
    static constexpr int kPartFloats = 8 * D + 16;                            // a partial result: O, M, l
    static constexpr int kVAt = kKStages * kTileBytes, kRing = kVAt + kVStages * kTileBytes;
    static constexpr int kQueryAt = kRing + 2 * kWeightBytes;
    static constexpr int kAsideAt = kQueryAt + kQueries * kQueryBytes;
    static constexpr int kControlAt = kAsideAt + 4 * kPartFloats * 4;         // [pair's parity][warpgroup]
};
static_assert(kThreads == 32 * (kFetchWarp + 2 * kFetchers), "a warp for each role");
static_assert(Cfg<128>::kQueryAt % 1024 == 0 && Cfg<64>::kQueryAt % 1024 == 0 && Cfg<128>::kControlAt % 16 == 0 && Cfg<64>::kControlAt % 16 == 0 &&
              Cfg<128>::kQueryBytes % 1024 == 0 && Cfg<64>::kQueryBytes % 1024 == 0, "operands and 16-byte accesses");

struct PageInfo {
    float k_scale, v_scale;
    int tokens, pad;                   // below the request's length; 0: absent
};

template <int D>
struct Control {
    PageInfo info[Cfg<D>::kVStages][kGroups];
    float power[kQueries][8];          // of each head: logit in powers of two = sum * power * s_K
    float top[2][2][4][8];             // largest w of a tile: [warpgroup][tile's parity][warp][head]
    float sum[2][4][8];                // sums of a pair's weights: [warpgroup][warp][head]
    uint64_t k_full[Cfg<D>::kKStages], k_empty[Cfg<D>::kKStages], v_full[Cfg<D>::kVStages], v_empty[Cfg<D>::kVStages], q_ready[kQueries], q_free[kQueries];
    uint64_t s_full[2][2], s_free[2][2], p_ready[2], o_done[2], exchange[2], aside[2], merged[2], drain[2];
    long long pre[kChunks + 1];
    long long sums[kThreads / 32];
    uint32_t tmem;
    int verdict, gave_up;
};

struct Args {
    const uint16_t *q;
    const float2 *scales;
    const int32_t *page_table, *seq_lens, *sel_idx, *sel_cnt;
    float *out, *lse, *partials;
    PromptControl *ctl;
    int B, H_q, H_kv, G, max_pages, P_phys, k_max;
    float scale_log2;
};

__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t addr, float *v) {
    __syncwarp();
    uint32_t *r = reinterpret_cast<uint32_t *>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const float *v) {
    __syncwarp();
    const uint32_t *r = reinterpret_cast<const uint32_t *>(v);
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr), "r"(r[0]),
                 "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
                 "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}
// e4m3 operand whose M or N runs along rows of `width` bytes (64 or 128; the swizzle as wide): K-neighbours are rows, atoms of 8 rows
__device__ __forceinline__ uint64_t smem_codes_mn(uint32_t addr, int width) {
    return (uint64_t)((addr & 0x3ffffu) >> 4) | (uint64_t)(16 >> 4) << 16 | (uint64_t)((8 * width) >> 4) << 32 | 1ull << 46 |
           (width == 128 ? 2ull : 4ull) << 61;
}

// ---- the list of tiles: pairs (request, kv-head) in order, each with its pages in eights ---------
struct Pairs {
    const Args &a;
    const long long *pre;              // shared: tiles before each chunk of `per` pairs, [chunks + 1]
    int per, chunks;

    __device__ __forceinline__ int pages(int pair) const {
        if (a.sel_cnt) return min(max(a.sel_cnt[pair], 0), a.k_max);
        const int len = a.seq_lens[pair / a.H_kv];
        return len < 0 || len > a.max_pages * kPage ? 0 : (len + kPage - 1) / kPage;
    }
    __device__ __forceinline__ int count(int pair) const { return (pages(pair) + kGroups - 1) / kGroups; }
    // the pair that holds tile u of the list, and its first tile
    __device__ __forceinline__ int find(long long u, long long &first) const {
        int lo = 0, hi = chunks;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (pre[mid] <= u) lo = mid; else hi = mid;
        }
        first = pre[lo];
        int x = lo * per;
        if (per > 1)
            for (int n = count(x); first + n <= u; n = count(++x)) first += n;
        return x;
    }
    __device__ __forceinline__ int count_known(int pair) const { return per > 1 ? count(pair) : (int)(pre[pair + 1] - pre[pair]); }
};

// A role's way through the pairs of its CTA's run: tiles begin .. end - 1 of the run belong to `pair`.
struct Walk {
    const Pairs &ps;
    long long u0, first;
    int n, pair, begin, end, ordinal;

    __device__ __forceinline__ Walk(const Pairs &ps, long long u0, int n) : ps(ps), u0(u0), n(n), begin(0), ordinal(0) {
        pair = ps.find(u0, first);
        end = (int)min((long long)n, first + ps.count_known(pair) - u0);
    }
    __device__ __forceinline__ bool next() {
        if (end == n) return false;
        first += ps.count_known(pair);
        while (ps.count_known(++pair) == 0) {}
        begin = end, ++ordinal;
        end = (int)min((long long)n, first + ps.count_known(pair) - u0);
        return true;
    }
};

// ---- pages ---------------------------------------------------------------------------
// What a lane of a fetching warp knows of a page, found in three steps that lie a block of 32 pages (four tiles) apart.
struct Found {
    int r, h, j, count, b, len;        // 1: request (-1: behind the run), head, place in the pair's list, entries of the list, logical page, length
    int row, tokens;                   // 2, 3: page * H_kv + head, -1: not present; tokens below the length
    float2 scale;                      // 3
};
// A lane's way through the pairs: tiles come in ascending order.
struct Cursor {
    int pair, count, r, h;
    long long first;

    __device__ __forceinline__ Cursor(const Args &a, const Pairs &ps, long long u) {
        pair = ps.find(u, first), count = ps.count_known(pair);
        r = pair / a.H_kv, h = pair - r * a.H_kv;
    }
    __device__ __forceinline__ void find_page(const Args &a, const Pairs &ps, long long u0, int n, int i, Found &f) {
        f.r = -1;
        if (i / kGroups >= n) return;
        while (u0 + i / kGroups >= first + count) {
            first += count, count = ps.count_known(++pair);
            if (++h == a.H_kv) h = 0, ++r;
        }
        f.r = r, f.h = h;
        f.j = (int)(u0 + i / kGroups - first) * kGroups + i % kGroups;
        f.len = a.seq_lens[r];
        // (nothing that is loaded here is used here)
        f.count = a.sel_cnt ? a.sel_cnt[pair] : 0;
        f.b = a.sel_idx ? a.sel_idx[(size_t)pair * a.k_max + min(f.j, a.k_max - 1)] : f.j;
    }
};
__device__ __forceinline__ void find_row(const Args &a, Found &f) {
    f.row = -1, f.tokens = 0;
    if (f.r < 0 || f.j >= (a.sel_cnt ? min(f.count, a.k_max) : (f.len + kPage - 1) / kPage)) return;
    if (f.b < 0 || f.b >= a.max_pages || f.b * kPage >= f.len) {           // (only a selection can be wrong here)
        atomicOr(&a.ctl->status, SE_DEV_BAD_SELECTION);
        return;
    }
    f.row = a.page_table[(size_t)f.r * a.max_pages + f.b];
    f.tokens = min(kPage, f.len - f.b * kPage);
}
template <bool OF_V>
__device__ __forceinline__ void find_scale(const Args &a, Found &f) {
    if (f.row >= a.P_phys) {
        if (OF_V) atomicOr(&a.ctl->status, SE_DEV_BAD_PAGE_ID);
        f.row = -1;
    }
    f.scale = make_float2(1.f, 1.f);
    if (f.row < 0) return;
    f.row = f.row * a.H_kv + f.h;
    if (OF_V) f.scale = a.scales[f.row];
}

// Two warps bring K, two V and what is to be known of the pages, each every second tile.  (One alone took 1550 cycles a tile, half of
// them for loads that a block ahead was not far enough for.)  The rings have even numbers of slots, so a slot belongs to one warp,
// which waits for it in every phase; a warpgroup's tiles are those of one V warp.
template <int D, bool OF_V>
__device__ __forceinline__ void fetch_role(const Args &a, const Pairs &ps, const CUtensorMap *map, Control<D> *ctl, uint32_t ring, long long u0, int n, int which,
                                           int lane) {
    using C = Cfg<D>;
    constexpr int kStages = OF_V ? C::kVStages : C::kKStages, kBlock = 32 / kGroups;
    static_assert(kFetchers == 2 && kStages % kFetchers == 0, "slots of a warp's own");
    volatile int *gave_up = &ctl->gave_up;
    const uint32_t full = smem_u32(OF_V ? ctl->v_full : ctl->k_full), empty = smem_u32(OF_V ? ctl->v_empty : ctl->k_empty);
    const bool chosen = elect_one();
    if (which >= n) return;
    Found now, next, later, last;
    // the lane's page of the warp's block b: place in the run's list
    auto place = [&](int b) { return ((b * kBlock + lane / kGroups) * kFetchers + which) * kGroups + lane % kGroups; };
    Cursor at_lane(a, ps, u0 + min(place(0) / kGroups, n - 1));
    at_lane.find_page(a, ps, u0, n, place(0), now);
    find_row(a, now);
    find_scale<OF_V>(a, now);
    bool ok = true;
    int i = which, m = 0;              // tile, and the warp's own count
    for (; i < n; i += kFetchers, ++m) {
        const int at = m % kBlock * kGroups;                               // the tile's pages are lanes at .. at + 7
        if (at == 0 && m) now = next, next = later, later = last;
        int row[kGroups];
#pragma unroll
        for (int pg = 0; pg < kGroups; ++pg) row[pg] = __shfl_sync(kFull, now.row, at + pg);
        const uint32_t slot = i % kStages, bar = full + 8 * slot, dst = ring + slot * C::kTileBytes;
        ok = warp_wait(empty + 8 * slot, (i / kStages & 1) ^ 1, gave_up, &a.ctl->status);
        if (!ok) break;
        if (OF_V) {
            if (lane >= at && lane < at + kGroups)
                ctl->info[slot][lane - at] = PageInfo{now.scale.x, now.scale.y, now.row >= 0 ? now.tokens : 0, 0};
            __syncwarp();
        }
        if (chosen) {
            mbar_expect_tx(bar, C::kTileBytes + (OF_V && i == 0 ? kTestExtraTx : 0));
#pragma unroll
            for (int pg = 0; pg < kGroups; ++pg)                           // absent: from behind the last row, zeros
                tma_load_2d(dst + pg * C::kPageBytes, map, 0, (row[pg] < 0 ? a.P_phys * a.H_kv : row[pg]) * kPage, bar);
        }
        __syncwarp();
        if (at == 0) {                 // what comes later is looked up behind the copies
            const int b = m / kBlock;
            if (b == 0) {
                at_lane.find_page(a, ps, u0, n, place(1), next), at_lane.find_page(a, ps, u0, n, place(2), later);
                find_row(a, next);
            }
            at_lane.find_page(a, ps, u0, n, place(b + 3), last);
            find_row(a, later);
            find_scale<OF_V>(a, next);
        }
    }
    // nothing may still be on its way to the CTA's shared memory, or arrive there, when the CTA ends
    for (int e = max(i - kStages, which); e < i; e += kFetchers) {
        ok = ok && warp_wait(empty + 8 * (e % kStages), e / kStages & 1, gave_up, &a.ctl->status);
        if (!ok) mbar_wait(full + 8 * (e % kStages), e / kStages & 1);
    }
}

// ---- q of a pair as codes, a pair ahead: lane (g, t) takes head g, channels 64 i + 16 t .. + 15 -------
template <int D>
__device__ __forceinline__ void query_role(const Args &a, const Pairs &ps, Control<D> *ctl, uint32_t q_at, long long u0, int n, int lane) {
    using C = Cfg<D>;
    volatile int *gave_up = &ctl->gave_up;
    const int g = lane >> 2, t = lane & 3;
    Walk w(ps, u0, n);
    do {
        const int place = w.ordinal % kQueries;
        const int r = w.pair / a.H_kv, h = w.pair - r * a.H_kv;
        uint4 raw[D / 32];
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
            const uint4 *src = reinterpret_cast<const uint4 *>(a.q + ((size_t)r * a.H_q + h * a.G + min(g, a.G - 1)) * D + 64 * i + 16 * t);
            raw[2 * i] = src[0], raw[2 * i + 1] = src[1];
        }
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) top = bmax2(top, largest8(raw[i]));
        top = max(top & 0xffffu, top >> 16);
        top = max(top, __shfl_xor_sync(kFull, top, 1));
        top = max(top, __shfl_xor_sync(kFull, top, 2));
        const int e = min(max((int)(top >> 7) - 135 + ((top & 127u) > 96u ? 1 : 0), -60), 110);    // least 2^e with the maximum at most 448 * 2^e
        const float down = g < a.G ? __uint_as_float((uint32_t)(127 - e) << 23) : 0.f;
        if (!warp_wait(smem_u32(&ctl->q_free[place]), (w.ordinal / kQueries & 1) ^ 1, gave_up, &a.ctl->status)) return;
#pragma unroll
        for (int i = 0; i < D / 64; ++i) {
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint4 &s = raw[2 * i + j / 2];
                const uint32_t x[2] = {j % 2 ? s.z : s.x, j % 2 ? s.w : s.y};
                uint32_t c[2], d[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float2 v = bf16x2_to_f2(x[k]);
                    v.x *= down, v.y *= down;
                    c[k] = e4m3x2(v.x, v.y);
                    const float2 back = float2_of_e4m3x2(c[k]);
                    d[k] = e4m3x2(v.x - back.x, v.y - back.y);
                }
                hi[j] = c[0] | c[1] << 16, lo[j] = d[0] | d[1] << 16;
            }
            const int chunk = t + 4 * i;
            const uint32_t at = q_at + place * C::kQueryBytes + g * D + ((D == 128 ? chunk ^ g : chunk ^ (g >> 1 & 3)) << 4);
            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(hi[0]), "r"(hi[1]), "r"(hi[2]), "r"(hi[3]) : "memory");
            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at + 8 * D), "r"(lo[0]), "r"(lo[1]), "r"(lo[2]), "r"(lo[3]) : "memory");
        }
        if (t == 0) ctl->power[place][g] = __uint_as_float((uint32_t)(127 + e) << 23) * a.scale_log2;
        fence_async_proxy();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ctl->q_ready[place]));
    } while (w.next());
    // (the products' arrivals for the last pairs)
    for (int o = max(w.ordinal + 1 - kQueries, 0); o <= w.ordinal; ++o)
        if (!warp_wait(smem_u32(&ctl->q_free[o % kQueries]), o / kQueries & 1, gave_up, &a.ctl->status)) return;
}

// ---- products --------------------------------------------------------------------------
// Tile i belongs to warpgroup i % 2, whose scores (of two tiles) and output have tensor memory of their own: S at columns 32 w and
// 32 w + 16, O at 64 + 64 w.  Scores are made up to four tiles ahead, so that a warpgroup finds those of its next tile ready.  (A
// barrier tells its phases apart by parity alone: each is waited for in every phase, or has one open phase at most.)
// A warp for each of the two products: with one for both, a tile took it 1100 cycles of issuing and waiting in order.
template <int D>
__device__ __forceinline__ void score_role(const Args &a, const Pairs &ps, Control<D> *ctl, uint32_t base, long long u0, int n, int lane) {
    using C = Cfg<D>;
    volatile int *gave_up = &ctl->gave_up;
    const uint32_t tmem = ctl->tmem;
    const bool chosen = elect_one();
    auto wait = [&](const uint64_t *bar, uint32_t parity) { return warp_wait(smem_u32(bar), parity & 1, gave_up, &a.ctl->status); };
    Walk w(ps, u0, n);
    bool fresh = true;                 // the pair has just begun
    for (int i = 0; i < n; ++i) {
        const int place = w.ordinal % kQueries;
        if (fresh && !wait(&ctl->q_ready[place], w.ordinal / kQueries)) break;
        if (!wait(&ctl->k_full[i % C::kKStages], i / C::kKStages)) break;
        if (i >= 4 && !wait(&ctl->s_free[i & 1][i >> 1 & 1], i / 4 - 1)) break;                 // the scores that lay there have been read
        tc_fence_after();
        const bool ends = i + 1 == w.end;
        if (chosen) {
            const uint64_t kd = smem_codes<D>(base + i % C::kKStages * C::kTileBytes);
            const uint64_t qd = smem_codes<D>(base + C::kQueryAt + place * C::kQueryBytes);
            const uint32_t to = tmem + (i & 1) * 32 + (i >> 1 & 1) * 16;
#pragma unroll
            for (int k = 0; k < D / 32; ++k) mma_ss_codes(to, kd + k * 2, qd + k * 2, mma_instr_codes(16), k > 0);
            mma_commit(smem_u32(&ctl->s_full[i & 1][i >> 1 & 1]));
            mma_commit(smem_u32(&ctl->k_empty[i % C::kKStages]));
            if (ends) mma_commit(smem_u32(&ctl->q_free[place]));
        }
        __syncwarp();
        fresh = ends && w.next();
    }
    // nothing may be running when tensor memory goes away
    if (chosen) mma_commit(smem_u32(&ctl->drain[0]));
    __syncwarp();
    mbar_wait(smem_u32(&ctl->drain[0]), 0);
}

template <int D>
__device__ __forceinline__ void out_role(const Args &a, const Pairs &ps, Control<D> *ctl, uint32_t base, long long u0, int n, int lane) {
    using C = Cfg<D>;
    constexpr int kWidth = 64;         // bytes of a token's row of weights
    volatile int *gave_up = &ctl->gave_up;
    const uint32_t tmem = ctl->tmem;
    const bool chosen = elect_one();
    const int columns = a.G > 4 ? 48 : 32;
    const uint32_t instr = 1u << 4 | 1u << 15 | 1u << 16 | (uint32_t)(columns >> 3) << 17 | (uint32_t)(D >> 4) << 24;     // A and B run along M and N
    auto wait = [&](const uint64_t *bar, uint32_t parity) { return warp_wait(smem_u32(bar), parity & 1, gave_up, &a.ctl->status); };
    Walk w(ps, u0, n);
    for (int i = 0; i < n; ++i) {
        if (!wait(&ctl->v_full[i % C::kVStages], i / C::kVStages) || !wait(&ctl->p_ready[i & 1], i / 2)) break;
        tc_fence_after();
        if (chosen) {
            const uint64_t vd = smem_codes_mn(base + C::kVAt + i % C::kVStages * C::kTileBytes, D);
            const uint64_t pd = smem_codes_mn(base + C::kRing + (i & 1) * C::kWeightBytes, kWidth);
            const bool first = i < w.begin + 2;                            // the pair's first tile of this warpgroup
#pragma unroll
            for (int k = 0; k < kTile / 32; ++k)
                mma_ss_codes(tmem + 64 + (i & 1) * 64, vd + k * (32 * D >> 4), pd + k * (32 * kWidth >> 4), instr, !first || k > 0);
            mma_commit(smem_u32(&ctl->o_done[i & 1]));
            mma_commit(smem_u32(&ctl->v_empty[i % C::kVStages]));
        }
        __syncwarp();
        if (i + 1 == w.end) w.next();
    }
    if (chosen) mma_commit(smem_u32(&ctl->drain[1]));
    __syncwarp();
    mbar_wait(smem_u32(&ctl->drain[1]), 0);
}

// ---- softmax ------------------------------------------------------------------------------
// Merges the parts of a pair that the runs c0 .. c1 have left, in their order; the whole CTA.
template <int D>
__device__ __noinline__ void merge_parts(const Args &a, int pair, int c0, int c1) {
    using C = Cfg<D>;
    const size_t row0 = (size_t)(pair / a.H_kv) * a.H_q + pair % a.H_kv * a.G;
    for (int e = threadIdx.x; e < a.G * (D / 4); e += kThreads) {
        const int head = e / (D / 4), ch = e % (D / 4) * 4;
        float M = -INFINITY, L = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int x = c0; x <= c1; ++x) {
            const float *src = a.partials + (size_t)(x * 2 + (x == c0 ? 1 : 0)) * C::kPartFloats;
            const float mx = __ldcg(src + 8 * D + head), lx = __ldcg(src + 8 * D + 8 + head);
            const float4 v = __ldcg(reinterpret_cast<const float4 *>(src + head * D + ch));
            const float top = fmaxf(M, mx), ref = top == -INFINITY ? 0.f : top;
            const float fo = ex2(M - ref), fx = ex2(mx - ref);
            M = top, L = L * fo + lx * fx;
            o.x = o.x * fo + v.x * fx, o.y = o.y * fo + v.y * fx, o.z = o.z * fo + v.z * fx, o.w = o.w * fo + v.w * fx;
        }
        const float inv = L == 0.f ? 0.f : 1.f / L;
        *reinterpret_cast<float4 *>(a.out + (row0 + head) * D + ch) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
        if (ch == 0) a.lse[row0 + head] = L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
    }
}

// H: heads that the code is laid out for, 4 or 8 (a.G of them are real).
template <int D, int H>
__device__ __forceinline__ void softmax_role(const Args &a, const Pairs &ps, Control<D> *ctl, uint8_t *smem, uint32_t base, long long u0, int n, long long size,
                                             int st) {
    using C = Cfg<D>;
    constexpr int kColumns = H > 4 ? 48 : 32;
    volatile int *gave_up = &ctl->gave_up;
    const int row = threadIdx.x & 127, lane = threadIdx.x & 31, warp = row >> 5;
    const uint32_t lanes = (uint32_t)(warp * 32) << 16;
    const uint32_t t_s = ctl->tmem + lanes + st * 32, t_o = ctl->tmem + lanes + 64 + st * 64;
    const uint32_t weights = base + C::kRing + st * C::kWeightBytes + row * 64, swizzle = (uint32_t)(row >> 1 & 3) << 4;
    auto wait = [&](const uint64_t *bar, uint32_t parity) { return warp_wait(smem_u32(bar), parity & 1, gave_up, &a.ctl->status); };
    int exchanges = 0;
    // the warps of the group have come here
    auto group_sync = [&] {
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ctl->exchange[st]));
        return wait(&ctl->exchange[st], exchanges++);
    };
    // output channel of the thread in tensor memory (64 rows lie in the lower halves of the four warps' lanes)
    const int ch = D == 128 ? row : warp * 16 + lane;
    const bool has_ch = D == 128 || lane < 16;
    Walk w(ps, u0, n);
    int i = st;                        // next tile of the group
    do {
        float f[H], M[H], l[H];
#pragma unroll
        for (int h = 0; h < H; ++h) M[h] = -INFINITY, l[h] = 0.f;
        bool any = false;
        for (; i < w.end; i += 2) {
            const uint32_t k = i / 2, slot = i % C::kVStages;
            if (!wait(&ctl->v_full[slot], i / C::kVStages) || !wait(&ctl->s_full[st][k & 1], k / 2)) return;
            tc_fence_after();
            float z[16];
            tmem_ld16(t_s + (k & 1) * 16, z);
            const PageInfo info = ctl->info[slot][row / kPage];
            if (!any) {
#pragma unroll
                for (int h = 0; h < H; ++h) f[h] = *(volatile float *)&ctl->power[w.ordinal % kQueries][h];
            }
            tmem_wait_ld();
            settle<16>(z);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&ctl->s_free[st][k & 1]));
            // w = logit + log2 of V's scale, in powers of two; largest of the tile
            const bool seen = row % kPage < info.tokens;
            const float shift = (float)((int)(__float_as_uint(info.v_scale) >> 23) - 127);
            // what lies behind the end of the request may be anything, and a weight of zero would not hide it
            if (!seen && info.tokens > 0) {
#pragma unroll
                for (int e = 0; e < D / 16; ++e)
                    asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(base + C::kVAt + slot * C::kTileBytes + row * D + e * 16), "r"(0) : "memory");
            }
            __syncwarp();
            float tile_top[H];
#pragma unroll
            for (int h = 0; h < H; ++h) {
                z[h] = seen ? fmaf(z[h] + z[8 + h], f[h] * info.k_scale, shift) : -INFINITY;     // hi and lo
                float x = z[h];
#pragma unroll
                for (int o = 16; o; o >>= 1) x = fmaxf(x, __shfl_xor_sync(kFull, x, o));
                tile_top[h] = x;
            }
            float *top = &ctl->top[st][k & 1][warp][0];
            if (lane == 0) {
#pragma unroll
                for (int h = 0; h < H; ++h) top[h] = tile_top[h];
            }
            if (!group_sync()) return;
            bool grown = false;
#pragma unroll
            for (int h = 0; h < H; ++h) {
#pragma unroll
                for (int x = 0; x < 4; ++x) tile_top[h] = fmaxf(tile_top[h], *(volatile float *)&ctl->top[st][k & 1][x][h]);
                grown = grown || tile_top[h] > M[h] + kSlack;
            }
            // the group's last product is done: its weights and its output may be written
            if (k > 0 && !wait(&ctl->o_done[st], k - 1)) return;
            if (grown) {                                                   // (the same for all threads of the group)
                float by[H];
#pragma unroll
                for (int h = 0; h < H; ++h) {
                    const float m = fmaxf(M[h], tile_top[h]);
                    by[h] = M[h] == -INFINITY ? 0.f : ex2(M[h] - m);
                    M[h] = m, l[h] *= by[h];
                }
                if (any) {
                    tc_fence_after();
#pragma unroll
                    for (int c = 0; c < kColumns; c += 16) {
                        float o[16];
                        tmem_ld16(t_o + c, o);
                        tmem_wait_ld();
                        settle<16>(o);
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] *= by[(c + e) % H];
                        tmem_st16(t_o + c, o);
                    }
                    tmem_wait_st();
                }
            }
            any = true;
            // weights as codes
            const float inv = __uint_as_float(0x7f000000u - __float_as_uint(info.v_scale));
            uint32_t code[kParts][H / 4];
#pragma unroll
            for (int h = 0; h < H; h += 2) {
                float r0 = M[h] == -INFINITY ? 0.f : ex2(z[h] - M[h]), r1 = M[h + 1] == -INFINITY ? 0.f : ex2(z[h + 1] - M[h + 1]);
                l[h] = fmaf(r0, inv, l[h]), l[h + 1] = fmaf(r1, inv, l[h + 1]);
#pragma unroll
                for (int part = 0; part < kParts; ++part) {
                    const uint32_t c = e4m3x2(r0, r1);
                    if (h % 4 == 0) code[part][h / 4] = c;
                    else code[part][h / 4] |= c << 16;
                    const float2 back = float2_of_e4m3x2(c);
                    r0 = fmaf(-16.f, back.x, 16.f * r0), r1 = fmaf(-16.f, back.y, 16.f * r1);
                }
            }
            // the token's row: part after part, the heads of each side by side
            uint32_t words[kColumns / 4];
#pragma unroll
            for (int e = 0; e < kColumns / 4; ++e) words[e] = e < kParts * (H / 4) ? code[e / (H / 4)][e % (H / 4)] : 0u;
#pragma unroll
            for (int c = 0; c < kColumns / 16; ++c)
                asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(weights + ((c << 4) ^ swizzle)), "r"(words[4 * c]), "r"(words[4 * c + 1]),
                             "r"(words[4 * c + 2]), "r"(words[4 * c + 3])
                             : "memory");
            fence_async_proxy();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&ctl->p_ready[st]));
            __syncwarp();
        }

        // ---- the pair's sums aside ----
        const int side = w.ordinal & 1;
        if (w.ordinal > 1 && !wait(&ctl->merged[side], w.ordinal / 2 - 1)) return;
        float *own = reinterpret_cast<float *>(smem + C::kAsideAt) + (side * 2 + st) * C::kPartFloats;
        if (any) {
#pragma unroll
            for (int h = 0; h < H; ++h) {
#pragma unroll
                for (int o = 16; o; o >>= 1) l[h] += __shfl_xor_sync(kFull, l[h], o);
                if (lane == 0) ctl->sum[st][warp][h] = l[h];
            }
            if (!group_sync() || !wait(&ctl->o_done[st], (i - 2) / 2)) return;
            tc_fence_after();
            float o[kColumns];
#pragma unroll
            for (int c = 0; c < kColumns; c += 16) tmem_ld16(t_o + c, o + c);
            tmem_wait_ld();
            settle<kColumns>(o);
            tc_fence_before();
            if (has_ch) {
#pragma unroll
                for (int h = 0; h < H; ++h) {
                    float v = o[(kParts - 1) * H + h];
#pragma unroll
                    for (int part = kParts - 2; part >= 0; --part) v = fmaf(v, 0.0625f, o[part * H + h]);
                    own[h * D + ch] = v;
                }
            }
            if (row < H) {
                float sum = 0.f;
#pragma unroll
                for (int x = 0; x < 4; ++x) sum += *(volatile float *)&ctl->sum[st][x][row];
                own[8 * D + 8 + row] = sum;
            }
        }
#pragma unroll
        for (int h = 0; h < H; ++h)
            if (row == h) own[8 * D + h] = any ? M[h] : -INFINITY;
        __syncwarp();
        if (lane == 0) {
            mbar_arrive(smem_u32(&ctl->aside[side]));
            mbar_arrive(smem_u32(&ctl->q_free[w.ordinal % kQueries]));     // (`power` has been read)
        }
        __syncwarp();
        if (side == st) {              // the groups take turns in merging
            if (!wait(&ctl->aside[side], w.ordinal / 2)) return;
            const float *both = reinterpret_cast<const float *>(smem + C::kAsideAt) + side * 2 * C::kPartFloats;
            const int pages = ps.count_known(w.pair), run = blockIdx.x;
            const int c0 = (int)(w.first / size), c1 = (int)((w.first + pages - 1) / size);        // runs that share the pair
            const size_t row0 = (size_t)(w.pair / a.H_kv) * a.H_q + w.pair % a.H_kv * a.G;
            float *part = a.partials + (size_t)(run * 2 + (c0 == run ? 1 : 0)) * C::kPartFloats;
            for (int e = row; e < a.G * D; e += 128) {
                const int h = e / D, c = e - h * D;
                const float ma = both[8 * D + h], mb = both[C::kPartFloats + 8 * D + h];
                const float top = fmaxf(ma, mb), ref = top == -INFINITY ? 0.f : top;
                const float fa = ex2(ma - ref), fb = ex2(mb - ref);
                // (a group without a tile of the pair has put nothing but -infinity)
                const float la = ma == -INFINITY ? 0.f : fa * both[8 * D + 8 + h], lb = mb == -INFINITY ? 0.f : fb * both[C::kPartFloats + 8 * D + 8 + h];
                const float oa = ma == -INFINITY ? 0.f : fa * both[h * D + c], ob = mb == -INFINITY ? 0.f : fb * both[C::kPartFloats + h * D + c];
                const float L = la + lb, o = oa + ob;
                if (c0 == c1) {
                    a.out[(row0 + h) * D + c] = L == 0.f ? 0.f : o / L;
                    if (c == 0) a.lse[row0 + h] = L == 0.f ? -INFINITY : (top + log2f(L)) * kLn2;
                } else {
                    part[h * D + c] = o;
                    if (c == 0) part[8 * D + h] = top, part[8 * D + 8 + h] = L;
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&ctl->merged[side]));
            __syncwarp();
        }
    } while (w.next());
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
kv8_decode_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const __grid_constant__ Args a) {
    using C = Cfg<D>;
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t base = smem_u32(smem);
    Control<D> *ctl = reinterpret_cast<Control<D> *>(smem + C::kControlAt);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    if ((base & 1023u) || *(volatile uint32_t *)&a.ctl->needs_init) {                   // the swizzle pattern hangs on the address
        if (tid == 0 && blockIdx.x == 0) atomicOr(&a.ctl->status, SE_DEV_WAIT_TIMEOUT);
        return;
    }
    if (tid < C::kKStages) mbar_init(smem_u32(&ctl->k_full[tid]), 1), mbar_init(smem_u32(&ctl->k_empty[tid]), 1);
    if (tid < C::kVStages) mbar_init(smem_u32(&ctl->v_full[tid]), 1), mbar_init(smem_u32(&ctl->v_empty[tid]), 1);
    if (tid < kQueries) mbar_init(smem_u32(&ctl->q_ready[tid]), 1), mbar_init(smem_u32(&ctl->q_free[tid]), 9);
    if (tid < 2) {
        mbar_init(smem_u32(&ctl->s_full[tid][0]), 1), mbar_init(smem_u32(&ctl->s_full[tid][1]), 1), mbar_init(smem_u32(&ctl->o_done[tid]), 1);
        mbar_init(smem_u32(&ctl->s_free[tid][0]), 4), mbar_init(smem_u32(&ctl->s_free[tid][1]), 4);
        mbar_init(smem_u32(&ctl->p_ready[tid]), 4), mbar_init(smem_u32(&ctl->exchange[tid]), 4), mbar_init(smem_u32(&ctl->merged[tid]), 4);
        mbar_init(smem_u32(&ctl->aside[tid]), 8);
    }
    if (tid == 0) {
        ctl->gave_up = 0;
        mbar_init(smem_u32(&ctl->drain[0]), 1), mbar_init(smem_u32(&ctl->drain[1]), 1);
        prefetch_map(&k_map), prefetch_map(&v_map);
    }
    mbar_fence_init();
    if (warp == kScoreWarp) tmem_alloc(smem_u32(&ctl->tmem), 256);

    // tiles before every pair (or every run of pairs, where there are more than 1024)
    const int pairs = a.B * a.H_kv;
    Pairs ps = {a, ctl->pre, (pairs + kChunks - 1) / kChunks, 0};
    ps.chunks = (pairs + ps.per - 1) / ps.per;
    {
        const int each = (ps.chunks + kThreads - 1) / kThreads;
        const int c0 = min(tid * each, ps.chunks), c1 = min(c0 + each, ps.chunks);
        long long sum = 0;
        for (int c = c0; c < c1; ++c) {
            ctl->pre[c] = sum;
            for (int x = c * ps.per; x < min((c + 1) * ps.per, pairs); ++x) {
                if (blockIdx.x == 0) {
                    const int len = a.seq_lens[x / a.H_kv];
                    if (len < 0 || len > a.max_pages * kPage) atomicOr(&a.ctl->status, SE_DEV_BAD_LENGTH);
                    if (a.sel_cnt && (a.sel_cnt[x] < 0 || a.sel_cnt[x] > a.k_max)) atomicOr(&a.ctl->status, SE_DEV_BAD_SELECTION);
                }
                sum += ps.count(x);
            }
        }
        long long inc = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long x = __shfl_up_sync(kFull, inc, o);
            if (lane >= o) inc += x;
        }
        if (lane == 31) ctl->sums[warp] = inc;
        __syncthreads();
        long long before = inc - sum;
        for (int w = 0; w < warp; ++w) before += ctl->sums[w];
        for (int c = c0; c < c1; ++c) ctl->pre[c] += before;
        if (tid == kThreads - 1) ctl->pre[ps.chunks] = before + sum;
    }
    fence_async_proxy();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const long long total = ctl->pre[ps.chunks];
    const long long size = (total + gridDim.x - 1) / gridDim.x;
    const long long u0 = size * blockIdx.x;
    const int n = (int)min(size, max(total - u0, 0ll));
    if (n) {
        if (warp >= kFetchWarp + kFetchers) fetch_role<D, true>(a, ps, &v_map, ctl, base + C::kVAt, u0, n, warp - kFetchWarp - kFetchers, lane);
        else if (warp >= kFetchWarp) fetch_role<D, false>(a, ps, &k_map, ctl, base, u0, n, warp - kFetchWarp, lane);
        else if (warp == kQueryWarp) query_role<D>(a, ps, ctl, base + C::kQueryAt, u0, n, lane);
        else if (warp == kScoreWarp) score_role<D>(a, ps, ctl, base, u0, n, lane);
        else if (warp == kOutWarp) out_role<D>(a, ps, ctl, base, u0, n, lane);
        else if (a.G > 4) softmax_role<D, 8>(a, ps, ctl, smem, base, u0, n, size, warp >> 2);
        else softmax_role<D, 4>(a, ps, ctl, smem, base, u0, n, size, warp >> 2);
        __syncwarp();
    }
    // pairs without a page
    for (int x0 = (blockIdx.x + warp * gridDim.x) * 32; x0 < pairs; x0 += 32 * (kThreads / 32) * gridDim.x) {
        unsigned none = __ballot_sync(kFull, x0 + lane < pairs && ps.count_known(min(x0 + lane, pairs - 1)) == 0);
        for (; none; none &= none - 1) {
            const int x = x0 + __ffs(none) - 1;
            const size_t row = (size_t)(x / a.H_kv) * a.H_q + x % a.H_kv * a.G;
            for (int e = lane; e < a.G * D; e += 32) a.out[row * D + e] = 0.f;
            if (lane < a.G) a.lse[row + lane] = -INFINITY;
        }
    }
    tc_fence_before();
    __threadfence();
    __syncthreads();
    if (warp == kScoreWarp) {
        tc_fence_after();
        tmem_free(ctl->tmem, 256);
    }
    if (n == 0) return;

    // The run's parts of pairs that other runs share (its first pair, its last) are written: one round of fence and tickets for both.
    long long first, first1;
    const int begun = ps.find(u0, first), ending = ps.find(u0 + n - 1, first1), run = blockIdx.x;
    const int b0 = (int)(first / size), b1 = (int)((first + ps.count_known(begun) - 1) / size);
    const int e0 = (int)(first1 / size), e1 = (int)((first1 + ps.count_known(ending) - 1) / size);
    const bool ask0 = b0 < run, ask1 = e0 == run && e1 > run;              // an earlier run began it; later runs go on with it
    if (!ask0 && !ask1) return;
    if (tid == 0) {
        __threadfence();
        int verdict = 0;
        if (!ctl->gave_up) {           // (a run without all of its parts is not counted)
            if (ask0 && atomicAdd(a.ctl->tickets + b0, 1u) == (uint32_t)(b1 - b0)) atomicExch(a.ctl->tickets + b0, 0u), verdict = 1;
            if (ask1 && atomicAdd(a.ctl->tickets + e0, 1u) == (uint32_t)(e1 - e0)) atomicExch(a.ctl->tickets + e0, 0u), verdict |= 2;
        }
        ctl->verdict = verdict;
        __threadfence();
    }
    __syncthreads();
    const int verdict = ctl->verdict;
    if (verdict & 1) merge_parts<D>(a, begun, b0, b1);
    if (verdict & 2) merge_parts<D>(a, ending, e0, e1);
}

template <int D>
cudaError_t launch(const se_params &p, const Kv8DecodeCall &c, cudaStream_t stream) {
    using C = Cfg<D>;
    CUtensorMap k_map, v_map;
    const long long rows = (long long)p.num_phys_pages * p.H_kv * kPage;
    if (!make_codes_map(&k_map, c.k_cache, D, rows, kPage) || !make_codes_map(&v_map, c.v_cache, D, rows, kPage)) return cudaErrorInvalidValue;
    Args a = {};
    a.q = static_cast<const uint16_t *>(c.q), a.scales = reinterpret_cast<const float2 *>(c.scales);
    a.page_table = c.page_table, a.seq_lens = c.seq_lens, a.sel_idx = c.sel_idx, a.sel_cnt = c.sel_cnt;
    a.out = c.out, a.lse = c.lse, a.partials = partials_of(c.workspace), a.ctl = reinterpret_cast<PromptControl *>(c.workspace);
    a.B = p.B, a.H_q = p.H_q, a.H_kv = p.H_kv, a.G = p.H_q / p.H_kv, a.max_pages = p.max_pages, a.P_phys = p.num_phys_pages;
    a.k_max = p.k_max, a.scale_log2 = effective_scale(p) * kLog2e;
    constexpr size_t kSmem = C::kControlAt + sizeof(Control<D>);
    static_assert(kSmem <= 227 * 1024, "shared memory of a CTA");
    static_assert(2 * C::kPartFloats <= 8 * (128 * D + 256), "partial results of a CTA fit where the prompt kernels keep theirs");
    auto kern = kv8_decode_kernel<D>;
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem);
    if (e != cudaSuccess) return e;
    kern<<<kPromptCtas, kThreads, kSmem, stream>>>(k_map, v_map, a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_kv8_decode(const se_params &p, const Kv8DecodeCall &c, cudaStream_t stream) {
    return p.D == 128 ? launch<128>(p, c, stream) : launch<64>(p, c, stream);
}

}  // namespace se
