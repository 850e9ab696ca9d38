// Attention of one token per request over an 8-bit paged cache (Appendix A, "Attention over Selected Positions", with K and V
// held as e4m3 codes with a power-of-two scale per page and kv-head): over the pages of a selection, or over all present pages.
//
// Mathematics.  For a page with scales s_K, s_V and codes c:  z_j = sm_scale s_K (q . c_j),  out = sum_j p_j s_V c_j / sum_j p_j,
// p_j = 2^(z_j log2 e - m).  The products run on mma.sync with halves, because a code is a half exactly; s_K multiplies the page's
// logits in fp32, s_V becomes a part of the exponent:
//   q     is brought to a maximum of 2^13..2^14 per head by a power of two; its 8 significant bits fit a half for everything
//         above 2^-30 of the maximum, so nothing that fp32 sums could show is lost
//   p s_V = 2^(w - m), w = z log2 e + log2 s_V, m 12 below the running maximum of w, enters as two halves, hi + lo (22 bits), as the
//         output is fp32: the largest are near 2^12 whatever the scales.  The sum of the weights takes s_V out again, in fp32.
//
// What bounds it: the bytes, 2 * D per token and kv-head, come at 0.70 of what a gather of the same pages without arithmetic reaches (43.1 us
// for the first case below), so neither HBM nor the pieces of 2 KB; a page and head takes a warp about 300 instructions at D = 128, 64 of
// them conversions of two codes each and 24 matrix instructions, and an issue slot in two is empty.
//
// Split.  The list of all (request, kv-head) pairs' pages is cut into 592 runs of equal length, one per group of four warps; a
// group's pages go round its warps, each of which keeps a ring of pages in flight (tensor copies, 128-byte swizzle) across the
// borders of pairs.  At the end of a pair's run the warps merge through shared memory; a pair that several groups share leaves
// partial results in the workspace, and the group that arrives last merges them in order.
//
// Measured (device time in graphs): 64 requests x 2048 selected tokens, 8 kv-heads x 4, D = 128: 60.5 us for 271 MB = 4.5 TB/s, 0.68 of a
// copy; 16 requests over 100-32767 tokens, 4 x 7: 55.7 us, 0.63; one request over 2048 tokens 10.3 us,
// one head over 65536 19.7, eight 61-66 over 131000.  On the first, with caches flushed:
// eight warps 91 us, sixteen on their own 77, groups of four 75; one warp that fetches for fifteen 142.  Both products on tcgen05 with
// tokens on the M side and weights as five codes: 65.0 us where this took 63.4 without flushes.
#include <math.h>

#include "se_internal.h"
#include "se_kv8.cuh"
#include "se_pieces.cuh"

namespace se {

namespace {

constexpr int kWarps = 16, kThreads = 32 * kWarps;
constexpr int kTeam = 4, kTeams = kWarps / kTeam;      // warps that share a run of pages, runs of a CTA
constexpr int kLeast = 2 * kTeam;      // pages of a run
constexpr int kChunks = 1024;          // prefix sums that a CTA keeps: of every pair, or of runs of pairs
// The largest weight is 2^12 when the maximum moves, and 2^15 at most until it moves again: the steps of small weights are 2^-36 of the
// largest, and 131072 of them that vanish 2^-20 of it (with the largest at 1 a row lost all tokens 17 below the first one's logit).
constexpr float kLift = 12.f, kTop = 15.f;
// Logits beyond this (in powers of two) are rounded like their maximum was before it is taken off: with one rounding less the largest
// weight would be off by what the maximum was rounded by, which reaches a power of two from 2^23 on and many of them later.
constexpr float kFar = 0x1p22f;
// The tensor cores cut a sum off after each product, always towards zero: sums over 1500 pages of a warp came out 1e-4 too small.  After
// this many pages they join those in the merge buffer, rounded to nearest: 2^-18 at most for two products a page, 5e-7 on average.
constexpr uint32_t kFold = 16;

template <int D>
struct Cfg {
    static constexpr int kPageBytes = kPage * D;                    // of K or of V, one head
    static constexpr int kStages = D == 128 ? 2 : 4;
    static constexpr int kRowsPerPage = kPageBytes / 128;
    static constexpr int kTiles = D / 16;                           // 16-channel tiles of the output
    static constexpr int kPitch = D + 4;                            // floats of a head's row in the merge buffer
    static constexpr int kPartFloats = 8 * D + 16;                  // a partial result: O, m, l
    static constexpr size_t kRing = (size_t)kWarps * kStages * 2 * kPageBytes;
    static constexpr size_t kMerge = (size_t)kWarps * (8 * kPitch + 16) * 4, kQ = (size_t)kTeams * 2 * 8 * D * 2;
    static constexpr size_t kSmem = kRing + kMerge + kQ + (kChunks + 1) * 8 + kWarps * kStages * 8 + 64 * 4;
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

// D(16x8, fp32) += A(16x16, half, row) * B(16x8, half, col)
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the same without an addend
__device__ __forceinline__ void mma_f16_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ uint4 lds128(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t at) {
    uint2 v;
    asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
    return v;
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
__device__ __forceinline__ uint32_t pack_half2(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float2 unpack_half2(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }

// ---- the list of pages: pairs (request, kv-head) in order, each with its pages ---------
struct Pairs {
    const Args &a;
    const long long *pre;              // shared: pages before each chunk of `per` pairs, [chunks + 1]
    int per, chunks;

    __device__ __forceinline__ int pages_of(int r) const {
        const int len = a.seq_lens[r];
        return len < 0 || len > a.max_pages * kPage ? 0 : (len + kPage - 1) / kPage;
    }
    __device__ __forceinline__ int count(int pair) const {
        if (!a.sel_cnt) return pages_of(pair / a.H_kv);
        return min(max(a.sel_cnt[pair], 0), a.k_max);
    }
    // the pair that holds page u of the list, and its first page
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

// what a lane knows of one page of its warp
struct Page {
    int row;                           // page * H_kv + head, -1: not present
    int tokens;                        // below the request's length, 1..16
    float2 scale;
};
__device__ __forceinline__ void team_sync(int team) { asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "n"(32 * kTeam) : "memory"); }
__device__ __forceinline__ Page look_up(const Args &a, const Pairs &ps, long long u0, int n, int i) {
    Page p = {-1, 0, make_float2(0.f, 0.f)};
    if (i >= n) return p;
    long long first;
    const int pair = ps.find(u0 + i, first);
    const int r = pair / a.H_kv, h = pair - r * a.H_kv;
    int b = (int)(u0 + i - first);
    const int chosen = a.sel_idx ? a.sel_idx[(size_t)pair * a.k_max + b] : b, len = a.seq_lens[r];
    b = chosen;
    if (b < 0 || b >= a.max_pages || b * kPage >= len) {                                 // (only a selection can be wrong here)
        atomicOr(&a.ctl->status, SE_DEV_BAD_SELECTION);
        return p;
    }
    const int pid = a.page_table[(size_t)r * a.max_pages + b];
    if (pid >= a.P_phys) atomicOr(&a.ctl->status, SE_DEV_BAD_PAGE_ID);
    if (pid < 0 || pid >= a.P_phys) return p;
    p.row = pid * a.H_kv + h;
    p.tokens = min(kPage, len - b * kPage);
    p.scale = a.scales[p.row];
    return p;
}

// A pair's query heads on their way to shared memory, by the team's threads.
template <int D>
__device__ __forceinline__ void fetch_q(const Args &a, int pair, uint32_t dst, int tt) {
    const int r = pair / a.H_kv, h = pair - r * a.H_kv;
    if (tt < a.G * D / 8)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + tt * 16), "l"(a.q + ((size_t)r * a.H_q + h * a.G) * D + tt * 8) : "memory");
    asm volatile("cp.async.commit_group;" ::: "memory");
}

// The parts of a pair that the runs c0 .. c1 have left.  Up to 31 are merged by whoever comes last.  More are merged in groups of 16
// neighbours (the last group of up to 31), each by the last of its runs, into the place of the group's first, and the groups by the
// last of them: where one team merged all 592 parts of a single head over 65536 tokens the call took 75 us, now 19; below 32 parts a
// second round of tickets costs what it saves.  Always in the order of the runs.
constexpr int kGroup = 16;
struct Parts {
    int c0, c1;
    __device__ __forceinline__ int groups() const { return max((c1 - c0 + 1) / kGroup, 1); }
    __device__ __forceinline__ int group_of(int run) const { return min((run - c0) / kGroup, groups() - 1); }
    __device__ __forceinline__ int size_of(int j) const { return j < groups() - 1 ? kGroup : c1 - c0 + 1 - j * kGroup; }
    // Counters: of the pair's parts or groups that of run c0; of group j that of its first run, of the first group that of the second
    // run.  The pair fills all runs between the first and the last, so no other pair begins in these.
    __device__ __forceinline__ int ticket_of(int j) const { return groups() == 1 ? c0 : j == 0 ? c0 + 1 : c0 + j * kGroup; }
    __device__ __forceinline__ size_t slot(int run) const { return (size_t)run * 2 + (run == c0 ? 1 : 0); }
};

// Merges n parts, of runs x0, x0 + step, ..., into the pair's output (LAST) or into the place of the first one.
template <int D, bool LAST>
__device__ __noinline__ void merge_parts(const Args &a, int pair, Parts ps, int x0, int step, int n, int tt) {
    using C = Cfg<D>;
    const size_t row0 = (size_t)(pair / a.H_kv) * a.H_q + pair % a.H_kv * a.G;
    static_assert(32 % (D / 4) == 0, "a head's statistics are read and written by one warp");
    for (int e0 = 0; e0 < a.G * (D / 4); e0 += 32 * kTeam) {
        const int e = e0 + tt, head = e / (D / 4), ch = e % (D / 4) * 4;
        const bool mine = e < a.G * (D / 4);
        float M = -INFINITY, L = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        constexpr int kBatch = 8;      // parts on their way at a time (with four: a dense layer 58.4 us instead of 56.6, a sparse one 61.7 for 63.1)
        for (int i0 = 0; i0 < (mine ? n : 0); i0 += kBatch) {
            float mx[kBatch], lx[kBatch];
            float4 v[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const float *src = a.partials + ps.slot(x0 + min(i0 + k, n - 1) * step) * C::kPartFloats;
                mx[k] = __ldcg(src + 8 * D + head), lx[k] = __ldcg(src + 8 * D + 8 + head);
                v[k] = __ldcg(reinterpret_cast<const float4 *>(src + head * D + ch));
            }
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const float at = i0 + k < n ? mx[k] : -INFINITY;                         // (a branch here, and each load waits for the last)
                const float top = fmaxf(M, at), ref = top == -INFINITY ? 0.f : top;
                const float fo = ex2(M - ref), fx = ex2(at - ref);
                M = top, L = L * fo + lx[k] * fx;
                o.x = o.x * fo + v[k].x * fx, o.y = o.y * fo + v[k].y * fx, o.z = o.z * fo + v[k].z * fx, o.w = o.w * fo + v[k].w * fx;
            }
        }
        __syncwarp();
        if (!mine) continue;
        if constexpr (LAST) {
            const float inv = L == 0.f ? 0.f : 1.f / L;
            *reinterpret_cast<float4 *>(a.out + (row0 + head) * D + ch) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
            if (ch == 0) a.lse[row0 + head] = L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
        } else {
            float *dst = a.partials + ps.slot(x0) * C::kPartFloats;
            __stcg(reinterpret_cast<float4 *>(dst + head * D + ch), o);
            if (ch == 0) __stcg(dst + 8 * D + head, M), __stcg(dst + 8 * D + 8 + head, L);
        }
    }
}

// The team whose run was the last of its group goes on with it, and perhaps with the groups.
template <int D>
__device__ __noinline__ void join_parts(const Args &a, int pair, Parts ps, int run, int tt, int team, int *said) {
    const int groups = ps.groups(), j = ps.group_of(run);
    if (groups == 1) {
        merge_parts<D, true>(a, pair, ps, ps.c0, 1, ps.size_of(0), tt);
        return;
    }
    merge_parts<D, false>(a, pair, ps, ps.c0 + j * kGroup, 1, ps.size_of(j), tt);
    __threadfence();
    team_sync(team);
    if (tt == 0) {
        __threadfence();
        const bool last = atomicAdd(a.ctl->tickets + ps.c0, 1u) == (uint32_t)(groups - 1);
        if (last) atomicExch(a.ctl->tickets + ps.c0, 0u);
        *said = last;
    }
    team_sync(team);
    if (*said) {
        __threadfence();
        merge_parts<D, true>(a, pair, ps, ps.c0, kGroup, groups, tt);
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
kv8_decode_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const __grid_constant__ Args a) {
    using C = Cfg<D>;
    extern __shared__ __align__(1024) uint8_t smem[];
    float *s_merge = reinterpret_cast<float *>(smem + C::kRing);                        // [warp][8][kPitch], then m and l
    const uint32_t s_q = smem_u32(smem) + (uint32_t)(C::kRing + C::kMerge);             // [team][2][8][D] bf16
    long long *s_pre = reinterpret_cast<long long *>(smem + C::kRing + C::kMerge + C::kQ);
    uint64_t *s_bars = reinterpret_cast<uint64_t *>(s_pre + kChunks + 1);
    int *s_misc = reinterpret_cast<int *>(s_bars + kWarps * C::kStages);                // sums of a scan, verdict of a merge
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int team = warp / kTeam, mate = warp % kTeam, tt = tid % (32 * kTeam);         // team, warp and thread of the team
    const int runs = gridDim.x * kTeams, run = team * gridDim.x + blockIdx.x;            // (few runs: on SMs of their own)
    const uint32_t ring = smem_u32(smem) + warp * (C::kStages * 2 * C::kPageBytes);
    const uint32_t bars = smem_u32(s_bars) + warp * (C::kStages * 8);

    if ((smem_u32(smem) & 1023u) || *(volatile uint32_t *)&a.ctl->needs_init) {         // the swizzle pattern hangs on the address
        if (tid == 0 && blockIdx.x == 0) atomicOr(&a.ctl->status, SE_DEV_WAIT_TIMEOUT);
        return;
    }
    if (lane < C::kStages) mbar_init(bars + 8 * lane, 1);
    if (tid == 0) prefetch_map(&k_map), prefetch_map(&v_map);
    mbar_fence_init();

    // pages before every pair (or every run of pairs, where there are more than 1024)
    const int pairs = a.B * a.H_kv;
    Pairs ps = {a, s_pre, (pairs + kChunks - 1) / kChunks, 0};
    ps.chunks = (pairs + ps.per - 1) / ps.per;
    {
        const int each = (ps.chunks + kThreads - 1) / kThreads;
        const int c0 = min(tid * each, ps.chunks), c1 = min(c0 + each, ps.chunks);
        long long sum = 0;
        for (int c = c0; c < c1; ++c) {
            s_pre[c] = sum;
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
        long long *tot = reinterpret_cast<long long *>(s_misc);
        if (lane == 31) tot[warp] = inc;
        __syncthreads();
        long long before = inc - sum;
        for (int w = 0; w < warp; ++w) before += tot[w];
        for (int c = c0; c < c1; ++c) s_pre[c] += before;
        if (tid == kThreads - 1) s_pre[ps.chunks] = before + sum;
        __syncthreads();
    }
    // pairs without a page
    for (int x0 = blockIdx.x * 32 + warp * 32 * gridDim.x; x0 < pairs; x0 += 32 * kWarps * gridDim.x) {
        unsigned none = __ballot_sync(kFull, x0 + lane < pairs && ps.count_known(min(x0 + lane, pairs - 1)) == 0);
        for (; none; none &= none - 1) {
            const int x = x0 + __ffs(none) - 1;
            const size_t row = (size_t)(x / a.H_kv) * a.H_q + x % a.H_kv * a.G;
            for (int e = lane; e < a.G * D; e += 32) a.out[row * D + e] = 0.f;
            if (lane < a.G) a.lse[row + lane] = -INFINITY;
        }
    }

    const long long total = s_pre[ps.chunks];
    const long long size = max((total + runs - 1) / runs, (long long)kLeast);
    const long long u0 = size * run;
    if (u0 >= total) return;
    const int n = (int)min(size, total - u0);
    const int mine = n > mate ? (n - mate + kTeam - 1) / kTeam : 0;                      // page k of the warp is page k * kTeam + mate of the run
    long long first;
    int pair = ps.find(u0, first);
    const uint32_t q_at = s_q + team * (2 * 8 * D * 2);
    fetch_q<D>(a, pair, q_at, tt);     // (ahead of the pages: behind the rings' first fill it took 4 us)
    Page now = look_up(a, ps, u0, n, lane * kTeam + mate), next = {-1, 0, make_float2(0.f, 0.f)};
    int block = 0, known = 32, issue = 0;                                                // block of 32 pages that `now` describes, pages looked up; next page to fetch
    uint32_t sent = 0, used = 0;       // pages fetched, pages consumed
    bool ok = true;
    const bool chosen = elect_one();
    auto send = [&] {
        while (ok && issue < mine && sent - used < C::kStages && issue < known) {
            const int row = __shfl_sync(kFull, issue / 32 == block ? now.row : next.row, issue & 31);
            if (row >= 0) {
                if (chosen) {
                    const uint32_t slot = sent % C::kStages, dst = ring + slot * (2 * C::kPageBytes);
                    mbar_expect_tx(bars + 8 * slot, 2 * C::kPageBytes + (sent == 0 ? kTestExtraTx : 0));
                    tma_load_2d(dst, &k_map, 0, row * C::kRowsPerPage, bars + 8 * slot);
                    tma_load_2d(dst + C::kPageBytes, &v_map, 0, row * C::kRowsPerPage, bars + 8 * slot);
                }
                __syncwarp();
                ++sent;
            }
            ++issue;
        }
    };
    send();

    if (mine > 32) next = look_up(a, ps, u0, n, (32 + lane) * kTeam + mate);
    known = 64;
    int k = 0;
    int begun = -1, begun_c0 = 0, begun_c1 = 0;        // the run's first pair, where earlier runs hold a part of it
    for (int done = 0, turn = 0;; ++turn) {
        const int pages = ps.count_known(pair);
        const int stop = (int)min((long long)n, first + pages - u0);                     // end of the pair's pages in the run
        // q is here, and the team has read the merge buffer; the next pair's q is on its way a whole pair ahead
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        team_sync(team);
        int after = pair;
        if (stop < n) {
            while (ps.count_known(++after) == 0) {}
            fetch_q<D>(a, after, q_at + (turn + 1 & 1) * (8 * D * 2), tt);
        }
        // q as halves: head g, channels 64 i + 16 t .. + 15
        uint32_t qh[D / 8];
        float f0, f1;                  // heads 2 t and 2 t + 1: logit in powers of two = sum * f * s_K
        {
            uint4 raw[D / 32];
            const uint32_t src = q_at + (turn & 1) * (8 * D * 2) + min(g, a.G - 1) * (2 * D) + 32 * t;
#pragma unroll
            for (int i = 0; i < D / 64; ++i) raw[2 * i] = lds128(src + 128 * i), raw[2 * i + 1] = lds128(src + 128 * i + 16);
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) top = bmax2(top, largest8(raw[i]));
            top = max(top & 0xffffu, top >> 16);
            top = max(top, __shfl_xor_sync(kFull, top, 1));
            top = max(top, __shfl_xor_sync(kFull, top, 2));
            const int e = max((int)(top >> 7), 20);                                      // maximum 1.x * 2^(e - 127)
            const float up = __uint_as_float((uint32_t)(140 - e + 127) << 23);           // 2^(140 - e)
            const float down = __uint_as_float((uint32_t)(e - 140 + 127) << 23);
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 x = bf16x2_to_f2(w[j]);
                    qh[4 * i + j] = g < a.G ? pack_half2(x.x * up, x.y * up) : 0u;
                }
            }
            const float f = down * a.scale_log2;
            f0 = __shfl_sync(kFull, f, 8 * t), f1 = __shfl_sync(kFull, f, 8 * t + 4);
        }
        float acc[C::kTiles][4];       // [tile]: channel (D / 8) g + 2 tile, heads 2 t, 2 t + 1; the channel behind it
#pragma unroll
        for (int i = 0; i < C::kTiles; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
        float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
        float *own = s_merge + warp * (8 * C::kPitch + 16);
        bool far = false;              // a maximum is above kFar
        bool folded = false;           // the merge buffer holds the sums of earlier pages, for the maxima that lie with them
        auto fold = [&] {
            float r0 = 0.f, r1 = 0.f;
            if (folded) r0 = ex2(own[8 * C::kPitch + 2 * t] - m0), r1 = ex2(own[8 * C::kPitch + 2 * t + 1] - m1);
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) l0 += __shfl_xor_sync(kFull, l0, o), l1 += __shfl_xor_sync(kFull, l1, o);
            __syncwarp();
            if (g == 0) {
                float *stats = own + 8 * C::kPitch + 2 * t;
                if (folded) l0 = fmaf(stats[8], r0, l0), l1 = fmaf(stats[9], r1, l1);
                stats[0] = m0, stats[1] = m1, stats[8] = l0, stats[9] = l1;
            }
#pragma unroll
            for (int j = 0; j < C::kTiles / 2; ++j) {
                float4 *at0 = reinterpret_cast<float4 *>(own + (2 * t) * C::kPitch + (D / 8) * g + 4 * j), *at1 = at0 + C::kPitch / 4;
                float4 x = make_float4(acc[2 * j][0], acc[2 * j][2], acc[2 * j + 1][0], acc[2 * j + 1][2]);
                float4 y = make_float4(acc[2 * j][1], acc[2 * j][3], acc[2 * j + 1][1], acc[2 * j + 1][3]);
                if (folded) {
                    const float4 u = *at0, w = *at1;
                    x = make_float4(fmaf(u.x, r0, x.x), fmaf(u.y, r0, x.y), fmaf(u.z, r0, x.z), fmaf(u.w, r0, x.w));
                    y = make_float4(fmaf(w.x, r1, y.x), fmaf(w.y, r1, y.y), fmaf(w.z, r1, y.z), fmaf(w.w, r1, y.w));
                }
                *at0 = x, *at1 = y;
            }
        };

        for (; k < mine && k * kTeam + mate < stop; ++k) {
            if (k / 32 != block) {
                ++block;
                now = next;
                next = look_up(a, ps, u0, n, ((block + 1) * 32 + lane) * kTeam + mate);
                known += 32;
                send();
            }
            const int row = __shfl_sync(kFull, now.row, k & 31);
            if (row < 0) continue;
            const int tokens = __shfl_sync(kFull, now.tokens, k & 31);
            const float sk = __shfl_sync(kFull, now.scale.x, k & 31), sv = __shfl_sync(kFull, now.scale.y, k & 31);
            const uint32_t slot = used % C::kStages, at = ring + slot * (2 * C::kPageBytes);
            if (ok && !__all_sync(kFull, mbar_wait(bars + 8 * slot, used / C::kStages & 1))) {
                ok = false;
                if (lane == 0) atomicExch(&a.ctl->needs_init, 1u), atomicOr(&a.ctl->status, SE_DEV_WAIT_TIMEOUT);
            }
            if (!ok) continue;
            // ---- logits: rows are tokens, columns are heads.  Row x of the product is token x for even x, x ^ 4 for odd x (and the
            // same 8 further on): with the swizzle, lanes that load at the same time then never meet in a bank, here and for V.
            const int tok = g & 1 ? g ^ 4 : g;
            float c[2][4];
#pragma unroll
            for (int i = 0; i < D / 64; ++i) {
                uint4 x, y;
                if constexpr (D == 128) {
                    const uint32_t off = at + tok * 128 + (((t + 4 * i) ^ tok) << 4);
                    x = lds128(off), y = lds128(off + 1024);
                } else {
                    const uint32_t line = tok >> 1, off = (((tok & 1) * 4 + t) ^ line) << 4;
                    x = lds128(at + line * 128 + off), y = lds128(at + 512 + line * 128 + (off ^ 64));
                }
                const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    uint32_t a0, a1, a2, a3;
                    halves_of_e4m3x4(xw[s], a0, a2), halves_of_e4m3x4(yw[s], a1, a3);
                    if (i == 0 && s < 2) mma_f16_first(c[s & 1], a0, a1, a2, a3, qh[8 * i + 2 * s], qh[8 * i + 2 * s + 1]);
                    else mma_f16(c[s & 1], a0, a1, a2, a3, qh[8 * i + 2 * s], qh[8 * i + 2 * s + 1]);
                }
            }
            const float g0 = fmaxf(f0 * sk, 1e-37f), g1 = fmaxf(f1 * sk, 1e-37f);        // (0 times a masked logit would be NaN)
            float z[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) z[e] = c[0][e] + c[1][e];
            if (tokens < kPage) {
                if (tok >= tokens) z[0] = z[1] = -INFINITY;
                if (tok + 8 >= tokens) z[2] = z[3] = -INFINITY;
            }
            // w = logit + log2 of V's scale, in powers of two: what the weights in the product with V are made of
            const float shift = (float)((int)(__float_as_uint(sv) >> 23) - 127), inv = __uint_as_float(0x7f000000u - __float_as_uint(sv));
            const float t0 = fmaf(fmaxf(z[0], z[2]), g0, shift), t1 = fmaf(fmaxf(z[1], z[3]), g1, shift);
            if (__any_sync(kFull, t0 - m0 > kTop || t1 - m1 > kTop)) {
                float n0 = fmaxf(m0, t0 - kLift), n1 = fmaxf(m1, t1 - kLift);
                if (t0 - n0 > kTop) n0 = t0;                                             // (where the steps of fp32 are 8 and 16)
                if (t1 - n1 > kTop) n1 = t1;
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) {
                    n0 = fmaxf(n0, __shfl_xor_sync(kFull, n0, o));
                    n1 = fmaxf(n1, __shfl_xor_sync(kFull, n1, o));
                }
                const float r0 = ex2(m0 - n0), r1 = ex2(m1 - n1);                        // (a page has a token, so n is a number)
                m0 = n0, m1 = n1;
                far = __any_sync(kFull, fabsf(m0) > kFar || fabsf(m1) > kFar);
                l0 *= r0, l1 *= r1;
#pragma unroll
                for (int i = 0; i < C::kTiles; ++i) acc[i][0] *= r0, acc[i][1] *= r1, acc[i][2] *= r0, acc[i][3] *= r1;
            }
            const float off0 = shift - m0, off1 = shift - m1;
            float w0 = fmaf(z[0], g0, off0), w1 = fmaf(z[1], g1, off1), w2 = fmaf(z[2], g0, off0), w3 = fmaf(z[3], g1, off1);
            if (far) w0 = fmaf(z[0], g0, shift) - m0, w1 = fmaf(z[1], g1, shift) - m1, w2 = fmaf(z[2], g0, shift) - m0, w3 = fmaf(z[3], g1, shift) - m1;
            const float p0 = ex2(w0), p1 = ex2(w1), p2 = ex2(w2), p3 = ex2(w3);
            l0 = fmaf(p0 + p2, inv, l0), l1 = fmaf(p1 + p3, inv, l1);
            // weights as hi + lo, two halves; transposed, they are the second operand: rows tokens, columns heads
            const uint32_t h0 = pack_half2(p0, p1), h1 = pack_half2(p2, p3);
            const float2 u = unpack_half2(h0), w = unpack_half2(h1);
            const uint32_t b0 = transpose8x8(h0), b1 = transpose8x8(h1);
            const uint32_t e0 = transpose8x8(pack_half2(p0 - u.x, p1 - u.y)), e1 = transpose8x8(pack_half2(p2 - w.x, p3 - w.y));
            // ---- output: rows are channels, columns are heads
            uint32_t va[D / 32], vb[D / 32], vc[D / 32], vd[D / 32];                     // tokens of columns 2 t, 2 t + 1, and 8 further on
            const int ta = 2 * t, tb = (2 * t + 1) ^ 4;
            auto fetch = [&](int tk, uint32_t (&dst)[D / 32]) {
                if constexpr (D == 128) {
                    const uint4 x = lds128(at + C::kPageBytes + tk * 128 + ((g ^ (tk & 7)) << 4));
                    dst[0] = x.x, dst[1] = x.y, dst[2] = x.z, dst[3] = x.w;
                } else {
                    const uint32_t line = tk >> 1;
                    const uint2 x = lds64(at + C::kPageBytes + line * 128 + ((((tk & 1) * 4 + (g >> 1)) ^ line) << 4) + (g & 1) * 8);
                    dst[0] = x.x, dst[1] = x.y;
                }
            };
            fetch(ta, va), fetch(tb, vb), fetch(ta + 8, vc), fetch(tb + 8, vd);
            __syncwarp();
            ++used;                    // the page's bytes are in registers: its slot may be filled again
            send();
            if (tokens < kPage) {      // what lies behind the end may be anything, and a weight of zero would not hide a NaN
#pragma unroll
                for (int j = 0; j < D / 32; ++j) {
                    if (ta >= tokens) va[j] = 0;
                    if (tb >= tokens) vb[j] = 0;
                    if (ta + 8 >= tokens) vc[j] = 0;
                    if (tb + 8 >= tokens) vd[j] = 0;
                }
            }
#pragma unroll
            for (int i = 0; i < C::kTiles; ++i) {                                        // rows g, g + 8: channels (D / 8) g + 2 i, + 1
                const uint32_t sel = i & 1 ? 0x7362u : 0x5140u;
                const uint32_t x = __byte_perm(va[i / 2], vb[i / 2], sel), y = __byte_perm(vc[i / 2], vd[i / 2], sel);
                uint32_t a0, a1, a2, a3;
                halves_of_e4m3x4(x, a0, a1), halves_of_e4m3x4(y, a2, a3);
                mma_f16(acc[i], a0, a1, a2, a3, e0, e1);
                mma_f16(acc[i], a0, a1, a2, a3, b0, b1);
            }
            if (used % kFold == 0) {
                fold();
                folded = true;
                l0 = l1 = 0.f;
#pragma unroll
                for (int i = 0; i < C::kTiles; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
                __syncwarp();
            }
        }

        // ---- end of the pair's pages in this run ----
        fold();
        const float *team_merge = s_merge + team * kTeam * (8 * C::kPitch + 16);
        team_sync(team);
        const int c0 = (int)(first / size), c1 = (int)((first + pages - 1) / size);      // runs that share the pair
        const int r = pair / a.H_kv, h = pair - r * a.H_kv;
        const size_t row0 = (size_t)r * a.H_q + h * a.G;
        float *part = a.partials + (size_t)(run * 2 + (c0 == run ? 1 : 0)) * C::kPartFloats;
        for (int e = tt; e < a.G * (D / 4); e += 32 * kTeam) {
            const int head = e / (D / 4), ch = e % (D / 4) * 4;
            float M = -INFINITY;
#pragma unroll
            for (int w = 0; w < kTeam; ++w) M = fmaxf(M, team_merge[w * (8 * C::kPitch + 16) + 8 * C::kPitch + head]);
            const float ref = M == -INFINITY ? 0.f : M;
            float L = 0.f;
            float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kTeam; ++w) {
                const float *src = team_merge + w * (8 * C::kPitch + 16);
                const float x = ex2(src[8 * C::kPitch + head] - ref);
                L = fmaf(x, src[8 * C::kPitch + 8 + head], L);
                const float4 v = *reinterpret_cast<const float4 *>(src + head * C::kPitch + ch);
                o.x = fmaf(x, v.x, o.x), o.y = fmaf(x, v.y, o.y), o.z = fmaf(x, v.z, o.z), o.w = fmaf(x, v.w, o.w);
            }
            if (c0 == c1) {
                const float inv = L == 0.f ? 0.f : 1.f / L;
                *reinterpret_cast<float4 *>(a.out + (row0 + head) * D + ch) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
                if (ch == 0) a.lse[row0 + head] = L == 0.f ? -INFINITY : (M + log2f(L)) * kLn2;
            } else {
                __stcg(reinterpret_cast<float4 *>(part + head * D + ch), o);
                if (ch == 0) __stcg(part + 8 * D + head, M), __stcg(part + 8 * D + 8 + head, L);
            }
        }
        if (c0 < run) begun = pair, begun_c0 = c0, begun_c1 = c1;
        done = stop;
        if (done == n) {
            // The parts of pairs that other runs share are all written: one round of fence and tickets for both (after each pair it
            // took the team 6 to 9 us, under load, with nothing else to do).
            const bool ends = c1 > run && c0 == run;                                     // later runs go on with a pair that begins here
            if (begun >= 0 || ends) {
                __threadfence();
                team_sync(team);
                if (tt == 0) {
                    __threadfence();
                    auto last = [&](Parts parts) {                                       // of the run's group
                        const int j = parts.group_of(run);
                        uint32_t *ticket = a.ctl->tickets + parts.ticket_of(j);
                        if (atomicAdd(ticket, 1u) != (uint32_t)(parts.size_of(j) - 1)) return false;
                        atomicExch(ticket, 0u);
                        return true;
                    };
                    s_misc[team] = (begun >= 0 && last(Parts{begun_c0, begun_c1}) ? 1 : 0) | (ends && last(Parts{c0, c1}) ? 2 : 0);
                }
                team_sync(team);
                const int verdict = s_misc[team];
                if (verdict) __threadfence();
                if (verdict & 1) join_parts<D>(a, begun, Parts{begun_c0, begun_c1}, run, tt, team, s_misc + team);
                if (verdict & 2) join_parts<D>(a, pair, Parts{c0, c1}, run, tt, team, s_misc + team);
            }
            break;
        }
        pair = after, first += pages;
    }
    // a wait that gave up: the copies that are still on their way end before the CTA does
    for (; used != sent; ++used) mbar_wait(bars + 8 * (used % C::kStages), used / C::kStages & 1);
}

// the cache as lines of 128 bytes, boxes of one page of one head
bool make_lines_map(CUtensorMap *map, const void *base, long long bytes, int lines) {
    EncodeTiledFn fn = encode_tiled();
    if (!fn) return false;
    const cuuint64_t dims[2] = {128, (cuuint64_t)(bytes / 128)};
    const cuuint64_t strides[1] = {128};
    const cuuint32_t box[2] = {128, (cuuint32_t)lines};
    const cuuint32_t estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D>
cudaError_t launch(const se_params &p, const Kv8DecodeCall &c, cudaStream_t stream) {
    using C = Cfg<D>;
    CUtensorMap k_map, v_map;
    const long long bytes = (long long)p.num_phys_pages * p.H_kv * C::kPageBytes;
    if (!make_lines_map(&k_map, c.k_cache, bytes, C::kRowsPerPage) || !make_lines_map(&v_map, c.v_cache, bytes, C::kRowsPerPage))
        return cudaErrorInvalidValue;
    Args a = {};
    a.q = static_cast<const uint16_t *>(c.q), a.scales = reinterpret_cast<const float2 *>(c.scales);
    a.page_table = c.page_table, a.seq_lens = c.seq_lens, a.sel_idx = c.sel_idx, a.sel_cnt = c.sel_cnt;
    a.out = c.out, a.lse = c.lse, a.partials = partials_of(c.workspace), a.ctl = reinterpret_cast<PromptControl *>(c.workspace);
    a.B = p.B, a.H_q = p.H_q, a.H_kv = p.H_kv, a.G = p.H_q / p.H_kv, a.max_pages = p.max_pages, a.P_phys = p.num_phys_pages;
    a.k_max = p.k_max, a.scale_log2 = effective_scale(p) * kLog2e;
    static_assert(C::kSmem <= 227 * 1024, "shared memory of a CTA");
    static_assert(2 * kTeams * C::kPartFloats <= 8 * (128 * D + 256), "partial results of a CTA fit where the prompt kernels keep theirs");
    static_assert(kTeams * kPromptCtas <= 2 * kMaxPieces, "a ticket per run");
    auto kern = kv8_decode_kernel<D>;
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::kSmem);
    if (e != cudaSuccess) return e;
    kern<<<kPromptCtas, kThreads, C::kSmem, stream>>>(k_map, v_map, a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_kv8_decode(const se_params &p, const Kv8DecodeCall &c, cudaStream_t stream) {
    return p.D == 128 ? launch<128>(p, c, stream) : launch<64>(p, c, stream);
}

}  // namespace se
