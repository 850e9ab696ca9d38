// The pool's pages: requests fork, end, shrink and grow (pages_update_kernel), and live pages move to the front of the pool
// (pages_compact_kernel).  (Appendix A, "Logical Positions and Physical Blocks": a page table maps logical blocks to physical
// ones, and several requests may map to one; the paper leaves the pool itself to the engine.)
//
// Both are one cooperative launch: a few passes over the tables, the reference counts and scratch of four bytes per page, with
// grid-wide barriers between them, then the copies of the pages that move, in all of the caller's buffers.  Everything that
// decides which page goes where is a prefix sum, so equal inputs give equal tables; atomics only add integers.
//
// update.  Slot r takes over the first keep = min(length of parent[r], new_lens[r]) tokens of its parent's row.
//   1  changes of the reference counts (entries that stay in their slot cost nothing), and for every row that ends inside a
//      page - an open page - how many rows are open on it, and the first of them
//   2  an open page that more than its open rows refer to, or that an earlier row is open on, is copied; pages that each slot
//      asks for; free pages of each CTA's part of the pool
//   3  the i-th free page of the pool goes to the i-th request for one (slot by slot, page by page)
//   4  the open pages' contents are copied
// compact.  With n live pages, the i-th live page with a number from n on moves to the i-th free one below n.
//
// What bounds them: barriers and dependent loads for the tables (about 2 us each; 64 requests over a pool of 64 K pages grow by a
// token in 11.7 us), HBM for the copies (40000 pages of four layers of codes compacted: 2.57 GB in 419 us, 6.1 TB/s).
#include <climits>

#include "se_internal.h"

namespace se {

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kCtas = 148;
constexpr int kPiece = 4096;           // bytes that a warp copies at a time: 8 x 16 bytes per lane in flight

struct Control {
    uint32_t status, needs_init, arrived, left, pad[60];
    int sums[256];                     // of each CTA
};

// What becomes of a slot.
struct Slot {
    int parent, keep, kept, pages, len, copy, asis, pad;   // parent (-1: none), tokens and pages taken over, pages and length afterwards, last
                                                       // page copied, row left as it is
};

struct Buffers {
    int n, units;                      // units: pieces of one page in all buffers
    se_page_buffer at[SE_MAX_PAGE_BUFFERS];
};

struct UpdateArgs {
    const int32_t *table, *lens, *refs, *parent, *new_lens;
    int32_t *table_out, *lens_out, *refs_out, *count;
    Control *ctl;
    int32_t *delta, *opens, *owner;    // [P_phys], zero between calls
    Slot *slots;                       // [B]
    int2 *copies;                      // [B] from, to
    int B, max_pages, P;
};

struct CompactArgs {
    const int32_t *table, *lens, *refs;
    int32_t *table_out, *refs_out, *map, *count;
    Control *ctl;
    int32_t *holes, *movers, *rank;    // [P_phys]
    int B, max_pages, P;
};

// For the test of the bounded barriers (a second build of the library, never the product): they wait for a CTA that does not exist.
#ifdef SE_TEST_SHORT_TX
constexpr uint32_t kTestExtraCtas = 1;
#else
constexpr uint32_t kTestExtraCtas = 0;
#endif

// All CTAs of the launch have come here, and see what the others wrote before.  False: the wait gave up.
__device__ __forceinline__ bool grid_sync(Control *ctl, int turn) {
    __shared__ int s_ok;
    __syncthreads();
    if (gridDim.x == 1) return true;
    if (threadIdx.x == 0) {
        __threadfence();
        atomicAdd(&ctl->arrived, 1u);
        const uint32_t want = (uint32_t)turn * gridDim.x + kTestExtraCtas;
        bool ok = false;
        const unsigned long long t0 = globaltimer_ns();
        for (int it = 0; !ok; ++it) {
            uint32_t seen;
            asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(&ctl->arrived) : "memory");
            ok = seen >= want;
            if (!ok && (it & 255) == 255 && globaltimer_ns() - t0 > kWaitLimitNs) break;
        }
        if (!ok) {
            atomicExch(&ctl->needs_init, 1u);
            atomicOr(&ctl->status, SE_DEV_WAIT_TIMEOUT);
        }
        __threadfence();
        s_ok = ok;
    }
    __syncthreads();
    return s_ok != 0;
}
// The last CTA leaves the barrier's counters as it found them.
__device__ __forceinline__ void grid_leave(Control *ctl) {
    if (gridDim.x > 1 && threadIdx.x == 0 && atomicAdd(&ctl->left, 1u) == gridDim.x - 1) {
        atomicExch(&ctl->arrived, 0u);
        atomicExch(&ctl->left, 0u);
    }
}

__device__ __forceinline__ int cta_sum(int v, int *s, int lane, int warp) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
    __syncthreads();
    if (lane == 0) s[warp] = v;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) all += s[w];
    return all;
}

// sums of the CTAs before this one, and of all
__device__ __forceinline__ void sums_before(const Control *ctl, int *s, int tid, int lane, int warp, int &before, int &all) {
    const int v = tid < (int)gridDim.x ? __ldcg(ctl->sums + tid) : 0;
    before = cta_sum(tid < (int)blockIdx.x ? v : 0, s, lane, warp);
    all = cta_sum(v, s, lane, warp);
}

// ---- copies ------------------------------------------------------------------------
__device__ __forceinline__ int pieces_of(const se_page_buffer &b) { return (int)((b.bytes_per_page + kPiece - 1) / kPiece); }

// Pages from(i) -> to(i), i < n, in all buffers, by all warps of the launch.
template <typename From, typename To>
__device__ __forceinline__ void copy_pages(const Buffers &buf, int n, From from, To to, int *first, int lane, int warp) {
    // pieces before each buffer
    __syncthreads();
    if (threadIdx.x == 0) {
        int at = 0;
        for (int k = 0; k < buf.n; ++k) first[k] = at, at += pieces_of(buf.at[k]);
        first[buf.n] = at;
    }
    __syncthreads();
    const long long units = (long long)n * buf.units;
    for (long long u = blockIdx.x * kWarps + warp; u < units; u += (long long)gridDim.x * kWarps) {
        const int i = (int)(u / buf.units), v = (int)(u - (long long)i * buf.units);
        int lo = 0, hi = buf.n;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (first[mid] <= v) lo = mid; else hi = mid;
        }
        const long long bytes = buf.at[lo].bytes_per_page, at = (long long)(v - first[lo]) * kPiece;
        const int len = (int)min((long long)kPiece, bytes - at);
        const uint8_t *src = static_cast<const uint8_t *>(buf.at[lo].base) + from(i) * bytes + at;
        uint8_t *dst = static_cast<uint8_t *>(buf.at[lo].base) + to(i) * bytes + at;
        if (bytes % 16 == 0) {
            uint4 x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if ((e * 32 + lane) * 16 < len) x[e] = __ldcs(reinterpret_cast<const uint4 *>(src) + e * 32 + lane);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if ((e * 32 + lane) * 16 < len) reinterpret_cast<uint4 *>(dst)[e * 32 + lane] = x[e];
        } else {
            for (int e = lane * 4; e < len; e += 128) *reinterpret_cast<uint32_t *>(dst + e) = *reinterpret_cast<const uint32_t *>(src + e);
        }
    }
}

// ---- update ------------------------------------------------------------------------
__device__ __forceinline__ bool in_range(const UpdateArgs &a, int n) { return n >= 0 && n <= a.max_pages * kPage; }
__device__ __forceinline__ int length_of(const UpdateArgs &a, int r) { return in_range(a, a.lens[r]) ? a.lens[r] : 0; }
__device__ __forceinline__ Slot plan_slot(const UpdateArgs &a, int r, bool report) {
    int s = a.parent ? a.parent[r] : r, n = a.new_lens[r];
    const int own = a.lens[r];
    Slot x = {};
    x.len = n;
    if (s < -1 || s >= a.B || !in_range(a, n) || !in_range(a, own) || (s >= 0 && !in_range(a, a.lens[s]))) {
        if (report) atomicOr(&a.ctl->status, SE_DEV_BAD_LENGTH);
        s = r, n = length_of(a, r), x.len = own, x.asis = 1;
    }
    x.parent = s;
    x.keep = s < 0 ? 0 : min(length_of(a, s), n);
    x.kept = (x.keep + kPage - 1) / kPage;
    x.pages = (n + kPage - 1) / kPage;
    return x;
}
__device__ __forceinline__ bool is_page(const UpdateArgs &a, int e) { return e >= 0 && e < a.P; }
// the page that the row ends inside of, -1: none
__device__ __forceinline__ int open_page(const UpdateArgs &a, const Slot &x) {
    if (x.asis || x.keep % kPage == 0) return -1;
    const int e = a.table[(size_t)x.parent * a.max_pages + x.keep / kPage];
    return is_page(a, e) ? e : -1;
}

__global__ void __launch_bounds__(kThreads, 2)
pages_update_kernel(const __grid_constant__ UpdateArgs a, const __grid_constant__ Buffers buf) {
    extern __shared__ int s_asked[];                   // [B + 1] pages asked for before each slot, [B + 1] copies
    __shared__ int s_red[kWarps], s_scan[32], s_first[SE_MAX_PAGE_BUFFERS + 1];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int *s_copies = s_asked + a.B + 1;
    if (*(volatile uint32_t *)&a.ctl->needs_init) {
        if (tid == 0 && blockIdx.x == 0) atomicOr(&a.ctl->status, SE_DEV_WAIT_TIMEOUT);
        return;
    }
    // (B * max_pages < 2^31, so 32 bits hold an index and the step beyond the last one)
    const uint32_t entries = (uint32_t)a.B * a.max_pages, stride = gridDim.x * kThreads, me = blockIdx.x * kThreads + tid;

    // 1: changes of the reference counts, open pages
    for (uint32_t i = me; i < entries; i += stride) {
        const int r = (int)(i / (uint32_t)a.max_pages), b = (int)(i - (uint32_t)r * a.max_pages);
        const Slot x = plan_slot(a, r, b == 0);
        const int held = (length_of(a, r) + kPage - 1) / kPage;
        if (b < held) {
            const int e = a.table[i];
            if (e >= a.P) atomicOr(&a.ctl->status, SE_DEV_BAD_PAGE_ID);
            else if (e >= 0 && (x.parent != r || b >= x.kept)) atomicAdd(a.delta + e, -1);
        }
        if (x.parent != r && b < x.kept) {
            const int e = a.table[(size_t)x.parent * a.max_pages + b];
            if (is_page(a, e)) atomicAdd(a.delta + e, 1);
        }
        if (b == 0) {
            const int e = open_page(a, x);
            if (e >= 0) atomicAdd(a.opens + e, 1), atomicMax(a.owner + e, a.B - r);
        }
    }
    if (!grid_sync(a.ctl, 1)) return;

    // 2: which open pages are copied, free pages of the CTA's part
    for (int r = (int)me; r < a.B; r += (int)stride) {
        Slot x = plan_slot(a, r, false);
        const int e = open_page(a, x);
        x.copy = e >= 0 && (a.refs[e] + __ldcg(a.delta + e) > __ldcg(a.opens + e) || __ldcg(a.owner + e) != a.B - r);
        a.slots[r] = x;
    }
    const int per = (a.P + gridDim.x - 1) / gridDim.x;
    const int p0 = min(per * (int)blockIdx.x, a.P), p1 = min(p0 + per, a.P);
    int free_here = 0;
    for (int p = p0 + tid; p < p1; p += kThreads) free_here += a.refs[p] + __ldcg(a.delta + p) <= 0;
    free_here = cta_sum(free_here, s_red, lane, warp);
    if (tid == 0) __stcg(a.ctl->sums + blockIdx.x, free_here);
    if (!grid_sync(a.ctl, 2)) return;

    // 3: who gets which page
    int before, all_free;
    sums_before(a.ctl, s_red, tid, lane, warp, before, all_free);
    int asked = 0, copies = 0;
    for (int r0 = 0; r0 < a.B; r0 += kThreads) {
        const int r = r0 + tid;
        int want = 0, copy = 0;
        if (r < a.B) {
            const Slot x = a.slots[r];
            copy = x.copy, want = max(x.pages - x.kept, 0) + copy;
        }
        __syncthreads();
        const int ex = cta_excl_scan<kWarps>(want, s_scan, lane, warp);
        int sum = 0;
        for (int w = 0; w < kWarps; ++w) sum += s_scan[w];
        __syncthreads();
        const int ec = cta_excl_scan<kWarps>(copy, s_scan, lane, warp);
        int sc = 0;
        for (int w = 0; w < kWarps; ++w) sc += s_scan[w];
        if (r < a.B) s_asked[r] = asked + ex, s_copies[r] = copies + ec;
        asked += sum, copies += sc;
    }
    if (tid == 0) s_asked[a.B] = asked, s_copies[a.B] = copies;
    __syncthreads();
    const bool enough = asked <= all_free;
    if (me == 0) {
        *a.count = all_free - asked;
        if (!enough) atomicOr(&a.ctl->status, SE_DEV_NO_PAGES);
    }
    for (int q0 = p0; q0 < p1; q0 += kThreads) {
        const int p = q0 + tid;
        int refs = 0, open = 0;
        if (p < p1) {
            const int old = a.refs[p], d = __ldcg(a.delta + p);
            open = __ldcg(a.opens + p);
            refs = enough ? old + d : old;
            if (d) a.delta[p] = 0;
            if (open) a.opens[p] = 0, a.owner[p] = 0;
        }
        if (!enough) {
            if (p < p1) a.refs_out[p] = refs;
            continue;
        }
        const bool is_free = p < p1 && refs <= 0;
        __syncthreads();
        const int i = before + cta_excl_scan<kWarps>(is_free, s_scan, lane, warp);
        int sum = 0;
        for (int w = 0; w < kWarps; ++w) sum += s_scan[w];
        before += sum;
        if (p >= p1) continue;
        if (is_free) {
            refs = 0;
            if (i < asked) {
                int lo = 0, hi = a.B;                  // the last slot that begins at or before i
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (s_asked[mid] <= i) lo = mid; else hi = mid;
                }
                const Slot x = a.slots[lo];
                int j = i - s_asked[lo], b;
                if (x.copy && j == 0) {
                    b = x.keep / kPage;
                    a.copies[s_copies[lo]] = make_int2(a.table[(size_t)x.parent * a.max_pages + b], p);
                } else {
                    b = x.kept + j - x.copy;
                }
                a.table_out[(size_t)lo * a.max_pages + b] = p;
                refs = 1;
            }
        } else if (open) {
            refs -= refs > open ? open : open - 1;     // the rows that go on with a copy
        }
        a.refs_out[p] = refs;
    }
    for (uint32_t i = me; i < entries; i += stride) {
        const int r = (int)(i / (uint32_t)a.max_pages), b = (int)(i - (uint32_t)r * a.max_pages);
        if (!enough) {
            a.table_out[i] = a.table[i];
            if (b == 0) a.lens_out[r] = a.lens[r];
            continue;
        }
        const Slot x = a.slots[r];
        if (b == 0) a.lens_out[r] = x.len;
        if (x.asis) {
            a.table_out[i] = a.table[i];
        } else if (b < x.kept) {
            if (!x.copy || b != x.keep / kPage) a.table_out[i] = a.table[(size_t)x.parent * a.max_pages + b];
        } else if (b >= x.pages) {
            a.table_out[i] = -1;
        }
    }
    if (enough && copies && buf.n) {
        if (!grid_sync(a.ctl, 3)) return;
        copy_pages(buf, copies, [&](int i) { return (long long)__ldcg(&a.copies[i].x); }, [&](int i) { return (long long)__ldcg(&a.copies[i].y); },
                   s_first, lane, warp);
    }
    grid_leave(a.ctl);
}

// ---- compact -----------------------------------------------------------------------
__global__ void __launch_bounds__(kThreads, 2)
pages_compact_kernel(const __grid_constant__ CompactArgs a, const __grid_constant__ Buffers buf) {
    __shared__ int s_red[kWarps], s_scan[32], s_first[SE_MAX_PAGE_BUFFERS + 1];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (*(volatile uint32_t *)&a.ctl->needs_init) {
        if (tid == 0 && blockIdx.x == 0) atomicOr(&a.ctl->status, SE_DEV_WAIT_TIMEOUT);
        return;
    }
    const int per = (a.P + gridDim.x - 1) / gridDim.x;
    const int p0 = min(per * (int)blockIdx.x, a.P), p1 = min(p0 + per, a.P);
    int live_here = 0;
    for (int p = p0 + tid; p < p1; p += kThreads) live_here += a.refs[p] > 0;
    live_here = cta_sum(live_here, s_red, lane, warp);
    if (tid == 0) __stcg(a.ctl->sums + blockIdx.x, live_here);
    if (!grid_sync(a.ctl, 1)) return;

    int before, n;
    sums_before(a.ctl, s_red, tid, lane, warp, before, n);
    // live pages below n: those of the parts before the one that n lies in, and of that part's beginning
    int below = 0;
    {
        const int c = min(n / per, (int)gridDim.x - 1);
        const int v = tid < c ? __ldcg(a.ctl->sums + tid) : 0;
        int some = v;
        for (int p = per * c + tid; p < min(n, a.P); p += kThreads) some += a.refs[p] > 0;
        below = cta_sum(some, s_red, lane, warp);
    }
    const int moving = n - below;
    // (every CTA has read what it needs of the counts, also where they are rewritten in place: a live page's count stays above 0 and a
    // free page's at 0 until the next barrier)
    for (int q0 = p0; q0 < p1; q0 += kThreads) {
        const int p = q0 + tid;
        const int refs = p < p1 ? a.refs[p] : 0;
        const bool live = refs > 0;
        __syncthreads();
        const int i = before + cta_excl_scan<kWarps>(live, s_scan, lane, warp);
        int sum = 0;
        for (int w = 0; w < kWarps; ++w) sum += s_scan[w];
        before += sum;
        if (p >= p1) continue;
        if (p < n) {
            if (live) a.refs_out[p] = refs, a.map[p] = p;
            else a.holes[p - i] = p, a.map[p] = -1;
        } else {
            if (live) a.movers[i - below] = p, a.rank[p] = i - below;
            else a.rank[p] = -1, a.refs_out[p] = 0, a.map[p] = -1;
        }
    }
    if (tid == 0 && blockIdx.x == 0) *a.count = n;
    if (!grid_sync(a.ctl, 2)) return;

    // (B * max_pages < 2^31, so 32 bits hold an index and the step beyond the last one)
    const uint32_t entries = (uint32_t)a.B * a.max_pages, stride = gridDim.x * kThreads, me = blockIdx.x * kThreads + tid;
    for (uint32_t i = me; i < (uint32_t)moving; i += stride) {
        const int from = __ldcg(a.movers + i), to = __ldcg(a.holes + i);
        const int refs = a.refs[from];
        a.map[from] = to;
        a.refs_out[to] = refs;
        a.refs_out[from] = 0;
    }
    for (uint32_t i = me; i < entries; i += stride) {
        const int r = (int)(i / (uint32_t)a.max_pages), b = (int)(i - (uint32_t)r * a.max_pages);
        const int len = a.lens[r];
        if (b == 0 && (len < 0 || len > a.max_pages * kPage)) atomicOr(&a.ctl->status, SE_DEV_BAD_LENGTH);
        int e = a.table[i];
        if (len <= a.max_pages * kPage && b < (len + kPage - 1) / kPage) {
            if (e >= a.P) {
                atomicOr(&a.ctl->status, SE_DEV_BAD_PAGE_ID);
            } else if (e >= n) {
                const int k = __ldcg(a.rank + e);
                if (k >= 0) e = __ldcg(a.holes + k);
            }
        }
        a.table_out[i] = e;
    }
    if (moving && buf.n)
        copy_pages(buf, moving, [&](int i) { return (long long)__ldcg(a.movers + i); }, [&](int i) { return (long long)__ldcg(a.holes + i); },
                   s_first, lane, warp);
    grid_leave(a.ctl);
}

// ---- host side ---------------------------------------------------------------------
size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
struct Layout {
    size_t delta, opens, owner, slots, copies, total;
    size_t zeroed;                     // bytes from the start that are zero between calls
};
Layout layout(const se_params &p) {
    Layout l;
    const size_t pages = align256((size_t)p.num_phys_pages * 4);
    size_t at = align256(sizeof(Control));
    l.delta = at, at += pages;
    l.opens = at, at += pages;
    l.owner = at, at += pages;
    l.zeroed = at;
    // compact's scratch (three numbers per page) lies where update's slots and copies do
    l.slots = at;
    l.copies = at + align256((size_t)p.B * sizeof(Slot));
    const size_t slots = align256((size_t)p.B * sizeof(Slot)) + align256((size_t)p.B * sizeof(int2));
    l.total = at + (slots > 3 * pages ? slots : 3 * pages);
    return l;
}

void fill(Buffers &b, const se_page_buffer *buffers, int n) {
    b.n = n, b.units = 0;
    for (int k = 0; k < n; ++k) {
        b.at[k] = buffers[k];
        b.units += (int)((buffers[k].bytes_per_page + kPiece - 1) / kPiece);
    }
}

// CTAs: a barrier among few is quicker, and tables and counts of a few thousand entries keep a CTA busy for less time than a
// barrier takes; copies want every SM.
int ctas_for(long long numbers, bool copies) {
    const long long n = copies ? kCtas : (numbers + 4095) / 4096;
    return (int)(n < 1 ? 1 : n > kCtas ? kCtas : n);
}

}  // namespace

size_t pages_workspace_bytes(const se_params &p) { return layout(p).total; }
size_t pages_workspace_zeroed_bytes(const se_params &p) { return layout(p).zeroed; }

cudaError_t launch_pages_update(const se_params &p, const PagesUpdateCall &c, cudaStream_t stream) {
    const Layout l = layout(p);
    UpdateArgs a = {};
    a.table = c.page_table, a.lens = c.seq_lens, a.refs = c.ref_count, a.parent = c.parent, a.new_lens = c.new_lens;
    a.table_out = c.page_table_out, a.lens_out = c.seq_lens_out, a.refs_out = c.ref_count_out, a.count = c.free_pages;
    a.ctl = reinterpret_cast<Control *>(c.workspace);
    a.delta = reinterpret_cast<int32_t *>(c.workspace + l.delta), a.opens = reinterpret_cast<int32_t *>(c.workspace + l.opens);
    a.owner = reinterpret_cast<int32_t *>(c.workspace + l.owner), a.slots = reinterpret_cast<Slot *>(c.workspace + l.slots);
    a.copies = reinterpret_cast<int2 *>(c.workspace + l.copies);
    a.B = p.B, a.max_pages = p.max_pages, a.P = p.num_phys_pages;
    static thread_local Buffers buf;   // (8 KB)
    fill(buf, c.buffers, c.n_buffers);
    const size_t smem = (size_t)(p.B + 1) * 8;
    cudaError_t e = cudaFuncSetAttribute(pages_update_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 8193 * 8);
    if (e != cudaSuccess) return e;
    void *args[] = {&a, &buf};
    return cudaLaunchCooperativeKernel((const void *)pages_update_kernel, dim3(ctas_for((long long)p.B * p.max_pages + 2ll * p.num_phys_pages, c.n_buffers > 0)),
                                       dim3(kThreads), args, smem, stream);
}

cudaError_t launch_pages_compact(const se_params &p, const PagesCompactCall &c, cudaStream_t stream) {
    const Layout l = layout(p);
    CompactArgs a = {};
    a.table = c.page_table, a.lens = c.seq_lens, a.refs = c.ref_count;
    a.table_out = c.page_table_out, a.refs_out = c.ref_count_out, a.map = c.page_map, a.count = c.live_pages;
    a.ctl = reinterpret_cast<Control *>(c.workspace);
    const size_t pages = align256((size_t)p.num_phys_pages * 4);
    a.holes = reinterpret_cast<int32_t *>(c.workspace + l.slots), a.movers = reinterpret_cast<int32_t *>(c.workspace + l.slots + pages);
    a.rank = reinterpret_cast<int32_t *>(c.workspace + l.slots + 2 * pages);
    a.B = p.B, a.max_pages = p.max_pages, a.P = p.num_phys_pages;
    static thread_local Buffers buf;
    fill(buf, c.buffers, c.n_buffers);
    void *args[] = {&a, &buf};
    return cudaLaunchCooperativeKernel((const void *)pages_compact_kernel, dim3(ctas_for((long long)p.B * p.max_pages + 2ll * p.num_phys_pages, c.n_buffers > 0)),
                                       dim3(kThreads), args, 0, stream);
}

}  // namespace se
