// New tokens enter the cache: rotary positions for q and k, K and V written into the pages, Quest summaries of the
// touched pages brought up to date (Appendix A, Quest summary equation and the incremental-update sentence after the
// score equation; the rotation itself is the usual one of rotary position embeddings with an axis per channel pair).
//
// For token t, channel pair c of a head:  phi = positions[axis(c)][t] * inv_freq[c],
//     (x, y) -> (x cos phi - y sin phi, y cos phi + x sin phi)         in fp32, rounded once to bf16.
// A far position times a frequency needs more than 24 bits before the full turns are taken off, so phi / 2pi is formed
// and reduced in fp64 and only the remaining fraction of a turn goes to sincospif.  One (token, pair) angle serves all
// H_q + H_kv heads, so this costs 16 * rot/2 evaluations per page of 16 tokens.
//
// Work item = one touched page of one request (up to 16 new tokens, all heads), because the page's summary needs all of
// its keys.  A CTA finds its items through a prefix sum of the requests' page counts in shared memory, fills the page's
// table of angles, and deals (head of q, k or v) rows to its warps: a lane holds two 16-byte pieces of a token's
// head (the two halves of eight rotation pairs), a warp reads all 16 tokens before it computes, so 8 x 16 bytes per
// lane are in flight.  The K warps fold min and max of what they wrote, and of the page's older keys, with shuffles.
//
// Bound by HBM for prompts: 24K tokens of 32 + 2 x 8 heads, D = 128, 122 us for 662 MB = 5.4 TB/s, 0.84 of a plain copy (124-125 us
// as calls on changing inputs).  Small calls are four dependent round trips: 64 single tokens 7.7 us.  (Loading the next rows
// while a row is turned, with the registers that takes, was slower: 8.2 us where 7.2 were taken, 128.5 us for 121.5.)
#include <type_traits>

#include "se_internal.h"

namespace se {

namespace {

constexpr int kRopeThreads = 256;

struct RopeArgs {
    const uint16_t *q, *k, *v;
    long long q_stride, k_stride, v_stride;      // elements between tokens
    const int32_t *cu, *seq_lens, *page_table, *positions, *pair_axis;
    const double *inv_freq;
    uint16_t *q_out, *k_out, *k_cache, *v_cache, *meta;
    uint32_t *status;
    int B, H_q, H_kv, T, max_pages, P_phys, n_axes, rot;
};

__device__ __forceinline__ void rotate8(uint4 &lo, uint4 &hi, const float2 *cs, bool interleaved) {
    uint32_t a[4] = {lo.x, lo.y, lo.z, lo.w}, b[4] = {hi.x, hi.y, hi.z, hi.w};
    float x[8], y[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 fa = bf16x2_to_f2(a[i]), fb = bf16x2_to_f2(b[i]);
        if (interleaved) {       // neighbours are a pair: lo holds pairs 0..3, hi pairs 4..7
            x[i] = fa.x, y[i] = fa.y, x[4 + i] = fb.x, y[4 + i] = fb.y;
        } else {                 // lo holds the first members of pairs 0..7, hi the second ones
            x[2 * i] = fa.x, x[2 * i + 1] = fa.y, y[2 * i] = fb.x, y[2 * i + 1] = fb.y;
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 t = cs[i];  // (cos, sin)
        const float u = x[i] * t.x - y[i] * t.y;
        y[i] = y[i] * t.x + x[i] * t.y;
        x[i] = u;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 fa = interleaved ? make_float2(x[i], y[i]) : make_float2(x[2 * i], x[2 * i + 1]);
        const float2 fb = interleaved ? make_float2(x[4 + i], y[4 + i]) : make_float2(y[2 * i], y[2 * i + 1]);
        const __nv_bfloat162 pa = __float22bfloat162_rn(fa), pb = __float22bfloat162_rn(fb);
        a[i] = *reinterpret_cast<const uint32_t *>(&pa);
        b[i] = *reinterpret_cast<const uint32_t *>(&pb);
    }
    lo = make_uint4(a[0], a[1], a[2], a[3]);
    hi = make_uint4(b[0], b[1], b[2], b[3]);
}

__device__ __forceinline__ void fold_min(uint4 &m, const uint4 &w) {
    m.x = bmin2(m.x, w.x); m.y = bmin2(m.y, w.y); m.z = bmin2(m.z, w.z); m.w = bmin2(m.w, w.w);
}
__device__ __forceinline__ void fold_max(uint4 &m, const uint4 &w) {
    m.x = bmax2(m.x, w.x); m.y = bmax2(m.y, w.y); m.z = bmax2(m.z, w.z); m.w = bmax2(m.w, w.w);
}
__device__ __forceinline__ uint4 shfl_xor4(const uint4 &w, int m) {
    return make_uint4(__shfl_xor_sync(kFull, w.x, m), __shfl_xor_sync(kFull, w.y, m), __shfl_xor_sync(kFull, w.z, m),
                      __shfl_xor_sync(kFull, w.w, m));
}

// CTAS per SM: a CTA's latency is shorter with two (128 registers), more bytes are in flight with three (80 registers).
template <int D, bool INTERLEAVED, int CTAS>
__global__ void __launch_bounds__(kRopeThreads, CTAS)
rope_append_kernel(const RopeArgs a) {
    constexpr int LPR = D / 16;            // lanes per token: two 16-byte pieces each
    constexpr int RP = 32 / LPR;           // tokens per warp pass
    constexpr int NP = kPage / RP;         // passes per page
    constexpr int NW = kRopeThreads / 32;
    extern __shared__ int s_first[];       // [B + 1] first item of each request
    __shared__ float2 s_cs[kPage * (D / 2)];
    __shared__ int s_tot[32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;

    // items (touched pages) of every request, prefix-summed
    int carry = 0;
    for (int r0 = 0; r0 < a.B; r0 += kRopeThreads) {
        const int r = r0 + tid;
        int n = 0;
        if (r < a.B) {
            const TokenRange tr = token_range(a.cu, a.seq_lens, r, a.T, a.max_pages * kPage);
            if (!tr.valid) {
                if (blockIdx.x == 0) atomicOr(a.status, SE_DEV_BAD_LENGTH);
            } else if (tr.n > 0) {
                n = (tr.past + tr.n + kPage - 1) / kPage - tr.past / kPage;
            }
        }
        const int ex = cta_excl_scan<NW>(n, s_tot, lane, warp);
        if (r < a.B) s_first[r] = carry + ex;
        int all = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) all += s_tot[w];
        carry += all;
        __syncthreads();
    }
    if (tid == 0) s_first[a.B] = carry;
    __syncthreads();

    const int half = a.rot / 2;
    const int HR = a.H_q + 2 * a.H_kv;
    for (int it = blockIdx.x; it < carry; it += gridDim.x) {
        int lo = 0, hi = a.B;              // request r with s_first[r] <= it < s_first[r + 1]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (s_first[mid] <= it) lo = mid; else hi = mid;
        }
        const int r = lo;
        const TokenRange tr = token_range(a.cu, a.seq_lens, r, a.T, a.max_pages * kPage);
        const int b = tr.past / kPage + (it - s_first[r]);
        const int s0 = max(tr.past - b * kPage, 0);                          // first slot that receives a new token
        const int s1 = min(tr.past + tr.n - b * kPage, kPage);               // one past the last
        const long long row0 = (long long)tr.start + b * kPage - tr.past;    // row of slot 0 (may lie before the request)
        const int pid = a.page_table[(size_t)r * a.max_pages + b];
        const bool cached = pid >= 0 && pid < a.P_phys;
        if (!cached && tid == 0) atomicOr(a.status, SE_DEV_BAD_PAGE_ID);
        for (int i = tid; i < kPage * half; i += kRopeThreads) {
            const int t = i / half, c = i - t * half;
            if (t < s0 || t >= s1) continue;
            int ax = a.pair_axis[c];
            if (ax < 0 || ax >= a.n_axes) {
                atomicOr(a.status, SE_DEV_BAD_LENGTH);
                ax = 0;
            }
            const double turns = (double)a.positions[(size_t)ax * a.T + row0 + t] * a.inv_freq[c] * 0.15915494309189533577;
            float sn, cs;
            sincospif(2.f * (float)(turns - rint(turns)), &sn, &cs);
            s_cs[t * (D / 2) + c] = make_float2(cs, sn);
        }
        __syncthreads();

        const int cp = lane % LPR, tq = lane / LPR;
        const bool turned = cp < a.rot / 16;
        int c_lo, c_hi;                    // the lane's two 16-byte pieces of a head's row
        if (INTERLEAVED) c_lo = 2 * cp, c_hi = 2 * cp + 1;
        else if (turned) c_lo = cp, c_hi = cp + a.rot / 16;
        else c_lo = a.rot / 8 + 2 * (cp - a.rot / 16), c_hi = c_lo + 1;
        for (int hr = warp; hr < HR; hr += NW) {
            const bool is_q = hr < a.H_q, is_k = !is_q && hr < a.H_q + a.H_kv;
            const int h = is_q ? hr : is_k ? hr - a.H_q : hr - a.H_q - a.H_kv;
            const uint16_t *src = (is_q ? a.q : is_k ? a.k : a.v) + (size_t)h * D;
            const long long stride = is_q ? a.q_stride : is_k ? a.k_stride : a.v_stride;
            const size_t page = ((size_t)max(pid, 0) * a.H_kv + h) * (kPage * D);
            const bool want_meta = is_k && a.meta && cached;
            uint4 x[NP], y[NP];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int t = i * RP + tq;
                if (t >= s0 && t < s1) {
                    const uint4 *row = reinterpret_cast<const uint4 *>(src + (row0 + t) * stride);
                    x[i] = row[c_lo], y[i] = row[c_hi];
                } else if (want_meta && t < s0) {          // older keys of the page
                    const uint4 *row = reinterpret_cast<const uint4 *>(a.k_cache + page + (size_t)t * D);
                    x[i] = row[c_lo], y[i] = row[c_hi];
                }
            }
            uint4 mnx = make_uint4(0x7f807f80u, 0x7f807f80u, 0x7f807f80u, 0x7f807f80u), mny = mnx;   // +inf pairs
            uint4 mxx = make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u), mxy = mxx;   // -inf pairs
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int t = i * RP + tq;
                if (t >= s0 && t < s1) {
                    if ((is_q || is_k) && turned) rotate8(x[i], y[i], s_cs + t * (D / 2) + cp * 8, INTERLEAVED);
                    if (is_q || (is_k && a.k_out)) {
                        uint4 *o = reinterpret_cast<uint4 *>(is_q ? a.q_out + ((row0 + t) * a.H_q + h) * D
                                                                  : a.k_out + ((row0 + t) * a.H_kv + h) * D);
                        o[c_lo] = x[i], o[c_hi] = y[i];
                    }
                    if (!is_q && cached) {
                        uint4 *o = reinterpret_cast<uint4 *>((is_k ? a.k_cache : a.v_cache) + page + (size_t)t * D);
                        o[c_lo] = x[i], o[c_hi] = y[i];
                    }
                }
                if (want_meta && t < s1) {
                    fold_min(mnx, x[i]), fold_min(mny, y[i]);
                    fold_max(mxx, x[i]), fold_max(mxy, y[i]);
                }
            }
            if (want_meta) {
#pragma unroll
                for (int m = LPR; m < 32; m <<= 1) {
                    fold_min(mnx, shfl_xor4(mnx, m)), fold_min(mny, shfl_xor4(mny, m));
                    fold_max(mxx, shfl_xor4(mxx, m)), fold_max(mxy, shfl_xor4(mxy, m));
                }
                uint4 *mp = reinterpret_cast<uint4 *>(a.meta + ((size_t)pid * a.H_kv + h) * (2 * D));
                if (tq == 0) mp[c_lo] = mnx, mp[c_hi] = mny;
                if (tq == 1) mp[D / 8 + c_lo] = mxx, mp[D / 8 + c_hi] = mxy;
            }
        }
        __syncthreads();                   // the table of angles is refilled for the next page
    }
}

}  // namespace

cudaError_t launch_rope_append(const se_params &p, const RopeCall &c, cudaStream_t stream) {
    RopeArgs a;
    a.q = (const uint16_t *)c.q, a.k = (const uint16_t *)c.k, a.v = (const uint16_t *)c.v;
    a.q_stride = c.q_stride, a.k_stride = c.k_stride, a.v_stride = c.v_stride;
    a.cu = c.cu_seqlens, a.seq_lens = c.seq_lens, a.page_table = c.page_table, a.positions = c.positions;
    a.pair_axis = c.pair_axis, a.inv_freq = c.inv_freq;
    a.q_out = (uint16_t *)c.q_out, a.k_out = (uint16_t *)c.k_out, a.k_cache = (uint16_t *)c.k_cache;
    a.v_cache = (uint16_t *)c.v_cache, a.meta = (uint16_t *)c.meta, a.status = c.status;
    a.B = p.B, a.H_q = p.H_q, a.H_kv = p.H_kv, a.T = c.total_tokens, a.max_pages = p.max_pages;
    a.P_phys = p.num_phys_pages, a.n_axes = c.n_axes, a.rot = c.rot_dim;
    // a request touches at most ceil((n + 15) / 16) pages
    const long long items = (long long)c.total_tokens / kPage + 2ll * p.B;
    const int sms = device_sm_count();
    // Side by side, 64 single tokens: 7.2 us with two CTAs per SM, 8.4 us with three; 24K tokens of prompts: 126.8 and 121.5 us.
    // (Until each CTA has several pages the latency of one counts.)
    const bool many = items > 8ll * sms;
    const long long cap = (many ? 3ll : 2ll) * sms;
    const unsigned grid = (unsigned)(items < cap ? items : cap);
    const size_t smem = ((size_t)p.B + 1) * sizeof(int);
    auto pick = [&](auto d, auto ctas) {
        constexpr int D = decltype(d)::value, CTAS = decltype(ctas)::value;
        return c.interleaved ? rope_append_kernel<D, true, CTAS> : rope_append_kernel<D, false, CTAS>;
    };
    using Two = std::integral_constant<int, 2>;
    using Three = std::integral_constant<int, 3>;
    using D64 = std::integral_constant<int, 64>;
    using D128 = std::integral_constant<int, 128>;
    auto kern = p.D == 128 ? (many ? pick(D128{}, Three{}) : pick(D128{}, Two{})) : (many ? pick(D64{}, Three{}) : pick(D64{}, Two{}));
    kern<<<grid, kRopeThreads, smem, stream>>>(a);
    return cudaGetLastError();
}

}  // namespace se
