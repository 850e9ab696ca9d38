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
// A warp takes a head of q, k or v of one touched page of one request (up to 16 new tokens), because the page's summary needs
// all of its keys.  A CTA finds its pages through a prefix sum of the requests' page counts in shared memory and fills the page's table
// of angles.  A lane holds two 16-byte pieces of a token's head (the two halves of eight rotation pairs); a warp reads all 16 tokens at
// once, 8 x 16 bytes per lane.  The K warps fold min and max of what they wrote, and of the page's older keys, with shuffles.  How the
// CTAs share the pages depends on how many there are and how full (Plan, below).
//
// Bound by HBM for prompts: 26655 tokens of 32 + 2 x 8 heads, D = 128, 114 us for 662 MB = 5.8 TB/s, 0.89 of a plain copy (116 us
// as calls on changing inputs).  Small calls are four dependent round trips: 64 single tokens 5.5 us, 6.3 with summaries.  (Angles in the
// order of their pairs, which the lanes then read from four banks: 23 % more over an 8-bit cache.)
//
// The same kernel fills a cache of e4m3 codes (KV8): a warp holds all tokens of a (page, head), so it has the page's largest
// magnitude after five shuffles, picks the power-of-two scale, quantises, and brings older codes of the page to a scale that
// has grown.  A power of two costs e4m3 no precision (its relative step is the same in every binade), makes the older codes'
// second rounding exact but for subnormal codes, and makes every dequantised value a bf16 number.  20158 tokens of prompts:
// 83 us for 459 MB (5.5 TB/s, 0.84); 20000 tokens in eight equal prompts 83.4 us, into a 16-bit cache 84.5; 64 single tokens 8.4 us.
#include <type_traits>

#include "se_internal.h"
#include "se_kv8.cuh"

namespace se {

namespace {

constexpr int kRopeThreads = 256;

// How the CTAs share the work, and what 32 + 2 x 8 heads at D = 128 with summaries took, 16-bit / 8-bit cache, in us:
//   kParts   the heads of a page are cut into equal parts for as many CTAs, two per SM: up to two pages per SM
//   kAhead   equal shares of the list of all (page, eight heads), two CTAs per SM, whose 128 registers hold a head's rows and the
//            next one's: many well filled pages at D = 128
//   kPages   a CTA takes whole pages, three CTAs per SM: many pages that get a few tokens each, whose time is that of a page's dependent
//            loads, and D = 64, where a page's rows are half the bytes
//                                   kParts         kAhead         kPages
//   64 tokens, a page each          6.3 / 8.4      7.3 / 8.7      6.5 / 7.4
//   256 tokens, a page each         9.9 / 11.9     13.5 / 14.9    12.5 / 14.9
//   2048 tokens, a page each        66 / 79        80 / 89        60 / 69
//   8 prompts of 2500 tokens        96 / 100       84.5 / 83.4    86 / 88
//   the same, 8 + 2 x 2 heads, D 64 20.9 / 22.5    20.6 / 22.3    16.2 / 17.4
enum Plan { kParts, kAhead, kPages };
template <int PLAN>
constexpr int kRopeCtas = PLAN == kPages ? 3 : 2;

struct RopeArgs {
    const uint16_t *q, *k, *v;
    long long q_stride, k_stride, v_stride;      // elements between tokens
    const int32_t *cu, *seq_lens, *page_table, *positions, *pair_axis;
    const double *inv_freq;
    uint16_t *q_out, *k_out;
    void *k_cache, *v_cache;                     // bf16, or e4m3 codes
    float *scales;                               // codes: [P_phys, H_kv, 2]
    uint16_t *meta;
    uint32_t *status;
    int B, H_q, H_kv, T, max_pages, P_phys, n_axes, rot;
    int part;                                    // kParts: groups of eight heads of a part
};

// (the angle of pair i is cs[i * STEP])
template <int STEP>
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
        const float2 t = cs[i * STEP];   // (cos, sin)
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

template <int D, bool INTERLEAVED, bool KV8, int PLAN>
__global__ void __launch_bounds__(kRopeThreads, kRopeCtas<PLAN>)
rope_append_kernel(const RopeArgs a) {
    constexpr int LPR = D / 16;            // lanes per token: two 16-byte pieces each
    constexpr int RP = 32 / LPR;           // tokens per warp pass
    constexpr int NP = kPage / RP;         // passes per page
    constexpr int NW = kRopeThreads / 32;
    extern __shared__ int s_first[];       // [B + 1] first item of each request
    // cos and sin of token t, pair c at t * kPitch + c % 8 * LPR + c / 8: the lanes of a warp, each with eight pairs in a row, read from all
    // banks (in the order of the pairs they met in four of them, which took the shared memory as long as all that the kernel does)
    constexpr int kPitch = D / 2 + LPR;
    __shared__ float2 s_cs[kPage * kPitch];
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
    const int groups = (HR + NW - 1) / NW;       // of NW heads
    [[maybe_unused]] long long u = 0, end = 0;   // kAhead: the CTA's share of the list of all (page, group)
    if constexpr (PLAN == kAhead) u = (long long)carry * groups * blockIdx.x / gridDim.x, end = (long long)carry * groups * (blockIdx.x + 1) / gridDim.x;
    for (int page = blockIdx.x; PLAN == kAhead ? u < end : page < carry; page += gridDim.x) {
        int it = page, g0 = 0, g1 = groups;
        if constexpr (PLAN == kAhead) {
            it = (int)(u / groups), g0 = (int)(u - (long long)it * groups);
            g1 = (int)min((long long)groups, g0 + (end - u));
            u += g1 - g0;
        } else if constexpr (PLAN == kParts) {
            g0 = blockIdx.y * a.part, g1 = min(g0 + a.part, groups);
        }
        const int hr0 = g0 * NW, hr1 = min(g1 * NW, HR);
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
        const int cp = lane % LPR, tq = lane / LPR;
        const bool turned = cp < a.rot / 16;
        int c_lo, c_hi;                    // the lane's two 16-byte pieces of a head's row
        if (INTERLEAVED) c_lo = 2 * cp, c_hi = 2 * cp + 1;
        else if (turned) c_lo = cp, c_hi = cp + a.rot / 16;
        else c_lo = a.rot / 8 + 2 * (cp - a.rot / 16), c_hi = c_lo + 1;
        auto fetch = [&](int hr, uint4 (&x)[NP], uint4 (&y)[NP], float &scale) {
            const bool is_q = hr < a.H_q, is_k = !is_q && hr < a.H_q + a.H_kv;
            const int h = is_q ? hr : is_k ? hr - a.H_q : hr - a.H_q - a.H_kv;
            const uint16_t *src = (is_q ? a.q : is_k ? a.k : a.v) + (size_t)h * D;
            const long long stride = is_q ? a.q_stride : is_k ? a.k_stride : a.v_stride;
            const size_t page = ((size_t)max(pid, 0) * a.H_kv + h) * (kPage * D);
            const bool old_rows = cached && (KV8 ? !is_q : is_k && a.meta);
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int t = i * RP + tq;
                if (t >= s0 && t < s1) {
                    const uint4 *row = reinterpret_cast<const uint4 *>(src + (row0 + t) * stride);
                    x[i] = row[c_lo], y[i] = row[c_hi];
                } else if (old_rows && t < s0) {                             // older tokens of the page
                    if constexpr (KV8) {
                        const uint2 *row = reinterpret_cast<const uint2 *>((const uint8_t *)(is_k ? a.k_cache : a.v_cache) + page + (size_t)t * D);
                        const uint2 u = row[c_lo], w = row[c_hi];
                        x[i] = make_uint4(u.x, u.y, 0, 0), y[i] = make_uint4(w.x, w.y, 0, 0);
                    } else {
                        const uint4 *row = reinterpret_cast<const uint4 *>((const uint16_t *)a.k_cache + page + (size_t)t * D);
                        x[i] = row[c_lo], y[i] = row[c_hi];
                    }
                }
            }
            if (KV8 && old_rows && s0 > 0) scale = a.scales[((size_t)pid * a.H_kv + h) * 2 + (is_k ? 0 : 1)];
        };
        // kAhead: the rows of a head are on their way while the warp's last head is turned, the first ones while the angles are found
        [[maybe_unused]] uint4 next_x[NP], next_y[NP];
        [[maybe_unused]] float next_scale = 0.f;
        if constexpr (PLAN == kAhead) {
            if (hr0 + warp < hr1) fetch(hr0 + warp, next_x, next_y, next_scale);
        }
        for (int i = tid; i < (hr0 < a.H_q + a.H_kv ? kPage * half : 0); i += kRopeThreads) {
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
            s_cs[t * kPitch + c % 8 * LPR + c / 8] = make_float2(cs, sn);
        }
        __syncthreads();

        for (int hr = hr0 + warp; hr < hr1; hr += NW) {
            const bool is_q = hr < a.H_q, is_k = !is_q && hr < a.H_q + a.H_kv;
            const int h = is_q ? hr : is_k ? hr - a.H_q : hr - a.H_q - a.H_kv;
            const size_t page = ((size_t)max(pid, 0) * a.H_kv + h) * (kPage * D);
            const bool want_meta = is_k && a.meta && cached;
            uint4 x[NP], y[NP];
            float old_scale = 0.f;
            if constexpr (PLAN == kAhead) {
#pragma unroll
                for (int i = 0; i < NP; ++i) x[i] = next_x[i], y[i] = next_y[i];
                old_scale = next_scale;
                if (hr + NW < hr1) fetch(hr + NW, next_x, next_y, next_scale);
            } else {
                fetch(hr, x, y, old_scale);
            }
            [[maybe_unused]] uint32_t top = 0;     // KV8: largest magnitudes so far, two bf16
            uint4 mnx = make_uint4(0x7f807f80u, 0x7f807f80u, 0x7f807f80u, 0x7f807f80u), mny = mnx;   // +inf pairs
            uint4 mxx = make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u), mxy = mxx;   // -inf pairs
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int t = i * RP + tq;
                if (t >= s0 && t < s1) {
                    if ((is_q || is_k) && turned) rotate8<LPR>(x[i], y[i], s_cs + t * kPitch + cp, INTERLEAVED);
                    if (is_q || (is_k && a.k_out)) {
                        uint4 *o = reinterpret_cast<uint4 *>(is_q ? a.q_out + ((row0 + t) * a.H_q + h) * D
                                                                  : a.k_out + ((row0 + t) * a.H_kv + h) * D);
                        o[c_lo] = x[i], o[c_hi] = y[i];
                    }
                    if constexpr (KV8) {
                        top = bmax2(top, bmax2(largest8(x[i]), largest8(y[i])));
                    } else if (!is_q && cached) {
                        uint4 *o = reinterpret_cast<uint4 *>((uint16_t *)(is_k ? a.k_cache : a.v_cache) + page + (size_t)t * D);
                        o[c_lo] = x[i], o[c_hi] = y[i];
                    }
                }
                if (!KV8 && want_meta && t < s1) {
                    fold_min(mnx, x[i]), fold_min(mny, y[i]);
                    fold_max(mxx, x[i]), fold_max(mxy, y[i]);
                }
            }
            if constexpr (KV8) {
                if (!is_q && cached) {
#pragma unroll
                    for (int m = 16; m; m >>= 1) top = bmax2(top, __shfl_xor_sync(kFull, top, m));
                    const float own = kv8_scale(max(top & 0xffffu, top >> 16));
                    const float scale = s0 > 0 ? fmaxf(old_scale, own) : own;      // (a scale that is no number counts as none)
                    const float inv = __uint_as_float(0x7f000000u - __float_as_uint(scale));     // 1 / 2^e
                    const bool grown = s0 > 0 && scale != old_scale;
                    const float again = old_scale * inv;
                    uint8_t *codes = (uint8_t *)(is_k ? a.k_cache : a.v_cache) + page;
#pragma unroll
                    for (int i = 0; i < NP; ++i) {
                        const int t = i * RP + tq;
                        if (t >= s1) continue;
                        uint2 u, w;
                        if (t >= s0) {
                            u = kv8_codes(x[i], inv), w = kv8_codes(y[i], inv);
                        } else {
                            u = make_uint2(x[i].x, x[i].y), w = make_uint2(y[i].x, y[i].y);
                            if (grown) u = kv8_again(u, again), w = kv8_again(w, again);
                        }
                        if (t >= s0 || grown) {
                            uint2 *o = reinterpret_cast<uint2 *>(codes + (size_t)t * D);
                            o[c_lo] = u, o[c_hi] = w;
                        }
                        if (want_meta) {
                            x[i] = kv8_values(u, scale), y[i] = kv8_values(w, scale);
                            fold_min(mnx, x[i]), fold_min(mny, y[i]);
                            fold_max(mxx, x[i]), fold_max(mxy, y[i]);
                        }
                    }
                    if (lane == 0) a.scales[((size_t)pid * a.H_kv + h) * 2 + (is_k ? 0 : 1)] = scale;
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
    a.q_out = (uint16_t *)c.q_out, a.k_out = (uint16_t *)c.k_out, a.k_cache = c.k_cache, a.v_cache = c.v_cache;
    a.scales = c.scales, a.meta = (uint16_t *)c.meta, a.status = c.status;
    a.B = p.B, a.H_q = p.H_q, a.H_kv = p.H_kv, a.T = c.total_tokens, a.max_pages = p.max_pages;
    a.P_phys = p.num_phys_pages, a.n_axes = c.n_axes, a.rot = c.rot_dim;
    // About as many pages as that are touched: a token per page, or a partly filled page per request.
    const int sms = device_sm_count(), groups = (p.H_q + 2 * p.H_kv + kRopeThreads / 32 - 1) / (kRopeThreads / 32);
    const long long T = c.total_tokens, pages = T < T / kPage + p.B ? T : T / kPage + p.B;
    const bool full = p.D == 128 && 2 * T >= 11 * pages;    // (5.3 tokens a page: 13.3 us whole pages, 15.4 shares; 5.8: 36 and 32)
    // (short pages: two rounds of two CTAs per SM where the second round of three would be nearly empty; 512 tokens 17.9 for 19.0 us)
    const bool two = full ? pages <= sms : pages <= 2 * sms || (pages > 3 * sms && pages <= 4 * sms);
    const int plan = two ? kParts : full ? kAhead : kPages;
    const size_t smem = ((size_t)p.B + 1) * sizeof(int);
    dim3 grid(2 * sms);
    if (plan == kParts) {
        const int most = pages < 2 * sms ? 2 * sms / (int)pages : 1;      // parts of a page, of equal size but for the last
        a.part = (groups + most - 1) / most;
        const int parts = (groups + a.part - 1) / a.part;
        // (a request's tokens may begin and end inside a page, so there may be more pages)
        const long long bound = T < T / kPage + 2ll * p.B ? T : T / kPage + 2ll * p.B, room = 2 * sms / parts;
        grid = dim3((unsigned)(bound < room ? bound : room), parts);
    } else if (plan == kPages) {
        grid = dim3(3 * sms);
    }
    auto pick = [&](auto d, auto n) {
        constexpr int D = decltype(d)::value, PLAN = decltype(n)::value;
        if (c.scales) return c.interleaved ? rope_append_kernel<D, true, true, PLAN> : rope_append_kernel<D, false, true, PLAN>;
        return c.interleaved ? rope_append_kernel<D, true, false, PLAN> : rope_append_kernel<D, false, false, PLAN>;
    };
    using D64 = std::integral_constant<int, 64>;
    using D128 = std::integral_constant<int, 128>;
    using Parts = std::integral_constant<int, kParts>;
    using Ahead = std::integral_constant<int, kAhead>;
    using Pages = std::integral_constant<int, kPages>;
    auto kern = p.D == 64 ? (plan == kParts ? pick(D64{}, Parts{}) : pick(D64{}, Pages{}))
                          : plan == kParts ? pick(D128{}, Parts{}) : plan == kAhead ? pick(D128{}, Ahead{}) : pick(D128{}, Pages{});
    kern<<<grid, kRopeThreads, smem, stream>>>(a);
    return cudaGetLastError();
}

}  // namespace se
