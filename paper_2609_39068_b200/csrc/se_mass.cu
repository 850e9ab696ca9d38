// Attention of a packed batch of new tokens (Appendix A, attention equations of "MHA, MQA, and GQA"), over the paged
// cache or over contiguous K and V, and the accumulated weights of a chunk (H2O accumulated score equation).
//
// First form: one warp per (token, query head) with an online softmax over the tokens it sees, and one warp per
// (cached token, kv-head) for the weights.  Right for every case, bound by its shuffles.
#include <math.h>

#include "se_internal.h"

namespace se {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

struct SimpleArgs {
    const uint16_t *q, *k, *v;
    long long q_stride, k_stride, v_stride;
    const int32_t *cu, *seq_lens, *page_table;
    uint16_t *out;
    float *lse, *accum;
    uint32_t *status;
    int B, H_q, H_kv, T, max_pages, P_phys;
    float scale_log2;
};

template <int D>
__device__ __forceinline__ void load_row(float (&x)[D / 32], const uint16_t *row, int lane) {
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
        const float2 f = bf16x2_to_f2(reinterpret_cast<const uint32_t *>(row)[i * 32 + lane]);
        x[2 * i] = f.x, x[2 * i + 1] = f.y;
    }
}

template <int D>
__device__ __forceinline__ float dot(const float (&x)[D / 32], const float (&y)[D / 32]) {
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < D / 32; ++i) s += x[i] * y[i];
#pragma unroll
    for (int m = 16; m; m >>= 1) s += __shfl_xor_sync(kFull, s, m);
    return s;
}

template <int D>
__global__ void accumulate_kernel(const SimpleArgs a) {
    const int lane = threadIdx.x & 31, G = a.H_q / a.H_kv;
    const long long w = (long long)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    const int h = (int)(w % a.H_kv), j = (int)(w / a.H_kv % (a.max_pages * kPage));
    const int r = (int)(w / a.H_kv / (a.max_pages * kPage));
    if (r >= a.B) return;
    const TokenRange tr = token_range(a.cu, a.seq_lens, r, a.T, a.max_pages * kPage);
    if (!tr.valid && lane == 0) atomicOr(a.status, SE_DEV_BAD_LENGTH);
    if (j >= tr.past + tr.n || tr.n == 0) return;
    const int pid = a.page_table[(size_t)r * a.max_pages + j / kPage];
    if (pid >= a.P_phys && lane == 0) atomicOr(a.status, SE_DEV_BAD_PAGE_ID);
    if (pid < 0 || pid >= a.P_phys) return;
    const size_t slot = ((size_t)pid * a.H_kv + h) * kPage + j % kPage;
    float k[D / 32], sum = 0.f;
    load_row<D>(k, a.k + slot * D, lane);
    for (int i = max(j - tr.past, 0); i < tr.n; ++i)
        for (int g = 0; g < G; ++g) {
            const size_t t = tr.start + i;
            float x[D / 32];
            load_row<D>(x, a.q + t * a.q_stride + (h * G + g) * D, lane);
            sum += exp2f(dot<D>(k, x) * a.scale_log2 - a.lse[t * a.H_q + h * G + g] * kLog2e);
        }
    if (lane == 0) a.accum[slot] += sum;
}

SimpleArgs simple_args(const se_params &p, const AttendCall &c) {
    SimpleArgs a = {};
    a.q = (const uint16_t *)c.q, a.k = (const uint16_t *)c.k, a.v = (const uint16_t *)c.v;
    a.q_stride = c.q_stride, a.k_stride = c.k_stride, a.v_stride = c.v_stride;
    a.cu = c.cu_seqlens, a.seq_lens = c.seq_lens, a.page_table = c.page_table;
    a.out = (uint16_t *)c.out, a.lse = c.lse, a.status = (uint32_t *)c.workspace;
    a.B = p.B, a.H_q = p.H_q, a.H_kv = p.H_kv, a.T = c.total_tokens, a.max_pages = p.max_pages;
    a.P_phys = p.num_phys_pages, a.scale_log2 = effective_scale(p) * kLog2e;
    return a;
}

}  // namespace

cudaError_t launch_h2o_accumulate(const se_params &p, const AttendCall &c, float *score_accum, cudaStream_t stream) {
    SimpleArgs a = simple_args(p, c);
    a.accum = score_accum;
    const unsigned grid = (unsigned)(((long long)p.B * p.max_pages * kPage * p.H_kv + 7) / 8);
    if (p.D == 128) accumulate_kernel<128><<<grid, 256, 0, stream>>>(a);
    else accumulate_kernel<64><<<grid, 256, 0, stream>>>(a);
    return cudaGetLastError();
}

}  // namespace se
