// Building blocks of the kernels on the fifth-generation tensor cores: tensor memory, tcgen05 PTX wrappers, operand
// and instruction descriptors, tensor copies, and waits that end for every role of a CTA once one of them gave up.
#pragma once

#include <cuda.h>

#include "se_device.cuh"

namespace se {

// Fault injection for the test of the bounded waits (a second build of the library, -DSE_TEST_SHORT_TX, never the product): a
// CTA's first copy of one kind announces 16 bytes more than it delivers, so the wait for it runs out.
#ifdef SE_TEST_SHORT_TX
constexpr uint32_t kTestExtraTx = 16;
#else
constexpr uint32_t kTestExtraTx = 0;
#endif

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// ---- tensor memory -----------------------------------------------------------------
// One warp allocates and later frees; the address of the first column lands in shared memory.
__device__ __forceinline__ void tmem_alloc(uint32_t smem_dst, uint32_t columns) {
    __syncwarp();
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_dst), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t columns) {
    __syncwarp();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(columns) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Values that an asynchronous load has delivered: no use of them moves above this point (tmem_wait_ld names no registers).
template <int N>
__device__ __forceinline__ void settle(float *v) {
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+f"(v[i]));
}

// 32 consecutive 32-bit columns of the warp's 32 lanes: lane i of the warp gets row i.  The access is one of the whole warp,
// which has to be converged; after a branch on the lane only a warp barrier makes sure of that (SYNC = false: none since the
// last one).
template <bool SYNC = true>
__device__ __forceinline__ void tmem_ld32(uint32_t addr, float *v) {
    if (SYNC) __syncwarp();
    uint32_t *r = reinterpret_cast<uint32_t *>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
}
template <bool SYNC = true>
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t *r) {
    if (SYNC) __syncwarp();
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(addr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
        "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]),
        "r"(r[31])
        : "memory");
}

// ---- matrix products ---------------------------------------------------------------
// Shared-memory operand with 128-byte swizzle: rows (K-major) or runs of 64 elements along M/N (MN-major) of 128 bytes,
// atoms of 8 rows = 1024 bytes.  `lead` is the distance in bytes between neighbouring 64-element blocks of an MN-major
// operand (not used for K-major), `stride` the distance between neighbouring atoms along the other axis.
__device__ __forceinline__ uint64_t smem_operand(uint32_t addr, uint32_t lead, uint32_t stride) {
    return (uint64_t)((addr & 0x3ffffu) >> 4) | (uint64_t)((lead >> 4) & 0x3fffu) << 16 | (uint64_t)((stride >> 4) & 0x3fffu) << 32 |
           1ull << 46 | 2ull << 61;
}
// bf16 x bf16 -> fp32, M = 128, N columns; b_mn: B is MN-major
__host__ __device__ constexpr uint32_t mma_instr(int N, bool b_mn) {
    return 1u << 4 | 1u << 7 | 1u << 10 | (b_mn ? 1u << 16 : 0u) | (uint32_t)(N >> 3) << 17 | (uint32_t)(128 >> 4) << 24;
}
// One instruction = 16 along K.  A in shared memory, or (ts) in tensor memory; issued by one thread.
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t instr, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(instr), "r"((uint32_t)accumulate)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t instr, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(instr), "r"((uint32_t)accumulate)
        : "memory");
}
// The same for e4m3 operands, both K-major; one instruction = 32 along K.  smem_codes: rows of D bytes (128- or 64-byte swizzle).
template <int D>
__device__ __forceinline__ uint64_t smem_codes(uint32_t addr) {
    return (uint64_t)((addr & 0x3ffffu) >> 4) | (uint64_t)(16 >> 4) << 16 | (uint64_t)((8 * D) >> 4) << 32 | 1ull << 46 |
           (D == 128 ? 2ull : 4ull) << 61;
}
__host__ __device__ constexpr uint32_t mma_instr_codes(int N) { return 1u << 4 | (uint32_t)(N >> 3) << 17 | (uint32_t)(128 >> 4) << 24; }
__device__ __forceinline__ void mma_ss_codes(uint32_t d, uint64_t a, uint64_t b, uint32_t instr, bool accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(instr), "r"((uint32_t)accumulate)
        : "memory");
}
// arrives on `bar` once every product issued so far by this thread is complete
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// one lane of a converged warp, always the same
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}

// ---- tensor copies -----------------------------------------------------------------
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap *map, int x, int y, int z, int w, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
        : "memory");
}
// the descriptor on its way before the first copy needs it
__device__ __forceinline__ void prefetch_map(const CUtensorMap *map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

// Wait of a warp of a role.  Gives up after 400 million cycles (200 ms at 1.97 GHz), or as soon as another role of the CTA has
// given up (*gave_up != 0, shared memory); the first one to give up reports it in the status word, and marks the workspace in
// the word behind it: the call's counters stay half counted, so no later call may use them.  False: leave the role's loop.
// The warp leaves it together: tensor copies and products take their operands from uniform registers, which lanes that ran ahead
// of the issuing lane would overwrite, and tensor memory is accessed by whole warps.  (A vote at every look took 2 to 10 % of
// the attention kernel's time.)
constexpr int kNeedsInitWord = 1;
constexpr long long kWaitLimitCycles = 400ll * 1000 * 1000;
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int *gave_up, uint32_t *status) {
    bool got = mbar_try_wait(bar, parity);
    if (!got) {
        const long long t0 = clock64();
        for (;;) {
#pragma unroll 1
            for (int it = 0; it < 64 && !got; ++it) got = mbar_try_wait(bar, parity);
            if (got || *gave_up) break;
            if (clock64() - t0 > kWaitLimitCycles) {
                *gave_up = 1;
                atomicExch(status + kNeedsInitWord, 1u);
                atomicOr(status, SE_DEV_WAIT_TIMEOUT);
                break;
            }
        }
    }
    return __all_sync(kFull, got);
}

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <int N>
__device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

// ---- tensor maps (host) --------------------------------------------------------------
typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                  CUtensorMapFloatOOBfill);

inline EncodeTiledFn encode_tiled() {
    static EncodeTiledFn fn = [] {
        void *sym = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &qres) != cudaSuccess ||
            qres != cudaDriverEntryPointSuccess)
            sym = nullptr;
        return reinterpret_cast<EncodeTiledFn>(sym);
    }();
    return fn;
}

// bf16 tensor [rows][heads][D], boxes of 64 channels x box_heads x box_rows, 128-byte swizzle, zeros outside
inline bool make_rows_map(CUtensorMap *map, const void *base, int D, long long heads, long long rows, long long stride, int box_heads,
                   int box_rows) {
    EncodeTiledFn fn = encode_tiled();
    if (!fn) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)heads, (cuuint64_t)rows};
    const cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)stride * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_heads, (cuuint32_t)box_rows};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(base), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// e4m3 codes [rows][D], boxes of whole rows x box_rows, swizzle as wide as a row, zeros outside
inline bool make_codes_map(CUtensorMap *map, const void *base, int D, long long rows, int box_rows) {
    EncodeTiledFn fn = encode_tiled();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)D, (cuuint64_t)rows};
    const cuuint64_t strides[1] = {(cuuint64_t)D};
    const cuuint32_t box[2] = {(cuuint32_t)D, (cuuint32_t)box_rows};
    const cuuint32_t estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The same tensor with the channels in blocks of 64, boxes of one head x box_rows x all blocks: [D/64][box_rows][64] in shared
// memory (the blocks are the slowest dimension of the box although their stride, 128 bytes, is the smallest).
inline bool make_split_map(CUtensorMap *map, const void *base, int D, long long heads, long long rows, long long stride, int box_rows) {
    EncodeTiledFn fn = encode_tiled();
    if (!fn) return false;
    const cuuint64_t dims[4] = {64, (cuuint64_t)heads, (cuuint64_t)rows, (cuuint64_t)(D / 64)};
    const cuuint64_t strides[3] = {(cuuint64_t)D * 2, (cuuint64_t)stride * 2, 128};
    const cuuint32_t box[4] = {64, 1, (cuuint32_t)box_rows, (cuuint32_t)(D / 64)};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(base), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace se
