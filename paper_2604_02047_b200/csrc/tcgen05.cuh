// PTX of the tensor-core kernels: mbarriers, TMA loads, tcgen05 instructions and their descriptors, tensor maps.
#pragma once

#include <cuda.h>

#include "goose_internal.cuh"

namespace goose {

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(unsigned long long* bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(count));
}
__device__ __forceinline__ void mbar_arrive(unsigned long long* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx(unsigned long long* bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(unsigned long long* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(smem_u32(bar)), "r"(parity) : "memory");
    return ok != 0;
}

__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

__device__ __forceinline__ void tma_load_4d(void* dst, const CUtensorMap* map, unsigned long long* bar,
                                            int c0, int c1, int c2, int c3) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(smem_u32(dst)), "l"(map), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}
__device__ __forceinline__ void tma_load_3d_hint(void* dst, const CUtensorMap* map, unsigned long long* bar,
                                                 int c0, int c1, int c2, unsigned long long policy) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint "
                 "[%0], [%1, {%3, %4, %5}], [%2], %6;"
                 ::"r"(smem_u32(dst)), "l"(map), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2), "l"(policy) : "memory");
}
// the same by one lane of a warp that runs converged (see umma_f16_by)
__device__ __forceinline__ void tma_load_3d_hint_by(bool leader, uint32_t dst, const CUtensorMap* map, unsigned long long* bar,
                                                    int c0, int c1, int c2, unsigned long long policy) {
    asm volatile("{\n\t.reg .pred e;\n\tsetp.ne.b32 e, %7, 0;\n\t"
                 "@e cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint "
                 "[%0], [%1, {%3, %4, %5}], [%2], %6;\n\t}"
                 ::"r"(dst), "l"(map), "r"(smem_u32(bar)), "r"(c0), "r"(c1), "r"(c2), "l"(policy), "r"((uint32_t)leader) : "memory");
}
// 16 bytes into shared memory by the generic proxy: what the tensor cores read of it is behind an arrival of cp_async_arrive() and a fence_proxy_async()
// of the thread that issues the product.  there == false: zeros, and nothing is read
__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src, bool there, unsigned long long policy) {
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;"
                 ::"r"(dst), "l"(src), "r"(there ? 16 : 0), "l"(policy) : "memory");
}
// an arrival when all this thread's copies have landed
__device__ __forceinline__ void cp_async_arrive(unsigned long long* bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// brings a box of a tensor map into L2: a hint; nothing reaches the SM, and a box outside the tensor touches nothing
__device__ __forceinline__ void tma_prefetch_3d(const CUtensorMap* map, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global [%0, {%1, %2, %3}];" ::"l"(map), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
// a load that may run beside the kernel that writes the word (it returns the old or the new value)
__device__ __forceinline__ int32_t load_early(const int32_t* p) {
    int32_t v;
    asm volatile("ld.relaxed.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ int64_t load_early(const int64_t* p) {
    int64_t v;
    asm volatile("ld.relaxed.gpu.global.s64 %0, [%1];" : "=l"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ unsigned long long l2_policy_evict_first() {
    unsigned long long pol;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(pol));
    return pol;
}
__device__ __forceinline__ unsigned long long l2_policy_evict_last() {
    unsigned long long pol;
    asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(pol));
    return pol;
}
__device__ __forceinline__ void prefetch_tmap(const CUtensorMap* map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// Shared-memory matrix descriptor, 128-byte swizzle (addresses and offsets in bytes): the half that holds the address (in a
// cluster the bits above say which CTA's: cut off), to which an offset / 16 may be added as long as the sum stays in shared
// memory, and the other half, the same for all.  One descriptor a tile and additions instead of sixteen built from scratch by
// the issuing thread, and tile counts and stages carried along instead of worked out tile by tile (with 64-bit list positions
// and divisions by five), stood between a tile's arrival and its scores: attention call 512 keys 8.5 -> 8.1, 1531 11.4 -> 11.0,
// 2k 12.7 -> 12.4, 8k 28.0 -> 27.4 (32 heads), 32 over 8 heads 3k 12.2 -> 11.9, 2 x 32 over 8 16.7 -> 16.4 us, with the
// multiplication of cluster_start(), to which the clusters owe most of it.
__device__ __forceinline__ uint32_t smem_desc_lo(uint32_t addr, uint32_t lbo) { return ((addr >> 4) & 0x3FFF) | ((lbo >> 4) << 16); }
__device__ __forceinline__ uint64_t smem_desc(uint32_t lo) {
    constexpr uint32_t hi = (1024u >> 4) /*SBO: the next eight rows*/ | (1u << 14) /*descriptor version*/ | (2u << 29) /*SWIZZLE_128B*/;
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(lo), "r"(hi));
    return d;
}
// instruction descriptor: bf16 x bf16 -> fp32, M = 128, N = 128, A K-major, B K-major or MN-major
__host__ __device__ constexpr uint32_t instr_desc(bool b_mn_major) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((b_mn_major ? 1u : 0u) << 16) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
}
__device__ __forceinline__ void umma_f16(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(acc) : "memory");
}
// same, with the A operand (M x 16 bf16, two per 32-bit column, lane = row) read from tensor memory
__device__ __forceinline__ void umma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(acc) : "memory");
}
__device__ __forceinline__ void umma_commit(unsigned long long* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

// The same for a whole warp that runs converged, of which the one elected lane acts (`leader`, the same one every time: a commit covers what its
// own thread has issued).  Descriptors and addresses then live in uniform registers, where the instructions take them from; issued from
// inside a branch of one lane they are moved there one by one, some 70 cycles an instruction, more than the tensor cores need for it.
__device__ __forceinline__ bool elect_leader() {
    uint32_t e;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
    return e != 0;
}
__device__ __forceinline__ void umma_f16_by(bool leader, uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n\t.reg .pred p, e;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 e, %5, 0;\n\t"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(acc), "r"((uint32_t)leader) : "memory");
}
__device__ __forceinline__ void umma_f16_ts_by(bool leader, uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t acc) {
    asm volatile("{\n\t.reg .pred p, e;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 e, %5, 0;\n\t"
                 "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(acc), "r"((uint32_t)leader) : "memory");
}
__device__ __forceinline__ void umma_commit_by(bool leader, unsigned long long* bar) {
    asm volatile("{\n\t.reg .pred e;\n\tsetp.ne.b32 e, %1, 0;\n\t"
                 "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
                 ::"r"(smem_u32(bar)), "r"((uint32_t)leader) : "memory");
}

// the cluster's barrier: orders the partials written by its CTAs before the reads behind it
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}
#define TMEM_LD32(taddr, v, off)                                                                                      \
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "                                                            \
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"                                          \
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"                           \
                 : "=r"(v[off + 0]), "=r"(v[off + 1]), "=r"(v[off + 2]), "=r"(v[off + 3]), "=r"(v[off + 4]),          \
                   "=r"(v[off + 5]), "=r"(v[off + 6]), "=r"(v[off + 7]), "=r"(v[off + 8]), "=r"(v[off + 9]),          \
                   "=r"(v[off + 10]), "=r"(v[off + 11]), "=r"(v[off + 12]), "=r"(v[off + 13]), "=r"(v[off + 14]),     \
                   "=r"(v[off + 15]), "=r"(v[off + 16]), "=r"(v[off + 17]), "=r"(v[off + 18]), "=r"(v[off + 19]),     \
                   "=r"(v[off + 20]), "=r"(v[off + 21]), "=r"(v[off + 22]), "=r"(v[off + 23]), "=r"(v[off + 24]),     \
                   "=r"(v[off + 25]), "=r"(v[off + 26]), "=r"(v[off + 27]), "=r"(v[off + 28]), "=r"(v[off + 29]),     \
                   "=r"(v[off + 30]), "=r"(v[off + 31])                                                               \
                 : "r"(taddr))
#define TMEM_ST32(taddr, v, off)                                                                                      \
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "                                                     \
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"                                          \
                 "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"                                  \
                 ::"r"(v[off + 0]), "r"(v[off + 1]), "r"(v[off + 2]), "r"(v[off + 3]), "r"(v[off + 4]),               \
                   "r"(v[off + 5]), "r"(v[off + 6]), "r"(v[off + 7]), "r"(v[off + 8]), "r"(v[off + 9]),               \
                   "r"(v[off + 10]), "r"(v[off + 11]), "r"(v[off + 12]), "r"(v[off + 13]), "r"(v[off + 14]),          \
                   "r"(v[off + 15]), "r"(v[off + 16]), "r"(v[off + 17]), "r"(v[off + 18]), "r"(v[off + 19]),          \
                   "r"(v[off + 20]), "r"(v[off + 21]), "r"(v[off + 22]), "r"(v[off + 23]), "r"(v[off + 24]),          \
                   "r"(v[off + 25]), "r"(v[off + 26]), "r"(v[off + 27]), "r"(v[off + 28]), "r"(v[off + 29]),          \
                   "r"(v[off + 30]), "r"(v[off + 31]), "r"(taddr) : "memory")

#define TMEM_LD16(taddr, v, off)                                                                                      \
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "                                                            \
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"                                    \
                 : "=r"(v[off + 0]), "=r"(v[off + 1]), "=r"(v[off + 2]), "=r"(v[off + 3]), "=r"(v[off + 4]),          \
                   "=r"(v[off + 5]), "=r"(v[off + 6]), "=r"(v[off + 7]), "=r"(v[off + 8]), "=r"(v[off + 9]),          \
                   "=r"(v[off + 10]), "=r"(v[off + 11]), "=r"(v[off + 12]), "=r"(v[off + 13]), "=r"(v[off + 14]),     \
                   "=r"(v[off + 15])                                                                                  \
                 : "r"(taddr))
#define TMEM_ST16(taddr, v, off)                                                                                      \
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], "                                                     \
                 "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"                                           \
                 ::"r"(v[off + 0]), "r"(v[off + 1]), "r"(v[off + 2]), "r"(v[off + 3]), "r"(v[off + 4]),               \
                   "r"(v[off + 5]), "r"(v[off + 6]), "r"(v[off + 7]), "r"(v[off + 8]), "r"(v[off + 9]),               \
                   "r"(v[off + 10]), "r"(v[off + 11]), "r"(v[off + 12]), "r"(v[off + 13]), "r"(v[off + 14]),          \
                   "r"(v[off + 15]), "r"(taddr) : "memory")

__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// bf16 queries [rows][Hkv][g][128] -> 4-D map, box = 64 x g x 1 x box_rows: the g query heads of one key/value
// head for box_rows consecutive nodes, landing as rows (node, member) of one 128-byte-swizzled tile
inline bool make_q_map(void* fn, CUtensorMap* map, const void* base, int64_t rows, int Hkv, int g, int box_rows) {
    cuuint64_t dims[4] = {(cuuint64_t)kHeadDim, (cuuint64_t)g, (cuuint64_t)Hkv, (cuuint64_t)rows};
    cuuint64_t strides[3] = {(cuuint64_t)kHeadDim * 2, (cuuint64_t)g * kHeadDim * 2, (cuuint64_t)Hkv * g * kHeadDim * 2};
    cuuint32_t box[4] = {64, (cuuint32_t)g, 1, (cuuint32_t)box_rows};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    CUresult r = reinterpret_cast<EncodeTiledFn>(fn)(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base),
                                                     dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                                     CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS;
}

// bf16 tensor [rows][H][128] -> 3-D map, box = 64 x 1 x box_rows, 128-byte swizzle, zero fill out of bounds
inline bool make_map(void* fn, CUtensorMap* map, const void* base, int64_t rows, int H, int box_rows) {
    cuuint64_t dims[3] = {(cuuint64_t)kHeadDim, (cuuint64_t)H, (cuuint64_t)rows};
    cuuint64_t strides[2] = {(cuuint64_t)kHeadDim * 2, (cuuint64_t)H * kHeadDim * 2};
    cuuint32_t box[3] = {64, 1, (cuuint32_t)box_rows};
    cuuint32_t estr[3] = {1, 1, 1};
    CUresult r = reinterpret_cast<EncodeTiledFn>(fn)(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base),
                                                     dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                                     CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS;
}

}  // namespace goose
