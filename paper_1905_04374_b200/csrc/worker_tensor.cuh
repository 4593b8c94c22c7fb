// Pieces shared by the worker-side kernels that run on the fifth-generation tensor cores in pairs of CTAs
// (clusters of two, cta_group::2): descriptors, the instructions' wrappers, the pair's barriers, TMA copies
// and tensor maps.
#pragma once
#include <cuda.h>

#include "mbar.cuh"
#include "worker_common.cuh"

namespace gar {
namespace worker {

// ---- tcgen05 ------------------------------------------------------------------------------------
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// Operand descriptor.  MN-major, 128-byte swizzle: blocks of 64 columns `lbo` bytes apart, groups of
// eight rows (of the contraction) `sbo` = 1024 bytes apart.  K-major, 128-byte swizzle: rows of 64 elements of the
// contraction, groups of eight rows `sbo` = 1024 bytes apart, lbo not looked at.  Bits [0,14) address / 16, [16,30) lbo / 16, [32,46) sbo / 16,
// [46,48) = 1 (version), [61,64) = 2 (128-byte swizzle).
__device__ __forceinline__ unsigned long long operand_desc(unsigned saddr, unsigned lbo, unsigned sbo, unsigned layout) {
    return static_cast<unsigned long long>((saddr >> 4) & 0x3fffu) | (static_cast<unsigned long long>(lbo >> 4) << 16) |
           (static_cast<unsigned long long>(sbo >> 4) << 32) | (1ull << 46) | (static_cast<unsigned long long>(layout) << 61);
}
// Instruction descriptor, kind::f16, of a pair's product of 256 rows and n columns: fp32 accumulators (1 at bit
// 4), both operands bf16 (1) or binary16 (0) at bits 7 and 10, MN-major operands (1) or K-major ones (0) at
// bits 15 and 16, N / 8 at bit 17, M / 16 at bit 24.
__host__ __device__ constexpr unsigned instruction_desc(int type, int n, bool a_mn = true, bool b_mn = true) {
    return (1u << 4) | (unsigned(type) << 7) | (unsigned(type) << 10) | (unsigned(a_mn) << 15) | (unsigned(b_mn) << 16) |
           (unsigned(n >> 3) << 17) | (256u >> 4 << 24);
}
__device__ __forceinline__ void mma_f16(unsigned d, unsigned long long a, unsigned long long b, unsigned idesc, unsigned accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// arrives on the barrier of both CTAs once the instructions issued so far have finished
__device__ __forceinline__ void mma_commit(unsigned long long* bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 ::"r"(kb_smem_u32(bar)), "h"(static_cast<unsigned short>(3)) : "memory");
}
// true in one lane of the warp
__device__ __forceinline__ bool elect_one() {
    unsigned r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
// ---- the pair -------------------------------------------------------------------------------------
__device__ __forceinline__ unsigned cta_rank() {
    unsigned r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void pair_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// this CTA's shared-memory address in CTA `rank` of the pair
__device__ __forceinline__ unsigned pair_address(unsigned addr, unsigned rank) {
    unsigned r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
// What is handed over lies in this CTA's own shared or tensor memory and is read by the tensor core
// (async proxy, after this CTA's own proxy or tcgen05 fence), so the arrival orders nothing at cluster
// scope: .release.cluster here waits for every load and store the warp has in flight, 1500 cycles a step.
__device__ __forceinline__ void arrive_at_leader(unsigned long long* bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(pair_address(kb_smem_u32(bar), 0)) : "memory");
}
// this thread's lane of tensor memory, 32 consecutive columns
__device__ __forceinline__ void tmem_ld32(unsigned taddr, float (&v)[32]) {
    unsigned r[32];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
                   "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
                   "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(taddr) : "memory");
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tma_load(unsigned dst, const CUtensorMap* map, int x, int y, int z, unsigned bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// into this CTA's shared memory, counted in on a barrier of either CTA of the pair
__device__ __forceinline__ void tma_load_pair(unsigned dst, const CUtensorMap* map, int x, int y, int z, unsigned bar) {
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}

// L2 policy of data that is not touched again: the result (738 MB for 11 workers of 4096 x 4096) passes
// through L2 without driving out the operands, which other tiles still read.
__device__ __forceinline__ unsigned long long evict_first() {
    unsigned long long p;
    asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
    return p;
}
// a piece of the result from shared memory (what lies outside the matrix is not written)
__device__ __forceinline__ void tma_store(const CUtensorMap* map, unsigned src, int x, int y, int z, unsigned long long policy) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group.L2::cache_hint [%0, {%2, %3, %4}], [%1], %5;"
                 ::"l"(map), "r"(src), "r"(x), "r"(y), "r"(z), "l"(policy) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
template <int LEFT> __device__ __forceinline__ void tma_store_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(LEFT) : "memory"); }
__device__ __forceinline__ void tma_store_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }

__device__ __forceinline__ void put_shared(unsigned at, const uint4& v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 get_shared(unsigned at) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}

// Slot of a running number in a ring of DEPTH buffers, and the parity of the slot's round.
template <int DEPTH> struct Ring {
    unsigned slot, parity;
    __device__ __forceinline__ explicit Ring(unsigned number) : slot(number % DEPTH), parity((number / DEPTH) & 1u) {}
};

// Programmatic launches: waits until the launches before this one on the stream have ended and what they wrote is there
// (at once where this one was launched plainly), then lets the next one's CTAs be set up as SMs get free.
__device__ __forceinline__ void grid_dependency() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
}

// The power of two that a coefficient (its bits, of either sign) is brought to 2^14 .. 2^15 with, and its inverse: |k| <= 120.  1 for 0, infinities and NaN.
__device__ __forceinline__ float power_for(unsigned top, bool inverse) {
    top &= 0x7fffffffu;
    if (top == 0u || top >= 0x7f800000u) return 1.f;
    const int k = max(-120, min(120, 14 - (int(top >> 23) - 127)));
    return __uint_as_float(unsigned(127 + (inverse ? -k : k)) << 23);
}

// ---- tensor maps (host) ---------------------------------------------------------------------------
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's entry point, looked up once.
inline EncodeTiled encode_tiled() {
    static const EncodeTiled found = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult how;
        const cudaError_t err = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &how);
        return err == cudaSuccess && how == cudaDriverEntryPointSuccess ? reinterpret_cast<EncodeTiled>(p) : nullptr;
    }();
    return found;
}

// [depth][rows][cols] with strides of `pitch` and `plane` bytes; boxes of box x box_rows
inline cudaError_t make_map(CUtensorMap* map, CUtensorMapDataType type, const void* base, int64_t cols, int64_t rows, int depth,
                     int64_t pitch, int64_t plane, int box, int box_rows, CUtensorMapSwizzle swizzle) {
    const EncodeTiled encode = encode_tiled();
    if (!encode) return cudaErrorNotSupported;
    const cuuint64_t dims[3] = {cuuint64_t(cols), cuuint64_t(rows), cuuint64_t(depth)};
    const cuuint64_t strides[2] = {cuuint64_t(pitch), cuuint64_t(plane)};
    const cuuint32_t boxes[3] = {cuuint32_t(box), cuuint32_t(box_rows), 1}, steps[3] = {1, 1, 1};
    const CUresult r = encode(map, type, 3, const_cast<void*>(base), dims, strides, boxes, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
                              swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}

}  // namespace worker
}  // namespace gar
