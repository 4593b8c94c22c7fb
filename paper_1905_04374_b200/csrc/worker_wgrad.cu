// Per-worker weight gradients from 8-bit checkpoints (gar_worker.h): dW_w = dY_w^T X'_w, written
// into the rows of the gradient block, on the fifth-generation tensor cores.
//
// A restored activation x' is a value of dy's own 16-bit type, so the products of the two are exact
// and tcgen05.mma (kind::f16, fp32 accumulators in tensor memory) sums them in fp32.  The contraction
// runs over tokens, which are the ROWS of both matrices: both operands are "MN-major" (the output
// dimension is the contiguous one), which the tensor core takes as they lie, no transpose.
//
// Pairs of CTAs (clusters of two, one CTA per SM) take tiles of 256 outputs x 256 inputs of one
// worker, 64 tokens a step, with the paired instruction (cta_group::2): each CTA holds 128 of the
// outputs of dy and 128 of the inputs of x', and its tensor memory gets its own 128 rows of the tile.
// One CTA alone (128 x 256, restoring all 256 columns) moved 128 KB through its shared memory per step,
// 1024 cycles against the 512 of the products; a CTA of the pair moves 80.
//   dy warp        TMA: two 64-column boxes per step, 128-byte swizzle, straight into the operand
//                  layout (and the same of x', where it was restored beforehand).  The tensor maps are
//                  three-dimensional (columns, tokens, workers): what lies past a worker's tokens arrives
//                  as zeros and no other worker's rows are read
//   codes warp     TMA: one box of 128 bytes per step
//   restore warps  groups of four take steps in turn: codes -> 16-bit values (byte permute into fp32,
//                  subtract, multiply by the row group's scale, one rounding) -> operand tile in shared
//                  memory, same layout
//   MMA warp       of the leading CTA: four 256 x 256 x 16 instructions per step
//   store warps    four: tensor memory -> shared memory -> TMA stores (where the result's rows do not start on
//                  16 bytes: shifted to aligned chunks and stored plainly, store_anywhere below), while the
//                  next tile's products run into the other half of tensor memory; where a tile has many tokens,
//                  first the sum of its chunks there (Chunk, Halves below)
// The bias is one more column tile whose second operand is a block of ones.
// Four ways for the operands to come (enum Mode below), and two for the tokens: a worker's tokens are cut
// into parts, joined in order by a second kernel, where there are too few tiles for the SMs.
//
// What bounds it (B200, 1 kW cap).  Long batches: power.  4 workers x 8192
// tokens, 4096 x 4096: 1.04 to 1.07 ms = 1.03 to 1.06 PFLOP/s for bf16 rows with the pass that restores x' (61 us of
// it), 1.09 to 1.11 ms for fp32 rows; 0.86 ms = 1.28 PFLOP/s for this kernel alone, bf16 rows, before the cap lowers
// the clock to 1.2 GHz; the library's bf16 product alone takes 0.79 to 0.87 ms.  Short batches: the rows of
// the block, 11 x 512 tokens: 0.26 to 0.27 ms for 738 MB of fp32 rows (0.11 ms at the copy's rate; bf16 rows take
// 58 to 62 us less, about the time of the 369 MB they save, so the stores do not hide), 11 x 128: 0.142 to 0.157 ms.
// Small layers: latency, 7 x 100 tokens, 500 x 800 with bias: 16 us.
//
// Hand-offs are mbarriers; every wait is bounded: a wait that gives up raises an error flag, all
// roles leave their loops once what they have in flight has landed, and the CTA's tiles become NaN.
#include <cuda.h>

#include <algorithm>
#include <atomic>

#include "gar_internal.cuh"
#include "mbar.cuh"
#include "worker_common.cuh"

namespace gar {
namespace worker {
namespace {

constexpr int WG_M = 128, WG_N = 256, WG_K = 64;      // rows of a CTA, columns of a pair, tokens per step
constexpr int WG_HALF = WG_N / 2;                     // columns a CTA restores
// How the operands come.
//   WG_PLAIN_DY  the restore warps load dy (its rows do not start on 16 bytes) and restore x, step by step
//   WG_FUSED     dy by TMA
//   WG_RESTORED  both by TMA, x restored beforehand in the caller's workspace
//   WG_PANEL     at most 512 tokens, so that the restored columns of x stay in shared memory while the
//                output tiles of one worker go by: each code is restored once per CTA, and a step moves
//                dy's 16 KB alone (the other modes are bound by the 32 KB a step moves from L2, 690 cycles
//                against the products' 512)
enum Mode { WG_PLAIN_DY = 0, WG_FUSED = 1, WG_RESTORED = 2, WG_PANEL = 3 };
constexpr int WG_PANEL_STEPS = 8;                     // 512 tokens
// Steps per accumulator.  The tensor core truncates what it adds to an accumulator: the sum loses 1e-9 of itself per
// token, up to 2.8e-9 where it grows steadily (measured: 4.4e-6 at 4096 random tokens, 5.6e-6 at 2048 positive ones;
// rounded additions lose a tenth).  Sums are therefore taken in chunks, joined by rounded additions in tensor memory, so
// that the loss has a bound however many tokens there are: 768 tokens for fp32 results (7e-7, growing sums 1.3e-6), 2048
// for 16-bit ones (growing sums 6e-6, a fortieth of binary16's rounding; the same at 32768 tokens).  A join holds the products up for 2000 cycles:
// 16-bit results at 768 tokens a chunk took 3 % longer with x restored beforehand and 10 to 13 % without.
template <typename G> struct Chunk { static constexpr int STEPS = sizeof(G) == 4 ? 12 : 32; };
template <int MODE> struct Plan {
    static constexpr int A_RING = MODE == WG_RESTORED || MODE == WG_PANEL ? 5 : 4;       // steps of dy in flight
    static constexpr int B_SLOTS = MODE == WG_PANEL ? WG_PANEL_STEPS : A_RING;    // restored tiles
    // Groups of four restore warps take steps in turn.  A step takes a group about 1500 cycles from its slot
    // being free to the arrival (waits, reads, 220 instructions, fence), three times what the products take.
    // A parity tells a barrier's round from the one before, so who waits for it has to know that the last but one is
    // over.  Of the operands' slots: a group's step before, GROUPS steps ago, found its slot free, so all steps up
    // to A_RING + GROUPS ago have been consumed, and the slot's last but one was 2 A_RING ago.  Of the slots of
    // codes, which change between the groups where a bias tile (steps without codes) goes by: they are waited for after the
    // step's slot has been found free, so all steps up to A_RING ago have been consumed, with their codes, and the
    // slot's last were Q_RING or more steps ago.
    static constexpr int GROUPS = MODE == WG_RESTORED ? 1 : MODE == WG_PANEL ? 2 : 3;
    // (WG_PANEL's restore warps read codes where they lie: no time to save, and its shared memory is full)
    static constexpr int Q_RING = MODE == WG_RESTORED ? 1 : MODE == WG_PANEL ? 2 : 6;
    static constexpr int Q_BYTES = MODE == WG_RESTORED || MODE == WG_PANEL ? 16 : 64 * 128;
    static constexpr int OUT = MODE == WG_PANEL ? 1 : 2;                     // staged pieces of a store warp
    static constexpr int THREADS = 32 * (8 + 4 * GROUPS);
    static_assert(GROUPS <= A_RING, "a group knows the rounds of the operands' slots");
    static_assert(MODE == WG_RESTORED || MODE == WG_PANEL || A_RING <= Q_RING, "a group knows the rounds of the slots of codes");
};
constexpr int WG_DY_WARP = 0, WG_MMA_WARP = 1, WG_ALLOC_WARP = 2, WG_CODES_WARP = 3;
constexpr int WG_STORE_WARP0 = 4;                     // 4..7: tensor-memory lanes 32 (warp % 4) ..
constexpr int WG_RESTORE_WARP0 = 8, WG_GROUP_WARPS = 4;
constexpr int WG_BLOCK = 64 * 128;                    // bytes of 64 tokens x 64 columns of an operand
constexpr int WG_A_BYTES = WG_M / 64 * WG_BLOCK, WG_B_BYTES = WG_HALF / 64 * WG_BLOCK, WG_Q_BYTES = WG_K * WG_HALF;
constexpr int WG_GROUP_M = 8;                         // (pair) row tiles that go round a column tile together
constexpr int WG_BIAS_N = 16;

template <int MODE> struct __align__(1024) WGSmem {
    typedef Plan<MODE> P;
    uint8_t  a[P::A_RING][WG_A_BYTES];
    uint8_t  b[P::B_SLOTS][WG_B_BYTES];
    float    out[4][P::OUT][32 * 32];                     // a store warp's pieces of the tile: 32 rows of 128 bytes
    uint8_t  q[P::Q_RING][P::Q_BYTES];
    uint16_t ones[512];
    // the operand slots are read (WG_PANEL: dy's; x's are b_empty); the codes are there, are read; dy's slot is
    // the restore warps' to fill; the accumulators are complete
    unsigned long long empty[P::A_RING], b_empty[P::B_SLOTS], q_full[P::Q_RING], q_empty[P::Q_RING], late[P::A_RING], acc_full[2];
    // the leading CTA's are used, for both: the operands are there; the accumulators are read
    unsigned long long a_full[P::A_RING], b_full[P::B_SLOTS], acc_empty[2];
    unsigned tmem_base;
    int      error, other_error;                          // a wait gave up, here or in the other CTA
};

struct WGArgs {
    const void*    dy;
    const int8_t*  q;
    const float*   scales;
    const int32_t* lengths;
    void *         dw, *db;
    int64_t        tokens, out, in, ld_dy, ldq, ld_grads, pitch;     // pitch: elements between the result's rows
    int            workers, groups, group_shift;
    int            mt, nt;                // pair row tiles, column tiles (the bias tile, if any, is one more)
    int            columns;               // nt + 1 with a bias
    int            splits;                // parts a worker's tokens are cut into, each with a result of its own
    int            wide;                  // the result's rows start on 16 bytes: stored by TMA
};

// ---- tcgen05 ------------------------------------------------------------------------------------
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// Operand descriptor.  MN-major, 128-byte swizzle: blocks of 64 columns `lbo` bytes apart, groups of
// eight tokens 1024 bytes apart.  Bits [0,14) address / 16, [16,30) lbo / 16, [32,46) sbo / 16,
// [46,48) = 1 (version), [61,64) = 2 (128-byte swizzle).
__device__ __forceinline__ unsigned long long operand_desc(unsigned saddr, unsigned lbo, unsigned sbo, unsigned layout) {
    return static_cast<unsigned long long>((saddr >> 4) & 0x3fffu) | (static_cast<unsigned long long>(lbo >> 4) << 16) |
           (static_cast<unsigned long long>(sbo >> 4) << 32) | (1ull << 46) | (static_cast<unsigned long long>(layout) << 61);
}
// Instruction descriptor, kind::f16: fp32 accumulators (1 at bit 4), both operands bf16 (1) or
// binary16 (0) at bits 7 and 10, both MN-major (bits 15, 16), N / 8 at bit 17, M / 16 at bit 24.
__host__ __device__ constexpr unsigned instruction_desc(int type, int n) {
    return (1u << 4) | (unsigned(type) << 7) | (unsigned(type) << 10) | (1u << 15) | (1u << 16) | (unsigned(n >> 3) << 17) |
           (unsigned(2 * WG_M >> 4) << 24);
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
// this thread's lane of tensor memory: 16 columns of either accumulator, there once the loads are waited for
__device__ __forceinline__ void load_columns(unsigned sum, unsigned part, float (&a)[16], float (&b)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=f"(a[0]), "=f"(a[1]), "=f"(a[2]), "=f"(a[3]), "=f"(a[4]), "=f"(a[5]), "=f"(a[6]), "=f"(a[7]), "=f"(a[8]), "=f"(a[9]),
                   "=f"(a[10]), "=f"(a[11]), "=f"(a[12]), "=f"(a[13]), "=f"(a[14]), "=f"(a[15])
                 : "r"(sum) : "memory");
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=f"(b[0]), "=f"(b[1]), "=f"(b[2]), "=f"(b[3]), "=f"(b[4]), "=f"(b[5]), "=f"(b[6]), "=f"(b[7]), "=f"(b[8]), "=f"(b[9]),
                   "=f"(b[10]), "=f"(b[11]), "=f"(b[12]), "=f"(b[13]), "=f"(b[14]), "=f"(b[15])
                 : "r"(part) : "memory");
}
__device__ __forceinline__ void loads_done(float (&a)[16], float (&b)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(a[0]), "+f"(a[1]), "+f"(a[2]), "+f"(a[3]), "+f"(a[4]), "+f"(a[5]), "+f"(a[6]), "+f"(a[7]), "+f"(a[8]), "+f"(a[9]),
                   "+f"(a[10]), "+f"(a[11]), "+f"(a[12]), "+f"(a[13]), "+f"(a[14]), "+f"(a[15]), "+f"(b[0]), "+f"(b[1]), "+f"(b[2]),
                   "+f"(b[3]), "+f"(b[4]), "+f"(b[5]), "+f"(b[6]), "+f"(b[7]), "+f"(b[8]), "+f"(b[9]), "+f"(b[10]), "+f"(b[11]),
                   "+f"(b[12]), "+f"(b[13]), "+f"(b[14]), "+f"(b[15]) :: "memory");
}
__device__ __forceinline__ void store_columns(unsigned at, const float (&a)[16], const float (&b)[16]) {
    float v[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __fadd_rn(a[i], b[i]);
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
                 ::"f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]), "f"(v[10]),
                   "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]), "r"(at) : "memory");
}
// `cols` columns of `part` added to those of `sum`, rounded to nearest; the next columns' loads are in flight while
// some are added.  Not inlined: its registers are no burden on the other paths.
__device__ __noinline__ void add_accumulator(unsigned sum, unsigned part, int cols) {
    float a0[16], b0[16], a1[16], b1[16];
    load_columns(sum, part, a0, b0);
    for (int c = 0; c < cols; c += 32) {
        loads_done(a0, b0);
        load_columns(sum + unsigned(c + 16), part + unsigned(c + 16), a1, b1);
        store_columns(sum + unsigned(c), a0, b0);
        loads_done(a1, b1);
        if (c + 32 < cols) load_columns(sum + unsigned(c + 32), part + unsigned(c + 32), a0, b0);
        store_columns(sum + unsigned(c + 16), a1, b1);
    }
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
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

// ---- tiles --------------------------------------------------------------------------------------
struct Tile {
    int     worker, m, n;        // n == nt: the bias
    int     steps;               // of WG_K tokens,
    int     first;               // from this one on
    int     plane;               // the result's place among the workers (and splits)
    int64_t len;                 // the worker's tokens that count
};
__device__ __forceinline__ int64_t worker_len(const WGArgs& a, int w) {
    if (!a.lengths) return a.tokens;
    const int64_t l = a.lengths[w];
    return l < 0 ? 0 : l < a.tokens ? l : a.tokens;
}
template <int MODE>
__device__ __forceinline__ Tile tile_at(const WGArgs& a, unsigned index) {
    Tile t;
    if (MODE == WG_PANEL) {              // the output tiles of a panel (a worker's column tile) one after the other
        const unsigned panel = index / unsigned(a.mt), worker = panel / unsigned(a.columns);
        t.m = int(index - panel * unsigned(a.mt));
        t.n = int(panel - worker * unsigned(a.columns));
        t.worker = int(worker);
        t.len = a.tokens;
        t.steps = int((t.len + WG_K - 1) / WG_K);
        t.first = 0;
        t.plane = t.worker;
        return t;
    }
    const unsigned split = a.splits > 1 ? index % unsigned(a.splits) : 0u;
    if (a.splits > 1) index /= unsigned(a.splits);
    const unsigned per = unsigned(a.mt) * unsigned(a.columns), worker = index / per, r = index - worker * per;
    const unsigned per_group = WG_GROUP_M * unsigned(a.columns), g = r / per_group, in_group = r - g * per_group;
    const unsigned rows = min(unsigned(WG_GROUP_M), unsigned(a.mt) - g * WG_GROUP_M);
    t.worker = int(worker);
    t.n = int(in_group / rows);
    t.m = int(g * WG_GROUP_M + in_group - unsigned(t.n) * rows);
    t.len = worker_len(a, t.worker);
    t.steps = int((t.len + WG_K - 1) / WG_K);
    t.first = 0;
    t.plane = t.worker;
    if (a.splits > 1) {
        // equal parts of the steps a full worker has
        const int part = (int((a.tokens + WG_K - 1) / WG_K) + a.splits - 1) / a.splits;
        t.first = int(split) * part;
        t.steps = max(0, min(part, t.steps - t.first));
        t.plane = int(split) * a.workers + t.worker;
    }
    return t;
}
__device__ __forceinline__ unsigned tile_count(const WGArgs& a) { return unsigned(a.workers) * unsigned(a.mt) * unsigned(a.columns) * unsigned(a.splits); }

// The tiles of a pair: every pairs-th one, or (WG_PANEL) a run of neighbours.
struct Walk {
    unsigned first, step, end;
};
template <int MODE>
__device__ __forceinline__ Walk walk_of(const WGArgs& a, unsigned pair, unsigned pairs) {
    const unsigned tiles = tile_count(a);                   // below 2^30: first + step does not wrap
    if (MODE != WG_PANEL) return {pair, pairs, tiles};
    return {unsigned(uint64_t(tiles) * pair / pairs), 1u, unsigned(uint64_t(tiles) * (pair + 1) / pairs)};
}

// Slot of a running number in a ring of DEPTH buffers, and the parity of the slot's round.
template <int DEPTH> struct Ring {
    unsigned slot, parity;
    __device__ __forceinline__ explicit Ring(unsigned number) : slot(number % DEPTH), parity((number / DEPTH) & 1u) {}
};

// The two halves of tensor memory as accumulators.  A tile's first chunk of tokens is summed in the half `sum`, where
// the store warps keep the tile's sum; its other chunks go through the other half, one after the other.  The next
// tile's half is the other one: free once the last chunk has been added, while this tile's is still being stored.
// Every use of a half is a round of its two barriers (acc_full, acc_empty).
struct Halves {
    unsigned bits = 0;                                    // 0, 1: the parity of half 0, 1; 2: the tile's half; 3: the current one
    __device__ __forceinline__ unsigned sum() const { return (bits >> 2) & 1u; }
    __device__ __forceinline__ unsigned half() const { return bits >> 3; }
    __device__ __forceinline__ unsigned parity() const { return (bits >> half()) & 1u; }
    __device__ __forceinline__ void used() { bits ^= 1u << half(); }
    __device__ __forceinline__ void other() { bits = (bits & 7u) | (((bits & 4u) ^ 4u) << 1); }
    __device__ __forceinline__ void next_tile() { bits = ((bits ^ 4u) & 7u) | (((bits & 4u) ^ 4u) << 1); }
};

// two codes' bytes of a word -> fp32 codes -> times the scale -> a pair of T
template <typename T>
__device__ __forceinline__ unsigned restore_pair(unsigned biased, unsigned sel0, unsigned sel1, f32x2 scale) {
    const f32x2 v = pack2(__uint_as_float(__byte_perm(biased, 0x4b000000u, sel0)), __uint_as_float(__byte_perm(biased, 0x4b000000u, sel1)));
    float x, y;
    unpack2(mul2(add2(v, pack2(-8388736.f, -8388736.f)), scale), x, y);
    if constexpr (sizeof(T) == 2 && std::is_same<T, __half>::value) {
        const __half2 h = __floats2half2_rn(x, y);
        return *reinterpret_cast<const unsigned*>(&h);
    } else {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
        return *reinterpret_cast<const unsigned*>(&h);
    }
}

// dy by plain loads into the operand layout, zeros past the worker's tokens: warp `w` of a group of
// restore warps fills tokens 16 w .. 16 w + 15.  VEC: rows start on 16 bytes.
template <bool VEC>
__device__ __forceinline__ void load_dy(const WGArgs& a, const Tile& t, int64_t o0, int step, uint8_t* tile, int w, int lane) {
    const unsigned short* dy = static_cast<const unsigned short*>(a.dy);
    if (VEC) {
        uint4 v[8];
        const int c = (lane % 16) * 8;                    // eight columns of tokens 16 w + lane / 16, + 2, + 4, ..
        const int64_t o = o0 + c;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int64_t token = int64_t(step) * WG_K + 16 * w + 2 * k + lane / 16;
            const unsigned short* src = dy + (int64_t(t.worker) * a.tokens + token) * a.ld_dy + o;
            v[k] = make_uint4(0, 0, 0, 0);
            if (token < t.len && o + 8 <= a.out) {
                v[k] = __ldg(reinterpret_cast<const uint4*>(src));
            } else if (token < t.len && o < a.out) {
                unsigned h[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) h[j] = o + j < a.out ? __ldg(src + j) : 0u;
                v[k] = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
            }
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int row = 16 * w + 2 * k + lane / 16;
            *reinterpret_cast<uint4*>(tile + (c / 64) * WG_BLOCK + row * 128 + ((((c % 64) / 8) ^ (row & 7)) << 4)) = v[k];
        }
    } else {
        // eight columns at any even address: the two aligned 16-byte words around them, shifted together;
        // single elements where a word would reach beyond the matrix
        const uintptr_t begin = reinterpret_cast<uintptr_t>(dy);
        const uintptr_t end = begin + 2 * uintptr_t((int64_t(a.workers) * a.tokens - 1) * a.ld_dy + a.out);
        const int c = (lane % 16) * 8;
        const int64_t o = o0 + c;
        const unsigned short* row0 = dy + (int64_t(t.worker) * a.tokens + int64_t(step) * WG_K + 16 * w + lane / 16) * a.ld_dy + o;
#pragma unroll
        for (int k0 = 0; k0 < 8; k0 += 4) {
            uint4 x[4], y[4];
            bool words[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int64_t token = int64_t(step) * WG_K + 16 * w + 2 * (k0 + k) + lane / 16;
                const uintptr_t word = reinterpret_cast<uintptr_t>(row0 + 2 * (k0 + k) * a.ld_dy) & ~uintptr_t(15);
                words[k] = token < t.len && o + 8 <= a.out && word >= begin && word + 32 <= end;
                if (words[k]) {
                    x[k] = __ldg(reinterpret_cast<const uint4*>(word));
                    y[k] = __ldg(reinterpret_cast<const uint4*>(word) + 1);
                }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int row = 16 * w + 2 * (k0 + k) + lane / 16;
                const unsigned short* src = row0 + 2 * (k0 + k) * a.ld_dy;
                uint4 v = make_uint4(0, 0, 0, 0);
                if (words[k]) {
                    const unsigned by = unsigned(reinterpret_cast<uintptr_t>(src) & 15);
                    unsigned h[8] = {x[k].x, x[k].y, x[k].z, x[k].w, y[k].x, y[k].y, y[k].z, y[k].w};
#pragma unroll
                    for (int j = 0; j < 6; ++j) h[j] = by & 8 ? h[j + 2] : h[j];
#pragma unroll
                    for (int j = 0; j < 5; ++j) h[j] = by & 4 ? h[j + 1] : h[j];
                    const unsigned bits = (by & 2) * 8;
                    v = make_uint4(__funnelshift_r(h[0], h[1], bits), __funnelshift_r(h[1], h[2], bits), __funnelshift_r(h[2], h[3], bits),
                                   __funnelshift_r(h[3], h[4], bits));
                } else if (int64_t(step) * WG_K + row < t.len && o < a.out) {
                    unsigned h[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) h[j] = o + j < a.out ? __ldg(src + j) : 0u;
                    v = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
                }
                *reinterpret_cast<uint4*>(tile + (c / 64) * WG_BLOCK + row * 128 + ((((c % 64) / 8) ^ (row & 7)) << 4)) = v;
            }
        }
    }
}

__device__ __forceinline__ void put_shared(unsigned at, const uint4& v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 get_shared(unsigned at) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}
// The elements of a chunk at `off` bytes of a row of `bytes` bytes that lie in the row.
template <typename G>
__device__ __forceinline__ void store_elements(char* dst, const uint4& v, int off, int bytes) {
    const unsigned w[4] = {v.x, v.y, v.z, v.w};
    constexpr int SIZE = int(sizeof(G));
#pragma unroll
    for (int e = 0; e < 16 / SIZE; ++e) {
        if (off + e * SIZE < 0 || off + e * SIZE >= bytes) continue;
        if constexpr (SIZE == 4) reinterpret_cast<float*>(dst)[e] = __uint_as_float(w[e]);
        else reinterpret_cast<unsigned short*>(dst)[e] = static_cast<unsigned short>(w[e / 2] >> 16 * (e & 1));
    }
}

// This lane's row of a piece of the accumulators (128 bytes), as G.
template <typename G>
__device__ __forceinline__ void read_piece(unsigned src, bool filled, unsigned* piece) {
    float v[32];
#pragma unroll
    for (int h = 0; h < 4 / int(sizeof(G)); ++h) {
        if (filled) {
            tmem_ld32(src + unsigned(32 * h), v);
        } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = 0.f;
        }
        if constexpr (sizeof(G) == 4) {
#pragma unroll
            for (int j = 0; j < 32; ++j) piece[j] = __float_as_uint(v[j]);
        } else {
#pragma unroll
            for (int j = 0; j < 32; j += 8) {
                const float f[8] = {v[j], v[j + 1], v[j + 2], v[j + 3], v[j + 4], v[j + 5], v[j + 6], v[j + 7]};
                const uint4 p = narrow16B(f, static_cast<const G*>(nullptr));
                piece[16 * h + j / 2] = p.x;
                piece[16 * h + j / 2 + 1] = p.y;
                piece[16 * h + j / 2 + 2] = p.z;
                piece[16 * h + j / 2 + 3] = p.w;
            }
        }
    }
}

// The accumulator's rows of a warp to the result through TMA, in pieces of 128 bytes a row staged in `STAGES` buffers
// in turn (piece `n`: the running number).  Not inlined: its registers are no burden on the other paths.
template <typename G, int STAGES>
__device__ __noinline__ unsigned store_aligned(unsigned src, bool filled, unsigned stages, unsigned n, const CUtensorMap* map, int x, int y, int z, int cols) {
    const int lane = threadIdx.x % 32;
    constexpr int COLS = 128 / int(sizeof(G));
    const unsigned long long policy = evict_first();
    for (int c0 = 0; c0 < cols; c0 += COLS, ++n) {
        unsigned piece[32];
        read_piece<G>(src + unsigned(c0), filled, piece);
        // the staging buffer's last copy out has been read; 16-byte chunks in the 128-byte swizzle
        const unsigned stage = stages + n % STAGES * 4096u;
        if (lane == 0) tma_store_read<STAGES - 1>();
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j)
            put_shared(stage + lane * 128 + ((j ^ (lane & 7)) << 4), make_uint4(piece[4 * j], piece[4 * j + 1], piece[4 * j + 2], piece[4 * j + 3]));
        fence_async_smem();
        __syncwarp();
        if (lane == 0) tma_store(map, stage, x + c0, y, z, policy);
    }
    return n;
}

// The accumulator's rows of a warp (cols = `bytes` of G) to rows of the result that start anywhere, `row_bytes`
// apart: each is moved up by what its start lies behind a multiple of 32 bytes, the words that move out of a piece
// are the next one's first, and what is written are whole aligned 16-byte chunks but for the row's ends.  Not
// inlined: its registers are no burden on the other paths.  Bound by the warp's own instructions, 1600 cycles a piece.
// Measured (odd row length; in brackets TMA stores, where rows start on 16 bytes): 11 x 512 tokens, 4096 x 4096: fp32
// 327 to 331 us (261 to 265), bf16 274 to 277 (199 to 205), by single elements from the staging buffer 414 and 546; 4 x
// 4096, 2048 x 2048, fp32 166 to 169 (163 to 166); 11 x 128, 2048 x 2048, fp32 70 (43).  A row's ends by the row's lane, or by eight lanes per row in a loop
// of their own, were slower (90 and 99 us for the last).
template <typename G>
__device__ __noinline__ void store_anywhere(unsigned src, bool filled, unsigned stage, char* first, int64_t row_bytes, int bytes, int rows) {
    const int lane = threadIdx.x % 32;
    const unsigned by = unsigned(reinterpret_cast<uintptr_t>(first + lane * row_bytes)) & 31u;
    unsigned carry[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) carry[j] = 0;
    for (int at = 0; at < bytes + 31; at += 128) {
        unsigned x[40];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = carry[j];
        if (at < bytes) {
            read_piece<G>(src + unsigned(at / int(sizeof(G))), filled, x + 8);
        } else {
#pragma unroll
            for (int j = 8; j < 40; ++j) x[j] = 0;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) carry[j] = x[32 + j];
        const unsigned skip = 7u - by / 4;
#pragma unroll
        for (int j = 0; j < 36; ++j) x[j] = skip & 4 ? x[j + 4] : x[j];
#pragma unroll
        for (int j = 0; j < 34; ++j) x[j] = skip & 2 ? x[j + 2] : x[j];
#pragma unroll
        for (int j = 0; j < 33; ++j) x[j] = skip & 1 ? x[j + 1] : x[j];
        const unsigned bits = sizeof(G) == 2 && (by & 2) ? 16u : 32u;
#pragma unroll
        for (int j = 0; j < 32; ++j) x[j] = __funnelshift_rc(x[j], x[j + 1], bits);
        __syncwarp();                          // the chunks before have been read
#pragma unroll
        for (int j = 0; j < 8; ++j)
            put_shared(stage + lane * 128 + ((j ^ (lane & 7)) << 4), make_uint4(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]));
        __syncwarp();
        const int j = lane % 8;
        const unsigned from = stage + lane / 8 * 128;
        char* begin = first + lane / 8 * row_bytes;
        if (at > 0 && at + 128 <= bytes && rows == 32) {
            // no row of the piece ends in it
            uint4 v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = get_shared(from + k * 512 + ((j ^ ((4 * k + lane / 8) & 7)) << 4));
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                *reinterpret_cast<uint4*>(reinterpret_cast<char*>(reinterpret_cast<uintptr_t>(begin) & ~uintptr_t(31)) + at + 16 * j) = v[k];
                begin += 4 * row_bytes;
            }
        } else {
#pragma unroll 2
            for (int k = 0; k < 8; ++k) {
                const int off = at + 16 * j - int(reinterpret_cast<uintptr_t>(begin) & 31u);
                if (4 * k + lane / 8 < rows && off > -16 && off < bytes) {
                    const uint4 v = get_shared(from + k * 512 + ((j ^ ((4 * k + lane / 8) & 7)) << 4));
                    if (off >= 0 && off + 16 <= bytes) *reinterpret_cast<uint4*>(begin + off) = v;
                    else store_elements<G>(begin + off, v, off, bytes);
                }
                begin += 4 * row_bytes;
            }
        }
    }
}

// map_x: the codes, or (WG_RESTORED) the restored activation.  Where dy comes by TMA the restore warps
// still load a worker's last step if only some of its tokens count.
template <typename T, typename G, int MODE>
__global__ void __launch_bounds__(Plan<MODE>::THREADS, 1) weight_grad_kernel(const WGArgs a, const __grid_constant__ CUtensorMap map_dy,
                                                                          const __grid_constant__ CUtensorMap map_x,
                                                                          const __grid_constant__ CUtensorMap map_dw) {
    typedef Plan<MODE> P;
    constexpr int WG_RING = P::A_RING, WG_Q_RING = P::Q_RING, WG_GROUPS = P::GROUPS, WG_THREADS = P::THREADS;
    constexpr bool TMA_A = MODE != WG_PLAIN_DY;
    constexpr int CHUNK = Chunk<G>::STEPS;
    typedef WGSmem<MODE> Smem;
    extern __shared__ uint8_t raw[];
    Smem& sm = *reinterpret_cast<Smem*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    volatile int* error = &sm.error;
    const unsigned rank = cta_rank();
    const unsigned pair = blockIdx.x / 2, pairs = gridDim.x / 2;
    if (tid == 0) {
        sm.error = sm.other_error = 0;
        for (int k = 0; k < WG_RING; ++k) {
            kb_init(&sm.empty[k], 1);
            kb_init(&sm.a_full[k], 1);
            kb_init(&sm.late[k], 1);
        }
        for (int k = 0; k < P::B_SLOTS; ++k) {
            kb_init(&sm.b_empty[k], 1);
            kb_init(&sm.b_full[k], 2 * WG_GROUP_WARPS);
        }
        for (int k = 0; k < WG_Q_RING; ++k) {
            kb_init(&sm.q_full[k], 1);
            kb_init(&sm.q_empty[k], WG_GROUP_WARPS);
        }
        for (int b = 0; b < 2; ++b) {
            kb_init(&sm.acc_full[b], 1);
            kb_init(&sm.acc_empty[b], 8);
        }
        kb_fence_init();
    }
    if (tid == 32) {
        prefetch_map(&map_x);
        if (TMA_A) prefetch_map(&map_dy);
        if (a.wide) prefetch_map(&map_dw);
    }
    for (int i = tid; i < 512; i += WG_THREADS) sm.ones[i] = std::is_same<T, __half>::value ? 0x3c00 : 0x3f80;
    fence_async_smem();
    if (warp == WG_ALLOC_WARP) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(kb_smem_u32(&sm.tmem_base)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    pair_sync();                              // the other CTA's barriers are initialised
    tc_fence_after();
    const unsigned tmem = sm.tmem_base;
    const Walk walk = walk_of<MODE>(a, pair, pairs);
    // step s of a tile is number g + s of all the CTA's steps; of those with codes, number gq + s
    unsigned g = 0, gq = 0;
    bool ok = true;

    if (warp == WG_DY_WARP) {
        if (TMA_A && lane == 0) {
            const unsigned leader_full = pair_address(kb_smem_u32(sm.a_full), 0);
            unsigned n_late = 0;
            for (unsigned i = walk.first; ok && i < walk.end; i += walk.step) {
                const Tile t = tile_at<MODE>(a, i);
                const int o0 = (2 * t.m + int(rank)) * WG_M;
                for (int s = 0; s < t.steps; ++s, ++g) {
                    const Ring<WG_RING> r(g);
                    if (!kb_wait(kb_smem_u32(&sm.empty[r.slot]), r.parity ^ 1u, error)) { ok = false; break; }
                    // dy's part of a step that the restore warps load is missing; a bias tile has no x
                    const int step = t.first + s;
                    const bool copy_dy = !(a.lengths && int64_t(step + 1) * WG_K > t.len), copy_x = MODE == WG_RESTORED && t.n < a.nt;
                    const unsigned bytes = (copy_dy ? WG_A_BYTES : 0) + (copy_x ? WG_B_BYTES : 0);
                    if (MODE == WG_RESTORED && !copy_dy) kb_arrive(&sm.late[n_late++ % WG_RING]);
                    if (rank == 0) {
                        if (bytes) kb_expect_tx(kb_smem_u32(&sm.a_full[r.slot]), 2 * bytes);
                        else kb_arrive(&sm.a_full[r.slot]);
                    }
                    const unsigned bar = leader_full + r.slot * 8;
                    if (copy_dy) {
                        const unsigned dst = kb_smem_u32(sm.a[r.slot]);
                        tma_load_pair(dst, &map_dy, o0, step * WG_K, t.worker, bar);
                        tma_load_pair(dst + WG_BLOCK, &map_dy, o0 + 64, step * WG_K, t.worker, bar);
                    }
                    if (copy_x) {
                        const unsigned dst = kb_smem_u32(sm.b[r.slot]);
                        const int c0 = t.n * WG_N + int(rank) * WG_HALF;
                        tma_load_pair(dst, &map_x, c0, step * WG_K, t.worker, bar);
                        tma_load_pair(dst + WG_BLOCK, &map_x, c0 + 64, step * WG_K, t.worker, bar);
                    }
                }
            }
            // after a wait that gave up: the copies in flight land (the leading CTA counts them in) before
            // either CTA's shared memory is given back
            for (unsigned k = 0; !ok && rank == 0 && k < WG_RING && k < g; ++k) {
                const Ring<WG_RING> r(g - 1 - k);
                kb_wait(kb_smem_u32(&sm.a_full[r.slot]), r.parity, error, true, 1u << 10);
            }
        }
    } else if (warp == WG_CODES_WARP) {
        if (MODE != WG_RESTORED && MODE != WG_PANEL && lane == 0) {
            for (unsigned i = walk.first; ok && i < walk.end; i += walk.step) {
                const Tile t = tile_at<MODE>(a, i);
                if (t.n == a.nt) continue;
                for (int s = 0; s < t.steps; ++s, ++gq) {
                    const Ring<WG_Q_RING> r(gq);
                    if (!kb_wait(kb_smem_u32(&sm.q_empty[r.slot]), r.parity ^ 1u, error)) { ok = false; break; }
                    const unsigned bar = kb_smem_u32(&sm.q_full[r.slot]);
                    kb_expect_tx(bar, WG_Q_BYTES);
                    tma_load(kb_smem_u32(sm.q[r.slot]), &map_x, t.n * WG_N + int(rank) * WG_HALF, (t.first + s) * WG_K, t.worker, bar);
                }
            }
            for (unsigned k = 0; !ok && k < WG_Q_RING && k < gq; ++k) {
                const Ring<WG_Q_RING> r(gq - 1 - k);
                kb_wait(kb_smem_u32(&sm.q_full[r.slot]), r.parity, error, true, 1u << 10);
            }
        }
    } else if (warp == WG_MMA_WARP) {
        // The whole warp walks the loop and one elected lane issues: what the instructions take is then the
        // same in every lane, and the compiler keeps it where they read it from.
        if (rank == 0) {
            const unsigned idesc = instruction_desc(std::is_same<T, __half>::value ? 0 : 1, WG_N);
            const unsigned idesc_bias = instruction_desc(std::is_same<T, __half>::value ? 0 : 1, WG_BIAS_N);
            const unsigned long long desc_a = operand_desc(kb_smem_u32(sm.a), WG_BLOCK, 1024, 2);
            const unsigned long long desc_b = operand_desc(kb_smem_u32(sm.b), WG_BLOCK, 1024, 2);
            // a block of ones needs no layout: every address the descriptor reaches holds 1
            const unsigned long long desc_ones = operand_desc(kb_smem_u32(sm.ones), 256, 256, 0);
            unsigned n_late = 0, panels = 0;
            Halves acc;
            for (unsigned i = walk.first; ok && i < walk.end; i += walk.step) {
                const Tile t = tile_at<MODE>(a, i);
                const int steps = __shfl_sync(0xffffffffu, t.steps, 0);
                const bool partial = t.len % WG_K != 0;
                const bool bias = t.n == a.nt;
                const bool panel_first = i == walk.first || t.m == 0, panel_last = i + 1 == walk.end || t.m + 1 == a.mt;
                unsigned d = 0;
                int begun = 0;                                   // the accumulator's first step
                for (int s = 0; s < steps; ++s, ++g) {
                    const Ring<WG_RING> r(g);
                    if (s == 0 || s - begun == CHUNK) {
                        // on to the tile's half, or from the chunk before to the other one
                        if (s > 0) {
                            if (elect_one()) mma_commit(&sm.acc_full[acc.half()]);
                            __syncwarp();
                            acc.used();
                            acc.other();
                        }
                        if (!kb_wait_warp(kb_smem_u32(&sm.acc_empty[acc.half()]), acc.parity() ^ 1u, error)) { ok = false; break; }
                        tc_fence_after();
                        d = tmem + acc.half() * WG_N;
                        begun = s;
                    }
                    if (TMA_A && !kb_wait_warp(kb_smem_u32(&sm.a_full[r.slot]), r.parity, error)) { ok = false; break; }
                    if (MODE == WG_PANEL) {
                        if (panel_first && !bias && !kb_wait_warp(kb_smem_u32(&sm.b_full[s]), panels & 1u, error)) { ok = false; break; }
                    } else if (MODE != WG_RESTORED && !kb_wait_warp(kb_smem_u32(&sm.b_full[r.slot]), r.parity, error)) {
                        ok = false;
                        break;
                    }
                    if (MODE == WG_RESTORED && a.lengths && s + 1 == steps && partial) {
                        const Ring<WG_RING> late(n_late++);
                        if (!kb_wait_warp(kb_smem_u32(&sm.b_full[late.slot]), late.parity, error)) { ok = false; break; }
                    }
                    tc_fence_after();
                    // 16 tokens are 2048 bytes; addresses count 16 bytes
                    const unsigned long long da = desc_a + r.slot * (WG_A_BYTES / 16);
                    const unsigned long long db = bias ? desc_ones : desc_b + (MODE == WG_PANEL ? unsigned(s) : r.slot) * (WG_B_BYTES / 16);
                    const unsigned kind = bias ? idesc_bias : idesc, db_step = bias ? 0u : 128u;
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < WG_K / 16; ++k) mma_f16(d, da + k * 128u, db + k * db_step, kind, s > begun || k > 0);
                        mma_commit(&sm.empty[r.slot]);
                        if (MODE == WG_PANEL && panel_last && !bias) mma_commit(&sm.b_empty[s]);
                    }
                    __syncwarp();
                }
                if (MODE == WG_PANEL && panel_last && !bias) ++panels;
                if (ok && steps > 0) {
                    if (elect_one()) mma_commit(&sm.acc_full[acc.half()]);
                    __syncwarp();
                    acc.used();
                    acc.next_tile();
                }
            }
            // nothing is in flight when the tensor memory is freed: on the good path the store warps have
            // seen every accumulator; after a wait that gave up, wait for what was issued
            if (!ok) {
                if (elect_one()) mma_commit(&sm.acc_full[acc.half()]);
                __syncwarp();
                kb_wait(kb_smem_u32(&sm.acc_full[acc.half()]), acc.parity(), error, true, 1u << 10);
            }
        }
    } else if (warp >= WG_RESTORE_WARP0 && MODE == WG_RESTORED) {
        // Only dy's last step of a worker whose length ends inside it.  These steps go round barriers on a
        // count of their own, and the dy warp says when the slot is free: a parity cannot be waited for by
        // who does not follow the slot from round to round.
        const int w = warp - WG_RESTORE_WARP0;
        unsigned n_late = 0;
        for (unsigned i = walk.first; a.lengths && i < walk.end; i += walk.step) {
            const Tile t = tile_at<MODE>(a, i);
            g += t.steps;
            if (t.len % WG_K == 0) continue;
            const Ring<WG_RING> r(g - 1), late(n_late++);
            if (!kb_wait_warp(kb_smem_u32(&sm.late[late.slot]), late.parity, error)) { ok = false; break; }
            load_dy<true>(a, t, int64_t(2 * t.m + int(rank)) * WG_M, t.steps - 1, sm.a[r.slot], w, lane);
            fence_async_smem();
            __syncwarp();
            if (lane == 0) arrive_at_leader(&sm.b_full[late.slot]);
        }
    } else if (warp >= WG_RESTORE_WARP0) {
        const int w = (warp - WG_RESTORE_WARP0) % WG_GROUP_WARPS, tl = lane & 7, sub = lane >> 3;
        const unsigned mine = unsigned(warp - WG_RESTORE_WARP0) / WG_GROUP_WARPS;
        const int row = 16 * w + tl;                              // this lane's tokens of a step: row and row + 8
        // the lane's two 16-column pieces of a row: a diagonal over the eight lanes of a phase, so that
        // neither the reads of the codes nor the swizzled stores meet in a bank
        const int piece[2] = {(tl + sub) & 7, (tl + sub + 4) & 7};
        const int q_at = row * WG_HALF;
        int b_at[2][2];                                           // the two halves of a piece in the operand tile
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                b_at[k][h] = row * 128 + (piece[k] >> 2) * WG_BLOCK + ((((piece[k] & 3) * 2 + h) ^ tl) << 4);
        unsigned panels = 0;
        for (unsigned i = walk.first; ok && i < walk.end; i += walk.step) {
            const Tile t = tile_at<MODE>(a, i);
            const bool bias = t.n == a.nt;
            if (MODE == WG_PANEL && (bias || (i != walk.first && t.m != 0))) continue;
            const int64_t c0 = int64_t(t.n) * WG_N + rank * WG_HALF;
            const int len = int(t.len);
            const float* scale_at[2];                             // of the first row, for each piece
            bool inside[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int64_t group = (c0 + piece[k] * 16) >> a.group_shift;
                inside[k] = !bias && group < a.groups;
                scale_at[k] = a.scales + (int64_t(t.worker) * a.tokens + row) * a.groups + group;
            }
            float next[4];
            auto fetch_scales = [&](int s) {
                const int64_t at = int64_t(t.first + s) * WG_K * a.groups;
                const int token = (t.first + s) * WG_K + row;
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    next[k] = inside[k & 1] && token + 8 * (k >> 1) < len ? __ldg(scale_at[k & 1] + at + 8 * (k >> 1) * a.groups) : 0.f;
            };
            // this group's first step of the tile; of a panel the group takes the same slots every time
            int s = MODE == WG_PANEL ? int(mine) : int((mine + WG_GROUPS - g % WG_GROUPS) % WG_GROUPS);
            if (s < t.steps) fetch_scales(s);
            bool ready = false;                                   // the step's slots have been seen free and filled
            for (; s < t.steps; s += WG_GROUPS) {
                Ring<WG_RING> r(g + s);
                Ring<WG_Q_RING> rq(gq + s);
                unsigned long long* free_slot = &sm.empty[r.slot % WG_RING];
                if (MODE == WG_PANEL) {
                    r.slot = unsigned(s);
                    r.parity = panels & 1u;
                    free_slot = &sm.b_empty[s];
                }
                float scale[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) scale[k] = next[k];
                if (s + WG_GROUPS < t.steps) fetch_scales(s + WG_GROUPS);
                uint4 c[4];
                if (MODE == WG_PANEL) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int token = s * WG_K + row + 8 * (k >> 1);
                        const int64_t col = c0 + piece[k & 1] * 16;
                        c[k] = make_uint4(0, 0, 0, 0);
                        if (token < len && col < a.in)       // rows of codes are padded to 16
                            c[k] = __ldg(reinterpret_cast<const uint4*>(a.q + (int64_t(t.worker) * a.tokens + token) * a.ldq + col));
                    }
                }
                if (!__all_sync(0xffffffffu, ready)) {
                    if (!kb_wait_warp(kb_smem_u32(free_slot), r.parity ^ 1u, error)) { ok = false; break; }
                    if (MODE != WG_PANEL && !bias && !kb_wait_warp(kb_smem_u32(&sm.q_full[rq.slot]), rq.parity, error)) { ok = false; break; }
                }
                if (MODE != WG_PANEL) {
                    // asked early, so that the answer is there when the next step of this group begins
                    const Ring<WG_RING> r2(g + s + WG_GROUPS);
                    const Ring<WG_Q_RING> rq2(gq + s + WG_GROUPS);
                    ready = s + WG_GROUPS < t.steps && !bias;
                    if (ready) {
                        const bool free = kb_test(kb_smem_u32(&sm.empty[r2.slot]), r2.parity ^ 1u);      // first: see Plan
                        ready = kb_test(kb_smem_u32(&sm.q_full[rq2.slot]), rq2.parity) & free;
                    }
                }
                if (!bias) {
                    const uint8_t* q = sm.q[rq.slot] + q_at;
                    uint8_t* b = sm.b[r.slot];
#pragma unroll
                    for (int k = 0; MODE != WG_PANEL && k < 4; ++k) c[k] = *reinterpret_cast<const uint4*>(q + (k >> 1) * 8 * WG_HALF + piece[k & 1] * 16);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const unsigned words[4] = {c[k].x ^ 0x80808080u, c[k].y ^ 0x80808080u, c[k].z ^ 0x80808080u, c[k].w ^ 0x80808080u};
                        const f32x2 sc = pack2(scale[k], scale[k]);
                        unsigned v[8];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            v[2 * j] = restore_pair<T>(words[j], 0x7440, 0x7441, sc);
                            v[2 * j + 1] = restore_pair<T>(words[j], 0x7442, 0x7443, sc);
                        }
                        *reinterpret_cast<uint4*>(b + (k >> 1) * 1024 + b_at[k & 1][0]) = make_uint4(v[0], v[1], v[2], v[3]);
                        *reinterpret_cast<uint4*>(b + (k >> 1) * 1024 + b_at[k & 1][1]) = make_uint4(v[4], v[5], v[6], v[7]);
                    }
                }
                const int64_t o0 = int64_t(2 * t.m + int(rank)) * WG_M;
                if (!TMA_A) load_dy<false>(a, t, o0, t.first + s, sm.a[r.slot], w, lane);
                else if (MODE != WG_PANEL && a.lengths && (t.first + s + 1) * WG_K > len) load_dy<true>(a, t, o0, t.first + s, sm.a[r.slot], w, lane);
                fence_async_smem();
                __syncwarp();
                if (lane == 0) {
                    arrive_at_leader(&sm.b_full[r.slot]);
                    if (MODE != WG_PANEL && !bias) kb_arrive(&sm.q_empty[rq.slot]);
                }
            }
            g += t.steps;
            if (!bias) gq += t.steps;
            ++panels;
        }
    } else if (warp >= WG_STORE_WARP0) {
        const int quarter = warp - WG_STORE_WARP0;               // == warp % 4: tensor-memory lanes 32 quarter ..
        unsigned n_piece = 0;
        Halves acc;
        for (unsigned i = walk.first; ok && i < walk.end; i += walk.step) {
            const Tile t = tile_at<MODE>(a, i);
            const int64_t o0 = int64_t(2 * t.m + int(rank)) * WG_M + quarter * 32;
            // the chunks of tokens in order, the later ones added to the first; a worker without tokens has none
            for (int s0 = 0; s0 < t.steps; s0 += CHUNK) {
                if (s0 > 0) acc.other();
                if (!kb_wait_warp(kb_smem_u32(&sm.acc_full[acc.half()]), acc.parity(), error)) { ok = false; break; }
                tc_fence_after();
                if (s0 == 0) {
                    acc.used();                                  // given back below, once it is stored
                    continue;
                }
                // what lies outside the matrix is added too and never stored
                add_accumulator(tmem + acc.sum() * WG_N + (unsigned(quarter * 32) << 16), tmem + acc.half() * WG_N + (unsigned(quarter * 32) << 16), t.n == a.nt ? 32 : WG_N);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) arrive_at_leader(&sm.acc_empty[acc.half()]);
                acc.used();
            }
            if (!ok) break;
            const unsigned src = tmem + acc.sum() * WG_N + (unsigned(quarter * 32) << 16);
            if (t.n == a.nt) {
                float v[32];
                if (t.steps) tmem_ld32(src, v);
                else v[0] = 0.f;
                if (o0 + lane < a.out) static_cast<G*>(a.db)[int64_t(t.plane) * a.ld_grads + o0 + lane] = Elem<G>::narrow(v[0]);
            } else {
                const int rows = int(min(int64_t(32), a.out - o0));
                const int64_t left = a.in - int64_t(t.n) * WG_N;
                const int cols = left < WG_N ? int(left) : WG_N;
                G* dw = static_cast<G*>(a.dw) + int64_t(t.plane) * a.ld_grads + o0 * a.pitch + int64_t(t.n) * WG_N;
                if (a.wide) {
                    if (rows > 0) n_piece = store_aligned<G, P::OUT>(src, t.steps > 0, kb_smem_u32(sm.out[quarter][0]), n_piece, &map_dw, t.n * WG_N, int(o0), t.plane, cols);
                } else if (rows > 0) {
                    store_anywhere<G>(src, t.steps > 0, kb_smem_u32(sm.out[quarter][0]), reinterpret_cast<char*>(dw),
                                      a.pitch * int64_t(sizeof(G)), cols * int(sizeof(G)), rows);
                }
            }
            if (t.steps) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) arrive_at_leader(&sm.acc_empty[acc.sum()]);
                acc.next_tile();
            }
        }
        if (lane == 0) tma_store_done();
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (tid == 0 && sm.error)
        asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(pair_address(kb_smem_u32(&sm.other_error), rank ^ 1u)), "r"(1) : "memory");
    __syncwarp();
    pair_sync();                              // the other CTA's products and arrivals have ended too
    tc_fence_after();
    if (warp == WG_ALLOC_WARP)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    if (sm.error || *static_cast<volatile int*>(&sm.other_error)) {
        // a wait gave up: nothing the pair was to write may look like a gradient
        for (unsigned i = walk.first; i < walk.end; i += walk.step) {
            const Tile t = tile_at<MODE>(a, i);
            for (int e = tid; e < WG_M * WG_N; e += WG_THREADS) {
                const int64_t o = int64_t(2 * t.m + int(rank)) * WG_M + e / WG_N, c = int64_t(t.n) * WG_N + e % WG_N;
                if (o >= a.out) continue;
                if (t.n == a.nt) {
                    if (e % WG_N == 0) static_cast<G*>(a.db)[int64_t(t.plane) * a.ld_grads + o] = Elem<G>::narrow(CUDART_NAN_F);
                } else if (c < a.in) {
                    static_cast<G*>(a.dw)[int64_t(t.plane) * a.ld_grads + o * a.pitch + c] = Elem<G>::narrow(CUDART_NAN_F);
                }
            }
        }
    }
}

// Rows of 16-bit elements copied to rows that start on 16 bytes (zeros behind the last column), eight
// elements per thread and turn.
__global__ void __launch_bounds__(256) align_rows_kernel(const unsigned short* src, int64_t ld, int64_t cols, int64_t pieces,
                                                         uint4* dst, int64_t per_row) {
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < pieces; i += int64_t(gridDim.x) * 256) {
        const int64_t row = i / per_row, c = (i - row * per_row) * 8;
        const unsigned short* p = src + row * ld + c;
        unsigned v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c + j < cols ? __ldg(p + j) : 0u;
        dst[i] = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
    }
}

// The parts of a cut worker (WGArgs.splits), added in order and rounded once: column c of row r of the
// result, c == in: the bias.
template <typename G>
__global__ void __launch_bounds__(128) join_parts_kernel(const float* parts, int64_t plane, int64_t pitch, int splits, int workers, int64_t out,
                                                         int64_t in, G* dw, G* db, int64_t ld) {
    const int64_t c = int64_t(blockIdx.x) * 128 + threadIdx.x, row = blockIdx.y, w = row / out, o = row - w * out;
    if (c > in || (c == in && !db)) return;
    const float* p = parts + w * plane + (c < in ? o * pitch + c : out * pitch + o);
    float sum = p[0];
    for (int k = 1; k < splits; ++k) sum += p[int64_t(k) * workers * plane];
    if (c < in) dw[w * ld + o * in + c] = Elem<G>::narrow(sum);
    else db[w * ld + o] = Elem<G>::narrow(sum);
}

// ---- launch -------------------------------------------------------------------------------------
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's entry point, looked up once.
EncodeTiled encode_tiled() {
    static const EncodeTiled found = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult how;
        const cudaError_t err = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &how);
        return err == cudaSuccess && how == cudaDriverEntryPointSuccess ? reinterpret_cast<EncodeTiled>(p) : nullptr;
    }();
    return found;
}

// [depth][rows][cols] with strides of `pitch` and `plane` bytes; boxes of box x box_rows
cudaError_t make_map(CUtensorMap* map, CUtensorMapDataType type, const void* base, int64_t cols, int64_t rows, int depth,
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
// the workers' tokens (at least one row, so that the map is valid; none is read without tokens)
cudaError_t make_token_map(CUtensorMap* map, CUtensorMapDataType type, const void* base, int64_t cols, int64_t tokens, int workers,
                           int64_t pitch, int box, CUtensorMapSwizzle swizzle) {
    const int64_t rows = tokens > 0 ? tokens : 1;
    return make_map(map, type, base, cols, rows, workers, pitch, pitch * rows, box, WG_K, swizzle);
}

template <typename T, typename G, int MODE>
cudaError_t launch(const WGArgs& a, const CUtensorMap& map_dy, const CUtensorMap& map_x, const CUtensorMap& map_dw, int sm_count, cudaStream_t stream) {
    constexpr int bytes = int(sizeof(WGSmem<MODE>)) + 1024;
    static_assert(bytes <= 232448, "a CTA's shared memory");
    auto kernel = weight_grad_kernel<T, G, MODE>;
    static std::atomic<uint64_t> allowed{0};           // devices on which the kernel may have that much
    int dev = 0;
    if (cudaError_t err = cudaGetDevice(&dev)) return err;
    if (dev >= 64 || !(allowed.load(std::memory_order_relaxed) >> dev & 1)) {
        if (cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes)) return err;
        if (dev < 64) allowed.fetch_or(uint64_t(1) << dev, std::memory_order_relaxed);
    }
    if (MODE == WG_PANEL && a.splits != 1) return cudaErrorInvalidConfiguration;      // its tiles know no parts
    const int64_t tiles = int64_t(a.workers) * a.mt * a.columns * a.splits;
    const int64_t pairs = sm_count / 2 > 1 ? sm_count / 2 : 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(unsigned(2 * (tiles < pairs ? tiles : pairs)));
    cfg.blockDim = dim3(Plan<MODE>::THREADS);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a, map_dy, map_x, map_dw);
}
template <typename T, int MODE>
cudaError_t launch_by_grads(int grads_dtype, const WGArgs& a, const CUtensorMap& map_dy, const CUtensorMap& map_x, const CUtensorMap& map_dw, int sm_count,
                            cudaStream_t stream) {
    if (grads_dtype == GAR_F32) return launch<T, float, MODE>(a, map_dy, map_x, map_dw, sm_count, stream);
    if (grads_dtype == GAR_BF16) return launch<T, __nv_bfloat16, MODE>(a, map_dy, map_x, map_dw, sm_count, stream);
    return launch<T, __half, MODE>(a, map_dy, map_x, map_dw, sm_count, stream);
}
template <typename T>
cudaError_t launch_by_mode(int mode, int grads_dtype, const WGArgs& a, const CUtensorMap& map_dy, const CUtensorMap& map_x,
                           const CUtensorMap& map_dw, int sm_count, cudaStream_t stream) {
    if (mode == WG_PANEL) return launch_by_grads<T, WG_PANEL>(grads_dtype, a, map_dy, map_x, map_dw, sm_count, stream);
    if (mode == WG_RESTORED) return launch_by_grads<T, WG_RESTORED>(grads_dtype, a, map_dy, map_x, map_dw, sm_count, stream);
    if (mode == WG_FUSED) return launch_by_grads<T, WG_FUSED>(grads_dtype, a, map_dy, map_x, map_dw, sm_count, stream);
    return launch_by_grads<T, WG_PLAIN_DY>(grads_dtype, a, map_dy, map_x, map_dw, sm_count, stream);
}

bool rows_on_16(const void* p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0; }
int64_t round8(int64_t v) { return (v + 7) / 8 * 8; }
// More than one output tile to reuse a panel for, tokens that fit one, and dy as TMA takes it: a length
// that ends inside a step needs dy's last step masked, which this mode does not do.
bool panel_applies(const gar_weight_grad_params_t& p, int64_t ld_dy) {
    return rows_on_16(p.dy, ld_dy) && !p.lengths && p.tokens <= WG_PANEL_STEPS * WG_K && p.out_features > 2 * WG_M;
}

// With few output tiles and many tokens the tokens are cut, so that every pair of SMs has a part, of four
// steps at least (a step takes a pair 0.6 to 2 us when no other tile hides its latencies, the join 4 us in
// all).  One worker, 4000 tokens, 200 x 300: 17 us, whole 47; 2 x 4096 tokens, 513 x 250: 29 us, whole 115.
// A panel's tokens stay whole (WG_PANEL's tiles know no parts).
constexpr int WG_PAIRS = 74;
int splits_of(const gar_weight_grad_params_t& p, int64_t ld_dy) {
    if (panel_applies(p, ld_dy)) return 1;
    const int64_t mt = (p.out_features + 2 * WG_M - 1) / (2 * WG_M), columns = (p.in_features + WG_N - 1) / WG_N + (p.bias_grads ? 1 : 0);
    if (mt > WG_PAIRS || columns > WG_PAIRS) return 1;
    const int64_t tiles = p.workers * mt * columns, steps = (p.tokens + WG_K - 1) / WG_K;
    const int64_t s = std::min<int64_t>(WG_PAIRS / tiles, steps / 4);
    return s > 1 ? int(std::min<int64_t>(s, 16)) : 1;
}
int64_t round4(int64_t v) { return (v + 3) / 4 * 4; }
// one part of one worker: weights with rows of whole 16 bytes, biases
int64_t part_floats(const gar_weight_grad_params_t& p) { return p.out_features * round4(p.in_features) + round4(p.out_features); }

template <typename G>
cudaError_t join_parts(const WGArgs& a, const gar_weight_grad_params_t& p, cudaStream_t stream) {
    const dim3 grid(unsigned((p.in_features + 1 + 127) / 128), unsigned(p.workers * p.out_features));
    join_parts_kernel<G><<<grid, 128, 0, stream>>>(static_cast<const float*>(a.dw), a.ld_grads, a.pitch, a.splits, p.workers, p.out_features,
                                                   p.in_features, static_cast<G*>(p.weight_grads), static_cast<G*>(p.bias_grads), p.ld_grads);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_weight_grad(const gar_weight_grad_params_t& p, int64_t ld_dy, int sm_count) {
    WGArgs a{};
    a.dy = p.dy;
    a.q = p.x_saved.q;
    a.scales = p.x_saved.scales;
    a.ldq = p.x_saved.ldq;
    a.lengths = p.lengths;
    a.dw = p.weight_grads;
    a.db = p.bias_grads;
    a.tokens = p.tokens;
    a.out = p.out_features;
    a.in = p.in_features;
    a.ld_dy = ld_dy;
    a.ld_grads = p.ld_grads;
    a.workers = p.workers;
    a.groups = int((p.in_features + p.group - 1) / p.group);
    a.group_shift = p.group == 32 ? 5 : p.group == 64 ? 6 : 7;
    a.mt = int((p.out_features + 2 * WG_M - 1) / (2 * WG_M));
    a.nt = int((p.in_features + WG_N - 1) / WG_N);
    a.columns = a.nt + (p.bias_grads ? 1 : 0);
    if (int64_t(a.mt) * a.columns >= (int64_t(1) << 30) / a.workers) return cudaErrorInvalidConfiguration;
    a.pitch = p.in_features;
    a.splits = p.workspace ? splits_of(p, ld_dy) : 1;
    // parts are fp32 results in the workspace
    int grads_dtype = p.grads_dtype;
    if (a.splits > 1) {
        grads_dtype = GAR_F32;
        a.dw = p.workspace;
        a.pitch = round4(p.in_features);
        a.ld_grads = part_floats(p);
        a.db = p.bias_grads ? static_cast<float*>(p.workspace) + p.out_features * a.pitch : nullptr;
    }
    const int64_t gs = grads_dtype == GAR_F32 ? 4 : 2;
    const int planes = p.workers * a.splits;
    a.wide = reinterpret_cast<uintptr_t>(a.dw) % 16 == 0 && (planes == 1 || a.ld_grads * gs % 16 == 0) && a.pitch * gs % 16 == 0;

    const CUtensorMapDataType type = p.dtype == GAR_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
    cudaStream_t stream = static_cast<cudaStream_t>(p.stream);
    CUtensorMap map_x, map_dy, map_dw;
    int mode = rows_on_16(p.dy, ld_dy) ? WG_FUSED : WG_PLAIN_DY;
    if (panel_applies(p, ld_dy)) mode = WG_PANEL;
    if (a.splits == 1 && mode != WG_PANEL && p.workspace && p.tokens > 0) {
        // x restored once (and dy copied, if its rows do not start on 16 bytes), then products of plain copies
        mode = WG_RESTORED;
        const int64_t rows = p.tokens * p.workers, ldx = round8(p.in_features);
        char* x = static_cast<char*>(p.workspace);
        if (cudaError_t err = launch_checkpoint_restore_masked(p, x, ldx, stream)) return err;
        if (cudaError_t err = make_token_map(&map_x, type, x, p.in_features, p.tokens, p.workers, ldx * 2, 64, CU_TENSOR_MAP_SWIZZLE_128B)) return err;
        if (!rows_on_16(p.dy, ld_dy)) {
            char* dy = x + gar::align256(size_t(rows) * size_t(ldx) * 2);
            const int64_t ld = round8(p.out_features);
            const int64_t pieces = rows * (ld / 8);
            const unsigned blocks = unsigned(min(int64_t(16 * sm_count), (pieces + 255) / 256));
            align_rows_kernel<<<blocks, 256, 0, stream>>>(static_cast<const unsigned short*>(p.dy), ld_dy, p.out_features, pieces,
                                                          reinterpret_cast<uint4*>(dy), ld / 8);
            if (cudaError_t err = cudaGetLastError()) return err;
            a.dy = dy;
            a.ld_dy = ld;
        }
    } else if (cudaError_t err = make_token_map(&map_x, CU_TENSOR_MAP_DATA_TYPE_UINT8, p.x_saved.q, p.in_features, p.tokens, p.workers,
                                          p.x_saved.ldq, WG_HALF, CU_TENSOR_MAP_SWIZZLE_NONE)) {
        return err;
    }
    if (mode == WG_PLAIN_DY) map_dy = map_x;      // not used
    else if (cudaError_t err = make_token_map(&map_dy, type, a.dy, p.out_features, p.tokens, p.workers, a.ld_dy * 2, 64, CU_TENSOR_MAP_SWIZZLE_128B)) return err;
    if (!a.wide) {
        map_dw = map_x;                           // not used
    } else {
        const CUtensorMapDataType gt = grads_dtype == GAR_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                       : grads_dtype == GAR_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
        const int64_t pitch = a.pitch * gs, plane = planes > 1 ? a.ld_grads * gs : pitch * p.out_features;
        if (cudaError_t err = make_map(&map_dw, gt, a.dw, p.in_features, p.out_features, planes, pitch, plane, int(128 / gs), 32,
                                       CU_TENSOR_MAP_SWIZZLE_128B)) return err;
    }
    const cudaError_t err = p.dtype == GAR_BF16 ? launch_by_mode<__nv_bfloat16>(mode, grads_dtype, a, map_dy, map_x, map_dw, sm_count, stream)
                                                : launch_by_mode<__half>(mode, grads_dtype, a, map_dy, map_x, map_dw, sm_count, stream);
    if (err != cudaSuccess || a.splits == 1) return err;
    return p.grads_dtype == GAR_F32    ? join_parts<float>(a, p, stream)
           : p.grads_dtype == GAR_BF16 ? join_parts<__nv_bfloat16>(a, p, stream) : join_parts<__half>(a, p, stream);
}

// Every 256 outputs restore the activation once more.  Measured, with a workspace against without (8 workers, 2048
// tokens, 4096 inputs): bf16 results 144 us against 126 at 768 outputs, 234 against 233 at 1536, 290 against 299 at
// 2048, 1045 against 1150 at 4 x 8192 tokens and 4096 outputs; fp32 results, whose chunks are joined more often, which
// holds the restore warps up, 116 against 105 at 512, 155 against 153 at 768, 181 against 189 at 1024, 316 against 366
// at 2048.  dy copied to aligned rows on the way (fp32 results): 191 against 382 at 1023 outputs, 125 against 253 at 499,
// where the rule, which looks at no other size, does without; 7 x 100 tokens, 500 x 800 19 against 13.
bool weight_grad_wants_workspace(const gar_weight_grad_params_t& p, int64_t ld_dy) {
    if (splits_of(p, ld_dy) > 1) return true;
    if (panel_applies(p, ld_dy)) return false;
    const bool chunks = p.grads_dtype == GAR_F32 && p.tokens > Chunk<float>::STEPS * WG_K;
    return p.out_features >= (chunks || !rows_on_16(p.dy, ld_dy) ? 768 : 2048);
}

size_t weight_grad_workspace_bytes(const gar_weight_grad_params_t& p, int64_t ld_dy) {
    if (splits_of(p, ld_dy) > 1) return gar::align256(size_t(splits_of(p, ld_dy)) * p.workers * size_t(part_floats(p)) * 4);
    if (panel_applies(p, ld_dy)) return 0;
    const int64_t rows = p.tokens * p.workers;
    size_t bytes = gar::align256(size_t(rows) * size_t(round8(p.in_features)) * 2);
    if (!rows_on_16(p.dy, ld_dy)) bytes += gar::align256(size_t(rows) * size_t(round8(p.out_features)) * 2);
    return bytes;
}

}  // namespace worker
}  // namespace gar
