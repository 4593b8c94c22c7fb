// Products with a worker's weights (gar_linear.h) and what is done with them while they are still in tensor
// memory: log probabilities of tokens without logits, their gradient at the logits, the gated feed-forward
// block with its checkpoints, and the gradients at the inputs.
//
// One kernel: C = A B^T for 16-bit matrices, pairs of CTAs (clusters of two, one CTA per SM) on tiles of
// 256 rows x 256 columns, 64 elements of the contraction a step, the paired instruction (cta_group::2) with
// fp32 accumulators in tensor memory, two tiles' worth of it.
//   copy warp      TMA, one lane: 128 rows of A and 128 rows of B per CTA and step, 128-byte swizzle; A and
//                  B lie with the contraction along their rows (K-major), or across them (MN-major: the
//                  gradient at the inputs, dz W, reads W as it lies, the gradient at the weights, dz^T x, both)
//   MMA warp       of the leading CTA: four 256 x 256 x 16 instructions per step
//   store warps    groups of four, each with its share of a tile's columns, while the next products run
//                  into the other half of tensor memory; a thread has one row, 32 columns at a time.  Two groups, or four
//                  where a column takes an exponential and one accumulator holds the sums (struct Shape)
// and four epilogues (LN_SUM's and LN_OUTER's are one; enum Epilogue).  A thread owning a row makes the softmax's statistics, the group
// maxima of the checkpoints and the row's target its own affair.
// Tiles are as wide as the rule in width_for makes them, 256 columns at most.
//
// The tensor core truncates what it adds: a product to a multiple of 2^-25 of the largest magnitude among the accumulator and the
// products it is added with, the accumulator to 24 bits (measured with single terms next to 1; mma.sync 2^-24).  Sums over k terms come out
// short by 1.0e-9 k of themselves (random signs; from k = 512 to 4096 lse off by -2.9e-6, -5.9e-6, -1.2e-5, -2.5e-5), by
// 1.4e-9 k (bf16) to 6e-9 k (binary16, whose products have more bits to lose) where the terms have one sign, by nothing where they are few.
// The logits, whose log probabilities are fp32 results, are therefore summed in chunks of 512 terms (up to 640 in one): the halves of
// tensor memory take a chunk each in turn, and the store warps add them up, rounded, in registers (linear_kernel's LONG).
// lse is then 2.2e-7 (binary16 3.0e-7) off, relative, from 512 to 16384 terms (5000 columns, random signs; in one accumulator
// 1.9e-6 at 4096), at the same speed.
//
// Every wait is bounded (mbar.cuh); a pair whose wait gave up fills its tiles with NaN.
#include <algorithm>
#include <atomic>

#include "gar_internal.cuh"
#include "worker_act.cuh"
#include "worker_linear.cuh"
#include "worker_tensor.cuh"
#include "worker_tiles.cuh"

namespace gar {
namespace worker {
namespace {

constexpr int LN_M = 128, LN_N = 256, LN_K = 64;      // rows of a CTA, columns of a pair, contraction per step
constexpr int LN_HALF = LN_N / 2;                     // rows of B that a CTA holds
constexpr int LN_TILE = LN_M * LN_K * 2;              // bytes of A (and, at full width, of B) per step and CTA
// Steps in flight: five of full width; narrow tiles have more in the same memory, since a step's copies take some 2000 cycles to come
// and a few narrow tiles wait for nothing else.
constexpr int LN_RING_BYTES = 5 * 2 * LN_TILE, LN_RING_MOST = 8;
constexpr int LN_BLOCK = 64 * 128;                    // bytes of 64 x 64 elements of an MN-major operand
constexpr int LN_COPY_WARP = 0, LN_MMA_WARP = 1, LN_ALLOC_WARP = 2;
constexpr int LN_STORE_WARP0 = 4;
constexpr int LN_PAIRS = 74;                          // pairs of SMs, for the rules that cut work into parts and tiles
// Steps of the contraction that a logit's accumulator takes where there are several (LONG), and up to which there is one.  A second chunk
// of a few steps would be over before the epilogue of 128 columns a thread: 4096 x 32000, scores and gradient with dx, 576 terms: 101 to 112 and
// 310 us in one accumulator, 138 and 338 in two; 640: 122 and 333, 142 and 346; 768: 142 and 369, 148 and 364; 1024: 190 and 457, 182 and 457.
// Chunks of 256 terms halve the loss and hold the products up: 8192 x 32000, 2048: 840 us instead of 765.
constexpr int LN_CHUNK = 8, LN_ONE = 10;

// What becomes of a tile.
//   LN_SCORES   z: maximum and sum of exponentials of each row's 256 columns, and the target's z
//   LN_DLOGITS  z: a ([j = t] - e^(z - lse)), stored in 16 bits
//   LN_GATED    128 columns of g and of u: act(g) u, stored, and the codes of g and u
//   LN_SUM      stored in 16 bits, or in fp32, or added to fp32 (parts of a longer contraction)
//   LN_OUTER    the same, of every worker's own contraction over its tokens
enum Epilogue { LN_SCORES = 0, LN_DLOGITS = 1, LN_GATED = 2, LN_SUM = 3, LN_OUTER = 4 };
enum Out { OUT_WIDE = 0, OUT_PLAIN = 1, OUT_PART = 2, OUT_ADD = 3, OUT_PLAIN32 = 4 };   // 16 bits by TMA or plainly; fp32 by TMA, added, plainly

struct LNArgs : Tiling {
    int64_t        rows, cols;            // of the result (LN_SCORES, LN_DLOGITS: columns from col0 on)
    int            width;                 // columns of a tile (LN_GATED: g's and u's together)
    int            ring, slot_bytes;      // steps in flight, what one takes in shared memory
    int            steps0;                // steps of the first pair of operands (`steps`: of both together)
    int            group_shift, groups, out;
    int64_t        col0;                  // first column of this launch
    const void *   bias, *bias2;          // 16-bit, or null
    const int64_t* targets;
    float2*        parts;                 // LN_SCORES [rows][nt]: maximum, sum
    float*         target_z;              // LN_SCORES [rows]
    const float *  lse, *lse_lo, *coef;   // LN_DLOGITS [rows]
    const unsigned* top;                  // every worker's largest |coef|, or (tokens = 1) every row's, as bits, where they carry a power of two; or null
    unsigned       tokens;                // rows of a worker, for `top`
    unsigned       fold;                  // LN_DLOGITS: dz in two parts, every worker's `fold` rows once more behind them for what the first left out; 0: one
    void*          y;                     // OUT_PLAIN, and the fill after a wait that gave up
    int64_t        ldy, plane;            // elements between the result's rows; its parts or workers
    gar_checkpoint_t s0, s1;              // of g and u
};

// Store warps, their staged pieces of a result (32 rows) and the biases they keep.  The logits' epilogues are bound by latency where the
// contraction is short (two warps on a scheduler issue in 37 % of the cycles): four groups, of fewer registers.  4096 x 32000, 128: 82.6 us,
// with four groups 73.0; the gradient 274 and 258.  LONG: a thread keeps the sums of its columns, 128 of them in two groups.
template <int EPI, bool LONG> struct Shape {
    static constexpr bool LOGITS = EPI == LN_SCORES || EPI == LN_DLOGITS;
    static_assert(LOGITS || !LONG, "chunks are the logits'");
    static constexpr int GROUPS = LOGITS && !LONG ? 4 : 2, STORE_WARPS = 4 * GROUPS, THREADS = 32 * (LN_STORE_WARP0 + STORE_WARPS);
    static constexpr int PIECE = EPI == LN_SCORES ? 16 : EPI == LN_DLOGITS ? 32 * 64 : 32 * 128, BIASES = LOGITS ? LN_N / GROUPS : LN_N;
};
template <int EPI, bool LONG> struct __align__(1024) LNSmem {
    typedef Shape<EPI, LONG> S;
    uint8_t  ring[LN_RING_BYTES];                         // slots: 128 rows of A, half the tile's rows of B
    uint8_t  out[S::STORE_WARPS][S::PIECE];               // a store warp's piece: 32 rows of 128 bytes (LN_DLOGITS: 64)
    float    add[S::STORE_WARPS][S::BIASES];              // a warp's biases
    float2   part[EPI == LN_SCORES ? 2 : 1][S::GROUPS][EPI == LN_SCORES ? LN_M : 1]; // the groups' maxima and sums, of two tiles in turn
    unsigned long long part_full[2];                      // they are there
    unsigned long long empty[LN_RING_MOST], acc_full[2];  // the slots are read; the accumulators are complete
    unsigned long long full[LN_RING_MOST], acc_empty[2];  // the leading CTA's are used, for both
    unsigned tmem_base;
    int      error, other_error;                          // a wait gave up, here or in the other CTA
};

// The ring's slots, one after the other.
struct Slot {
    unsigned slot = 0, parity = 0;
    __device__ __forceinline__ void next(const LNArgs& a) {
        if (++slot == unsigned(a.ring)) {
            slot = 0;
            parity ^= 1u;
        }
    }
};

template <int EPI>
__device__ __forceinline__ Place place_at(const LNArgs& a, unsigned index) { return place_in<EPI == LN_OUTER>(a, index); }

// 32 columns of this thread's row of the accumulators: asked for, there once waited for
__device__ __forceinline__ void ask32(unsigned taddr, float (&v)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
                   "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]),
                   "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]),
                   "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void wait32(float (&v)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]),
                   "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(v[16]),
                   "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]), "+f"(v[24]),
                   "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31]) :: "memory");
}
// f(v, c0) for the columns 0 .. cols of a tile, 32 at a time (cols is the warp's own number); the next are on
// their way while some are worked on
template <typename F>
__device__ __forceinline__ void over_columns(unsigned src, int cols, F f) {
    float v0[32], v1[32];
    ask32(src, v0);
    for (int c0 = 0; c0 < cols; c0 += 64) {
        wait32(v0);
        if (c0 + 32 < cols) ask32(src + unsigned(c0 + 32), v1);
        f(v0, c0);
        if (c0 + 32 >= cols) break;
        wait32(v1);
        if (c0 + 64 < cols) ask32(src + unsigned(c0 + 64), v0);
        f(v1, c0 + 32);
    }
}
__device__ __forceinline__ void ask16(unsigned taddr, float (&v)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]),
                   "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void wait16(float (&a)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(a[0]), "+f"(a[1]), "+f"(a[2]), "+f"(a[3]), "+f"(a[4]), "+f"(a[5]), "+f"(a[6]), "+f"(a[7]), "+f"(a[8]), "+f"(a[9]),
                   "+f"(a[10]), "+f"(a[11]), "+f"(a[12]), "+f"(a[13]), "+f"(a[14]), "+f"(a[15]) :: "memory");
}
// What a thread has of its row's logits: its columns of the accumulators, 32 at a time (four warps of a scheduler take turns);
// or (LONG) the sums of the chunks so far, all its columns of them.
template <bool LONG> struct Logits {
    unsigned src;
    __device__ __forceinline__ void chunk(unsigned from, int, bool) { src = from; }
    template <typename F> __device__ __forceinline__ void each(int cols, F f) {
#pragma unroll 1
        for (int c0 = 0; c0 < cols; c0 += 32) {
            float v[32];
            ask32(src + unsigned(c0), v);
            wait32(v);
            f(v, c0);
        }
    }
};
template <> struct Logits<true> {
    float sum[4][32];
    // a chunk's accumulators, from `from` on (cols is the warp's own number)
    __device__ __forceinline__ void chunk(unsigned from, int cols, bool first) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (32 * k >= cols) break;
            if (first) {
                ask32(from + unsigned(32 * k), sum[k]);
                wait32(sum[k]);
                continue;
            }
#pragma unroll
            for (int h = 0; h < 32; h += 16) {
                float v[16];
                ask16(from + unsigned(32 * k + h), v);
                wait16(v);
#pragma unroll
                for (int j = 0; j < 16; j += 2) unpack2(add2(pack2(sum[k][h + j], sum[k][h + j + 1]), pack2(v[j], v[j + 1])), sum[k][h + j], sum[k][h + j + 1]);
            }
        }
    }
    template <typename F> __device__ __forceinline__ void each(int cols, F f) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (32 * k >= cols) break;
            f(sum[k], 32 * k);
        }
    }
};
__device__ __forceinline__ void add32(float (&v)[32], const float* add) {
#pragma unroll
    for (int j = 0; j < 32; j += 4) {
        const float4 b = *reinterpret_cast<const float4*>(add + j);
        unpack2(add2(pack2(v[j], v[j + 1]), pack2(b.x, b.y)), v[j], v[j + 1]);
        unpack2(add2(pack2(v[j + 2], v[j + 3]), pack2(b.z, b.w)), v[j + 2], v[j + 3]);
    }
}

// 32 values as T to the first or second half of this lane's row of the staged piece
template <typename T>
__device__ __forceinline__ void stage32(unsigned stage, int lane, int half, const float (&v)[32]) {
#pragma unroll
    for (int j = 0; j < 32; j += 8) {
        const float f[8] = {v[j], v[j + 1], v[j + 2], v[j + 3], v[j + 4], v[j + 5], v[j + 6], v[j + 7]};
        put_shared(stage + lane * 128 + (((half * 4 + j / 8) ^ (lane & 7)) << 4), narrow16B(f, static_cast<const T*>(nullptr)));
    }
}
__device__ __forceinline__ void tma_add(const CUtensorMap* map, unsigned src, int x, int y, int z) {
    asm volatile("cp.reduce.async.bulk.tensor.3d.global.shared::cta.add.tile.bulk_group [%0, {%2, %3, %4}], [%1];"
                 ::"l"(map), "r"(src), "r"(x), "r"(y), "r"(z) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
__device__ __forceinline__ void tma_put(const CUtensorMap* map, unsigned src, int x, int y, int z) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%2, %3, %4}], [%1];"
                 ::"l"(map), "r"(src), "r"(x), "r"(y), "r"(z) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// The staged piece (32 rows of 64 16-bit elements) to rows that start anywhere, eight rows' loads and stores at a time.
__device__ __forceinline__ void store_plain(unsigned stage, int lane, unsigned short* dst, int64_t ld, int rows, int cols) {
    const int c = 2 * lane;
    dst += c;
    if (rows == 32 && cols >= 64 && ((reinterpret_cast<uintptr_t>(dst) | (ld << 1)) & 2) == 0) {
        // A whole piece of rows that start on 4 bytes: nothing to check (14 workers x 95 tokens, 11558 outputs x 250 inputs, whole
        // backward pass without dx: 70.8 -> 62.4 us). Odd rows put together from shuffled words were slower than the halves
        // below (251 inputs: 74.5 -> 85.3 us).
#pragma unroll 1
        for (int r0 = 0; r0 < 32; r0 += 8) {
            unsigned w[8];
#pragma unroll
            for (int k = 0; k < 8; ++k)
                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[k]) : "r"(stage + (r0 + k) * 128 + (((lane / 4) ^ k) << 4) + (lane & 3) * 4));
#pragma unroll
            for (int k = 0; k < 8; ++k) *reinterpret_cast<unsigned*>(dst + k * ld) = w[k];
            dst += 8 * ld;
        }
        return;
    }
#pragma unroll 1
    for (int r0 = 0; r0 < rows; r0 += 8) {
        unsigned w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[k]) : "r"(stage + (r0 + k) * 128 + (((lane / 4) ^ k) << 4) + (lane & 3) * 4));
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (r0 + k >= rows) break;
            if (c + 1 < cols && (reinterpret_cast<uintptr_t>(dst) & 2) == 0) {
                *reinterpret_cast<unsigned*>(dst) = w[k];
            } else {
                if (c < cols) dst[0] = static_cast<unsigned short>(w[k]);
                if (c + 1 < cols) dst[1] = static_cast<unsigned short>(w[k] >> 16);
            }
            dst += ld;
        }
    }
}

// The same of a piece of 32 rows of 32 fp32 elements, one per lane.
__device__ __forceinline__ void store_plain32(unsigned stage, int lane, float* dst, int64_t ld, int rows, int cols) {
    dst += lane;
#pragma unroll 1
    for (int r0 = 0; r0 < rows; r0 += 8) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v[k]) : "r"(stage + (r0 + k) * 128 + (((lane / 4) ^ k) << 4) + (lane & 3) * 4));
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (r0 + k < rows && lane < cols) *dst = v[k];
            dst += ld;
        }
    }
}

// N columns' biases from column c0 on, 0 where there is no column
template <typename T, int N>
__device__ __forceinline__ void fetch_biases(const void* bias, int64_t c0, int64_t cols, float* add, int lane) {
    float v[N / 32];
#pragma unroll
    for (int k = 0; k < N / 32; ++k) {
        const int64_t c = c0 + 32 * k + lane;
        v[k] = bias && c < cols ? Elem<T>::widen(static_cast<const T*>(bias)[c]) : 0.f;
    }
#pragma unroll
    for (int k = 0; k < N / 32; ++k) add[32 * k + lane] = v[k];
}

// ---- epilogues: one warp's 32 rows and its group's columns of a tile -------------------------------
struct Warp {
    unsigned src, stage;             // its lanes of the accumulators; its staging buffer
    float*   add;
    int      lane, group, quarter;
    int64_t  row0;                   // the first of its rows
};
// A group's columns of the `cols` a tile has: from, to; whole multiples of `unit` but for the tile's end
struct Columns {
    int from, to;
    template <int GROUPS, int UNIT> static __device__ __forceinline__ Columns of(int cols, int group) {
        const int each = (cols + GROUPS * UNIT - 1) / (GROUPS * UNIT) * UNIT;
        return Columns{min(group * each, cols), min((group + 1) * each, cols)};
    }
};

// Rows in two parts: a worker's `fold` rows, then the same once more.  Which of the caller's rows one is, and of which part.
struct Folded {
    unsigned row;
    bool     rest;
};
__device__ __forceinline__ Folded unfold(unsigned row, unsigned fold) {
    const unsigned worker = row / (2 * fold), at = row - worker * 2 * fold;
    return at < fold ? Folded{worker * fold + at, false} : Folded{worker * fold + at - fold, true};
}

// What a thread reads for its row of a tile from memory: asked for a tile ahead, looked at when it is the tile's turn.
struct RowInputs {
    int64_t target;
    float   coef, lse, lo;
    bool    rest;                    // the row of the second part of dz
};
template <int EPI>
__device__ __forceinline__ RowInputs ask_inputs(const LNArgs& a, const Place& t, unsigned rank, int quarter, int lane) {
    RowInputs in{-1, 0.f, 0.f, 0.f, false};
    if (EPI != LN_SCORES && EPI != LN_DLOGITS) return in;
    const int64_t row = int64_t(2 * t.m + int(rank)) * LN_M + quarter * 32 + lane;
    if (row >= a.rows) return in;
    if (EPI == LN_SCORES) {
        if (a.targets) in.target = a.targets[row];
        return in;
    }
    int64_t token = row;
    if (a.fold) {
        const Folded f = unfold(unsigned(row), a.fold);
        token = f.row;
        in.rest = f.rest;
    }
    in.target = a.targets[token];
    in.coef = a.coef[row];
    in.lse = a.lse[token];
    if (a.lse_lo) in.lo = a.lse_lo[token];
    return in;
}
// The biases of a warp's columns of a tile, into its piece of shared memory, while the tile's products still run.
template <typename T, int EPI, bool LONG>
__device__ __forceinline__ void fetch_tile_biases(const LNArgs& a, const Place& t, const Warp& w) {
    if (w.row0 >= a.rows) return;
    if (EPI == LN_GATED && (a.bias || a.bias2)) {
        const int64_t c0 = int64_t(t.n) * (a.width / 2);
        fetch_biases<T, LN_HALF>(a.bias, c0, a.cols, w.add, w.lane);
        fetch_biases<T, LN_HALF>(a.bias2, c0, a.cols, w.add + LN_HALF, w.lane);
    }
    if (EPI == LN_SCORES || EPI == LN_DLOGITS) {
        const int64_t c0 = int64_t(t.n) * a.width, left = a.cols - c0;
        if (a.bias) {
            typedef Shape<EPI, LONG> S;
            const Columns mine = Columns::of<S::GROUPS, 32>(left < a.width ? int(left) : a.width, w.group);
            fetch_biases<T, S::BIASES>(a.bias, a.col0 + c0 + mine.from, a.col0 + a.cols, w.add, w.lane);
        }
    }
}

// A group's columns of a tile of logits
template <int GROUPS>
__device__ __forceinline__ Columns logits_columns(const LNArgs& a, const Place& t, int group) {
    const int64_t left = a.cols - int64_t(t.n) * a.width;
    return Columns::of<GROUPS, 32>(left < a.width ? int(left) : a.width, group);
}

// The group's maximum and sum of this thread's row
template <bool LONG>
__device__ __forceinline__ float2 scores_tile(const LNArgs& a, const Place& t, const Warp& w, const RowInputs& in, const Columns& mine, Logits<LONG>& logits) {
    const int64_t c0 = int64_t(t.n) * a.width, row = w.row0 + w.lane;
    const int cols = mine.to - mine.from;
    const bool adds = a.bias != nullptr;
    const int64_t t64 = in.target - a.col0 - c0 - mine.from;
    const int target = in.target >= 0 && t64 >= 0 && t64 < cols ? int(t64) : -1;
    float m = -CUDART_INF_F, s = 0.f;
    if (cols > 0 && w.row0 < a.rows)
        logits.each(cols, [&](float (&v)[32], int at) {
            if (adds) add32(v, w.add + at);
            if (at + 32 > cols) {                        // columns that do not exist (0 times an infinity of the row is NaN there)
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = at + j < cols ? v[j] : -CUDART_INF_F;
            }
            if (__any_sync(0xffffffffu, target >= at && target < at + 32)) {
                float z = 0.f;
#pragma unroll
                for (int j = 0; j < 32; ++j) z = target == at + j ? v[j] : z;
                if (target >= at && target < at + 32) a.target_z[row] = z;
            }
            float top[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
            for (int j = 4; j < 32; ++j) top[j & 3] = fmaxf(top[j & 3], v[j]);
            const float higher = fmaxf(m, fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])));
            if (higher > m) {
                s *= ex2((m - higher) * kLog2e);
                m = higher;
            }
            // z - m is rounded once and the exponent's unit comes after it: masks of the lowest value do not overflow
            const float base = m == -CUDART_INF_F ? 0.f : m;
            const f32x2 minus = pack2(-base, -base), unit = pack2(kLog2e, kLog2e);
            f32x2 sum0 = pack2(0.f, 0.f), sum1 = sum0;
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
                float e0, e1, e2, e3;
                unpack2(mul2(add2(pack2(v[j], v[j + 1]), minus), unit), e0, e1);
                unpack2(mul2(add2(pack2(v[j + 2], v[j + 3]), minus), unit), e2, e3);
                sum0 = add2(sum0, pack2(ex2(e0), ex2(e1)));
                sum1 = add2(sum1, pack2(ex2(e2), ex2(e3)));
            }
            float p, q;
            unpack2(add2(sum0, sum1), p, q);
            s += p + q;
        });
    return make_float2(m, s);
}
// The groups' parts of a row as one
template <int GROUPS>
__device__ __forceinline__ float2 join_groups(const float2 (&p)[GROUPS][LN_M], int row) {
    float m = p[0][row].x;
#pragma unroll
    for (int k = 1; k < GROUPS; ++k) m = fmaxf(m, p[k][row].x);
    const float base = m == -CUDART_INF_F ? 0.f : m;
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) s += p[k][row].y * ex2((p[k][row].x - base) * kLog2e);      // a part without entries is -inf, 0
    return make_float2(m, s);
}

// 64 columns at a time to the result, staged
__device__ __forceinline__ void stage_free(const Warp& w) {
    if (w.lane == 0) tma_store_read<0>();
    __syncwarp();
}
// the staged piece, 64 columns from `col` on, `cols` of which exist
__device__ __forceinline__ void put_piece(const LNArgs& a, const Warp& w, const CUtensorMap* map, int64_t col, int cols, int z) {
    if (a.out == OUT_WIDE) {
        fence_async_smem();
        __syncwarp();
        if (w.lane == 0) tma_put(map, w.stage, int(col), int(w.row0), z);
    } else {
        const int64_t left = a.rows - w.row0;
        __syncwarp();
        store_plain(w.stage, w.lane, static_cast<unsigned short*>(a.y) + z * a.plane + w.row0 * a.ldy + col, a.ldy, left < 32 ? int(left) : 32, cols);
        __syncwarp();
    }
}

template <typename T, bool LONG>
__device__ __forceinline__ void dlogits_tile(const LNArgs& a, const Place& t, const Warp& w, const RowInputs& in, const Columns& mine, Logits<LONG>& logits,
                                             const CUtensorMap* map) {
    const int cols = mine.to - mine.from;
    if (w.row0 >= a.rows || cols <= 0) return;
    const int64_t first = int64_t(t.n) * a.width + mine.from;
    const bool adds = a.bias != nullptr;
    float coef = in.coef;
    if (a.top && w.row0 + w.lane < a.rows) coef *= power_for(a.top[unsigned(w.row0 + w.lane) / a.tokens], false);
    const float lse = in.lse, lo = in.lo;
    const int64_t t64 = in.target - a.col0 - first;
    const int target = in.target >= 0 && t64 >= 0 && t64 < cols ? int(t64) : -1;
    const bool nothing = coef == 0.f;
    const f32x2 minus = pack2(-lse, -lse), unit = pack2(kLog2e, kLog2e), minus_lo = pack2(-lo * kLog2e, -lo * kLog2e), by = pack2(-coef, -coef);
    logits.each(cols, [&](float (&v)[32], int at) {
        if (adds) add32(v, w.add + at);
#pragma unroll
        for (int j = 0; j < 32; j += 2) {
            float e0, e1;
            unpack2(fma2(add2(pack2(v[j], v[j + 1]), minus), unit, minus_lo), e0, e1);
            unpack2(mul2(pack2(ex2(e0), ex2(e1)), by), v[j], v[j + 1]);
        }
        if (__any_sync(0xffffffffu, target >= at && target < at + 32)) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = target == at + j ? v[j] + coef : v[j];
        }
        if (__any_sync(0xffffffffu, nothing)) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = nothing ? 0.f : v[j];
        }
        if (a.fold && __any_sync(0xffffffffu, in.rest)) {
            // what the first part's rounding left out; nothing of what it holds as an infinity
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                const float kept = Elem<T>::widen(Elem<T>::narrow(v[j]));
                if (in.rest) v[j] = fabsf(kept) <= 3.402823466e38f ? v[j] - kept : 0.f;
            }
        }
        stage_free(w);
        // rows of 64 bytes, 16-byte chunks in the 64-byte swizzle
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float f[8] = {v[8 * j], v[8 * j + 1], v[8 * j + 2], v[8 * j + 3], v[8 * j + 4], v[8 * j + 5], v[8 * j + 6], v[8 * j + 7]};
            put_shared(w.stage + w.lane * 64 + ((j ^ ((w.lane >> 1) & 3)) << 4), narrow16B(f, static_cast<const T*>(nullptr)));
        }
        fence_async_smem();
        __syncwarp();
        if (w.lane == 0) tma_put(map, w.stage, int(first) + at, int(w.row0), 0);
    });
}

// (LN_OUTER: the result is not touched again and would drive the operands out of L2)
template <typename T, int EPI>
__device__ __forceinline__ void sum_tile(const LNArgs& a, const Place& t, const Warp& w, const CUtensorMap* map) {
    const int64_t c0 = int64_t(t.n) * a.width;
    const int64_t left = a.cols - c0;
    const Columns mine = Columns::of<2, 64>(left < a.width ? int(left) : a.width, w.group);
    const int cols = mine.to - mine.from;
    if (w.row0 >= a.rows || cols <= 0) return;
    const int64_t first = c0 + mine.from;
    const unsigned src = w.src + unsigned(mine.from);
    // (LN_SUM: a row of the result is a token's)
    float by = 1.f;
    if (a.top && (EPI == LN_OUTER || w.row0 + w.lane < a.rows)) by = power_for(a.top[EPI == LN_OUTER ? unsigned(t.split) : unsigned(w.row0 + w.lane) / a.tokens], true);
    const unsigned long long policy = EPI == LN_OUTER ? evict_first() : 0;
    if (a.out >= OUT_PART) {
        over_columns(src, cols, [&](float (&v)[32], int at) {
            if (a.top) {
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] *= by;
            }
            stage_free(w);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                put_shared(w.stage + w.lane * 128 + ((j ^ (w.lane & 7)) << 4),
                           make_uint4(__float_as_uint(v[4 * j]), __float_as_uint(v[4 * j + 1]), __float_as_uint(v[4 * j + 2]), __float_as_uint(v[4 * j + 3])));
            if (EPI == LN_OUTER && a.out == OUT_PLAIN32) {
                const int64_t below = a.rows - w.row0;
                __syncwarp();
                store_plain32(w.stage, w.lane, static_cast<float*>(a.y) + t.split * a.plane + w.row0 * a.ldy + first + at, a.ldy, below < 32 ? int(below) : 32,
                              cols - at);
                __syncwarp();
                return;
            }
            fence_async_smem();
            __syncwarp();
            if (w.lane == 0) {
                if (EPI == LN_OUTER) tma_store(map, w.stage, int(first) + at, int(w.row0), t.split, policy);
                else if (a.out == OUT_ADD) tma_add(map, w.stage, int(first) + at, int(w.row0), t.split);
                else tma_put(map, w.stage, int(first) + at, int(w.row0), t.split);
            }
        });
        return;
    }
    int half = 0;
    over_columns(src, cols, [&](float (&v)[32], int at) {
        if (a.top) {
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] *= by;
        }
        if (half == 0) stage_free(w);
        stage32<T>(w.stage, w.lane, half, v);
        if (half == 1 || at + 32 >= cols) {
            if (EPI == LN_OUTER && a.out == OUT_WIDE) {
                fence_async_smem();
                __syncwarp();
                if (w.lane == 0) tma_store(map, w.stage, int(first) + (at & ~63), int(w.row0), t.split, policy);
            } else {
                put_piece(a, w, map, first + (at & ~63), cols - (at & ~63), EPI == LN_OUTER ? t.split : 0);
            }
        }
        half ^= 1;
    });
}

// 32 columns' codes of this thread's row to the checkpoint
__device__ __forceinline__ void store_codes(const float (&v)[32], const Step& step, int8_t* q, int count) {
    unsigned w[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float f[8] = {v[8 * j], v[8 * j + 1], v[8 * j + 2], v[8 * j + 3], v[8 * j + 4], v[8 * j + 5], v[8 * j + 6], v[8 * j + 7]};
        codes8(f, step, w[2 * j], w[2 * j + 1]);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if (16 * k + 16 <= count) {
            reinterpret_cast<uint4*>(q)[k] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
        } else {
#pragma unroll
            for (int j = 16 * k; j < 16 * k + 16; ++j)
                if (j < count) q[j] = int8_t((w[j / 4] >> 8 * (j & 3)) & 0xff);
        }
    }
}

// act(g) u of 32 columns as T to a half of this lane's row of the staged piece
template <typename T, int ACT>
__device__ __forceinline__ void gate32(unsigned stage, int lane, int half, const float (&g)[32], const float (&u)[32]) {
#pragma unroll
    for (int j = 0; j < 32; j += 8) {
        const float x[8] = {g[j], g[j + 1], g[j + 2], g[j + 3], g[j + 4], g[j + 5], g[j + 6], g[j + 7]};
        float y[8];
        act8<ACT>(x, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] *= u[j + i];
        put_shared(stage + lane * 128 + (((half * 4 + j / 8) ^ (lane & 7)) << 4), narrow16B(y, static_cast<const T*>(nullptr)));
    }
}
// 32 columns of g or u: the accumulators and the biases
__device__ __forceinline__ void ask_and_add(unsigned src, bool adds, const float* add, float (&v)[32]) {
    ask32(src, v);
    wait32(v);
    if (adds) add32(v, add);
}
__device__ __forceinline__ unsigned top32(const float (&v)[32]) {           // the largest magnitude, as bits: NaN above infinity
    unsigned t[4] = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 32; ++j) t[j & 3] = max(t[j & 3], __float_as_uint(v[j]) & 0x7fffffffu);
    return max(max(t[0], t[1]), max(t[2], t[3]));
}

// A store group has 64 columns of g and the same 64 of u (fewer at the end).  The maxima of checkpoints' groups are found in
// a pass of their own over tensor memory; for groups of 128 columns either store group looks at all of them.
template <typename T, int ACT>
__device__ __forceinline__ void gated_tile(const LNArgs& a, const Place& t, const Warp& w, const CUtensorMap* map) {
    const int half_width = a.width / 2;
    const int64_t c0 = int64_t(t.n) * half_width, row = w.row0 + w.lane;
    const int64_t left = a.cols - c0;
    const int all = left < half_width ? int(left) : half_width;
    const Columns mine = Columns::of<2, 64>(all, w.group);
    const int cols = mine.to - mine.from;
    if (w.row0 >= a.rows || cols <= 0) return;
    const int64_t first = c0 + mine.from;
    const bool adds = a.bias || a.bias2, saves = a.s0.q || a.s1.q, live = row < a.rows;
    const unsigned src_g = w.src, src_u = w.src + unsigned(half_width);
    unsigned top_g[2] = {0, 0}, top_u[2] = {0, 0};
    float g[32], u[32];
    if (saves) {
        const bool whole = a.group_shift == 7;
        const int from = whole ? 0 : mine.from, to = whole ? all : mine.to;
#pragma unroll 1
        for (int c = from; c < to; c += 32) {
            ask32(src_g + unsigned(c), g);
            ask32(src_u + unsigned(c), u);
            wait32(g);
            wait32(u);
            if (adds) {
                add32(g, w.add + c);
                add32(u, w.add + LN_HALF + c);
            }
            const int k = (c >> 5) & 1;
            const unsigned tg = top32(g), tu = top32(u);
            if (k == 0 || whole) { top_g[0] = max(top_g[0], tg); top_u[0] = max(top_u[0], tu); }
            else { top_g[1] = tg; top_u[1] = tu; }
        }
        if (whole) {
            top_g[1] = top_g[0];
            top_u[1] = top_u[0];
        } else if (a.group_shift == 6) {
            top_g[0] = top_g[1] = max(top_g[0], top_g[1]);
            top_u[0] = top_u[1] = max(top_u[0], top_u[1]);
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if (32 * k >= cols) break;
        const int64_t c = first + 32 * k, group = row * a.groups + (c >> a.group_shift);
        const bool begins = (c & ((1 << a.group_shift) - 1)) == 0;
        ask_and_add(src_g + unsigned(mine.from + 32 * k), adds, w.add + mine.from + 32 * k, g);
        if (a.s0.q && live) {
            const Step step(__uint_as_float(top_g[k]));
            if (begins) a.s0.scales[group] = step.scale(__uint_as_float(top_g[k]));
            store_codes(g, step, a.s0.q + row * a.s0.ldq + c, cols - 32 * k);
        }
        ask_and_add(src_u + unsigned(mine.from + 32 * k), adds, w.add + LN_HALF + mine.from + 32 * k, u);
        if (a.s1.q && live) {
            const Step step(__uint_as_float(top_u[k]));
            if (begins) a.s1.scales[group] = step.scale(__uint_as_float(top_u[k]));
            store_codes(u, step, a.s1.q + row * a.s1.ldq + c, cols - 32 * k);
        }
        if (k == 0) stage_free(w);
        gate32<T, ACT>(w.stage, w.lane, k, g, u);
    }
    put_piece(a, w, map, first, cols, 0);
}

template <typename T, int EPI, int ACT, bool LONG>
__global__ void __launch_bounds__(Shape<EPI, LONG>::THREADS, 1) linear_kernel(const LNArgs a, const __grid_constant__ CUtensorMap map_a0,
                                                              const __grid_constant__ CUtensorMap map_b0, const __grid_constant__ CUtensorMap map_a1,
                                                              const __grid_constant__ CUtensorMap map_b1, const __grid_constant__ CUtensorMap map_out) {
    constexpr bool A_MN = EPI == LN_OUTER, B_MN = EPI == LN_SUM || EPI == LN_OUTER;
    extern __shared__ uint8_t raw[];
    typedef Shape<EPI, LONG> S;
    constexpr int STORE_WARPS = S::STORE_WARPS, THREADS = S::THREADS;
    LNSmem<EPI, LONG>& sm = *reinterpret_cast<LNSmem<EPI, LONG>*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    volatile int* error = &sm.error;
    const unsigned rank = cta_rank();
    const unsigned pair = blockIdx.x / 2, pairs = gridDim.x / 2;
    if (tid == 0) {
        sm.error = sm.other_error = 0;
        for (int k = 0; k < LN_RING_MOST; ++k) {
            kb_init(&sm.empty[k], 1);
            kb_init(&sm.full[k], 1);
        }
        for (int b = 0; b < 2; ++b) {
            kb_init(&sm.acc_full[b], 1);
            kb_init(&sm.acc_empty[b], 2 * STORE_WARPS);
            kb_init(&sm.part_full[b], STORE_WARPS);
        }
        kb_fence_init();
    }
    if (tid == 32) {
        prefetch_map(&map_a0);
        prefetch_map(&map_b0);
        if (EPI != LN_SCORES && a.out != OUT_PLAIN && a.out != OUT_PLAIN32) prefetch_map(&map_out);
    }
    if (warp == LN_ALLOC_WARP) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(kb_smem_u32(&sm.tmem_base)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    pair_sync();                              // the other CTA's barriers are initialised
    tc_fence_after();
    // what the launches before it on the stream have written is there; the next one's CTAs may be set up
    grid_dependency();
    const unsigned tmem = sm.tmem_base;
    const unsigned tiles = unsigned(a.mt) * unsigned(a.nt) * unsigned(a.splits);      // below 2^30
    bool ok = true;

    if (warp == LN_COPY_WARP) {
        if (lane == 0) {
            const unsigned leader_full = pair_address(kb_smem_u32(sm.full), 0);
            unsigned g = 0;                                  // steps of all tiles so far
            Slot r;
            for (unsigned i = pair; ok && i < tiles; i += pairs) {
                const Place t = place_at<EPI>(a, i);
                const int y = (2 * t.m + int(rank)) * LN_M;
                // this CTA's half of the tile's columns; past 2^31, where there are none, it wraps to below 0, where there are none either
                const int x = int(unsigned(t.n) * unsigned(a.width) + rank * unsigned(a.width / 2));
                for (int s = 0; s < t.steps; ++s, ++g, r.next(a)) {
                    if (!kb_wait(kb_smem_u32(&sm.empty[r.slot]), r.parity ^ 1u, error)) { ok = false; break; }
                    if (rank == 0) kb_expect_tx(kb_smem_u32(&sm.full[r.slot]), 2 * LN_TILE + unsigned(a.width) * (LN_K * 2));
                    const unsigned bar = leader_full + r.slot * 8, da = kb_smem_u32(sm.ring) + r.slot * unsigned(a.slot_bytes), db = da + LN_TILE;
                    const int step = t.first + s;
                    const bool second = step >= a.steps0;
                    const int k = (second ? step - a.steps0 : step) * LN_K;
                    const int z = EPI == LN_OUTER ? t.split : 0;
                    if (A_MN) {
                        tma_load_pair(da, &map_a0, y, k, z, bar);
                        tma_load_pair(da + LN_BLOCK, &map_a0, y + 64, k, z, bar);
                    } else {
                        tma_load_pair(da, second ? &map_a1 : &map_a0, k, y, 0, bar);
                    }
                    if (B_MN) {
                        const CUtensorMap* map = second ? &map_b1 : &map_b0;
                        tma_load_pair(db, map, x, k, z, bar);
                        if (a.width == LN_N) tma_load_pair(db + LN_BLOCK, map, int(unsigned(x) + 64u), k, z, bar);
                    } else if (EPI == LN_GATED) {
                        tma_load_pair(db, rank == 0 ? &map_b0 : &map_b1, k, t.n * (a.width / 2), 0, bar);
                    } else {
                        tma_load_pair(db, &map_b0, k, x, 0, bar);
                    }
                }
            }
            // after a wait that gave up: the copies in flight land (the leading CTA counts them in) before
            // either CTA's shared memory is given back
            for (unsigned k = 0; !ok && rank == 0 && k < unsigned(a.ring) && k < g; ++k) {
                const unsigned step = g - 1 - k;
                kb_wait(kb_smem_u32(&sm.full[step % unsigned(a.ring)]), (step / unsigned(a.ring)) & 1u, error, true, 1u << 10);
            }
        }
    } else if (warp == LN_MMA_WARP) {
        // The whole warp walks the loop and one elected lane issues.
        if (rank == 0) {
            const unsigned idesc = instruction_desc(std::is_same<T, __half>::value ? 0 : 1, a.width, A_MN, B_MN);
            const unsigned long long desc_a = operand_desc(kb_smem_u32(sm.ring), A_MN ? LN_BLOCK : 16, 1024, 2);
            const unsigned long long desc_b = operand_desc(kb_smem_u32(sm.ring) + LN_TILE, B_MN ? LN_BLOCK : 16, 1024, 2);
            // 16 elements of the contraction: 32 bytes along a K-major row, 16 rows of 128 bytes of an MN-major block
            constexpr unsigned STEP_A = A_MN ? 128 : 2, STEP_B = B_MN ? 128 : 2;
            unsigned done = 0;
            Slot r;
            const unsigned slot_step = unsigned(a.slot_bytes) / 16;
            for (unsigned i = pair; ok && i < tiles; i += pairs) {
                const Place t = place_at<EPI>(a, i);
                const int steps = __shfl_sync(0xffffffffu, t.steps, 0);
                // an accumulator after the other, of the whole contraction or (LONG) of a chunk of it
                for (int s0 = 0; s0 < steps; s0 += LONG ? LN_CHUNK : steps, ++done) {
                    const unsigned half = done & 1u, round = (done >> 1) & 1u, d = tmem + half * LN_N;
                    if (!kb_wait_warp(kb_smem_u32(&sm.acc_empty[half]), round ^ 1u, error)) { ok = false; break; }
                    tc_fence_after();
                    const int here = LONG ? min(LN_CHUNK, steps - s0) : steps;
                    for (int s = 0; s < here; ++s, r.next(a)) {
                        if (!kb_wait_warp(kb_smem_u32(&sm.full[r.slot]), r.parity, error)) { ok = false; break; }
                        tc_fence_after();
                        const unsigned long long da = desc_a + r.slot * slot_step, db = desc_b + r.slot * slot_step;
                        if (elect_one()) {
#pragma unroll
                            for (int k = 0; k < LN_K / 16; ++k) mma_f16(d, da + k * STEP_A, db + k * STEP_B, idesc, s > 0 || k > 0);
                            mma_commit(&sm.empty[r.slot]);
                        }
                        __syncwarp();
                    }
                    if (!ok) break;
                    if (elect_one()) mma_commit(&sm.acc_full[half]);
                    __syncwarp();
                }
            }
            // nothing is in flight when the tensor memory is freed: on the good path the store warps have
            // seen every accumulator; after a wait that gave up, wait for what was issued
            if (!ok) {
                const unsigned half = done & 1u, round = (done >> 1) & 1u;
                if (elect_one()) mma_commit(&sm.acc_full[half]);
                __syncwarp();
                kb_wait(kb_smem_u32(&sm.acc_full[half]), round, error, true, 1u << 10);
            }
        }
    } else if (warp >= LN_STORE_WARP0) {
        Warp w;
        w.group = (warp - LN_STORE_WARP0) / 4;
        w.quarter = warp % 4;                                // its lanes of tensor memory: 32 quarter ..
        w.stage = kb_smem_u32(sm.out[warp - LN_STORE_WARP0]);
        w.add = sm.add[warp - LN_STORE_WARP0];
        w.lane = lane;
        unsigned done = 0, turn = 0;                         // accumulators and tiles so far
        Place t = place_at<EPI>(a, pair);                    // (a pair has a tile at least)
        RowInputs in = ask_inputs<EPI>(a, t, rank, w.quarter, lane);
        for (unsigned i = pair; ok && i < tiles; i += pairs, ++turn) {
            if (LONG && i != pair) {                         // (its first chunk is long enough to wait for them)
                t = place_at<EPI>(a, i);
                in = ask_inputs<EPI>(a, t, rank, w.quarter, lane);
            }
            w.row0 = int64_t(2 * t.m + int(rank)) * LN_M + w.quarter * 32;
            fetch_tile_biases<T, EPI, LONG>(a, t, w);
            Place next = t;
            RowInputs next_in = in;
            if (!LONG && i + pairs < tiles) {
                next = place_at<EPI>(a, i + pairs);
                next_in = ask_inputs<EPI>(a, next, rank, w.quarter, lane);
            }
            [[maybe_unused]] Logits<LONG> logits;
            [[maybe_unused]] Columns mine{0, 0};
            if constexpr (S::LOGITS) mine = logits_columns<S::GROUPS>(a, t, w.group);
            // the accumulators of the chunks, or the one there is: its half is given back when it has been read
            for (int s0 = 0;;) {
                const unsigned half = done & 1u;
                if (!kb_wait_warp(kb_smem_u32(&sm.acc_full[half]), (done >> 1) & 1u, error)) { ok = false; break; }
                tc_fence_after();
                __syncwarp();                                // the warp's biases are there
                w.src = tmem + half * LN_N + (unsigned(w.quarter * 32) << 16);
                if constexpr (S::LOGITS) logits.chunk(w.src + unsigned(mine.from), w.row0 < a.rows ? mine.to - mine.from : 0, s0 == 0);
                if (!LONG) break;
                tc_fence_before();
                __syncwarp();
                if (lane == 0) arrive_at_leader(&sm.acc_empty[half]);
                ++done;
                s0 += LN_CHUNK;
                if (s0 >= t.steps) break;
            }
            if (!ok) break;
            if constexpr (EPI == LN_SCORES) {
                const int own = w.quarter * 32 + lane;
                const unsigned at = turn & 1u;
                sm.part[at][w.group][own] = scores_tile<LONG>(a, t, w, in, mine, logits);
                __syncwarp();
                if (lane == 0) kb_arrive(&sm.part_full[at]);
                if (w.group == 0) {
                    if (!kb_wait_warp(kb_smem_u32(&sm.part_full[at]), (turn >> 1) & 1u, error)) break;
                    const int64_t row = w.row0 + lane;
                    if (row < a.rows) a.parts[row * a.nt + t.n] = join_groups<S::GROUPS>(sm.part[at], own);
                }
            }
            if constexpr (EPI == LN_DLOGITS) dlogits_tile<T, LONG>(a, t, w, in, mine, logits, &map_out);
            if constexpr (EPI == LN_GATED) gated_tile<T, ACT>(a, t, w, &map_out);
            if constexpr (EPI == LN_SUM || EPI == LN_OUTER) sum_tile<T, EPI>(a, t, w, &map_out);
            if (!LONG) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) arrive_at_leader(&sm.acc_empty[done & 1u]);
                ++done;
            }
            if (!LONG) {
                t = next;
                in = next_in;
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
    if (warp == LN_ALLOC_WARP)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    if (sm.error || *static_cast<volatile int*>(&sm.other_error)) {
        // a wait gave up: nothing the pair was to write may look like a result
        const int WIDTH = EPI == LN_SCORES ? 1 : EPI == LN_GATED ? a.width / 2 : a.width;
        for (unsigned i = pair; i < tiles; i += pairs) {
            const Place t = place_at<EPI>(a, i);
            for (int e = tid; e < LN_M * WIDTH; e += THREADS) {
                const int64_t row = int64_t(2 * t.m + int(rank)) * LN_M + e / WIDTH, c = int64_t(t.n) * WIDTH + e % WIDTH;
                if (row >= a.rows) continue;
                if constexpr (EPI == LN_SCORES) a.parts[row * a.nt + t.n] = make_float2(CUDART_NAN_F, CUDART_NAN_F);
                else if (c < a.cols) {
                    const int64_t at = int64_t(t.split) * a.plane + row * a.ldy + c;
                    if (a.out >= OUT_PART) static_cast<float*>(a.y)[at] = CUDART_NAN_F;
                    else static_cast<T*>(a.y)[at] = Elem<T>::narrow(CUDART_NAN_F);
                    if (EPI == LN_GATED && (c & ((1 << a.group_shift) - 1)) == 0) {
                        if (a.s0.q) a.s0.scales[row * a.groups + (c >> a.group_shift)] = CUDART_NAN_F;
                        if (a.s1.q) a.s1.scales[row * a.groups + (c >> a.group_shift)] = CUDART_NAN_F;
                    }
                }
            }
        }
    }
}

// ---- around the products ----------------------------------------------------------------------------
// The parts of a row joined: a warp per row.
__global__ void __launch_bounds__(256) join_scores_kernel(const float2* parts, const float* target_z, const int64_t* targets, int64_t rows, int nt,
                                                          int64_t vocab, float* logprobs, float* lse, float* lse_lo) {
    grid_dependency();
    const int64_t row = int64_t(blockIdx.x) * 8 + threadIdx.x / 32;
    const int lane = threadIdx.x % 32;
    if (row >= rows) return;
    const float2* p = parts + row * nt;
    float m = -CUDART_INF_F, s = 0.f;
    for (int k = lane; k < nt; k += 32) {
        const float2 q = p[k];
        const float higher = fmaxf(m, q.x);
        if (higher == -CUDART_INF_F) {
            s += q.y;                          // 0, or NaN
        } else {
            // a part without a finite maximum adds 0; NaN stays
            s = s * ex2((m - higher) * kLog2e) + q.y * ex2((q.x - higher) * kLog2e);
            m = higher;
        }
    }
    float top = m;
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (top != -CUDART_INF_F) s *= ex2((m - top) * kLog2e);
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (lane) return;
    // the sum of a row without entries is 0, of one with NaN or +inf NaN
    const float l = logf(s);
    const float hi = top == -CUDART_INF_F ? (s == 0.f ? top : CUDART_NAN_F) : top + l;
    if (lse) lse[row] = hi;
    if (lse_lo) {
        // two-sum: top + l = hi + lo
        const float bb = hi - top;
        const float lo = (top - (hi - bb)) + (l - bb);
        lse_lo[row] = fabsf(hi) <= 3.402823466e38f ? lo : 0.f;
    }
    if (logprobs) {
        const int64_t t = targets[row];
        float lp = 0.f;
        if (t >= vocab) lp = CUDART_NAN_F;
        else if (t >= 0) lp = top == -CUDART_INF_F ? hi : (target_z[row] - top) - l;
        logprobs[row] = lp;
    }
}

// Rows of 16-bit elements copied to rows that start on 16 bytes, eight elements per thread and turn; up to four matrices,
// one per blockIdx.y.  A job with targets is the rows of a head: those whose coefficient is 0 are copied as zeros, and the coefficients
// (the gradient at a row's log probability; 0 without a target and in a row masked throughout, whatever comes in; NaN for a target
// outside the vocabulary) are written.  Where the
// largest one's magnitude is asked for, the blocks behind the jobs find it, a worker each: one for all workers would let one
// worker's coefficients push the others' dz below binary16's range.
struct CopyJob {
    const unsigned short* src;
    int64_t        ld, cols, pieces, per_row;
    uint4*         dst;
    int            aligned;                // the source's rows start on 16 bytes
};
struct CopyArgs {
    CopyJob        job[4];
    int            jobs;
    const int64_t* targets;                // of the first job; or null
    const float *  grad, *lse;
    int64_t        vocab, tokens;
    int            workers;
    unsigned       fold;                   // the first job's rows are written twice, worker by worker (unfold); 0: once
    float*         coef;
    unsigned*      top;                    // [workers]; null: not asked for
};
__device__ __forceinline__ float coefficient(const CopyArgs& a, int64_t row) {
    const int64_t t = a.targets[row];
    return t < 0 || a.lse[row] == -CUDART_INF_F ? 0.f : t >= a.vocab ? CUDART_NAN_F : a.grad[row];
}
__global__ void __launch_bounds__(256) copy_rows_kernel(const CopyArgs a) {
    grid_dependency();
    if (blockIdx.y == unsigned(a.jobs)) {
        __shared__ unsigned most[8];
        for (int w = int(blockIdx.x); w < a.workers; w += int(gridDim.x)) {
            unsigned top = 0;
#pragma unroll 8
            for (int64_t i = threadIdx.x; i < a.tokens; i += 256) {
                const unsigned bits = __float_as_uint(coefficient(a, w * a.tokens + i)) & 0x7fffffffu;
                if (bits < 0x7f800000u) top = max(top, bits);
            }
            top = __reduce_max_sync(0xffffffffu, top);
            if (threadIdx.x % 32 == 0) most[threadIdx.x / 32] = top;
            __syncthreads();
            if (threadIdx.x == 0) {
                for (int k = 1; k < 8; ++k) top = max(top, most[k]);
                a.top[w] = top;
            }
            __syncthreads();                           // `most` has been read
        }
        return;
    }
    const CopyJob& j = a.job[blockIdx.y];
    const bool head = a.targets && blockIdx.y == 0;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < j.pieces; i += int64_t(gridDim.x) * 256) {
        const int64_t row = i / j.per_row, c = (i - row * j.per_row) * 8;
        bool zero = false;
        int64_t from = row;
        if (head) {
            if (a.fold) from = unfold(unsigned(row), a.fold).row;
            const float coef = coefficient(a, from);
            zero = coef == 0.f;
            if (c == 0) a.coef[row] = coef;
        }
        const unsigned short* p = j.src + from * j.ld + c;
        uint4 w = make_uint4(0, 0, 0, 0);
        if (!zero) {
            if (j.aligned && c + 8 <= j.cols) {
                w = __ldg(reinterpret_cast<const uint4*>(p));
            } else {
                unsigned v[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = c + k < j.cols ? __ldg(p + k) : 0u;
                w = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
            }
        }
        j.dst[i] = w;
    }
}

// Bias gradients: the columns of a worker's dz added up, eight columns and every SLICES-th token per thread, the slices in order.
constexpr int LN_SLICES = 32;
template <typename T, typename G>
__global__ void __launch_bounds__(32 * LN_SLICES) column_sums_kernel(const T* dz, int64_t ld, int64_t tokens, int64_t cols, const unsigned* top, G* db,
                                                                    int64_t ld_grads) {
    __shared__ float sums[LN_SLICES][32][9];
    grid_dependency();
    const int64_t c = (int64_t(blockIdx.x) * 32 + threadIdx.x % 32) * 8;
    const int slice = threadIdx.x / 32;
    float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    const T* p = dz + int64_t(blockIdx.y) * tokens * ld + c;
    // (rows of dz are padded to whole pieces; what lies behind the last column is added and not stored)
    if (c < cols) {
#pragma unroll 4
        for (int64_t t = slice; t < tokens; t += LN_SLICES) {
            float v[8];
            widen16B(__ldg(reinterpret_cast<const uint4*>(p + t * ld)), v, static_cast<const T*>(nullptr));
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j] += v[j];
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[slice][threadIdx.x % 32][j] = s[j];
    __syncthreads();
    const int64_t mine = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (threadIdx.x >= 256 || mine >= cols) return;
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < LN_SLICES; ++k) sum += sums[k][threadIdx.x / 8][threadIdx.x % 8];
    if (top) sum *= power_for(top[blockIdx.y], true);
    db[int64_t(blockIdx.y) * ld_grads + mine] = Elem<G>::narrow(sum);
}

// The parts of a sum, added in order and rounded once, four columns per thread and turn.  fold: a row's sum and that of its second
// part, `fold` rows behind it.
template <typename T>
__global__ void __launch_bounds__(256) join_parts_kernel(const float* parts, int64_t plane, int64_t pitch, int splits, int64_t rows, int64_t cols,
                                                         const unsigned* top, unsigned tokens, unsigned fold, T* y, int64_t ldy) {
    grid_dependency();
    const int64_t per_row = (cols + 3) / 4, pieces = rows * per_row;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < pieces; i += int64_t(gridDim.x) * 256) {
        const int64_t row = i / per_row, c = (i - row * per_row) * 4;
        const int64_t at = fold ? row + row / fold * fold : row;
        const float* p = parts + at * pitch + c;
        const float by = top ? power_for(top[unsigned(at) / tokens], true) : 1.f;
        float4 s = __ldcs(reinterpret_cast<const float4*>(p));
        for (int k = 1; k < splits; ++k) {
            const float4 q = __ldcs(reinterpret_cast<const float4*>(p + k * plane));
            s.x += q.x; s.y += q.y; s.z += q.z; s.w += q.w;
        }
        for (int k = 0; fold && k < splits; ++k) {
            const float4 q = __ldcs(reinterpret_cast<const float4*>(p + fold * pitch + k * plane));
            s.x += q.x; s.y += q.y; s.z += q.z; s.w += q.w;
        }
        T out[4] = {Elem<T>::narrow(s.x * by), Elem<T>::narrow(s.y * by), Elem<T>::narrow(s.z * by), Elem<T>::narrow(s.w * by)};
        T* dst = y + row * ldy + c;
        if (c + 4 <= cols && reinterpret_cast<uintptr_t>(dst) % 8 == 0) {
            *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(out);
        } else {
            for (int j = 0; j < 4; ++j)
                if (c + j < cols) dst[j] = out[j];
        }
    }
}

// ---- launches ---------------------------------------------------------------------------------------
bool on_16(const void* p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0; }
int64_t up_to(int64_t v, int64_t m) { return (v + m - 1) / m * m; }
int64_t parts_of(int64_t v, int64_t m) { return (v + m - 1) / m; }
CUtensorMapDataType map_type(int dtype) { return dtype == GAR_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16; }

// A 16-bit matrix as the tensor maps take it: rows that start on 16 bytes.
struct Operand {
    const char* p;
    int64_t     rows, cols, ld;
};
cudaError_t operand_map(CUtensorMap* map, int dtype, const Operand& m, int box_cols, int box_rows,
                        CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B) {
    const int64_t pitch = 2 * (m.rows > 1 ? m.ld : up_to(m.cols, 8));         // (a single row's stride may be anything)
    return make_map(map, map_type(dtype), m.p, m.cols, m.rows, 1, pitch, pitch * m.rows, box_cols, box_rows, swizzle);
}

// A workspace handed out piece by piece; without memory it only counts.
class Space {
public:
    explicit Space(void* base) : base_(static_cast<char*>(base)) {}
    char* take(size_t bytes) {
        char* p = base_ ? base_ + used_ : nullptr;
        used_ += gar::align256(bytes);
        return p;
    }
    size_t used() const { return used_; }

private:
    char*  base_;
    size_t used_ = 0;
};

double products(int64_t rows, int64_t hidden, int64_t wide) { return double(rows) * double(hidden) * double(wide); }
unsigned copy_blocks(int64_t pieces, int sm_count) { return unsigned(std::min<int64_t>(int64_t(16) * sm_count, parts_of(pieces, 256))); }

// A launch that may be set up while the one before it on the stream ends: every kernel here waits for that one's
// results first (grid_dependency).
template <int THREADS = 256, typename... P, typename... A>
cudaError_t launch_small(void (*kernel)(P...), dim3 grid, cudaStream_t stream, A... args) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(THREADS);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

// A matrix of the caller's as an operand: where it lies, or copied to the space reserved for it.  It is copied where TMA does not take
// it, and where its rows start between the sectors of 32 bytes, if enough tiles read it: a box's rows of 128 bytes then touch five
// sectors instead of four.  1000 x 50001, 1000 elements a row, scores: 115 us, with x copied 100; 8192 x 20000 306, with x and W copied 279;
// with W read by eight tiles its copy costs more than it saves (2048 x 20000, gated 163, copied 175).
constexpr int64_t LN_PITCH = 16;                       // elements: rows of copies start on 32 bytes
struct Input {
    Operand m;
    char*   copy = nullptr;
    bool    copied;
    // reads: tiles that read each of its elements; work: products of the call
    Input(Space& space, const void* p, int64_t rows, int64_t cols, int64_t ld, int64_t reads, double work)
        : m{static_cast<const char*>(p), rows, cols, ld}, copied(!on_16(p, ld)) {
        const bool split = rows > 1 && (reinterpret_cast<uintptr_t>(p) % 32 != 0 || ld % 16 != 0);
        if (split && reads >= 16 && work >= 8e9) copied = true;
        if (copied) copy = space.take(size_t(rows) * size_t(up_to(cols, LN_PITCH)) * 2);
    }
};
CopyJob copy_job(const Operand& src, void* dst, int64_t ld) {
    return CopyJob{reinterpret_cast<const unsigned short*>(src.p), src.ld, src.cols, src.rows * (ld / 8), ld / 8, static_cast<uint4*>(dst), on_16(src.p, src.ld)};
}
// The copies of a call, in one launch.
struct Copies {
    CopyArgs a{};
    int      n = 0;
    int64_t  most = 0;
    void add(const CopyJob& j) {
        a.job[n++] = j;
        most = std::max(most, j.pieces);
    }
    void add(Input& in) {
        if (!in.copied) return;
        const int64_t ld = up_to(in.m.cols, LN_PITCH);
        add(copy_job(in.m, in.copy, ld));
        in.m.p = in.copy;
        in.m.ld = ld;
    }
    cudaError_t launch(int sm_count, cudaStream_t stream) {
        a.jobs = n;
        return most > 0 ? launch_small(copy_rows_kernel, dim3(copy_blocks(most, sm_count), unsigned(n + (a.top ? 1 : 0))), stream, a) : cudaSuccess;
    }
};

struct Maps {
    CUtensorMap a0, b0, a1, b1, out;
};

template <typename T, int EPI, int ACT, bool LONG>
cudaError_t launch_as(LNArgs a, const Maps& maps, int sm_count, cudaStream_t stream) {
    constexpr int bytes = int(sizeof(LNSmem<EPI, LONG>)) + 1024;
    static_assert(bytes <= 232448, "a CTA's shared memory");
    auto kernel = linear_kernel<T, EPI, ACT, LONG>;
    static std::atomic<uint64_t> allowed{0};           // devices on which the kernel may have that much
    int dev = 0;
    if (cudaError_t err = cudaGetDevice(&dev)) return err;
    if (dev >= 64 || !(allowed.load(std::memory_order_relaxed) >> dev & 1)) {
        if (cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes)) return err;
        if (dev < 64) allowed.fetch_or(uint64_t(1) << dev, std::memory_order_relaxed);
    }
    // (an outer product's tiles go along its rows, which are then written whole: 11 x 128 tokens, 32000 x 1024, fp32 rows, whole backward
    // pass without dx 370 us, row tiles in groups of 64 396; in other runs 410 to 420)
    a.group_m = EPI == LN_OUTER ? 1 : group_rows(a.steps, a.mt);
    a.slot_bytes = LN_TILE + a.width * LN_K;
    a.ring = std::min(LN_RING_MOST, LN_RING_BYTES / a.slot_bytes);
    const int64_t tiles = int64_t(a.mt) * a.nt * a.splits;
    if (tiles >= int64_t(1) << 30) return cudaErrorInvalidConfiguration;
    const int64_t pairs = sm_count / 2 > 1 ? sm_count / 2 : 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(unsigned(2 * std::min(tiles, pairs)));
    cfg.blockDim = dim3(Shape<EPI, LONG>::THREADS);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 2;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a, maps.a0, maps.b0, maps.a1, maps.b1, maps.out);
}
template <int EPI, int ACT = 0, bool LONG = false>
cudaError_t launch(int dtype, const LNArgs& a, const Maps& maps, int sm_count, cudaStream_t stream) {
    return dtype == GAR_BF16 ? launch_as<__nv_bfloat16, EPI, ACT, LONG>(a, maps, sm_count, stream) : launch_as<__half, EPI, ACT, LONG>(a, maps, sm_count, stream);
}
template <int EPI>
cudaError_t launch_logits(int dtype, const LNArgs& a, const Maps& maps, int sm_count, cudaStream_t stream) {
    return a.steps > LN_ONE ? launch<EPI, 0, true>(dtype, a, maps, sm_count, stream) : launch<EPI>(dtype, a, maps, sm_count, stream);
}

// Columns of a tile, a multiple of `unit` up to 256.  A step's copies come at some 47 bytes per cycle and SM, 16 KB of A and 64
// bytes per column of B, and the last tile's epilogue, some 22 cycles per column, is hidden by nothing: the width with the
// least of (rounds of the pairs) x steps x (348 + 1.36 width) + 22 width.  Few tiles get narrow ones, one for each pair; many
// get 256 columns, or what leaves no part of the last round idle.
int width_for(int64_t mt, int64_t cols, int64_t steps, int unit, int columns_of = 1) {
    int best = LN_N;
    double least = 0;
    for (int w = LN_N; w >= unit; w -= unit) {
        const double rounds = double(parts_of(mt * parts_of(cols, w / columns_of), LN_PAIRS));
        const double t = rounds * double(steps) * (348 + 1.36 * w) + 22.0 * w;
        if (w == LN_N || t < least) {
            least = t;
            best = w;
        }
    }
    return best;
}

// z = x W^T over `rows` rows and the columns of `w`: the operands' part of a launch, tiles of a multiple of `unit` columns
cudaError_t logits_maps(Maps& maps, LNArgs& a, int dtype, const Operand& x, const Operand& w, int unit) {
    a.rows = x.rows;
    a.cols = w.rows;
    a.mt = int(parts_of(x.rows, 2 * LN_M));
    a.splits = 1;
    a.steps0 = a.steps = int(parts_of(x.cols, LN_K));
    a.width = width_for(a.mt, a.cols, a.steps, unit);
    a.nt = int(parts_of(w.rows, a.width));
    if (cudaError_t err = operand_map(&maps.a0, dtype, x, LN_K, LN_M)) return err;
    if (cudaError_t err = operand_map(&maps.b0, dtype, w, LN_K, a.width / 2)) return err;
    maps.a1 = maps.b1 = maps.out = maps.a0;            // not used unless set
    return cudaSuccess;
}

// Parts a sum over a long contraction is cut into, `least` at least, so that the tiles fill the rounds of the pairs: the least of
// rounds x (steps of a part + 6), a step taking some 0.28 us, and of the parts' way through L2 and back (8 bytes at 4 TB/s).
// Two workers x 2048 tokens, 131072 x 4096: 256 tiles are 3.5 rounds, in two parts 6.9.
int splits_for(int64_t rows, int64_t cols, int64_t steps, int64_t least, bool parts_anyway) {
    const int64_t tiles = parts_of(rows, 2 * LN_M) * parts_of(cols, LN_N);
    int64_t best = least;
    double cost = 0;
    for (int64_t s = least; s <= std::max<int64_t>(16, least); ++s) {
        if (s > least && steps < 8 * s) break;
        const double through = s > 1 || parts_anyway ? double(s) * double(rows) * double(cols) * 8 / 4e6 : 0;          // us
        const double t = double(parts_of(tiles * s, LN_PAIRS)) * double(parts_of(steps, s) + 6) * 0.28 + through;
        if (s == least || t < cost) {
            cost = t;
            best = s;
        }
    }
    return int(parts_of(steps, parts_of(steps, best)));        // no part is empty
}

// dx, or a part of it, in fp32 parts or as it is wanted.
struct SumTarget {
    int      dtype;
    void*    dx;
    int64_t  rows, cols, ld;
    float*   parts;                                    // [splits][rows][pitch]; null: straight to dx
    int64_t  pitch;
    int      splits;
    const unsigned* top;                               // dz carries power_for(top[row / tokens]); or null
    unsigned tokens, fold;                             // fold: dz in two parts (LNArgs::fold); always with `parts`
};
cudaError_t launch_sum(const SumTarget& d, const Operand& a0, const Operand& b0, const Operand* a1, const Operand* b1, bool add, int sm_count, cudaStream_t stream) {
    Maps maps;
    LNArgs a{};
    a.rows = d.rows;
    a.cols = d.cols;
    a.mt = int(parts_of(d.rows, 2 * LN_M));
    a.steps0 = int(parts_of(a0.cols, LN_K));
    a.steps = a.steps0 + (a1 ? int(parts_of(a1->cols, LN_K)) : 0);
    // (a shorter last piece of the contraction may have steps for fewer parts)
    const int part = (a.steps + d.splits - 1) / d.splits;
    a.splits = (a.steps + part - 1) / part;
    a.width = width_for(int64_t(a.mt) * a.splits, d.cols, part, 128);
    a.nt = int(parts_of(d.cols, a.width));
    if (cudaError_t err = operand_map(&maps.a0, d.dtype, a0, LN_K, LN_M)) return err;
    if (cudaError_t err = operand_map(&maps.b0, d.dtype, b0, 64, LN_K)) return err;
    maps.a1 = maps.a0;
    maps.b1 = maps.b0;
    if (a1) {
        if (cudaError_t err = operand_map(&maps.a1, d.dtype, *a1, LN_K, LN_M)) return err;
        if (cudaError_t err = operand_map(&maps.b1, d.dtype, *b1, 64, LN_K)) return err;
    }
    maps.out = maps.a0;
    if (d.parts) {
        a.out = add ? OUT_ADD : OUT_PART;
        a.y = d.parts;
        a.ldy = d.pitch;
        a.plane = d.pitch * d.rows;
        if (cudaError_t err = make_map(&maps.out, CU_TENSOR_MAP_DATA_TYPE_FLOAT32, d.parts, d.cols, d.rows, d.splits, d.pitch * 4, d.pitch * 4 * d.rows, 32, 32,
                                       CU_TENSOR_MAP_SWIZZLE_128B)) return err;
    } else {
        a.out = on_16(d.dx, d.ld) ? OUT_WIDE : OUT_PLAIN;
        a.y = d.dx;
        a.ldy = d.ld;
        a.top = d.top;
        a.tokens = d.tokens;
        if (a.out == OUT_WIDE)
            if (cudaError_t err = operand_map(&maps.out, d.dtype, Operand{static_cast<const char*>(d.dx), d.rows, d.cols, d.ld}, 64, 32)) return err;
    }
    return launch<LN_SUM>(d.dtype, a, maps, sm_count, stream);
}
cudaError_t join_sum(const SumTarget& d, int sm_count, cudaStream_t stream) {
    const int64_t rows = d.fold ? d.rows / 2 : d.rows;
    const dim3 grid(copy_blocks(rows * parts_of(d.cols, 4), sm_count));
    if (d.dtype == GAR_BF16)
        return launch_small(join_parts_kernel<__nv_bfloat16>, grid, stream, d.parts, d.rows * d.pitch, d.pitch, d.splits, rows, d.cols, d.top, d.tokens, d.fold,
                            static_cast<__nv_bfloat16*>(d.dx), d.ld);
    return launch_small(join_parts_kernel<__half>, grid, stream, d.parts, d.rows * d.pitch, d.pitch, d.splits, rows, d.cols, d.top, d.tokens, d.fold,
                        static_cast<__half*>(d.dx), d.ld);
}

// ---- weight gradients -------------------------------------------------------------------------------
// the block's rows as TMA stores them
bool block_on_16(const DenseWeightGrad& g) {
    const int64_t gs = g.grads_dtype == GAR_F32 ? 4 : 2;
    return reinterpret_cast<uintptr_t>(g.dw) % 16 == 0 && (g.workers == 1 || g.ld_grads * gs % 16 == 0) && g.in * gs % 16 == 0;
}
}  // namespace
// Where this kernel makes them: sums short enough for one accumulator (see gar_linear_weight_grad's chunks).  Two store groups, and a
// pair's next tile in the other half of tensor memory, keep up with the block's rows where there are few tokens to a tile:
// 11 workers x 128 tokens, 16128 x 1024, bf16 rows: 70 us, 98 by weight_grad_kernel's four store warps.  Rows that start anywhere are
// stored in words of 4 bytes (whole backward pass without dx, weight_grad_kernel in brackets): 11 x 128, 100 x 512 15.4 us (22.5); 7 x 100,
// 2000 x 501, fp32 25.2 (30.8); 2 x 2000, 16000 x 2047, bf16 483 (525); 4 x 700, 8000 x 2050, fp32 260 (269); but 11 x 128, 32000 x 1024, fp32,
// 1.4 GB of rows with little to compute, 668 (525 to 546): those are left to the latter, which shifts rows to 16-byte chunks.
bool outer_applies(const DenseWeightGrad& g) {
    const int64_t gs = g.grads_dtype == GAR_F32 ? 4 : 2;
    if (g.tokens < 1 || g.tokens > (gs == 4 ? 768 : 2048)) return false;
    if (gs == 4 && g.tokens < 512 && !block_on_16(g) && g.out * g.in * g.workers > (int64_t(16) << 20)) return false;
    return (gs == 4 || g.grads_dtype == g.dtype) && parts_of(g.out, 2 * LN_M) * parts_of(g.in, LN_N) < (int64_t(1) << 30) / g.workers / 2;
}
namespace {
cudaError_t token_map(CUtensorMap* map, int dtype, const void* p, int64_t cols, int64_t ld, const DenseWeightGrad& g) {
    return make_map(map, map_type(dtype), p, cols, g.tokens, g.workers, ld * 2, ld * 2 * g.tokens, 64, LN_K, CU_TENSOR_MAP_SWIZZLE_128B);
}
}  // namespace
cudaError_t launch_outer(const DenseWeightGrad& g, int sm_count, cudaStream_t stream) {
    Maps maps;
    LNArgs a{};
    const bool wide = g.grads_dtype == GAR_F32;
    const int64_t gs = wide ? 4 : 2;
    a.rows = g.out;
    a.cols = g.in;
    a.mt = int(parts_of(g.out, 2 * LN_M));
    a.splits = g.workers;
    a.steps0 = a.steps = int(parts_of(g.tokens, LN_K));
    a.width = width_for(int64_t(a.mt) * g.workers, g.in, a.steps, 128);
    a.nt = int(parts_of(g.in, a.width));
    const bool by_tma = block_on_16(g);
    a.out = wide ? (by_tma ? OUT_PART : OUT_PLAIN32) : by_tma ? OUT_WIDE : OUT_PLAIN;
    a.top = g.top;
    a.y = g.dw;
    a.ldy = g.in;
    a.plane = g.ld_grads;
    if (cudaError_t err = token_map(&maps.a0, g.dtype, g.dy, g.out, g.ld_dy, g)) return err;
    if (cudaError_t err = token_map(&maps.b0, g.dtype, g.x, g.in, g.ldx, g)) return err;
    maps.a1 = maps.b1 = maps.a0;                       // not used
    maps.out = maps.a0;
    const int64_t plane = g.workers > 1 ? g.ld_grads * gs : g.in * g.out * gs;
    if (!by_tma) return launch<LN_OUTER>(g.dtype, a, maps, sm_count, stream);
    if (cudaError_t err = make_map(&maps.out, wide ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : map_type(g.dtype), g.dw, g.in, g.out, g.workers, g.in * gs, plane,
                                   int(128 / gs), 32, CU_TENSOR_MAP_SWIZZLE_128B)) return err;
    return launch<LN_OUTER>(g.dtype, a, maps, sm_count, stream);
}
namespace {
template <typename T>
cudaError_t column_sums(const DenseWeightGrad& g, cudaStream_t stream) {
    const dim3 grid(unsigned(parts_of(g.out, 256)), unsigned(g.workers));
    const T* dz = static_cast<const T*>(g.dy);
    if (g.grads_dtype == GAR_F32) return launch_small<32 * LN_SLICES>(column_sums_kernel<T, float>, grid, stream, dz, g.ld_dy, g.tokens, g.out, g.top, static_cast<float*>(g.db), g.ld_grads);
    if (g.grads_dtype == GAR_BF16)
        return launch_small<32 * LN_SLICES>(column_sums_kernel<T, __nv_bfloat16>, grid, stream, dz, g.ld_dy, g.tokens, g.out, g.top, static_cast<__nv_bfloat16*>(g.db), g.ld_grads);
    return launch_small<32 * LN_SLICES>(column_sums_kernel<T, __half>, grid, stream, dz, g.ld_dy, g.tokens, g.out, g.top, static_cast<__half*>(g.db), g.ld_grads);
}
cudaError_t weight_grad(DenseWeightGrad g, int sm_count, cudaStream_t stream) {
    if (!outer_applies(g)) return launch_dense_weight_grad(g, sm_count, stream);
    if (cudaError_t err = launch_outer(g, sm_count, stream)) return err;
    if (!g.db) return cudaSuccess;
    return g.dtype == GAR_BF16 ? column_sums<__nv_bfloat16>(g, stream) : column_sums<__half>(g, stream);
}

// ---- log probabilities ------------------------------------------------------------------------------
constexpr int64_t LN_PARTS_BYTES = int64_t(64) << 20, LN_PIECE_BYTES = int64_t(96) << 20;
constexpr int64_t LN_TERMS = 32768;                            // of a sum on the tensor cores
constexpr int64_t LN_FEW_PARTS = 512;                          // CTAs of a few rows' kernel at most: two per SM
constexpr int LN_UNIT = 32;                                    // columns of a thread's turn
// rows of a launch, so that its parts take 64 MB or so
int64_t rows_at_once(int64_t rows, int64_t vocab) {
    const int64_t most = std::max<int64_t>(256, LN_PARTS_BYTES / (8 * parts_of(vocab, LN_N)) / 256 * 256);
    return std::min(rows, most);
}
int64_t scores_tiles(int64_t rows, int64_t hidden, int64_t vocab) {
    return parts_of(vocab, width_for(parts_of(rows, 2 * LN_M), vocab, parts_of(hidden, LN_K), LN_UNIT));
}
struct ScoresPlan {
    Space   space;
    Input   x, w;
    int64_t rows;
    float2* parts;
    float*  target_z;
    ScoresPlan(const gar_linear_logprobs_params_t& p, int64_t ldx, int64_t ldw)
        : space(p.workspace), x(space, p.x, p.rows, p.hidden, ldx, parts_of(p.vocab, LN_N), products(p.rows, p.hidden, p.vocab)),
          w(space, p.weight, p.vocab, p.hidden, ldw, parts_of(p.rows, 2 * LN_M), products(p.rows, p.hidden, p.vocab)), rows(rows_at_once(p.rows, p.vocab)) {
        // (the last rows, if they are fewer, may have narrower tiles; a few rows have a part per CTA)
        const int64_t last = (p.rows - 1) % rows + 1;
        const int64_t most = p.rows <= 16 ? std::max(p.rows * scores_tiles(p.rows, p.hidden, p.vocab), p.rows * LN_FEW_PARTS)
                                          : std::max(rows * scores_tiles(rows, p.hidden, p.vocab), last * scores_tiles(last, p.hidden, p.vocab));
        parts = reinterpret_cast<float2*>(space.take(size_t(most) * 8));
        target_z = reinterpret_cast<float*>(space.take(size_t(rows) * 4));
    }
};

// Columns of a piece of the vocabulary: dz of up to 96 MB (L2 holds it).  Of the sizes between that and half of it the one with the
// least of (rounds of the pairs over all pieces) x (steps x 0.28 + 1.5 us) and 8 us a piece, for its launches and their ends.
// Two workers x 2048 tokens, 131072 x 4096: 46 tiles of columns (10 rounds each) instead of 47 (11).
int64_t piece_of(int64_t rows, int64_t hidden, int64_t vocab) {
    const int64_t mt = parts_of(rows, 2 * LN_M), all = parts_of(vocab, LN_N);
    const int64_t most = std::min(all, std::max<int64_t>(1, LN_PIECE_BYTES / (2 * rows) / LN_N));
    const double round = double(parts_of(hidden, LN_K)) * 0.28 + 1.5;
    int64_t best = most;
    double cost = 0;
    for (int64_t n = most; n >= std::max<int64_t>(1, most / 2); --n) {
        const int64_t full = all / n, last = all % n;
        const double t = double(full * parts_of(mt * n, LN_PAIRS) + parts_of(mt * last, LN_PAIRS)) * round + 8.0 * double(full + (last > 0));
        if (n == most || t < cost) {
            cost = t;
            best = n;
        }
    }
    return best * LN_N;
}
// Rows up to which dz, which is rounded to 16 bits, comes in two parts, the second of what rounding the first left out, a row each: a
// pair's tile of 256 rows has room for both, at no product's cost.  Few coefficients decide a gradient there, whose roundings do not
// average out: 8 workers x 2 tokens, 10 columns, bf16: gradients 2.6e-3 off in the mean, 1.7e-3 with both parts, which is the rounding of the result.
constexpr int64_t LN_TWO_PARTS = LN_M;
struct GradPlan {
    Space     space;
    unsigned  fold;                        // dz in two parts
    int64_t   tokens, rows, piece, ld_dz, ldx;            // of a worker, of all: of dz, in both parts
    int       splits;
    Input     w;
    char*     x_rows;                      // x with rows that do not count as zeros
    float*    coef;
    unsigned* top = nullptr;               // a number per worker; without weight gradients no rows are added up and every row goes by its own
    unsigned  tops = 0;                    // rows that share one
    char*     dz;
    float*    parts = nullptr;
    int64_t   pitch;
    char*     weight_space = nullptr;
    size_t    weight_bytes = 0;
    GradPlan(const gar_linear_logprobs_grad_params_t& p, int64_t ldw)
        : space(p.workspace), fold(p.workers * p.tokens <= LN_TWO_PARTS ? unsigned(p.tokens) : 0u), tokens(fold ? 2 * p.tokens : p.tokens), rows(p.workers * tokens), piece(piece_of(std::max<int64_t>(rows, 1), p.hidden, p.vocab)), ld_dz(up_to(piece, 8)), ldx(up_to(p.hidden, LN_PITCH)),
          w(space, p.weight, p.vocab, p.hidden, ldw, 2 * parts_of(rows, 2 * LN_M), products(rows, p.hidden, p.vocab)) {
        x_rows = space.take(size_t(rows) * size_t(ldx) * 2);
        coef = reinterpret_cast<float*>(space.take(size_t(rows) * 4));
        if (p.dtype == GAR_F16) {
            top = p.weight_grads ? reinterpret_cast<unsigned*>(space.take(size_t(p.workers) * 4)) : reinterpret_cast<unsigned*>(coef);
            tops = p.weight_grads ? unsigned(tokens) : 1u;
        }
        dz = space.take(size_t(rows) * size_t(ld_dz) * 2);
        pitch = up_to(p.hidden, 4);
        // (sums of 2^15 terms at most)
        const int64_t terms = std::min(piece, p.vocab);
        splits = splits_for(std::max<int64_t>(rows, 1), p.hidden, parts_of(terms, LN_K), parts_of(terms, LN_TERMS), piece < p.vocab || fold);
        if (p.dx && (splits > 1 || piece < p.vocab || fold)) parts = reinterpret_cast<float*>(space.take(size_t(splits) * size_t(rows) * size_t(pitch) * 4));
        if (p.weight_grads) {
            // (the last piece, if it is shorter, may be cut into more parts)
            const int64_t last = (p.vocab - 1) % piece + 1;
            weight_bytes = std::max(dense_weight_grad_workspace_bytes(p.workers, tokens, std::min(piece, p.vocab), p.hidden, p.bias_grads != nullptr),
                                    dense_weight_grad_workspace_bytes(p.workers, tokens, last, p.hidden, p.bias_grads != nullptr));
            weight_space = space.take(weight_bytes);
        }
    }
};

}  // namespace

size_t linear_logprobs_workspace_bytes(const gar_linear_logprobs_params_t& p, int64_t ldx, int64_t ldw) {
    gar_linear_logprobs_params_t q = p;
    q.workspace = nullptr;
    return ScoresPlan(q, ldx, ldw).space.used();
}

cudaError_t launch_linear_logprobs(const gar_linear_logprobs_params_t& p, int64_t ldx, int64_t ldw, int sm_count) {
    cudaStream_t stream = static_cast<cudaStream_t>(p.stream);
    ScoresPlan plan(p, ldx, ldw);
    if (few_rows_applies(p.rows, p.hidden, p.weight, ldw, nullptr, 0) && few_scores_parts(sm_count) <= LN_FEW_PARTS) {
        int count = 0;
        if (cudaError_t err = launch_few_scores(p, ldx, ldw, plan.parts, plan.target_z, &count, sm_count)) return err;
        return launch_small(join_scores_kernel, dim3(unsigned(parts_of(p.rows, 8))), stream, plan.parts, plan.target_z, p.logprobs ? p.targets : nullptr, p.rows,
                            count, p.vocab, p.logprobs, p.lse, p.lse_lo);
    }
    Copies copies;
    copies.add(plan.x);
    copies.add(plan.w);
    if (cudaError_t err = copies.launch(sm_count, stream)) return err;
    for (int64_t r0 = 0; r0 < p.rows; r0 += plan.rows) {
        Operand x = plan.x.m;
        x.p += r0 * x.ld * 2;
        x.rows = std::min(plan.rows, p.rows - r0);
        Maps maps;
        LNArgs a{};
        if (cudaError_t err = logits_maps(maps, a, p.dtype, x, plan.w.m, LN_UNIT)) return err;
        a.bias = p.bias;
        a.targets = p.logprobs ? p.targets + r0 : nullptr;
        a.parts = plan.parts;
        a.target_z = plan.target_z;
        if (cudaError_t err = launch_logits<LN_SCORES>(p.dtype, a, maps, sm_count, stream)) return err;
        if (cudaError_t err = launch_small(join_scores_kernel, dim3(unsigned(parts_of(x.rows, 8))), stream, plan.parts, plan.target_z, a.targets, x.rows, a.nt,
                                           p.vocab, p.logprobs ? p.logprobs + r0 : nullptr, p.lse ? p.lse + r0 : nullptr,
                                           p.lse_lo ? p.lse_lo + r0 : nullptr)) return err;
    }
    return cudaSuccess;
}

size_t linear_logprobs_backward_workspace_bytes(const gar_linear_logprobs_grad_params_t& p, int64_t ldw) {
    gar_linear_logprobs_grad_params_t q = p;
    q.workspace = nullptr;
    return GradPlan(q, ldw).space.used();
}

cudaError_t launch_linear_logprobs_backward(const gar_linear_logprobs_grad_params_t& p, int64_t ldx, int64_t ldw, int sm_count) {
    cudaStream_t stream = static_cast<cudaStream_t>(p.stream);
    GradPlan plan(p, ldw);
    const Operand x{plan.x_rows, plan.rows, p.hidden, plan.ldx};
    if (plan.rows > 0) {
        Copies copies;
        copies.add(copy_job(Operand{static_cast<const char*>(p.x), plan.rows, p.hidden, ldx}, plan.x_rows, plan.ldx));
        copies.add(plan.w);
        copies.a.targets = p.targets;
        copies.a.grad = p.grad_logprobs;
        copies.a.lse = p.lse;
        copies.a.vocab = p.vocab;
        copies.a.tokens = p.tokens;
        copies.a.workers = p.workers;
        copies.a.fold = plan.fold;
        copies.a.coef = plan.coef;
        copies.a.top = p.weight_grads ? plan.top : nullptr;
        if (cudaError_t err = copies.launch(sm_count, stream)) return err;
    }
    SumTarget d{p.dtype, p.dx, plan.rows, p.hidden, p.lddx ? p.lddx : p.hidden, plan.parts, plan.pitch, plan.splits, plan.top, plan.tops, plan.fold};
    for (int64_t v0 = 0; v0 < p.vocab; v0 += plan.piece) {
        Operand w = plan.w.m;
        w.p += v0 * w.ld * 2;
        w.rows = std::min(plan.piece, p.vocab - v0);
        const Operand dz{plan.dz, plan.rows, w.rows, plan.ld_dz};
        if (plan.rows > 0) {
            Maps maps;
            LNArgs a{};
            if (cudaError_t err = logits_maps(maps, a, p.dtype, x, w, LN_UNIT)) return err;
            a.bias = p.bias;
            a.col0 = v0;
            a.targets = p.targets;
            a.lse = p.lse;
            a.lse_lo = p.lse_lo;
            a.coef = plan.coef;
            a.top = plan.top;
            a.tokens = plan.tops;
            a.fold = plan.fold;
            a.out = OUT_WIDE;
            a.y = plan.dz;
            a.ldy = plan.ld_dz;
            if (cudaError_t err = operand_map(&maps.out, p.dtype, dz, 32, 32, CU_TENSOR_MAP_SWIZZLE_64B)) return err;
            if (cudaError_t err = launch_logits<LN_DLOGITS>(p.dtype, a, maps, sm_count, stream)) return err;
            if (p.dx)
                if (cudaError_t err = launch_sum(d, dz, w, nullptr, nullptr, v0 > 0, sm_count, stream)) return err;
        }
        if (p.weight_grads) {
            DenseWeightGrad g{};
            g.dtype = p.dtype;
            g.grads_dtype = p.grads_dtype;
            g.workers = p.workers;
            g.tokens = plan.tokens;
            g.out = w.rows;
            g.in = p.hidden;
            g.dy = plan.dz;
            g.ld_dy = plan.ld_dz;
            g.x = plan.x_rows;
            g.ldx = plan.ldx;
            const size_t gs = p.grads_dtype == GAR_F32 ? 4 : 2;
            g.dw = static_cast<char*>(p.weight_grads) + size_t(v0) * size_t(p.hidden) * gs;
            g.db = p.bias_grads ? static_cast<char*>(p.bias_grads) + size_t(v0) * gs : nullptr;
            g.ld_grads = p.ld_grads;
            g.top = plan.top;
            g.workspace = plan.weight_space;
            if (cudaError_t err = weight_grad(g, sm_count, stream)) return err;
        }
    }
    return d.parts && plan.rows > 0 ? join_sum(d, sm_count, stream) : cudaSuccess;
}

// ---- the gated block --------------------------------------------------------------------------------
namespace {
struct GatedPlan {
    Space space;
    Input x, gate, up;
    GatedPlan(const gar_gated_linear_params_t& p)
        : space(p.workspace), x(space, p.x, p.rows, p.hidden, p.ldx, parts_of(p.inner, LN_HALF), work(p)),
          gate(space, p.w_gate, p.inner, p.hidden, p.ld_gate, parts_of(p.rows, 2 * LN_M), work(p)),
          up(space, p.w_up, p.inner, p.hidden, p.ld_up, parts_of(p.rows, 2 * LN_M), work(p)) {}
    static double work(const gar_gated_linear_params_t& p) { return 2 * products(p.rows, p.hidden, p.inner); }
};
struct GatedGradPlan {
    Space   space;
    Input   gate, up, dgate, dup;
    int     splits;
    int64_t pitch;
    float*  parts = nullptr;
    GatedGradPlan(const gar_gated_linear_grad_params_t& p)
        : space(p.workspace), gate(space, p.w_gate, p.inner, p.hidden, p.ld_gate, parts_of(p.rows, 2 * LN_M), work(p)),
          up(space, p.w_up, p.inner, p.hidden, p.ld_up, parts_of(p.rows, 2 * LN_M), work(p)),
          dgate(space, p.dgate, p.rows, p.inner, p.ld_dgate, parts_of(p.hidden, LN_N), work(p)),
          dup(space, p.dup, p.rows, p.inner, p.ld_dup, parts_of(p.hidden, LN_N), work(p)),
          splits(splits_for(std::max<int64_t>(p.rows, 1), p.hidden, 2 * parts_of(p.inner, LN_K), 1, false)), pitch(up_to(p.hidden, 4)) {
        if (splits > 1) parts = reinterpret_cast<float*>(space.take(size_t(splits) * size_t(p.rows) * size_t(pitch) * 4));
    }
    static double work(const gar_gated_linear_grad_params_t& p) { return 2 * products(p.rows, p.hidden, p.inner); }
};
}  // namespace

size_t gated_linear_workspace_bytes(const gar_gated_linear_params_t& p) {
    gar_gated_linear_params_t q = p;
    q.workspace = nullptr;
    return GatedPlan(q).space.used();
}

cudaError_t launch_gated_linear_forward(const gar_gated_linear_params_t& p, int sm_count) {
    cudaStream_t stream = static_cast<cudaStream_t>(p.stream);
    GatedPlan plan(p);
    if (!p.gate_saved.q && !p.up_saved.q && !p.y_saved.q && few_rows_applies(p.rows, p.hidden, p.w_gate, p.ld_gate, p.w_up, p.ld_up))
        return launch_few_gated(p, sm_count);
    Copies copies;
    for (Input* in : {&plan.x, &plan.gate, &plan.up}) copies.add(*in);
    if (cudaError_t err = copies.launch(sm_count, stream)) return err;
    Maps maps;
    LNArgs a{};
    a.rows = p.rows;
    a.cols = p.inner;
    a.mt = int(parts_of(p.rows, 2 * LN_M));
    a.splits = 1;
    a.steps0 = a.steps = int(parts_of(p.hidden, LN_K));
    // half the columns are g's; a tile has whole groups of a checkpoint
    a.width = (p.gate_saved.q || p.up_saved.q) && p.group == 128 ? LN_N : width_for(a.mt, p.inner, a.steps, 128, 2);
    a.nt = int(parts_of(p.inner, a.width / 2));
    if (cudaError_t err = operand_map(&maps.a0, p.dtype, plan.x.m, LN_K, LN_M)) return err;
    if (cudaError_t err = operand_map(&maps.b0, p.dtype, plan.gate.m, LN_K, a.width / 2)) return err;
    if (cudaError_t err = operand_map(&maps.b1, p.dtype, plan.up.m, LN_K, a.width / 2)) return err;
    maps.a1 = maps.out = maps.a0;                      // not used unless set
    a.group_shift = p.group == 32 ? 5 : p.group == 64 ? 6 : 7;
    a.groups = int(parts_of(p.inner, p.group));
    a.bias = p.b_gate;
    a.bias2 = p.b_up;
    a.s0 = p.gate_saved;
    a.s1 = p.up_saved;
    a.y = p.y;
    a.ldy = p.ldy;
    a.out = on_16(p.y, p.ldy) ? OUT_WIDE : OUT_PLAIN;
    if (a.out == OUT_WIDE)
        if (cudaError_t err = operand_map(&maps.out, p.dtype, Operand{static_cast<const char*>(p.y), p.rows, p.inner, p.ldy}, 64, 32)) return err;
    const cudaError_t ran = p.act == GAR_ACT_SILU   ? launch<LN_GATED, GAR_ACT_SILU>(p.dtype, a, maps, sm_count, stream)
                            : p.act == GAR_ACT_GELU ? launch<LN_GATED, GAR_ACT_GELU>(p.dtype, a, maps, sm_count, stream)
                            : p.act == GAR_ACT_RELU ? launch<LN_GATED, GAR_ACT_RELU>(p.dtype, a, maps, sm_count, stream)
                                                    : launch<LN_GATED, GAR_ACT_IDENTITY>(p.dtype, a, maps, sm_count, stream);
    if (ran != cudaSuccess) return ran;
    if (!p.y_saved.q) return cudaSuccess;
    gar_activation_params_t c{};
    c.dtype = p.dtype;
    c.act = GAR_ACT_IDENTITY;
    c.group = p.group;
    c.rows = p.rows;
    c.cols = p.inner;
    c.x = p.y;
    c.ldx = p.ldy;
    c.x_saved = p.y_saved;
    c.stream = p.stream;
    return launch_activation_forward(c);
}

size_t gated_linear_backward_workspace_bytes(const gar_gated_linear_grad_params_t& p) {
    if (!p.dx) return 0;
    gar_gated_linear_grad_params_t q = p;
    q.workspace = nullptr;
    return GatedGradPlan(q).space.used();
}

cudaError_t launch_gated_linear_backward(const gar_gated_linear_grad_params_t& p, int sm_count) {
    cudaStream_t stream = static_cast<cudaStream_t>(p.stream);
    gar_activation_grad_params_t c{};
    c.dtype = p.dtype;
    c.act = p.act;
    c.group = p.group;
    c.rows = p.rows;
    c.cols = p.inner;
    c.dy = p.dy;
    c.lddy = p.lddy;
    c.x_saved = p.gate_saved;
    c.up_saved = p.up_saved;
    c.dx = p.dgate;
    c.lddx = p.ld_dgate;
    c.dup = p.dup;
    c.lddup = p.ld_dup;
    c.stream = p.stream;
    if (cudaError_t err = launch_activation_backward(c)) return err;
    if (!p.dx) return cudaSuccess;
    GatedGradPlan plan(p);
    Copies copies;
    for (Input* in : {&plan.gate, &plan.up, &plan.dgate, &plan.dup}) copies.add(*in);
    if (cudaError_t err = copies.launch(sm_count, stream)) return err;
    SumTarget d{p.dtype, p.dx, p.rows, p.hidden, p.lddx, plan.parts, plan.pitch, plan.splits, nullptr, 1, 0};
    if (cudaError_t err = launch_sum(d, plan.dgate.m, plan.gate.m, &plan.dup.m, &plan.up.m, false, sm_count, stream)) return err;
    return plan.parts ? join_sum(d, sm_count, stream) : cudaSuccess;
}

}  // namespace worker
}  // namespace gar
