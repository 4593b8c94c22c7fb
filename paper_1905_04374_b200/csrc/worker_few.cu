// Products of a few rows with a worker's weights (gar_linear.h), as when single tokens are scored: the weights are read
// once from memory and nothing else takes time, so they go straight from memory into the registers of
// mma.sync (m16n8k16, fp32 accumulators), sixteen weight rows at a time as A, the rows of x (up to eight, or sixteen) as B.
// tcgen05's tiles are of 256 rows of x and stage the weights in shared memory; its copies of 128 bytes a row and step reach
// 4.7 TB/s where a warp here reads 256 consecutive bytes of sixteen rows at a time.
//
// The order of the contraction within 32 elements is free as long as A and B agree on it: a lane takes 16 consecutive bytes of
// a weight row (and of a row of x), which are the elements of two instructions.
// Warps split a long contraction between them where there are few weight rows (joined in shared memory, in order).
#include <algorithm>
#include <atomic>

#include "worker_act.cuh"
#include "worker_linear.cuh"
#include "worker_tensor.cuh"

namespace gar {
namespace worker {
namespace {

constexpr int FW_WARPS = 8, FW_THREADS = 32 * FW_WARPS;
constexpr int FW_UNIT = 128;                          // elements of the contraction a warp takes at a time: 256 bytes of a row
constexpr int FW_SMEM = 100 << 10;                    // x in shared memory: two CTAs on an SM

struct FewArgs {
    const void*    x;
    int64_t        ldx;
    const void *   w0, *w1;               // w1: gated, the other projection
    int64_t        ld0, ld1;
    const void *   b0, *b1;
    int            rows, units, pitch;    // of x; of FW_UNIT; bytes between rows of x in shared memory
    int            split;                 // warps that share a contraction: 1, 2, 4, 8
    int64_t        hidden, wide, tiles;   // wide: weight rows (of each projection)
    const int64_t* targets;
    float2*        parts;                 // [rows][gridDim.x]
    float*         target_z;
    void*          y;
    int64_t        ldy;
};

template <typename T>
__device__ __forceinline__ void mma_16x8x16(float (&d)[4], unsigned a0, unsigned a1, unsigned a2, unsigned a3, unsigned b0, unsigned b1) {
    if constexpr (std::is_same<T, __half>::value)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// eight elements of a row from k on, zeros behind its end; WIDE: rows start on 16 bytes
template <bool WIDE = true>
__device__ __forceinline__ uint4 weight8(const unsigned short* row, int64_t k, int64_t hidden) {
    if (WIDE && k + 8 <= hidden) return load_stream(row + k);
    unsigned v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = k + j < hidden ? row[k + j] : 0u;
    return make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
}

// NT: rows of x / 8.  GATED: a tile is eight rows of either projection, otherwise sixteen weight rows.
template <typename T, int NT, bool GATED, int ACT>
__global__ void __launch_bounds__(FW_THREADS, 2) few_rows_kernel(const FewArgs a) {
    extern __shared__ uint4 raw4[];
    uint8_t* xs = reinterpret_cast<uint8_t*>(raw4);
    __shared__ float joined[FW_WARPS][NT][4][32];
    __shared__ float2 ends[FW_WARPS][NT * 8];
    grid_dependency();
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, g = lane / 4, t = lane % 4;
    const int sets = FW_WARPS / a.split, set = warp / a.split, part = warp % a.split;      // tiles at a time; this warp's
    const unsigned short *w0 = static_cast<const unsigned short*>(a.w0), *w1 = static_cast<const unsigned short*>(GATED ? a.w1 : a.w0);
    const int64_t ld0 = a.ld0, ld1 = GATED ? a.ld1 : a.ld0;
    // the warp's weight rows of a tile, and the unit of them that is on its way
    const unsigned short *p0, *p1;
    bool live0, live1;
    int64_t r0, r1;
    uint4 next[4][2];
    auto fetch = [&](int u) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int64_t k = int64_t(u) * FW_UNIT + 32 * c + 8 * t;
            next[c][0] = live0 && k < a.hidden ? weight8(p0, k, a.hidden) : make_uint4(0, 0, 0, 0);
            next[c][1] = live1 && k < a.hidden ? weight8(p1, k, a.hidden) : make_uint4(0, 0, 0, 0);
        }
    };
    auto begin = [&](int64_t tile) {
        r0 = GATED ? tile * 8 + g : tile * 16 + g;
        r1 = GATED ? r0 : r0 + 8;
        live0 = tile < a.tiles && r0 < a.wide;
        live1 = tile < a.tiles && r1 < a.wide;
        p0 = w0 + r0 * ld0;
        p1 = w1 + r1 * ld1;
        fetch(part);                               // (units >= split)
    };
    begin(int64_t(blockIdx.x) * sets + set);
    {
        // x, zeros behind its rows and columns
        const unsigned short* x = static_cast<const unsigned short*>(a.x);
        const bool aligned = reinterpret_cast<uintptr_t>(x) % 16 == 0 && a.ldx % 8 == 0;
        const int per_row = a.units * (FW_UNIT / 8);
        for (int r = 0; r < NT * 8; ++r)
            for (int i = tid; i < per_row; i += FW_THREADS) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (r < a.rows) {
                    const unsigned short* p = x + r * a.ldx;
                    if (aligned && 8 * i + 8 <= a.hidden) v = __ldg(reinterpret_cast<const uint4*>(p) + i);
                    else v = weight8<false>(p, 8 * i, a.hidden);
                }
                *reinterpret_cast<uint4*>(xs + r * a.pitch + 16 * i) = v;
            }
    }
    __syncthreads();
    float m[NT][2], s[NT][2];
    int64_t target[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            m[n][c] = -CUDART_INF_F;
            s[n][c] = 0.f;
            const int r = n * 8 + 2 * t + c;
            target[n][c] = !GATED && a.targets && r < a.rows ? a.targets[r] : -1;
        }

    for (int64_t first = int64_t(blockIdx.x) * sets; first < a.tiles; first += int64_t(gridDim.x) * sets) {
        const int64_t tile = first + set;
        // the tensor core truncates what it adds: its sums are of a unit, which are added up rounded
        float sum[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < 4; ++c) sum[n][c] = 0.f;
        for (int u = part; u < a.units; u += a.split) {
            uint4 w[4][2];
#pragma unroll
            for (int c = 0; c < 4; ++c) { w[c][0] = next[c][0]; w[c][1] = next[c][1]; }
            if (u + a.split < a.units) fetch(u + a.split);
            const uint8_t* xk = xs + g * a.pitch + (u * FW_UNIT + 8 * t) * 2;
            float acc[NT][4];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[n][c] = 0.f;
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const uint4 b = *reinterpret_cast<const uint4*>(xk + n * 8 * a.pitch + c * 64);
                    mma_16x8x16<T>(acc[n], w[c][0].x, w[c][1].x, w[c][0].y, w[c][1].y, b.x, b.y);
                    mma_16x8x16<T>(acc[n], w[c][0].z, w[c][1].z, w[c][0].w, w[c][1].w, b.z, b.w);
                }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < 4; ++c) sum[n][c] += acc[n][c];
        }
        // the next tile's first unit is on its way while this one is finished
        const bool mine0 = live0, mine1 = live1;
        const int64_t v0 = r0, v1 = r1;
        begin(tile + int64_t(gridDim.x) * sets);
        if (a.split > 1) {
            __syncthreads();                       // the parts before have been read
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < 4; ++c) joined[warp][n][c][lane] = sum[n][c];
            __syncthreads();
            if (part == 0)
                for (int k = 1; k < a.split; ++k)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int c = 0; c < 4; ++c) sum[n][c] += joined[warp + k][n][c][lane];
        }
        if (part != 0 || tile >= a.tiles) continue;
        if constexpr (GATED) {
            if (!mine0) continue;
            const float bg = a.b0 ? Elem<T>::widen(static_cast<const T*>(a.b0)[v0]) : 0.f, bu = a.b1 ? Elem<T>::widen(static_cast<const T*>(a.b1)[v0]) : 0.f;
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float x[8] = {sum[n][0] + bg, sum[n][1] + bg, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                float y[8];
                act8<ACT>(x, y);
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int r = n * 8 + 2 * t + c;
                    if (r < a.rows) static_cast<T*>(a.y)[r * a.ldy + v0] = Elem<T>::narrow(y[c] * (sum[n][2 + c] + bu));
                }
            }
        } else {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int64_t v = half ? v1 : v0;
                if (!(half ? mine1 : mine0)) continue;
                const float bias = a.b0 ? Elem<T>::widen(static_cast<const T*>(a.b0)[v]) : 0.f;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const float z = sum[n][2 * half + c] + bias;
                        if (target[n][c] == v) a.target_z[n * 8 + 2 * t + c] = z;
                        const float higher = fmaxf(m[n][c], z);
                        const float base = higher == -CUDART_INF_F ? 0.f : higher;
                        s[n][c] = s[n][c] * ex2((m[n][c] - base) * kLog2e) + ex2((z - base) * kLog2e);
                        m[n][c] = higher;
                    }
            }
        }
    }
    if constexpr (!GATED) {
        // over the lanes of a row of x, then over the warps
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float top = m[n][c], sum = s[n][c];
                for (int o = 4; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                const float base = top == -CUDART_INF_F ? 0.f : top;
                sum *= ex2((m[n][c] - base) * kLog2e);
                for (int o = 4; o < 32; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                if (g == 0) ends[warp][n * 8 + 2 * t + c] = make_float2(top, sum);
            }
        __syncthreads();
        if (tid < a.rows) {
            float top = -CUDART_INF_F, sum = 0.f;
            for (int k = 0; k < FW_WARPS; ++k) top = fmaxf(top, ends[k][tid].x);
            const float base = top == -CUDART_INF_F ? 0.f : top;
            for (int k = 0; k < FW_WARPS; ++k) sum += ends[k][tid].y * ex2((ends[k][tid].x - base) * kLog2e);
            a.parts[int64_t(tid) * gridDim.x + blockIdx.x] = make_float2(top, sum);
        }
    }
}

template <typename T, int NT, bool GATED, int ACT>
cudaError_t launch_as(const FewArgs& a, unsigned blocks, cudaStream_t stream) {
    auto kernel = few_rows_kernel<T, NT, GATED, ACT>;
    const int bytes = NT * 8 * a.pitch;
    static std::atomic<uint64_t> allowed{0};           // devices on which the kernel may have its shared memory
    int dev = 0;
    if (cudaError_t err = cudaGetDevice(&dev)) return err;
    if (dev >= 64 || !(allowed.load(std::memory_order_relaxed) >> dev & 1)) {
        if (cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, FW_SMEM)) return err;
        if (dev < 64) allowed.fetch_or(uint64_t(1) << dev, std::memory_order_relaxed);
    }
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(blocks);
    cfg.blockDim = dim3(FW_THREADS);
    cfg.dynamicSmemBytes = size_t(bytes);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, a);
}
template <bool GATED, int ACT>
cudaError_t launch(int dtype, const FewArgs& a, unsigned blocks, cudaStream_t stream) {
    if (dtype == GAR_BF16)
        return a.rows <= 8 ? launch_as<__nv_bfloat16, 1, GATED, ACT>(a, blocks, stream) : launch_as<__nv_bfloat16, 2, GATED, ACT>(a, blocks, stream);
    return a.rows <= 8 ? launch_as<__half, 1, GATED, ACT>(a, blocks, stream) : launch_as<__half, 2, GATED, ACT>(a, blocks, stream);
}

int64_t units_of(int64_t hidden) { return (hidden + FW_UNIT - 1) / FW_UNIT; }
// bytes between rows of x in shared memory: neighbours half a bank row apart
int64_t pitch_of(int64_t hidden) { return units_of(hidden) * FW_UNIT * 2 + 64; }
bool on_16(const void* p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0; }
int64_t most_blocks(int sm_count) { return 2 * int64_t(sm_count); }

// the sizes' part of the arguments, and the CTAs
unsigned plan(FewArgs& a, int rows, int64_t hidden, int64_t wide, int64_t tiles, int sm_count) {
    a.rows = rows;
    a.hidden = hidden;
    a.wide = wide;
    a.tiles = tiles;
    a.units = int(units_of(hidden));
    a.pitch = int(pitch_of(hidden));
    const int64_t warps = most_blocks(sm_count) * FW_WARPS;
    a.split = 1;
    while (a.split < FW_WARPS && tiles * 2 * a.split <= warps && a.units >= 2 * a.split) a.split *= 2;
    const int64_t sets = FW_WARPS / a.split;
    return unsigned(std::min((tiles + sets - 1) / sets, most_blocks(sm_count)));
}

}  // namespace

bool few_rows_applies(int64_t rows, int64_t hidden, const void* w0, int64_t ld0, const void* w1, int64_t ld1) {
    return rows <= 16 && (rows <= 8 ? 8 : 16) * pitch_of(hidden) <= FW_SMEM && on_16(w0, ld0) && (!w1 || on_16(w1, ld1));
}
int64_t few_scores_parts(int sm_count) { return most_blocks(sm_count); }

cudaError_t launch_few_scores(const gar_linear_logprobs_params_t& p, int64_t ldx, int64_t ldw, float2* parts, float* target_z, int* count,
                              int sm_count) {
    FewArgs a{};
    const unsigned blocks = plan(a, int(p.rows), p.hidden, p.vocab, (p.vocab + 15) / 16, sm_count);
    a.x = p.x;
    a.ldx = ldx;
    a.w0 = p.weight;
    a.ld0 = ldw;
    a.b0 = p.bias;
    a.targets = p.logprobs ? p.targets : nullptr;
    a.parts = parts;
    a.target_z = target_z;
    *count = int(blocks);
    return launch<false, 0>(p.dtype, a, blocks, static_cast<cudaStream_t>(p.stream));
}

cudaError_t launch_few_gated(const gar_gated_linear_params_t& p, int sm_count) {
    FewArgs a{};
    const unsigned blocks = plan(a, int(p.rows), p.hidden, p.inner, (p.inner + 7) / 8, sm_count);
    a.x = p.x;
    a.ldx = p.ldx;
    a.w0 = p.w_gate;
    a.ld0 = p.ld_gate;
    a.w1 = p.w_up;
    a.ld1 = p.ld_up;
    a.b0 = p.b_gate;
    a.b1 = p.b_up;
    a.y = p.y;
    a.ldy = p.ldy;
    cudaStream_t stream = static_cast<cudaStream_t>(p.stream);
    return p.act == GAR_ACT_SILU   ? launch<true, GAR_ACT_SILU>(p.dtype, a, blocks, stream)
           : p.act == GAR_ACT_GELU ? launch<true, GAR_ACT_GELU>(p.dtype, a, blocks, stream)
           : p.act == GAR_ACT_RELU ? launch<true, GAR_ACT_RELU>(p.dtype, a, blocks, stream) : launch<true, GAR_ACT_IDENTITY>(p.dtype, a, blocks, stream);
}

}  // namespace worker
}  // namespace gar
