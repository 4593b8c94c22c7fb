// Per-worker weight gradients from 8-bit checkpoints (gar_worker.h): dW_w = dY_w^T X'_w, written
// into the rows of the gradient block.
//
// Plain tiled form: a CTA forms a 64 x 64 tile of one worker's gradient, 16 tokens at a time
// through shared memory, 4 x 4 fp32 accumulators per thread.
#include "worker_common.cuh"

namespace gar {
namespace worker {
namespace {

constexpr int WG_TILE = 64, WG_K = 16, WG_THREADS = 256;

struct WeightGradArgs {
    const void*    dy;
    const int8_t*  q;
    const float*   scales;
    const int32_t* lengths;
    void *         dw, *db;
    int64_t        tokens, out, in, ld_dy, ldq, ld_grads;
    int            groups, group_shift;
};

template <typename G> __device__ __forceinline__ void put(G* p, float v) { *p = Elem<G>::narrow(v); }

template <typename T, typename G>
__global__ void __launch_bounds__(WG_THREADS) weight_grad_kernel(const WeightGradArgs a) {
    __shared__ float sa[WG_K][WG_TILE], sb[WG_K][WG_TILE];
    const int tid = threadIdx.x, tx = tid % 16, ty = tid / 16;
    const int64_t i0 = int64_t(blockIdx.x) * WG_TILE, o0 = int64_t(blockIdx.y) * WG_TILE;
    const int w = blockIdx.z;
    int64_t len = a.tokens;
    if (a.lengths) {
        const int64_t l = a.lengths[w];
        len = l < 0 ? 0 : l < len ? l : len;
    }
    float acc[4][4] = {}, bias[4] = {};
    for (int64_t t0 = 0; t0 < len; t0 += WG_K) {
        for (int e = tid; e < WG_K * WG_TILE; e += WG_THREADS) {
            const int k = e / WG_TILE, c = e % WG_TILE;
            const int64_t t = t0 + k, row = int64_t(w) * a.tokens + t;
            sa[k][c] = t < len && o0 + c < a.out ? Elem<T>::widen(static_cast<const T*>(a.dy)[row * a.ld_dy + o0 + c]) : 0.f;
            float x = 0.f;
            if (t < len && i0 + c < a.in)
                x = Elem<T>::widen(Elem<T>::narrow(float(a.q[row * a.ldq + i0 + c]) * a.scales[row * a.groups + ((i0 + c) >> a.group_shift)]));
            sb[k][c] = x;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < WG_K; ++k) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float d = sa[k][ty * 4 + i];
                bias[i] += d;
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(d, sb[k][tx * 4 + j], acc[i][j]);
            }
        }
        __syncthreads();
    }
    G* dw = static_cast<G*>(a.dw) + int64_t(w) * a.ld_grads;
    for (int i = 0; i < 4; ++i) {
        const int64_t o = o0 + ty * 4 + i;
        if (o >= a.out) break;
        for (int j = 0; j < 4; ++j) {
            const int64_t c = i0 + tx * 4 + j;
            if (c < a.in) put(dw + o * a.in + c, acc[i][j]);
        }
        if (a.db && blockIdx.x == 0 && tx == 0) put(static_cast<G*>(a.db) + int64_t(w) * a.ld_grads + o, bias[i]);
    }
}

template <typename T>
cudaError_t weight_grad(const WeightGradArgs& a, int workers, int grads_dtype, cudaStream_t stream) {
    const dim3 grid(unsigned((a.in + WG_TILE - 1) / WG_TILE), unsigned((a.out + WG_TILE - 1) / WG_TILE), unsigned(workers));
    if (grads_dtype == GAR_F32) weight_grad_kernel<T, float><<<grid, WG_THREADS, 0, stream>>>(a);
    else if (grads_dtype == GAR_BF16) weight_grad_kernel<T, __nv_bfloat16><<<grid, WG_THREADS, 0, stream>>>(a);
    else weight_grad_kernel<T, __half><<<grid, WG_THREADS, 0, stream>>>(a);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_weight_grad(const gar_weight_grad_params_t& p, int64_t ld_dy, int) {
    const WeightGradArgs a{p.dy, p.x_saved.q, p.x_saved.scales, p.lengths, p.weight_grads, p.bias_grads, p.tokens,
                           p.out_features, p.in_features, ld_dy, p.x_saved.ldq, p.ld_grads,
                           int((p.in_features + p.group - 1) / p.group), p.group == 32 ? 5 : p.group == 64 ? 6 : 7};
    cudaStream_t s = static_cast<cudaStream_t>(p.stream);
    return p.dtype == GAR_BF16 ? weight_grad<__nv_bfloat16>(a, p.workers, p.grads_dtype, s)
                               : weight_grad<__half>(a, p.workers, p.grads_dtype, s);
}

}  // namespace worker
}  // namespace gar
