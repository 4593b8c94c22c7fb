// Launchers behind gar_linear.h (arguments checked by the C entry points; row strides filled in).
#pragma once
#include "gar_linear.h"
#include "worker_common.cuh"

namespace gar {
namespace worker {

size_t linear_logprobs_workspace_bytes(const gar_linear_logprobs_params_t& p, int64_t ldx, int64_t ldw);
cudaError_t launch_linear_logprobs(const gar_linear_logprobs_params_t& p, int64_t ldx, int64_t ldw, int sm_count);
size_t linear_logprobs_backward_workspace_bytes(const gar_linear_logprobs_grad_params_t& p, int64_t ldw);
cudaError_t launch_linear_logprobs_backward(const gar_linear_logprobs_grad_params_t& p, int64_t ldx, int64_t ldw, int sm_count);
size_t gated_linear_workspace_bytes(const gar_gated_linear_params_t& p);
cudaError_t launch_gated_linear_forward(const gar_gated_linear_params_t& p, int sm_count);
size_t gated_linear_backward_workspace_bytes(const gar_gated_linear_grad_params_t& p);
cudaError_t launch_gated_linear_backward(const gar_gated_linear_grad_params_t& p, int sm_count);
cudaError_t launch_dropout(const gar_dropout_params_t& p, unsigned limit, float scale);

// A few rows (worker_few.cu): whether it applies, the parts a row's scores come in at most, the launches.
bool few_rows_applies(int64_t rows, int64_t hidden, const void* w0, int64_t ld0, const void* w1, int64_t ld1);
int64_t few_scores_parts(int sm_count);
cudaError_t launch_few_scores(const gar_linear_logprobs_params_t& p, int64_t ldx, int64_t ldw, float2* parts, float* target_z, int* count,
                              int sm_count);
cudaError_t launch_few_gated(const gar_gated_linear_params_t& p, int sm_count);

// Weight and bias gradients as gar_linear_weight_grad's, from x in 16 bits: dw[w][o][i] = sum_t dy[w, t, o] x[w, t, i].
// Rows of dy and x start on 16 bytes; dw's o-rows follow one another, `ld_grads` elements between workers.
struct DenseWeightGrad {
    int             dtype, grads_dtype, workers;
    int64_t         tokens, out, in;
    const void *    dy, *x;
    int64_t         ld_dy, ldx;
    void *          dw, *db;
    int64_t         ld_grads;
    const unsigned* top;              // a worker's dy carries power_for(top[worker]); or null
    void*           workspace;        // of dense_weight_grad_workspace_bytes
};
// By the product with two store groups (worker_linear.cu): whether it applies, and the launch (weights only).
bool outer_applies(const DenseWeightGrad& g);
cudaError_t launch_outer(const DenseWeightGrad& g, int sm_count, cudaStream_t stream);
// By weight_grad_kernel.
size_t dense_weight_grad_workspace_bytes(int workers, int64_t tokens, int64_t out, int64_t in, bool bias);
cudaError_t launch_dense_weight_grad(const DenseWeightGrad& g, int sm_count, cudaStream_t stream);

}  // namespace worker
}  // namespace gar
