// C entry points of a worker's layers (gar_linear.h): argument checks, then the launches.
#include <cmath>

#include "worker_checks.cuh"
#include "worker_linear.cuh"

using namespace gar::worker;
using gar::cuda_status;

namespace {

constexpr int64_t kRows = int64_t(1) << 30, kWidth = int64_t(1) << 31, kWeights = int64_t(1) << 56;

bool half_type(int dtype) { return dtype == GAR_BF16 || dtype == GAR_F16; }
// sizes a launch can index
bool sizes_fit(int64_t rows, int64_t hidden, int64_t wide) {
    return rows < kRows && hidden < kWidth && wide < kWidth && hidden * wide <= kWeights;
}
Span vec(const void* p, int64_t n, size_t es) { return span(p, 1, n, 0, es); }
Span space(const void* p, size_t bytes) { return span(p, 1, int64_t(bytes), 0, 1); }
// a workspace as it has to be: GAR_OK, or what is wrong
int workspace_ok(const void* p, size_t have, size_t need, const Span* rest, int n) {
    if (need == 0 && !p) return GAR_OK;
    if (!p) return GAR_ERR_WORKSPACE;
    if (!aligned(p, 256) || have < need) return GAR_ERR_WORKSPACE;
    const Span ws[1] = {space(p, have)};
    return clash(ws, 1, rest, n) ? GAR_ERR_INVALID_ARG : GAR_OK;
}

// ---- log probabilities ----
int scores_ok(const gar_linear_logprobs_params_t* p, int64_t* ldx, int64_t* ldw) {
    if (!p || !dtype_ok(p->dtype) || !p->x || !p->weight) return GAR_ERR_INVALID_ARG;
    *ldx = p->ldx;
    *ldw = p->ldw;
    if (!shape_ok(p->rows, p->hidden, ldx) || !shape_ok(p->vocab, p->hidden, ldw) || p->vocab < 1) return GAR_ERR_INVALID_ARG;
    if (!half_type(p->dtype) || !sizes_fit(p->rows, p->hidden, p->vocab)) return GAR_ERR_UNSUPPORTED;
    return GAR_OK;
}
int scores_grad_ok(const gar_linear_logprobs_grad_params_t* p, int64_t* ldx, int64_t* ldw) {
    if (!p || !dtype_ok(p->dtype) || !dtype_ok(p->grads_dtype) || !p->x || !p->weight || p->workers < 1 || p->tokens < 0) return GAR_ERR_INVALID_ARG;
    *ldx = p->ldx;
    *ldw = p->ldw;
    if (p->workers > GAR_MAX_N || p->tokens >= kRows / p->workers) return GAR_ERR_UNSUPPORTED;
    if (!shape_ok(p->workers * p->tokens, p->hidden, ldx) || !shape_ok(p->vocab, p->hidden, ldw) || p->vocab < 1) return GAR_ERR_INVALID_ARG;
    if (!half_type(p->dtype) || !sizes_fit(p->workers * p->tokens, p->hidden, p->vocab)) return GAR_ERR_UNSUPPORTED;
    return GAR_OK;
}

// ---- the gated block: row strides filled in ----
int gated_ok(gar_gated_linear_params_t* p) {
    if (!dtype_ok(p->dtype) || !act_ok(p->act) || !group_ok(p->group) || !p->x || !p->w_gate || !p->w_up || !p->y) return GAR_ERR_INVALID_ARG;
    if (!shape_ok(p->rows, p->hidden, &p->ldx) || !shape_ok(p->inner, p->hidden, &p->ld_gate) || !shape_ok(p->inner, p->hidden, &p->ld_up) ||
        !shape_ok(p->rows, p->inner, &p->ldy)) return GAR_ERR_INVALID_ARG;
    if (!half_type(p->dtype) || !sizes_fit(p->rows, p->hidden, p->inner)) return GAR_ERR_UNSUPPORTED;
    return GAR_OK;
}
int gated_grad_ok(gar_gated_linear_grad_params_t* p) {
    if (!dtype_ok(p->dtype) || !act_ok(p->act) || !group_ok(p->group) || !p->dy || !p->w_gate || !p->w_up || !p->dgate || !p->dup) return GAR_ERR_INVALID_ARG;
    if (!shape_ok(p->rows, p->inner, &p->lddy) || !shape_ok(p->inner, p->hidden, &p->ld_gate) || !shape_ok(p->inner, p->hidden, &p->ld_up) ||
        !shape_ok(p->rows, p->inner, &p->ld_dgate) || !shape_ok(p->rows, p->inner, &p->ld_dup)) return GAR_ERR_INVALID_ARG;
    if (p->dx && !shape_ok(p->rows, p->hidden, &p->lddx)) return GAR_ERR_INVALID_ARG;
    if (!half_type(p->dtype) || !sizes_fit(p->rows, p->hidden, p->inner)) return GAR_ERR_UNSUPPORTED;
    return GAR_OK;
}

}  // namespace

extern "C" {

size_t gar_linear_logprobs_workspace_bytes(const gar_linear_logprobs_params_t* p) {
    int64_t ldx, ldw;
    return scores_ok(p, &ldx, &ldw) == GAR_OK && p->rows > 0 ? linear_logprobs_workspace_bytes(*p, ldx, ldw) : 0;
}

int gar_linear_logprobs(const gar_linear_logprobs_params_t* p) {
    int64_t ldx, ldw;
    if (int rc = scores_ok(p, &ldx, &ldw)) return rc;
    if (!aligned(p->x, 2) || !aligned(p->weight, 2) || !aligned(p->bias, 2) || !aligned(p->targets, 8)) return GAR_ERR_INVALID_ARG;
    if (!aligned(p->logprobs, 4) || !aligned(p->lse, 4) || !aligned(p->lse_lo, 4)) return GAR_ERR_INVALID_ARG;
    if ((p->logprobs && !p->targets) || (!p->logprobs && !p->lse && !p->lse_lo)) return GAR_ERR_INVALID_ARG;
    const Span all[7] = {vec(p->logprobs, p->rows, 4), vec(p->lse, p->rows, 4), vec(p->lse_lo, p->rows, 4), span(p->x, p->rows, p->hidden, ldx, 2),
                         span(p->weight, p->vocab, p->hidden, ldw, 2), vec(p->bias, p->vocab, 2), vec(p->targets, p->rows, 8)};
    if (clash(all, 3, all + 3, 4)) return GAR_ERR_INVALID_ARG;
    if (p->rows == 0) return GAR_OK;
    if (int rc = workspace_ok(p->workspace, p->workspace_bytes, linear_logprobs_workspace_bytes(*p, ldx, ldw), all, 7)) return rc;
    int sms = 0;
    if (int rc = sm_count(&sms)) return rc;
    return cuda_status(launch_linear_logprobs(*p, ldx, ldw, sms));
}

size_t gar_linear_logprobs_backward_workspace_bytes(const gar_linear_logprobs_grad_params_t* p) {
    int64_t ldx, ldw;
    return scores_grad_ok(p, &ldx, &ldw) == GAR_OK ? linear_logprobs_backward_workspace_bytes(*p, ldw) : 0;
}

int gar_linear_logprobs_backward(const gar_linear_logprobs_grad_params_t* p) {
    int64_t ldx, ldw;
    if (int rc = scores_grad_ok(p, &ldx, &ldw)) return rc;
    const int64_t rows = p->workers * p->tokens, weights = p->vocab * p->hidden;
    const size_t gs = esize(p->grads_dtype);
    if (!p->targets || !p->lse || !p->grad_logprobs || (!p->dx && !p->weight_grads) || (p->bias_grads && !p->weight_grads)) return GAR_ERR_INVALID_ARG;
    if (!aligned(p->x, 2) || !aligned(p->weight, 2) || !aligned(p->bias, 2) || !aligned(p->dx, 2) || !aligned(p->weight_grads, gs) ||
        !aligned(p->bias_grads, gs) || !aligned(p->targets, 8) || !aligned(p->lse, 4) || !aligned(p->lse_lo, 4) ||
        !aligned(p->grad_logprobs, 4)) return GAR_ERR_INVALID_ARG;
    int64_t lddx = p->lddx;
    if (p->dx && !shape_ok(rows, p->hidden, &lddx)) return GAR_ERR_INVALID_ARG;
    if (p->weight_grads) {
        if (p->ld_grads < 0 || p->ld_grads > (int64_t(1) << 59) / p->workers) return GAR_ERR_INVALID_ARG;
        if (p->workers > 1 && (p->ld_grads < weights || p->ld_grads < p->vocab)) return GAR_ERR_INVALID_ARG;
    }
    const Span all[10] = {span(p->dx, rows, p->hidden, lddx, 2), span(p->weight_grads, p->workers, weights, p->ld_grads, gs),
                          span(p->bias_grads, p->workers, p->vocab, p->ld_grads, gs), span(p->x, rows, p->hidden, ldx, 2),
                          span(p->weight, p->vocab, p->hidden, ldw, 2), vec(p->bias, p->vocab, 2), vec(p->targets, rows, 8), vec(p->lse, rows, 4),
                          vec(p->lse_lo, rows, 4), vec(p->grad_logprobs, rows, 4)};
    if (clash(all, 3, all + 3, 7)) return GAR_ERR_INVALID_ARG;
    if (rows == 0 && !p->weight_grads) return GAR_OK;
    if (int rc = workspace_ok(p->workspace, p->workspace_bytes, linear_logprobs_backward_workspace_bytes(*p, ldw), all, 10)) return rc;
    int sms = 0;
    if (int rc = sm_count(&sms)) return rc;
    return cuda_status(launch_linear_logprobs_backward(*p, ldx, ldw, sms));
}

size_t gar_gated_linear_workspace_bytes(const gar_gated_linear_params_t* params) {
    if (!params) return 0;
    gar_gated_linear_params_t p = *params;
    return gated_ok(&p) == GAR_OK && p.rows > 0 ? gated_linear_workspace_bytes(p) : 0;
}

int gar_gated_linear_forward(const gar_gated_linear_params_t* params) {
    if (!params) return GAR_ERR_INVALID_ARG;
    gar_gated_linear_params_t p = *params;
    if (int rc = gated_ok(&p)) return rc;
    for (const void* m : {p.x, p.w_gate, p.w_up, p.b_gate, p.b_up, static_cast<const void*>(p.y)})
        if (!aligned(m, 2)) return GAR_ERR_INVALID_ARG;
    for (const gar_checkpoint_t* s : {&p.gate_saved, &p.up_saved, &p.y_saved})
        if (s->q && !saved_ok(*s, p.inner)) return GAR_ERR_INVALID_ARG;
    const Span all[12] = {span(p.y, p.rows, p.inner, p.ldy, 2),
                          codes(p.gate_saved, p.rows, p.inner), scales(p.gate_saved, p.rows, p.inner, p.group),
                          codes(p.up_saved, p.rows, p.inner), scales(p.up_saved, p.rows, p.inner, p.group),
                          codes(p.y_saved, p.rows, p.inner), scales(p.y_saved, p.rows, p.inner, p.group),
                          span(p.x, p.rows, p.hidden, p.ldx, 2), span(p.w_gate, p.inner, p.hidden, p.ld_gate, 2),
                          span(p.w_up, p.inner, p.hidden, p.ld_up, 2), vec(p.b_gate, p.inner, 2), vec(p.b_up, p.inner, 2)};
    if (clash(all, 7, all + 7, 5)) return GAR_ERR_INVALID_ARG;
    if (p.rows == 0) return GAR_OK;
    if (int rc = workspace_ok(p.workspace, p.workspace_bytes, gated_linear_workspace_bytes(p), all, 12)) return rc;
    int sms = 0;
    if (int rc = sm_count(&sms)) return rc;
    return cuda_status(launch_gated_linear_forward(p, sms));
}

size_t gar_gated_linear_backward_workspace_bytes(const gar_gated_linear_grad_params_t* params) {
    if (!params) return 0;
    gar_gated_linear_grad_params_t p = *params;
    return gated_grad_ok(&p) == GAR_OK && p.rows > 0 ? gated_linear_backward_workspace_bytes(p) : 0;
}

int gar_gated_linear_backward(const gar_gated_linear_grad_params_t* params) {
    if (!params) return GAR_ERR_INVALID_ARG;
    gar_gated_linear_grad_params_t p = *params;
    if (int rc = gated_grad_ok(&p)) return rc;
    for (const void* m : {p.dy, p.w_gate, p.w_up, static_cast<const void*>(p.dgate), static_cast<const void*>(p.dup), static_cast<const void*>(p.dx)})
        if (!aligned(m, 2)) return GAR_ERR_INVALID_ARG;
    if (!saved_ok(p.gate_saved, p.inner) || !saved_ok(p.up_saved, p.inner)) return GAR_ERR_INVALID_ARG;
    const bool in_place = p.dgate == p.dy && p.ld_dgate == p.lddy;
    const Span dy = span(p.dy, p.rows, p.inner, p.lddy, 2);
    const Span all[10] = {span(p.dgate, p.rows, p.inner, p.ld_dgate, 2), span(p.dup, p.rows, p.inner, p.ld_dup, 2), span(p.dx, p.rows, p.hidden, p.lddx, 2),
                          codes(p.gate_saved, p.rows, p.inner), scales(p.gate_saved, p.rows, p.inner, p.group),
                          codes(p.up_saved, p.rows, p.inner), scales(p.up_saved, p.rows, p.inner, p.group),
                          span(p.w_gate, p.inner, p.hidden, p.ld_gate, 2), span(p.w_up, p.inner, p.hidden, p.ld_up, 2), dy};
    if (clash(all, 3, all + 3, 6) || (!in_place && overlap(all[0], dy)) || overlap(all[1], dy) || overlap(all[2], dy)) return GAR_ERR_INVALID_ARG;
    if (p.rows == 0) return GAR_OK;
    if (int rc = workspace_ok(p.workspace, p.workspace_bytes, gated_linear_backward_workspace_bytes(p), all, 10)) return rc;
    int sms = 0;
    if (int rc = sm_count(&sms)) return rc;
    return cuda_status(launch_gated_linear_backward(p, sms));
}

int gar_dropout(const gar_dropout_params_t* params) {
    if (!params) return GAR_ERR_INVALID_ARG;
    gar_dropout_params_t p = *params;
    if (!dtype_ok(p.dtype) || !p.x || !p.y || !(p.p >= 0.f && p.p <= 1.f)) return GAR_ERR_INVALID_ARG;
    const size_t es = esize(p.dtype);
    if (!aligned(p.x, es) || !aligned(p.residual, es) || !aligned(p.y, es) || !aligned(p.counter, 8)) return GAR_ERR_INVALID_ARG;
    if (!shape_ok(p.rows, p.cols, &p.ldx) || !shape_ok(p.rows, p.cols, &p.ldy)) return GAR_ERR_INVALID_ARG;
    if (p.residual && !shape_ok(p.rows, p.cols, &p.ld_residual)) return GAR_ERR_INVALID_ARG;
    if (p.cols >= int64_t(1) << 32) return GAR_ERR_UNSUPPORTED;
    const Span y = span(p.y, p.rows, p.cols, p.ldy, es), x = span(p.x, p.rows, p.cols, p.ldx, es), r = span(p.residual, p.rows, p.cols, p.ld_residual, es);
    const bool on_x = p.y == p.x && p.ldy == p.ldx, on_r = p.y == p.residual && p.ldy == p.ld_residual;
    if ((!on_x && overlap(y, x)) || (!on_r && overlap(y, r)) || overlap(y, vec(p.counter, 1, 8))) return GAR_ERR_INVALID_ARG;
    if (p.rows == 0) return GAR_OK;
    // dropped: 16 bits below this many of 2^16; kept elements are scaled by what keeps the expectation
    const unsigned limit = unsigned(std::lrint(double(p.p) * 65536.0));
    const float scale = limit < 65536u ? float(65536.0 / double(65536u - limit)) : 0.f;
    return cuda_status(launch_dropout(p, limit, scale));
}

}  // extern "C"
