// C entry points of the worker-side operators: argument checks, then one launch.
#include "worker_checks.cuh"
#include "worker_common.cuh"

using namespace gar::worker;
using gar::cuda_status;

extern "C" {

int gar_token_logprobs(const gar_logprobs_params_t* p) {
    if (!p || !dtype_ok(p->dtype) || !p->logits || !aligned(p->logits, esize(p->dtype))) return GAR_ERR_INVALID_ARG;
    int64_t ld = p->ld;
    if (!shape_ok(p->rows, p->vocab, &ld)) return GAR_ERR_INVALID_ARG;
    if (p->top < 0 || p->top > GAR_MAX_TOP || p->top > p->vocab) return GAR_ERR_INVALID_ARG;
    if (p->logprobs && !p->targets) return GAR_ERR_INVALID_ARG;
    if ((p->top > 0) != (p->top_logprobs != nullptr) || (p->top > 0) != (p->top_index != nullptr)) return GAR_ERR_INVALID_ARG;
    if (!p->logprobs && !p->entropy && !p->lse && !p->lse_lo && !p->top) return GAR_ERR_INVALID_ARG;
    if (p->vocab >= (int64_t(1) << 31)) return GAR_ERR_UNSUPPORTED;
    const Span outs[6] = {span(p->logprobs, 1, p->rows, 0, 4), span(p->lse_lo, 1, p->rows, 0, 4), span(p->entropy, 1, p->rows, 0, 4), span(p->lse, 1, p->rows, 0, 4),
                          span(p->top_logprobs, p->rows, p->top, p->top, 4), span(p->top_index, p->rows, p->top, p->top, 8)};
    const Span ins[2] = {span(p->logits, p->rows, p->vocab, ld, esize(p->dtype)), span(p->targets, 1, p->rows, 0, 8)};
    if (clash(outs, 6, ins, 2)) return GAR_ERR_INVALID_ARG;
    if (p->rows == 0) return GAR_OK;
    int sms = 0;
    if (int rc = sm_count(&sms)) return rc;
    return cuda_status(gar::worker::launch_logprobs(*p, ld, sms));
}

int gar_token_logprobs_backward(const gar_logprobs_grad_params_t* p) {
    if (!p || !dtype_ok(p->dtype) || !p->logits || !p->dlogits || !p->lse) return GAR_ERR_INVALID_ARG;
    if (!aligned(p->logits, esize(p->dtype)) || !aligned(p->dlogits, esize(p->dtype))) return GAR_ERR_INVALID_ARG;
    int64_t ld = p->ld, ldo = p->ld_dlogits;
    if (!shape_ok(p->rows, p->vocab, &ld) || !shape_ok(p->rows, p->vocab, &ldo)) return GAR_ERR_INVALID_ARG;
    if (p->top < 0 || p->top > GAR_MAX_TOP || p->top > p->vocab) return GAR_ERR_INVALID_ARG;
    if ((p->top > 0) != (p->grad_top != nullptr) || (p->top > 0 && !p->top_index)) return GAR_ERR_INVALID_ARG;
    if ((p->grad_logprobs && !p->targets) || (p->grad_entropy && !p->entropy)) return GAR_ERR_INVALID_ARG;
    if (p->vocab >= (int64_t(1) << 31)) return GAR_ERR_UNSUPPORTED;
    const size_t es = esize(p->dtype);
    const bool in_place = p->dlogits == p->logits && ldo == ld;
    const Span outs[1] = {span(p->dlogits, p->rows, p->vocab, ldo, es)};
    const Span ins[9] = {in_place ? Span{} : span(p->logits, p->rows, p->vocab, ld, es), span(p->targets, 1, p->rows, 0, 8),
                         span(p->lse, 1, p->rows, 0, 4), span(p->lse_lo, 1, p->rows, 0, 4), span(p->entropy, 1, p->rows, 0, 4),
                         span(p->top_index, p->rows, p->top, p->top, 8), span(p->grad_logprobs, 1, p->rows, 0, 4),
                         span(p->grad_entropy, 1, p->rows, 0, 4), span(p->grad_top, p->rows, p->top, p->top, 4)};
    if (clash(outs, 1, ins, 9)) return GAR_ERR_INVALID_ARG;
    if (p->rows == 0) return GAR_OK;
    int sms = 0;
    if (int rc = sm_count(&sms)) return rc;
    return cuda_status(gar::worker::launch_logprobs_backward(*p, ld, ldo, sms));
}

int gar_activation_forward(const gar_activation_params_t* params) {
    if (!params) return GAR_ERR_INVALID_ARG;
    gar_activation_params_t p = *params;
    if (!dtype_ok(p.dtype) || !act_ok(p.act) || !group_ok(p.group) || !p.x) return GAR_ERR_INVALID_ARG;
    const size_t es = esize(p.dtype);
    if (!aligned(p.x, es) || !aligned(p.up, es) || !aligned(p.y, es)) return GAR_ERR_INVALID_ARG;
    if (!shape_ok(p.rows, p.cols, &p.ldx)) return GAR_ERR_INVALID_ARG;
    if (p.up && !shape_ok(p.rows, p.cols, &p.ldup)) return GAR_ERR_INVALID_ARG;
    if (p.y && !shape_ok(p.rows, p.cols, &p.ldy)) return GAR_ERR_INVALID_ARG;
    if (p.x_saved.q && !saved_ok(p.x_saved, p.cols)) return GAR_ERR_INVALID_ARG;
    if (p.up_saved.q && (!p.up || !saved_ok(p.up_saved, p.cols))) return GAR_ERR_INVALID_ARG;
    if (p.y_saved.q && !saved_ok(p.y_saved, p.cols)) return GAR_ERR_INVALID_ARG;
    if (!p.y && !p.x_saved.q && !p.up_saved.q && !p.y_saved.q) return GAR_ERR_INVALID_ARG;
    const bool in_place = p.y == p.x && p.ldy == p.ldx;
    const Span outs[7] = {in_place ? Span{} : span(p.y, p.rows, p.cols, p.ldy, es),
                          codes(p.x_saved, p.rows, p.cols), scales(p.x_saved, p.rows, p.cols, p.group),
                          codes(p.up_saved, p.rows, p.cols), scales(p.up_saved, p.rows, p.cols, p.group),
                          codes(p.y_saved, p.rows, p.cols), scales(p.y_saved, p.rows, p.cols, p.group)};
    const Span ins[2] = {span(p.x, p.rows, p.cols, p.ldx, es), span(p.up, p.rows, p.cols, p.ldup, es)};
    if (clash(outs, 7, ins, 2) || (in_place && overlap(ins[0], ins[1]))) return GAR_ERR_INVALID_ARG;
    if (p.rows == 0) return GAR_OK;
    return cuda_status(gar::worker::launch_activation_forward(p));
}

int gar_activation_backward(const gar_activation_grad_params_t* params) {
    if (!params) return GAR_ERR_INVALID_ARG;
    gar_activation_grad_params_t p = *params;
    if (!dtype_ok(p.dtype) || !act_ok(p.act) || !group_ok(p.group) || !p.dy || !p.dx) return GAR_ERR_INVALID_ARG;
    const size_t es = esize(p.dtype);
    if (!aligned(p.dy, es) || !aligned(p.dx, es) || !aligned(p.dup, es)) return GAR_ERR_INVALID_ARG;
    if (!shape_ok(p.rows, p.cols, &p.lddy) || !shape_ok(p.rows, p.cols, &p.lddx)) return GAR_ERR_INVALID_ARG;
    if (!saved_ok(p.x_saved, p.cols)) return GAR_ERR_INVALID_ARG;
    if ((p.up_saved.q != nullptr) != (p.dup != nullptr)) return GAR_ERR_INVALID_ARG;
    if (p.dup && (!saved_ok(p.up_saved, p.cols) || !shape_ok(p.rows, p.cols, &p.lddup))) return GAR_ERR_INVALID_ARG;
    const bool in_place = p.dx == p.dy && p.lddx == p.lddy;
    const Span outs[2] = {span(p.dx, p.rows, p.cols, p.lddx, es), span(p.dup, p.rows, p.cols, p.lddup, es)};
    const Span dy = span(p.dy, p.rows, p.cols, p.lddy, es);
    const Span ins[4] = {codes(p.x_saved, p.rows, p.cols), scales(p.x_saved, p.rows, p.cols, p.group),
                         codes(p.up_saved, p.rows, p.cols), scales(p.up_saved, p.rows, p.cols, p.group)};
    if (clash(outs, 2, ins, 4) || (!in_place && overlap(outs[0], dy)) || overlap(outs[1], dy)) return GAR_ERR_INVALID_ARG;
    if (p.rows == 0) return GAR_OK;
    return cuda_status(gar::worker::launch_activation_backward(p));
}

int gar_checkpoint_pack(int dtype, const void* x, int64_t rows, int64_t cols, int64_t ldx, int group,
                        const gar_checkpoint_t* saved, void* stream) {
    if (!saved || !saved->q) return GAR_ERR_INVALID_ARG;
    gar_activation_params_t p{};
    p.dtype = dtype; p.act = GAR_ACT_IDENTITY; p.group = group;
    p.rows = rows; p.cols = cols;
    p.x = x; p.ldx = ldx;
    p.x_saved = *saved;
    p.stream = stream;
    return gar_activation_forward(&p);
}

int gar_checkpoint_unpack(int dtype, const gar_checkpoint_t* saved, int64_t rows, int64_t cols, int group, void* x,
                          int64_t ldx, void* stream) {
    if (!saved || !x || !dtype_ok(dtype) || !group_ok(group) || !aligned(x, esize(dtype))) return GAR_ERR_INVALID_ARG;
    if (!shape_ok(rows, cols, &ldx) || !saved_ok(*saved, cols)) return GAR_ERR_INVALID_ARG;
    const Span outs[1] = {span(x, rows, cols, ldx, esize(dtype))};
    const Span ins[2] = {codes(*saved, rows, cols), scales(*saved, rows, cols, group)};
    if (clash(outs, 1, ins, 2)) return GAR_ERR_INVALID_ARG;
    if (rows == 0) return GAR_OK;
    return cuda_status(gar::worker::launch_checkpoint_unpack(dtype, *saved, rows, cols, group, x, ldx,
                                                             static_cast<cudaStream_t>(stream)));
}

static bool sizes_ok(const gar_weight_grad_params_t* p) {
    const int64_t limit = int64_t(1) << 31;
    if (!p || p->workers < 1 || p->workers > GAR_MAX_N || p->tokens < 0 || p->tokens >= limit / 2 / p->workers) return false;
    return p->out_features >= 1 && p->in_features >= 1 && p->out_features < limit && p->in_features < limit;
}
size_t gar_weight_grad_workspace_bytes(const gar_weight_grad_params_t* p) {
    return sizes_ok(p) ? gar::worker::weight_grad_workspace_bytes(*p, p->ld_dy ? p->ld_dy : p->out_features) : 0;
}
int gar_weight_grad_wants_workspace(const gar_weight_grad_params_t* p) {
    return sizes_ok(p) && gar::worker::weight_grad_wants_workspace(*p, p->ld_dy ? p->ld_dy : p->out_features);
}

int gar_linear_weight_grad(const gar_weight_grad_params_t* p) {
    if (!p || !dtype_ok(p->dtype) || !dtype_ok(p->grads_dtype) || !group_ok(p->group)) return GAR_ERR_INVALID_ARG;
    if (p->workers < 1 || p->tokens < 0 || p->out_features < 1 || p->in_features < 1) return GAR_ERR_INVALID_ARG;
    if (!p->dy || !p->weight_grads) return GAR_ERR_INVALID_ARG;
    if (p->workers > GAR_MAX_N || p->dtype == GAR_F32) return GAR_ERR_UNSUPPORTED;
    const size_t es = esize(p->dtype), gs = esize(p->grads_dtype);
    if (!aligned(p->dy, es) || !aligned(p->weight_grads, gs) || !aligned(p->bias_grads, gs)) return GAR_ERR_INVALID_ARG;
    // sizes a launch can index: tokens of all workers below 2^30, both widths below 2^31
    const int64_t limit = int64_t(1) << 31;
    if (p->tokens >= limit / 2 / p->workers || p->out_features >= limit || p->in_features >= limit) return GAR_ERR_UNSUPPORTED;
    int64_t ld_dy = p->ld_dy;
    if (p->ld_grads < 0 || p->ld_grads > (int64_t(1) << 59) / p->workers) return GAR_ERR_INVALID_ARG;
    const int64_t rows = p->tokens * p->workers, weights = p->out_features * p->in_features;
    if (weights > int64_t(1) << 56) return GAR_ERR_UNSUPPORTED;
    if (!shape_ok(rows, p->out_features, &ld_dy) || !saved_ok(p->x_saved, p->in_features)) return GAR_ERR_INVALID_ARG;
    if (p->workers > 1 && (p->ld_grads < weights || p->ld_grads < p->out_features)) return GAR_ERR_INVALID_ARG;
    const Span dw = span(p->weight_grads, p->workers, weights, p->ld_grads, gs);
    const Span db = span(p->bias_grads, p->workers, p->out_features, p->ld_grads, gs);
    const int64_t g = (p->in_features + p->group - 1) / p->group;
    const Span outs[2] = {dw, db};
    const Span ins[4] = {span(p->dy, rows, p->out_features, ld_dy, es), span(p->x_saved.q, rows, p->in_features, p->x_saved.ldq, 1),
                         span(p->x_saved.scales, rows, g, g, 4), span(p->lengths, 1, p->workers, 0, 4)};
    if (clash(outs, 2, ins, 4)) return GAR_ERR_INVALID_ARG;
    if (p->workspace) {
        if (!aligned(p->workspace, 256) || p->workspace_bytes < gar_weight_grad_workspace_bytes(p)) return GAR_ERR_WORKSPACE;
        const Span ws[1] = {span(p->workspace, 1, int64_t(p->workspace_bytes), 0, 1)};
        const Span rest[6] = {dw, db, ins[0], ins[1], ins[2], ins[3]};
        if (clash(ws, 1, rest, 6)) return GAR_ERR_INVALID_ARG;
    }
    int sms = 0;
    if (int rc = sm_count(&sms)) return rc;
    return cuda_status(gar::worker::launch_weight_grad(*p, ld_dy, sms));
}

}  // extern "C"
