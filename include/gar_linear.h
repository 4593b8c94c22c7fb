/*
 * gar_linear.h -- C ABI of a worker's layers (NVIDIA B200, sm_100a): log
 * probabilities of tokens straight from the hidden states, without the logits
 * ever being kept, and their gradients; the gated feed-forward block, both
 * projections, activation and product in one kernel, with its backward pass;
 * and dropout whose mask is computed again instead of stored.
 *
 * Conventions are those of gar_worker.h: device pointers of the current
 * device, all buffers owned by the caller, every call asynchronous on
 * `stream`, argument errors returned before anything is launched, GAR_ERR_CUDA
 * for launch failures, no exceptions, no CPU fallback, bit-identical output
 * for the same call.  (How a call's work is cut up goes by its sizes, so that a
 * row's last bits may differ between calls of different numbers of rows, a token
 * scored alone and in a batch for instance.)  Matrices are row-major with unit
 * column stride and a row stride `ld` in elements (0 means the number of
 * columns), at any alignment of the element type.  A call with no rows writes no
 * rows.
 *
 * The matrix products are those of 16-bit elements (GAR_BF16 or GAR_F16; GAR_F32 is
 * GAR_ERR_UNSUPPORTED except for dropout), exact, summed in fp32 on the tensor
 * cores, which truncate where they add: a sum over k terms is short by some
 * 1e-9 k of itself, where it grows steadily by 1.4e-9 k (bfloat16) to 6e-9 k
 * (binary16), where nothing is cut off by nothing; at the very most by 4e-8 k (up
 * to 16 rows 7e-8 k) of the terms' magnitudes.  Logits are summed in chunks of 512
 * terms (up to 640 in one; of up to 16 rows mostly 128), whose sums are added in
 * fp32, rounded; the sums over `hidden` and `inner` that end in 16 bits or in
 * checkpoints are whole; other sums have 2^15 terms at most before they are added,
 * rounded, to the rest.  Everything after a product is fp32, each output rounded once.
 *
 * Workspaces: 256-byte aligned, of at least the bytes the sizes call returns
 * for the same parameters (host, pure; 0 on invalid ones).  Nothing in them
 * is kept from one call for the next; two calls that may run at the same time, replays of captured graphs
 * among them, need one each.  Matrices whose rows do not start
 * on 16 bytes (in large products: on 32) are copied there first, at the cost of
 * reading and writing them once more.
 */
#ifndef GAR_LINEAR_H_
#define GAR_LINEAR_H_

#include "gar_worker.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Log probabilities of given tokens under a linear head: z = x W^T + b,
 *     lse = log sum_j e^(z_j),   logprob = z_t - lse
 * as gar_token_logprobs has them for logits z, which exist one tile at a time only.
 *   - A negative target means "none": logprob 0.  A target >= vocab: logprob NaN.
 *   - A bias of -inf or of the type's lowest value masks a column (its weights have to be finite all the same).  A row masked
 *     throughout by -inf: lse = logprob = -inf.
 *   - A row whose logits hold a NaN or +inf: lse and logprob NaN.
 * The softmax cross entropy of a token is -logprob.  rows < 2^30, hidden and vocab < 2^31 (GAR_ERR_UNSUPPORTED beyond).
 */
typedef struct gar_linear_logprobs_params_t {
    int32_t        dtype;         /* GAR_BF16 or GAR_F16: of x, weight and bias */
    int64_t        rows, hidden, vocab;
    const void*    x;             /* dev [rows, hidden] */
    int64_t        ldx;
    const void*    weight;        /* dev [vocab, hidden] */
    int64_t        ldw;
    const void*    bias;          /* dev [vocab]; NULL: 0 */
    const int64_t* targets;       /* dev [rows]; may be NULL when logprobs is */
    float*         logprobs;      /* dev [rows]; may be NULL */
    float*         lse;           /* dev [rows]; may be NULL */
    float*         lse_lo;        /* dev [rows]; may be NULL: what rounding lse to fp32 left out */
    void*          workspace;
    size_t         workspace_bytes;
    void*          stream;
} gar_linear_logprobs_params_t;
int gar_linear_logprobs(const gar_linear_logprobs_params_t* params);
size_t gar_linear_logprobs_workspace_bytes(const gar_linear_logprobs_params_t* params);

/*
 * Gradients of the above for `workers` workers at once, row w * tokens + t being worker w's token
 * t, from the saved lse and the gradient a at the log probabilities: with
 *     dz_ij = a_i ([j = t_i] - e^(z_ij - lse_i))         (z computed again, dz rounded to x's type; of up to 128 rows
 *                                                         what that leaves out is rounded and used besides)
 *     dx = dz W,    dW_w = dz_w^T x_w,    db_w[j] = sum_i dz_ij over the worker's rows
 * the latter two stored at weight_grads[w * ld_grads + j * hidden + k] and bias_grads[w * ld_grads + j], as by
 * gar_linear_weight_grad.  The vocabulary is gone through in pieces, whose dz is kept in the workspace: up to 96 MB of
 * it, or 256 columns where those take more.  binary16 dz carry a power of two taken from the largest |a| of their worker (of their
 * row, where no weight gradients are asked for), so that small gradients do not underflow: dz have all their bits down to 2^-28 of that
 * |a|, what is below 2^-39 of it is lost.
 *   - A row without a target, or with a = 0, gets dx 0 and nothing it holds, NaN included, reaches a weight gradient.
 *     The same holds for a row masked throughout, lse = -inf, whatever its coefficient and its target.
 *   - In any other row a target >= vocab gives NaN, in dx and in its worker's gradients; no row reaches another worker's.
 *   - No tokens: weight and bias gradients of zeros.
 * 1 <= workers <= GAR_MAX_N; workers * tokens < 2^30.
 */
typedef struct gar_linear_logprobs_grad_params_t {
    int32_t        dtype;         /* GAR_BF16 or GAR_F16: of x, weight, bias and dx */
    int32_t        grads_dtype;   /* gar_dtype_t of the weight and bias gradients */
    int32_t        workers;
    int64_t        tokens, hidden, vocab;
    const void*    x;             /* dev [workers * tokens, hidden] */
    int64_t        ldx;
    const void*    weight;        /* dev [vocab, hidden] */
    int64_t        ldw;
    const void*    bias;          /* dev [vocab]; NULL: 0 */
    const int64_t* targets;       /* dev [workers * tokens] */
    const float*   lse;           /* dev [workers * tokens] */
    const float*   lse_lo;        /* dev [workers * tokens]; NULL: 0 */
    const float*   grad_logprobs; /* dev [workers * tokens] */
    void*          dx;            /* dev [workers * tokens, hidden]; NULL: not asked for */
    int64_t        lddx;
    void*          weight_grads;  /* dev; NULL: not asked for */
    void*          bias_grads;    /* dev; NULL: not asked for; needs weight_grads */
    int64_t        ld_grads;      /* elements between workers; >= vocab * hidden when workers > 1 */
    void*          workspace;
    size_t         workspace_bytes;
    void*          stream;
} gar_linear_logprobs_grad_params_t;
int gar_linear_logprobs_backward(const gar_linear_logprobs_grad_params_t* params);
size_t gar_linear_logprobs_backward_workspace_bytes(const gar_linear_logprobs_grad_params_t* params);

/*
 * The gated feed-forward block: g = x Wg^T + bg, u = x Wu^T + bu, y = act(g) * u, with 8-bit checkpoints
 * of g, u and of the stored, rounded y where they are asked for (gar_worker.h; g and u are coded from their fp32
 * values: one as near the border between two codes as its sum is off gets either, and is restored a whole step away from
 * where the other would be; ReLU's derivative next to 0 goes with it).  g and u themselves are not kept.
 */
typedef struct gar_gated_linear_params_t {
    int32_t          dtype, act, group;       /* GAR_BF16 or GAR_F16; gar_act_t; of the checkpoints */
    int64_t          rows, hidden, inner;
    const void*      x;           /* dev [rows, hidden] */
    int64_t          ldx;
    const void*      w_gate;      /* dev [inner, hidden] */
    int64_t          ld_gate;
    const void*      w_up;        /* dev [inner, hidden] */
    int64_t          ld_up;
    const void*      b_gate;      /* dev [inner]; NULL: 0 */
    const void*      b_up;        /* dev [inner]; NULL: 0 */
    void*            y;           /* dev [rows, inner] */
    int64_t          ldy;
    gar_checkpoint_t gate_saved, up_saved, y_saved;
    void*            workspace;   /* may be NULL where the size is 0 */
    size_t           workspace_bytes;
    void*            stream;
} gar_gated_linear_params_t;
int gar_gated_linear_forward(const gar_gated_linear_params_t* params);
size_t gar_gated_linear_workspace_bytes(const gar_gated_linear_params_t* params);

/*
 * Its backward pass from the checkpoints, g' and u' being the restored values:
 *     dg = dy u' act'(g'),   du = dy act(g')       (as gar_activation_backward)
 *     dx = dg Wg + du Wu
 * dg and du are outputs: gar_linear_weight_grad turns them into the workers' weight and bias gradients.
 */
typedef struct gar_gated_linear_grad_params_t {
    int32_t          dtype, act, group;
    int64_t          rows, hidden, inner;
    const void*      dy;          /* dev [rows, inner] */
    int64_t          lddy;
    gar_checkpoint_t gate_saved, up_saved;
    const void*      w_gate;      /* dev [inner, hidden] */
    int64_t          ld_gate;
    const void*      w_up;        /* dev [inner, hidden] */
    int64_t          ld_up;
    void*            dgate;       /* dev [rows, inner]; may be exactly dy (same ld) */
    int64_t          ld_dgate;
    void*            dup;         /* dev [rows, inner] */
    int64_t          ld_dup;
    void*            dx;          /* dev [rows, hidden]; NULL: not asked for */
    int64_t          lddx;
    void*            workspace;   /* may be NULL where the size is 0 */
    size_t           workspace_bytes;
    void*            stream;
} gar_gated_linear_grad_params_t;
int gar_gated_linear_backward(const gar_gated_linear_grad_params_t* params);
size_t gar_gated_linear_backward_workspace_bytes(const gar_gated_linear_grad_params_t* params);

/*
 * Dropout: y = [residual +] keep * x / (1 - p'), p' being p rounded to a multiple of 2^-16.  Whether an element is kept
 * is a function of (seed, offset, row, column) alone, so the backward pass is the same call on the gradient:
 * Philox 4x32-10 (Salmon, Moraes, Dror, Shaw 2011) with the 64-bit key `seed` and the counter
 * (low, high word of row * ceil(cols / 8) + column / 8; low, high word of the offset) gives four 32-bit words for eight
 * columns, column j taking half j % 2 (the low one first) of word j / 2; an element is dropped where its 16 bits are
 * below 2^16 p'.  A dropped element counts as 0 whatever it holds; p = 1 drops everything.
 * Calls that are to be independent differ in the seed or the offset.  `counter`, where given, is a number on the device
 * that is added to the offset when the call runs: in a captured graph, advance it between replays.
 */
typedef struct gar_dropout_params_t {
    int32_t         dtype;        /* gar_dtype_t of x, residual and y */
    float           p;            /* 0 .. 1 */
    int64_t         rows, cols;
    const void*     x;            /* dev */
    int64_t         ldx;
    const void*     residual;     /* dev; NULL: none */
    int64_t         ld_residual;
    void*           y;            /* dev; may be exactly x or the residual (same ld); any other overlap is refused */
    int64_t         ldy;
    uint64_t        seed, offset;
    const uint64_t* counter;      /* dev; NULL: 0 */
    void*           stream;
} gar_dropout_params_t;
int gar_dropout(const gar_dropout_params_t* params);

#ifdef __cplusplus
}
#endif
#endif /* GAR_LINEAR_H_ */
