/*
 * gar_worker.h -- C ABI of the operators a worker runs before its gradient is
 * aggregated (NVIDIA B200, sm_100a): token log probabilities and their
 * gradient, activation checkpoints in 8 bits with the activation's forward and
 * backward pass, and the per-worker weight gradients, written straight into
 * the rows of the n x d gradient block that gar_aggregate reads.
 *
 * Conventions are those of gar.h: device pointers of the current device, all
 * buffers owned by the caller, every call asynchronous on `stream`, argument
 * errors returned before anything is launched, GAR_ERR_CUDA for launch
 * failures, no exceptions, no CPU fallback, bit-identical output for the same
 * input.  Matrices are row-major with unit column stride and a
 * row stride `ld` in elements (0 means the number of columns); any alignment
 * of the element type is accepted unless stated otherwise.  Element types are
 * a gar_dtype_t; all arithmetic and every sum are fp32 and each output is
 * rounded once.  A call with no rows succeeds and writes nothing.  The paper
 * has no counterpart of these calls: it starts from the workers' gradients.
 */
#ifndef GAR_WORKER_H_
#define GAR_WORKER_H_

#include "gar.h"

#ifdef __cplusplus
extern "C" {
#endif

#define GAR_MAX_TOP 32            /* most alternatives a call returns per row */

/*
 * Log probabilities of given tokens.  For a row x of `vocab` logits with target t,
 *     m = max x,  s = sum_j e^(x_j - m),  lse = m + log s,
 *     logprob = x_t - lse,   entropy = -sum_j p_j log p_j,  p_j = e^(x_j - lse)
 * and, for top > 0, the `top` largest entries in descending order (equal entries: lowest index
 * first; NaN entries last) as log probabilities and indices.
 *   - A negative target means "none": logprob 0.  A target >= vocab: logprob NaN.
 *   - A row that is -inf everywhere: lse = logprob = top_logprobs = -inf, entropy 0.
 *   - A row that holds a NaN or +inf: lse, logprob, entropy and top_logprobs are NaN.
 * One pass over the logits.  vocab < 2^31 (GAR_ERR_UNSUPPORTED beyond).
 */
typedef struct gar_logprobs_params_t {
    int32_t        dtype;         /* gar_dtype_t of logits */
    int32_t        top;           /* 0 .. min(vocab, GAR_MAX_TOP) */
    int64_t        rows, vocab, ld;
    const void*    logits;        /* dev */
    const int64_t* targets;       /* dev [rows]; may be NULL when logprobs is */
    float*         logprobs;      /* dev [rows]; may be NULL */
    float*         entropy;       /* dev [rows]; may be NULL */
    float*         lse;           /* dev [rows]; may be NULL */
    float*         lse_lo;        /* dev [rows]; may be NULL: what rounding lse to fp32 left out (m + log s = lse + lse_lo) */
    float*         top_logprobs;  /* dev [rows * top]; NULL iff top == 0 */
    int64_t*       top_index;     /* dev [rows * top]; NULL iff top == 0 */
    void*          stream;
} gar_logprobs_params_t;
int gar_token_logprobs(const gar_logprobs_params_t* params);

/*
 * Gradient of the above at the logits.  With a, c, b_i the gradients at logprob, entropy and
 * top_logprobs[i]:
 *     dx_j = -p_j (a + sum_i b_i + c (log p_j + entropy)) + a [j = t] + sum_i b_i [j = top_index_i]
 * from the logits and the saved lse (and entropy, when grad_entropy is given).  A row without a
 * target has a = 0.  An empty row has gradient 0 whatever a, c, b_i, its target and its indices are;
 * in any other row a target or index outside the vocabulary gives a row of NaN.  dlogits has the logits' type and may be the logits themselves (same ld); any other
 * overlap is refused.
 */
typedef struct gar_logprobs_grad_params_t {
    int32_t        dtype;
    int32_t        top;           /* entries per row of top_index / grad_top; 0: none */
    int64_t        rows, vocab, ld;
    const void*    logits;        /* dev */
    const int64_t* targets;       /* dev [rows]; may be NULL when grad_logprobs is */
    const float*   lse;           /* dev [rows] */
    const float*   lse_lo;        /* dev [rows]; NULL: 0.  Without it p is off by up to 2^-24 |lse| relative, which
                                     matters for logits of large magnitude (all masked by the lowest value, say) */
    const float*   entropy;       /* dev [rows]; needed with grad_entropy */
    const int64_t* top_index;     /* dev [rows * top] */
    const float*   grad_logprobs; /* dev [rows]; NULL: 0 */
    const float*   grad_entropy;  /* dev [rows]; NULL: 0 */
    const float*   grad_top;      /* dev [rows * top]; NULL iff top == 0 */
    void*          dlogits;       /* dev, row stride ld_dlogits */
    int64_t        ld_dlogits;
    void*          stream;
} gar_logprobs_grad_params_t;
int gar_token_logprobs_backward(const gar_logprobs_grad_params_t* params);

/*
 * Activation checkpoints in 8 bits.  Every `group` (32, 64 or 128) consecutive columns of a row
 * share one fp32 scale; with A the largest magnitude of the group
 *     scale = A / 127,   q = rint(x * ((1 / A) * 127))   (int8, ties to even, each step rounded to fp32),
 * and a restored value is q * scale rounded once to the activation's element type, at most half a
 * step (and 2e-5 of one for the two roundings of q, plus that rounding) from the original.  (The scale is at most the largest number that 127 can be
 * multiplied with: A / 127 of the largest finite fp32 value, a mask, say, would be restored as infinity.)
 * A group with A < 2^-100 is stored as zeros; a
 * group that holds a NaN or an infinity gets scale NaN and is restored as NaN throughout.
 *   q       dev, 16-byte aligned, row stride ldq (a multiple of 16, >= columns; the padding is not touched)
 *   scales  dev [rows * ceil(columns / group)]
 */
typedef struct gar_checkpoint_t {
    int8_t* q;                    /* NULL: no checkpoint */
    float*  scales;
    int64_t ldq;
} gar_checkpoint_t;
int gar_checkpoint_pack(int dtype, const void* x, int64_t rows, int64_t cols, int64_t ldx, int group,
                        const gar_checkpoint_t* saved, void* stream);
int gar_checkpoint_unpack(int dtype, const gar_checkpoint_t* saved, int64_t rows, int64_t cols, int group,
                          void* x, int64_t ldx, void* stream);

typedef enum {
    GAR_ACT_IDENTITY = 0,
    GAR_ACT_RELU     = 1,
    GAR_ACT_SILU     = 2,         /* x / (1 + e^-x)                */
    GAR_ACT_GELU     = 3          /* x / 2 (1 + erf(x / sqrt 2))   */
} gar_act_t;

/*
 * y = act(x), or y = act(x) * up, with the checkpoints of x, up and y (of the stored, rounded y)
 * that are asked for, in one pass.
 */
typedef struct gar_activation_params_t {
    int32_t          dtype, act, group;
    int64_t          rows, cols;
    const void*      x;           /* dev */
    int64_t          ldx;
    const void*      up;          /* dev; NULL: not gated */
    int64_t          ldup;
    void*            y;           /* dev; must not overlap x or up, except exactly x (same ld) */
    int64_t          ldy;
    gar_checkpoint_t x_saved, up_saved, y_saved;
    void*            stream;
} gar_activation_params_t;
int gar_activation_forward(const gar_activation_params_t* params);

/*
 * The backward pass from the checkpoints, x' and up' being the restored values:
 *     dx = dy act'(x') [up'],   dup = dy act(x')        (relu'(0) = 0)
 * dx may be exactly dy (same ld); any other overlap is refused.
 */
typedef struct gar_activation_grad_params_t {
    int32_t          dtype, act, group;
    int64_t          rows, cols;
    const void*      dy;          /* dev */
    int64_t          lddy;
    gar_checkpoint_t x_saved;
    gar_checkpoint_t up_saved;    /* q NULL: not gated */
    void*            dx;          /* dev */
    int64_t          lddx;
    void*            dup;         /* dev; NULL iff not gated */
    int64_t          lddup;
    void*            stream;
} gar_activation_grad_params_t;
int gar_activation_backward(const gar_activation_grad_params_t* params);

/*
 * Weight (and bias) gradients of a linear layer y = x W^T + b for `workers` workers at once, from
 * the gradient at y and the 8-bit checkpoint of x: for worker w
 *     dW_w[o, i] = sum_t dy[w, t, o] x'[w, t, i],    db_w[o] = sum_t dy[w, t, o]
 * stored at weight_grads[w * ld_grads + o * in_features + i] and bias_grads[w * ld_grads + o]: with
 * ld_grads = d and pointers into the block these are the layer's pieces of the n gradient rows.
 * Row w * tokens + t of dy and of the checkpoint is worker w's token t.  Only a worker's first
 * lengths[w] tokens count (clamped to 0 .. tokens); nothing a later token or another worker holds,
 * NaN included, reaches its sums.  No tokens: zeros.
 * dy is bf16 or binary16 (GAR_ERR_UNSUPPORTED for fp32) and x' is restored in the same type; the
 * products are exact and summed in fp32 on the tensor cores.  These truncate where they add: a sum is
 * short by 1e-9 of itself per token, up to 2.8e-9 where it grows steadily.  It is therefore taken over
 * 768 tokens at a time (16-bit gradients: 2048) and the parts are added rounded: before its own rounding
 * a gradient is off by some 1e-6 (16-bit: 6e-6) of the sum of its terms' magnitudes at most, at any length.
 * 1 <= workers <= GAR_MAX_N.
 */
typedef struct gar_weight_grad_params_t {
    int32_t          dtype;       /* GAR_BF16 or GAR_F16: type of dy and of the restored x */
    int32_t          grads_dtype; /* gar_dtype_t of the gradients */
    int32_t          group;       /* of the checkpoint */
    int32_t          workers;
    int64_t          tokens, out_features, in_features;
    const void*      dy;          /* dev [workers * tokens, out_features] */
    int64_t          ld_dy;
    gar_checkpoint_t x_saved;     /* [workers * tokens, in_features] */
    const int32_t*   lengths;     /* dev [workers]; NULL: all tokens */
    void*            weight_grads;/* dev */
    void*            bias_grads;  /* dev; NULL: none */
    int64_t          ld_grads;    /* elements between workers; >= out_features * in_features when workers > 1 */
    void*            workspace;   /* dev, 256-byte aligned, >= gar_weight_grad_workspace_bytes; NULL: none.  With one, a
                                     call with few output tiles and many tokens cuts the tokens into parts, whose fp32
                                     sums are kept there and added in order; another restores x' into it once (and
                                     copies dy there if its rows do not start on 16 bytes) instead of per tile */
    size_t           workspace_bytes;
    void*            stream;
} gar_weight_grad_params_t;
int gar_linear_weight_grad(const gar_weight_grad_params_t* params);
/* Bytes of that workspace (host, pure; the sizes, dy's alignment, and whether lengths and biases are given
 * are looked at).  0 on invalid sizes and where none is used: up to 512 tokens, without lengths and with
 * dy's rows on 16 bytes, every CTA restores the columns it works on once by itself. */
size_t gar_weight_grad_workspace_bytes(const gar_weight_grad_params_t* params);
/* 1 where the call is faster with a workspace than without (measured rule; grads_dtype is looked at too). */
int gar_weight_grad_wants_workspace(const gar_weight_grad_params_t* params);

#ifdef __cplusplus
}
#endif
#endif /* GAR_WORKER_H_ */
