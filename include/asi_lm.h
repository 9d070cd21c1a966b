/*
 * asi_lm.h - the operators of a language model's fine-tuning step that stand beside the compressed
 * layers of asi.h: token log probabilities with entropy and top alternatives and their gradient,
 * embedding lookup and its gradient, norms of queries and keys with the position rotation and their
 * gradient, and an AdamW step over many tensors with states in 32 or in 8 bits.
 *
 * The conventions of asi.h hold: device pointers, no allocation, no state between calls, kernels are
 * only enqueued on `stream`, argument errors are returned and enqueue nothing, scratch is the
 * caller's and 256-byte aligned.  Types are ASI_F32 and ASI_BF16 (asi_dtype); every sum, statistic,
 * norm and angle product is in fp32 whatever the types, and a result in bf16 is rounded once, to nearest.
 * Strides are in elements; the innermost dimension is always contiguous.  Pointers need the alignment
 * of their element type only.  Inputs must not overlap outputs except where that is stated.
 */
#ifndef ASI_LM_H
#define ASI_LM_H

#include "asi.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- Token log probabilities -------------------------------------------------------------------
 * For a row x of `vocab` logits:  z = scale * x,  lse = log sum_i exp(z_i),  p_i = exp(z_i - lse),
 *     logprob = z_target - lse        entropy = - sum_i p_i log p_i
 *     top: the `top` largest logits in descending order, equal ones by ascending index.
 * A logit of -infinity has probability 0 and adds nothing.  A row of nothing but -infinity has lse and
 * logprob -infinity, entropy 0 and gradient 0.  A row that holds NaN or +infinity gives NaN.
 * In the order of the top alternatives NaN comes first. */
#define ASI_LOGPROB_MAX_TOP 64
typedef struct {
    int64_t rows, vocab;
    int64_t row_stride;        /* of logits, >= vocab (rows may be padded) */
    int64_t grad_stride;       /* of dlogits, >= vocab; read by asi_token_logprobs_grad only */
    int64_t ignore_index;      /* a row with this target has none: logprob 0 and no gradient from it */
    int32_t dtype;             /* of logits and dlogits */
    int32_t top;               /* 0 .. min(vocab, ASI_LOGPROB_MAX_TOP); read by asi_token_logprobs only */
    float scale;               /* 1e-20 .. 1e20: the inverse of a temperature */
    int32_t reserved;          /* 0 */
} asi_logprob_desc;

/* Scratch bytes of asi_token_logprobs (0 where it needs none; ws may then be NULL). */
size_t asi_token_logprobs_workspace_bytes(const asi_logprob_desc* desc);

/*   targets      in  device int64 (rows), nullable if logprob is; a target outside [0, vocab) that is not
 *                    ignore_index gives NaN
 *   logprob      out device fp32 (rows), nullable
 *   entropy      out device fp32 (rows), nullable
 *   lse          out device fp32 (rows), nullable
 *   top_logprob  out device fp32 (rows, top), top_index out device int64 (rows, top); both if top > 0 */
asi_status asi_token_logprobs(const asi_logprob_desc* desc, const void* logits, const int64_t* targets, float* logprob,
                              float* entropy, float* lse, float* top_logprob, int64_t* top_index, void* ws,
                              size_t ws_bytes, asi_stream_t stream);

/* The gradient of sum_t a_t logprob_t + b_t entropy_t, and both values, in one pass:
 *     dlogits_i = scale * ( a (delta_{i,target} - p_i) - b p_i (log p_i + entropy) )
 *   grad_logprob  in  device fp32 (rows): a, nullable (all zero)
 *   grad_entropy  in  device fp32 (rows): b, nullable (all zero)
 *   dlogits       out device (rows, vocab), dtype per desc; may be `logits` itself, with the same stride
 *   logprob, entropy  out device fp32 (rows), nullable
 * A row whose target is ignore_index takes a = 0; one whose target is out of range gets NaN. */
asi_status asi_token_logprobs_grad(const asi_logprob_desc* desc, const void* logits, const int64_t* targets,
                                   const float* grad_logprob, const float* grad_entropy, void* dlogits, float* logprob,
                                   float* entropy, asi_stream_t stream);

/* ---- Embedding ---------------------------------------------------------------------------------
 * out[t] = scale * table[token_t];     dtable[v] = scale * sum over t with token_t = v of grad_out[t],
 * the sum taken in an order that depends on the tokens alone, so that equal calls give equal bits. */
typedef struct {
    int64_t tokens, vocab, dim;    /* tokens < 2^30, vocab <= 2^24 */
    int64_t table_stride;      /* of table / dtable, >= dim */
    int64_t out_stride;        /* of out / grad_out, >= dim */
    int64_t padding_index;     /* a token whose row gets no gradient; -1: none */
    int32_t table_dtype;       /* of table / dtable */
    int32_t out_dtype;         /* of out / grad_out */
    float scale;
    int32_t reserved;          /* 0 */
} asi_embedding_desc;

/*   tokens  in  device int64 (tokens); one outside [0, vocab) gives a row of NaN */
asi_status asi_embedding(const asi_embedding_desc* desc, const int64_t* tokens, const void* table, void* out,
                         asi_stream_t stream);

size_t asi_embedding_grad_workspace_bytes(const asi_embedding_desc* desc);

/*   dtable  out device (vocab, dim): overwritten, rows without a token with zeros; with accumulate != 0 the
 *               rows that have tokens are added to and no other is touched
 * Tokens outside [0, vocab) and padding_index count for nothing.  ASI_ERR_UNSUPPORTED where one launch has not enough
 * workgroups: above some 2^38 entries of grad_out, or 2^32 in up to 1024 rows. */
asi_status asi_embedding_grad(const asi_embedding_desc* desc, const int64_t* tokens, const void* grad_out, void* dtable,
                              int accumulate, void* ws, size_t ws_bytes, asi_stream_t stream);

/* ---- Norms of queries and keys with the position rotation ------------------------------------------
 * For every head x of q (gain q_gain) and of k (gain k_gain) at position s = positions[b, t]:
 *     r = 1 / sqrt(mean_i x_i^2 + eps);   n_i = x_i r gain_i
 *     (y_i, y_j) = (n_i cos[s, e] - n_j sin[s, e], n_j cos[s, e] + n_i sin[s, e])
 * on the pairs (i, j) = (e, e + rot_dim / 2), or (2 e, 2 e + 1) if interleaved, e < rot_dim / 2; the rest of
 * the head, y_i = n_i, is not turned.  There is no form without the norm: without gains x_i r is turned. */
typedef struct {
    int64_t batch, tokens;
    int64_t max_position;      /* rows of cos and sin */
    int64_t position_stride;   /* between batch entries of positions; 0: the same positions for all */
    int64_t q_stride[3], k_stride[3];           /* (batch, token, head) of q, k */
    int64_t q_out_stride[3], k_out_stride[3];   /* of q_out, k_out, or of their gradients */
    int64_t dq_stride[3], dk_stride[3];         /* of dq, dk; read by asi_qk_norm_rotate_grad only */
    int32_t q_heads, k_heads;  /* 0 allowed: that side is left out */
    int32_t head_dim;          /* 1 .. 1024 */
    int32_t rot_dim;           /* even, 0 .. head_dim */
    int32_t interleaved;       /* 0 or 1 */
    int32_t dtype;             /* of q, k, their outputs and gradients */
    int32_t gain_dtype;        /* of q_gain, k_gain */
    float eps;                 /* >= 0 */
} asi_qk_desc;

/*   q_gain, k_gain  in  device (head_dim), nullable (all one)
 *   positions       in  device int64 (batch, tokens), nullable: 0 .. tokens - 1; one outside [0, max_position) gives NaN
 *   cos, sin        in  device fp32 (max_position, rot_dim / 2), not read if rot_dim = 0
 *   q_out, k_out    out device; may be q, k themselves, with the same strides */
asi_status asi_qk_norm_rotate(const asi_qk_desc* desc, const void* q, const void* k, const void* q_gain, const void* k_gain,
                              const int64_t* positions, const float* cos, const float* sin, void* q_out, void* k_out,
                              asi_stream_t stream);

size_t asi_qk_norm_rotate_grad_workspace_bytes(const asi_qk_desc* desc);

/*   q, k            in  what the forward call read
 *   grad_q, grad_k  in  gradients of q_out, k_out (strides q_out_stride, k_out_stride)
 *   dq, dk          out gradients of q, k; may be q, k or grad_q, grad_k themselves, with the same strides
 *   dq_gain, dk_gain  out device fp32 (head_dim), nullable; summed over batch, tokens and heads in a fixed order */
asi_status asi_qk_norm_rotate_grad(const asi_qk_desc* desc, const void* q, const void* k, const void* q_gain,
                                   const void* k_gain, const int64_t* positions, const float* cos, const float* sin,
                                   const void* grad_q, const void* grad_k, void* dq, void* dk, float* dq_gain,
                                   float* dk_gain, void* ws, size_t ws_bytes, asi_stream_t stream);

/* ---- AdamW over many tensors -------------------------------------------------------------------
 * With g' = g * *grad_scale, and every product, sum, quotient and root rounded to fp32 by itself:
 *     m = beta1 m + (1 - beta1) g';   v = beta2 v + (1 - beta2) g'^2
 *     p = (1 - lr weight_decay) p - lr / (1 - beta1^step) * m / (sqrt(v) / sqrt(1 - beta2^step) + eps)
 * States of 8 bits: m and sqrt(v) are held as 8-bit floats (1 sign bit, 4 of exponent, 3 of mantissa, no
 * infinities) times an fp32 scale for each ASI_ADAMW_BLOCK consecutive elements, the largest finite magnitude of the
 * block / 448.  Rounding is to nearest, except that a positive root is never held as zero (the next step divides by
 * it).  A block whose scale would be below 2^-126 is held as zeros; a value that is not finite is held as NaN. */
#define ASI_ADAMW_BLOCK 256
typedef struct {
    void* param;               /* in/out, param_dtype */
    const void* grad;          /* in, grad_dtype */
    float* master;             /* in/out fp32, nullable: the parameter's value; param is then only written, rounded */
    void* exp_avg;             /* in/out: m, fp32 or 8-bit codes */
    void* exp_avg_sq;          /* in/out: v in fp32, or sqrt(v) as 8-bit codes */
    float* exp_avg_scale;      /* in/out, (count + 255) / 256 entries; 8 bits only */
    float* exp_avg_sq_scale;   /* in/out, the same of sqrt(v); 8 bits only */
    int64_t count;             /* elements, 0 .. 2^40 */
    int32_t param_dtype, grad_dtype;
    double lr, weight_decay;
} asi_adamw_tensor;

/*   tensors     HOST array of `count` tensors; they must not overlap
 *   state_bits  32 or 8, of all of them
 *   step        1 for the first step
 *   grad_scale  device fp32 (1), nullable (1): what every gradient is multiplied by, e.g. to clip their norm
 *   skip        device int32 (1), nullable: if it is not zero when the kernels run, nothing is changed */
asi_status asi_adamw(int32_t count, const asi_adamw_tensor* tensors, int32_t state_bits, double beta1, double beta2,
                     double eps, int64_t step, const float* grad_scale, const int32_t* skip, asi_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* ASI_LM_H */
