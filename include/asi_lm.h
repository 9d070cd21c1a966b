/*
 * asi_lm.h - the operators of a language model's fine-tuning step that stand beside the compressed
 * layers of asi.h: token log probabilities with entropy and top alternatives and their gradient,
 * embedding lookup and its gradient, norms of queries and keys with the position rotation and their
 * gradient, an AdamW step over many tensors with states in 32 or in 8 bits; and what spares a step
 * the rest of its memory: the same log probabilities and gradients without the logits, dropout without a
 * stored mask, the edge between two blocks in one pass.
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

/* ---- Token log probabilities without the logits -------------------------------------------------
 * The values of asi_token_logprobs for the logits x = H W^T, H the hidden states (rows, dim) and W the
 * weights of the output layer (vocab, dim), and the gradients of sum_t a_t logprob_t + b_t entropy_t:
 *     dz = scale ( a (delta_target - p) - b p (log p + entropy) )       dH = dz W        dW = dz^T H
 * The logits are made in tiles and used up there; for the gradients they are made a second time, in pieces of
 * the vocabulary, or kept in the workspace where the whole vocabulary is one piece (for few rows, 64 at most, always; otherwise up to 96 MiB
 * and where `given` is 0).  Weights that cannot be multiplied as they lie (fp32; bf16 whose rows are no whole vectors or no multiple of
 * 64 entries) are copied into the workspace by pieces of up to 768 MiB, so that it may be larger than the logits of few rows.  Kept
 * between the two calls are two numbers a row: the largest logit x_max (before the scale) and log sum_i exp(scale (x_i - x_max)).
 * A row whose target is ignore_index is left out: whatever it holds, it has logprob, entropy and gradient 0 and adds nothing
 * to dW.  A target out of range otherwise gives NaN, as a row does that holds NaN or +infinity among its logits.  A logit of
 * -infinity has probability 0; where a weight is infinite, dH has 0 times infinity, NaN, in its column.
 * ASI_ERR_UNSUPPORTED where a launch has not enough workgroups: above 2^23 tiles of 128 x 128 logits, 2^23 of dW, or 2^32
 * entries of H with gradients (2^35 without).
 * Products of fp32 inputs are exact to about the rounding of fp32 (each side as three bf16 numbers, six products of
 * them, sums in fp32).  For bf16 inputs dz is held to 2^-16 of itself (as two parts of bf16; in
 * fp32 for few rows) when it is multiplied, and dH and dW are rounded once at the end. */
typedef struct {
    int64_t rows, dim, vocab;  /* rows < 2^24, dim < 2^18, vocab < 2^28 */
    int64_t hidden_stride;     /* of H, >= dim */
    int64_t weight_stride;     /* of W, >= dim; dH and dW are dense */
    int64_t ignore_index;
    int32_t dtype;             /* of H, W, dH and dW */
    float scale;               /* 1e-20 .. 1e20 */
    int32_t any_address;       /* 0: weight lies at a multiple of 16 bytes; 1: it may not (bf16 weights are then copied by pieces) */
    int32_t reserved;          /* 0 */
} asi_linear_logprob_desc;

size_t asi_linear_logprobs_workspace_bytes(const asi_linear_logprob_desc* desc);

/*   targets  in  device int64 (rows), nullable if logprob is: then no row is left out
 *   logprob, entropy  out device fp32 (rows), nullable
 *   stats    out device fp32 (rows, 2): x_max and the logarithm, for asi_linear_logprobs_grad; nullable */
asi_status asi_linear_logprobs(const asi_linear_logprob_desc* desc, const void* hidden, const void* weight,
                               const int64_t* targets, float* logprob, float* entropy, float* stats, void* ws,
                               size_t ws_bytes, asi_stream_t stream);

size_t asi_linear_logprobs_grad_workspace_bytes(const asi_linear_logprob_desc* desc);

/*   given    0: the values are computed first, and written where logprob and entropy are not NULL; stats is not used
 *            1: stats and entropy are those of asi_linear_logprobs for the same descriptor; entropy is read only if grad_entropy is given
 *   targets       in  nullable if grad_logprob is
 *   grad_logprob  in  device fp32 (rows): a, nullable (all zero)
 *   grad_entropy  in  device fp32 (rows): b, nullable (all zero)
 *   dhidden  out device (rows, dim), dweight  out device (vocab, dim), both dense, either nullable */
asi_status asi_linear_logprobs_grad(const asi_linear_logprob_desc* desc, int given, const void* hidden, const void* weight,
                                    const int64_t* targets, const float* stats, float* logprob, float* entropy,
                                    const float* grad_logprob, const float* grad_entropy, void* dhidden, void* dweight,
                                    void* ws, size_t ws_bytes, asi_stream_t stream);

/* ---- Dropout without a stored mask ----------------------------------------------------------------
 *     y_i = x_i * 2^16 / (2^16 - t) if u_i >= t, else 0;      t = round(p * 2^16)
 * i counts the elements of (rows, dim) in order.  u_i are 16 of the 128 bits that Philox4x32-10 (Salmon et al., SC
 * 2011) gives with the seed as its key on the counter (i / 8 mod 2^32, i / 8 div 2^32, offset mod 2^32, offset div 2^32):
 * of word (i mod 8) / 2 the low half for even i, the high half for odd i.  The gradient is the same call on the
 * gradient of y.  An element that is dropped is 0 whatever it held.  Different offsets are independent. */
typedef struct {
    int64_t rows, dim;
    int64_t x_stride, y_stride;    /* of rows, >= dim */
    int64_t seed;              /* read if no pointer to a seed is given */
    int64_t offset;            /* which layer's, say */
    double p;                  /* 0 <= p, t < 2^16 */
    int32_t dtype;
    int32_t reserved;          /* 0 */
} asi_dropout_desc;

/*   seed  in  device int64 (1), nullable: read when the kernel runs, so that a captured call takes new numbers
 *   y     out device; may be x itself, with the same stride */
asi_status asi_dropout(const asi_dropout_desc* desc, const void* x, const int64_t* seed, void* y, asi_stream_t stream);

/* ---- The edge between two blocks ------------------------------------------------------------------
 * For every row x of the stream and y of a block's output:
 *     u = y / sqrt(mean_i y_i^2 + eps) if post_norm, else y;     n = u post_gain
 *     s = x + scale gate dropout(n), rounded to the stream's type;     out = s / sqrt(mean_i s_i^2 + eps) pre_gain
 * dropout as above, over (rows, dim).  Without y the stream is taken as it is, s = x: a norm alone.
 * gate has gate_rows rows of dim entries (0: no gate); each serves rows / gate_rows consecutive rows. */
typedef struct {
    int64_t rows, dim;         /* dim <= ASI_RESIDUAL_MAX_DIM */
    int64_t x_stride;          /* of x; of s in the backward pass */
    int64_t y_stride;
    int64_t gate_rows;         /* 0, or a divisor of rows; gate, stream, out and the gradients are dense */
    int64_t seed, offset;      /* as asi_dropout_desc */
    double p;
    int32_t stream_dtype;      /* of x, s and their gradients */
    int32_t dtype;             /* of y, out and their gradients: ASI_BF16, or both ASI_F32 */
    int32_t gain_dtype;        /* of the gains and the gate */
    int32_t post_norm;         /* 0 or 1 */
    float scale, eps;          /* eps >= 0 */
} asi_residual_desc;
#define ASI_RESIDUAL_MAX_DIM 16384

/*   y        in  nullable
 *   post_gain, pre_gain  in  device (dim), nullable (all one); post_gain only with post_norm
 *   gate     in  device (gate_rows, dim), NULL if and only if gate_rows is 0
 *   stream   out device (rows, dim): s; NULL if and only if y is; may be x itself, with x_stride = dim
 *   out      out device (rows, dim), nullable if stream is not: no norm of the stream */
asi_status asi_residual_norm(const asi_residual_desc* desc, const void* x, const void* y, const void* post_gain,
                             const void* gate, const void* pre_gain, const int64_t* seed, void* stream_out, void* out,
                             asi_stream_t stream);

size_t asi_residual_norm_grad_workspace_bytes(const asi_residual_desc* desc);

/*   grad_stream, grad_out  in  gradients of s and out, dense, one of them nullable (zero; without grad_out: no norm)
 *   s        in  the forward call's stream (x where there is no y), stride x_stride; nullable if grad_out is
 *   dx, dy   out gradients of x and y, dense; dx nullable, dy NULL if and only if y is
 *   dpost_gain, dpre_gain  out device fp32 (dim), nullable; dgate  out device fp32 (gate_rows, dim), nullable
 * Sums over rows are in an order that the shape alone decides. */
asi_status asi_residual_norm_grad(const asi_residual_desc* desc, const void* grad_stream, const void* grad_out, const void* s,
                                  const void* y, const void* post_gain, const void* gate, const void* pre_gain,
                                  const int64_t* seed, void* dx, void* dy, float* dpost_gain, float* dgate, float* dpre_gain,
                                  void* ws, size_t ws_bytes, asi_stream_t stream);

#ifdef __cplusplus
}
#endif
#endif /* ASI_LM_H */
