/*
 * jorge_lm.h - C ABI of the operators of a language model's training step that
 * stand beside the Jorge step (jorge.h) in libjorge.so: layer norm, embedding
 * lookup, softmax cross entropy over a vocabulary, linear and gated linear
 * layers, attention, and AdamW with the global gradient norm for the parameters
 * that Jorge does not precondition (gains, biases, tables wider than
 * JORGE_MAX_DIM). Each has its forward and backward pass where it has one.
 *
 * The calls keep no state: what a step keeps (moments, saved statistics) lies in
 * the caller's buffers, and temporaries in a workspace that the caller lends and
 * whose size the matching _workspace call tells (a multiple of 256; it may be
 * reused as soon as the stream has executed the call, and need not be cleared).
 * Every call queues its work on hip_stream (a hipStream_t; NULL = the null
 * stream) of the current device and returns without waiting. Nothing is
 * allocated, so the calls may be captured into a graph; what they take by value
 * is fixed then, which for jorge_adamw_step is t and the rates (see there).
 *
 * Pointers are device pointers unless the comment says "host". Matrices are
 * row-major with a row stride in elements (ld* >= columns), but for attention's,
 * which have three strides (jorge_heads). Elements are fp32 or
 * bfloat16 (JORGE_F32, JORGE_BF16); pointers need the alignment of their element,
 * workspaces 256 bytes, and every speed remark assumes 16. Whatever the type of
 * the elements, sums, softmax statistics and norms are held in fp32 or wider and
 * a result is rounded once, to nearest, unless the comment says otherwise. An
 * output may not overlap an input, other than where the comment allows it.
 *
 * Every call returns a jorge_status (jorge.h). Arguments are checked before any
 * work is queued: a call that is refused writes nothing. jorge_lm_last_error
 * tells why the calling thread's last refused or failed call was. No C++
 * exception crosses the ABI. Sums are formed in an order that timing has no part
 * in: the same inputs at the same alignment and strides give the same bits. The
 * order follows from the shapes; for the embedding's gradient also from the
 * tokens, and for the forward loss of bfloat16 inputs also from whether weight
 * can be read in place (cols a multiple of 64, ldw of 8, 16-byte alignment).
 */
#ifndef JORGE_LM_H
#define JORGE_LM_H

#include <stdint.h>

#include "jorge.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
#define JORGE_F32  0
#define JORGE_BF16 1

/* Why the calling thread's last refused or failed call of this header was; "" before any. */
const char* jorge_lm_last_error(void);

/* ---------------------------------------------------------------- layer norm
 * Per row x of `cols` elements: mean = sum(x) / cols, rstd = 1 / sqrt(sum((x -
 * mean)^2) / cols + eps), y = (x - mean) rstd weight + bias. */

/* Largest cols. */
#define JORGE_NORM_MAX_COLS 16384

/* x, y: rows x cols of dtype. weight, bias: cols elements of param_dtype each, or NULL (a gain
 * of one, a bias of zero; one may be NULL alone). mean, rstd: rows floats each, what the
 * backward pass needs; both NULL: not written. y may be x. eps >= 0, finite; with eps 0 a
 * constant row gives infinities and NaN, as the formula does. rows >= 0. */
jorge_status jorge_layernorm_forward(const void* x, int64_t ldx, int32_t dtype, const void* weight, const void* bias,
                                     int32_t param_dtype, void* y, int64_t ldy, float* mean, float* rstd, int64_t rows,
                                     int64_t cols, double eps, void* hip_stream);

/* Bytes of workspace of jorge_layernorm_backward (host pointer). */
jorge_status jorge_layernorm_workspace(int64_t rows, int64_t cols, int64_t* bytes);

/* With xhat = (x - mean) rstd and g = dy weight (per row, means over its cols):
 *   dx = rstd (g - mean(g) - xhat mean(g xhat)),
 *   dweight = sum over rows of dy xhat,  dbias = sum over rows of dy.
 * dy, x, dx: rows x cols of dtype; dx may be dy. weight: as in the forward pass (NULL: ones).
 * dweight, dbias: cols elements of param_dtype, each written unless NULL (zeros when rows is 0).
 * workspace: needed unless both are NULL. */
jorge_status jorge_layernorm_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, int32_t dtype,
                                      const float* mean, const float* rstd, const void* weight, int32_t param_dtype,
                                      void* dx, int64_t lddx, void* dweight, void* dbias, int64_t rows, int64_t cols,
                                      void* workspace, int64_t workspace_bytes, void* hip_stream);

/* ---------------------------------------------------------------- embedding
 * out[i] = scale table[tokens[i]]; dtable[v] = scale * sum over the i with tokens[i] = v of
 * dout[i]. A token outside [0, vocab), or equal to padding in the backward pass, stands for no
 * token: its row of out is zero (padding's row is read like any other), and it takes no part in
 * dtable. */

/* Largest number of tokens, of rows of a table and of its columns. */
#define JORGE_EMBED_MAX_TOKENS (1 << 24)
#define JORGE_EMBED_MAX_VOCAB  (1 << 24)
#define JORGE_EMBED_MAX_COLS   32768

/* tokens: count of them, int64. table: vocab x cols, out: count x cols, of dtype. cols >= 1. */
jorge_status jorge_embedding_forward(const int64_t* tokens, int64_t count, const void* table, int64_t ldt,
                                     int32_t dtype, int64_t vocab, int64_t cols, double scale, void* out,
                                     int64_t ldo, void* hip_stream);

/* Bytes of workspace of jorge_embedding_backward (host pointer). */
jorge_status jorge_embedding_workspace(int64_t count, int64_t vocab, int64_t cols, int64_t* bytes);

/* dout: count x cols, dtable: vocab x cols, of dtype; every row of dtable is written (zeros where
 * no token takes it). The tokens are sorted first (a token's positions ascending), each run of
 * equal tokens is summed in fp32 in an order that its place among the sorted tokens fixes, and no
 * atomics are used. padding: a token without a gradient; negative for none. */
jorge_status jorge_embedding_backward(const void* dout, int64_t lddo, const int64_t* tokens, int64_t count,
                                      int32_t dtype, int64_t vocab, int64_t cols, double scale, int64_t padding,
                                      void* dtable, int64_t lddt, void* workspace, int64_t workspace_bytes,
                                      void* hip_stream);

/* ---------------------------------------------------------------- cross entropy
 * Of logits z = hidden weight^T (tokens x vocab), which are formed piece by piece and never kept:
 *   lse_i = log sum_v exp(z_iv),
 *   loss_i = lse_i - (1 - e) z_i,target_i - (e / vocab) sum_v z_iv,  e the label smoothing.
 * A target outside [0, vocab), or equal to ignore_index, is no target: loss_i = 0, and the row
 * takes no part in the sums and gradients (its lse_i is written). */

/* Largest tokens, vocab, cols and row strides; tokens * cols ends at 2^35. */
#define JORGE_LOSS_MAX_TOKENS (1 << 21)
#define JORGE_LOSS_MAX_VOCAB  (1 << 22)
#define JORGE_LOSS_MAX_COLS   32768
#define JORGE_LOSS_MAX_STRIDE (1 << 22)

/* What grad of the backward pass is the gradient of. */
#define JORGE_LOSS_ROWS 0 /* of every loss_i: tokens floats        */
#define JORGE_LOSS_SUM  1 /* of total[0], the sum: one float       */
#define JORGE_LOSS_MEAN 2 /* of total[2], the mean: one float      */

typedef struct jorge_loss_shape {
    int64_t tokens, cols, vocab; /* >= 1 (tokens may be 0)                            */
    int64_t ldh, ldw;            /* row strides of hidden (and dhidden), of weight (and dweight) */
    int32_t dtype;               /* of hidden, weight and their gradients             */
    int32_t reserved;            /* 0 */
    int64_t ignore_index;
    double  label_smoothing;     /* e, in [0, 1]                                      */
} jorge_loss_shape;

/* Bytes of workspace of the forward (backward = 0) or backward pass (host pointers). */
jorge_status jorge_cross_entropy_workspace(const jorge_loss_shape* shape, int32_t backward, int64_t* bytes);

/* shape: host. hidden: tokens x cols, weight: vocab x cols, targets: tokens of int64. loss, lse: tokens
 * floats each. total: three floats: the sum of the losses, the number of rows with a target, and the mean
 * over them (0 without any). */
jorge_status jorge_cross_entropy_forward(const jorge_loss_shape* shape, const void* hidden, const void* weight,
                                         const int64_t* targets, float* loss, float* lse, float* total,
                                         void* workspace, int64_t workspace_bytes, void* hip_stream);

/* lse, total: as the forward pass wrote them. kind: JORGE_LOSS_*; grad: see there. With g_i the gradient of
 * loss_i (0 without a target) and p = exp(z - lse):
 *   dz_iv = g_i (p_iv - (1 - e) [v = target_i] - e / vocab),
 *   dhidden = dz weight,  dweight = dz^T hidden.
 * dhidden, dweight: written whole; either may be NULL. A row of dhidden without a target is 0, whatever grad and
 * weight hold, and so is all of both where no row has a target. bfloat16 inputs: dz (without g where that is one
 * number) is rounded to bfloat16 for the two products, whose sums are fp32: rows of dweight of words that are
 * no row's target, sums of such rounded terms alone, err by some 2.2e-3 of their size instead of the 1.7e-3 of
 * their own rounding; dhidden and the other rows by 1.7e-3. fp32 inputs: every product is formed from three-term
 * bfloat16 splits as the Jorge step's are (jorge.h), dz included: values above 3.39e38 count as infinite, a
 * product of two infinities or a sum beyond fp32's range may be NaN, and a sum over K elements takes 6 K / 32
 * roundings of its fp32 accumulator. */
jorge_status jorge_cross_entropy_backward(const jorge_loss_shape* shape, const float* grad, int32_t kind,
                                          const void* hidden, const void* weight, const int64_t* targets,
                                          const float* lse, const float* total, void* dhidden, void* dweight,
                                          void* workspace, int64_t workspace_bytes, void* hip_stream);

/* ---------------------------------------------------------------- linear layers
 * With act one of JORGE_ACT_* (gelu with the error function, silu(z) = z sigmoid(z)):
 *   linear:        z = x weight^T + bias,  y = act(z) + residual;
 *   gated linear:  g = x gate^T,  u = x up^T,  y = act(g) u.
 * Gradients, with z, g and u formed again from x:
 *   linear:        dz = dy act'(z),  dx = dz weight,  dweight = dz^T x,  dbias = sum over tokens of dz
 *                  (the residual's gradient is dy);
 *   gated linear:  dg = dy u act'(g),  du = dy act(g),  dx = dg gate + du up,  dgate = dg^T x,  dup = du^T x.
 * relu's derivative at 0 is 0. gelu's normal distribution errs in fp32 by at most 20 roundings of itself, also in its
 * tails, and in bfloat16 by 3e-7 of 1, which shows below arguments of -5. bfloat16: dz, dg and du are rounded to bfloat16
 * for the products, whose sums are fp32 (dbias is summed before that); a gradient then errs by some 2.4e-3 of its size
 * instead of the 1.7e-3 of its own rounding. fp32: up to JORGE_LINEAR_FEW_TOKENS forward are multiplied in fp32; the
 * other products are formed from three-term bfloat16 splits as the Jorge step's are (jorge.h): values above 3.39e38
 * count as infinite, and a product of two infinities or a sum beyond fp32's range may be NaN. Their sums over more than
 * 1024 terms (2048 where z is formed again) are formed in up to eight ranges, of which a call's workspace holds up to
 * 1 GiB at a time. */
#define JORGE_ACT_NONE    0
#define JORGE_ACT_RELU    1
#define JORGE_ACT_GELU    2
#define JORGE_ACT_SILU    3
#define JORGE_ACT_SIGMOID 4

/* Up to so many tokens the forward passes need no workspace. */
#define JORGE_LINEAR_FEW_TOKENS 64

/* Largest tokens, cols, outs and row strides; tokens * max(cols, outs) ends at 2^34. */
#define JORGE_LINEAR_MAX_TOKENS (1 << 21)
#define JORGE_LINEAR_MAX_COLS   32768
#define JORGE_LINEAR_MAX_OUTS   (1 << 18)
#define JORGE_LINEAR_MAX_STRIDE (1 << 22)

typedef struct jorge_linear_shape {
    int64_t tokens, cols, outs;  /* >= 1 (tokens may be 0); x: tokens x cols, a weight: outs x cols  */
    int64_t ldx, ldw, ldu;       /* row strides of x, of weight (gate), of up (gated linear)         */
    int64_t ldy, ldr;            /* of y (forward) or dy (backward), of residual                     */
    int32_t dtype, bias_dtype;   /* of x, the weights, residual, y and their gradients; of bias and dbias */
    int32_t activation;          /* JORGE_ACT_*                                                      */
    int32_t reserved;            /* 0 */
} jorge_linear_shape;

/* Bytes of workspace of the forward (backward = 0) or backward pass of the linear (gated = 0) or gated linear layer
 * (host pointers), of any addresses and with all gradients; 0 where none is needed. */
jorge_status jorge_linear_workspace(const jorge_linear_shape* shape, int32_t gated, int32_t backward, int64_t* bytes);

/* The gradients that a call of the backward pass asks for (DWEIGHT: of both weights of the gated linear layer). */
#define JORGE_LINEAR_DX      1
#define JORGE_LINEAR_DWEIGHT 2
#define JORGE_LINEAR_DBIAS   4

/* Bytes of workspace of one call, of the linear (up NULL) or gated linear layer, forward (dy NULL) or backward with the
 * gradients `wanted`: at most what jorge_linear_workspace tells. A call needs no copies of bfloat16 operands whose rows
 * and strides are whole multiples of 64 (rows) and 8 (strides) elements, at 16-byte alignment (gate and up: of one
 * stride). The pointers are not followed. */
jorge_status jorge_linear_call_workspace(const jorge_linear_shape* shape, const void* dy, const void* x,
                                         const void* weight, const void* up, int32_t wanted, int64_t* bytes);

/* shape: host. bias: outs elements, residual: tokens x outs; each may be NULL. y may be residual (with ldy = ldr). */
jorge_status jorge_linear_forward(const jorge_linear_shape* shape, const void* x, const void* weight, const void* bias,
                                  const void* residual, void* y, void* workspace, int64_t workspace_bytes,
                                  void* hip_stream);

/* dx: tokens x cols, dweight: outs x cols, dbias: outs; each written whole unless NULL (dweight and dbias zeros where
 * tokens is 0). ldr is not read. */
jorge_status jorge_linear_backward(const jorge_linear_shape* shape, const void* dy, const void* x, const void* weight,
                                   const void* bias, void* dx, int64_t lddx, void* dweight, int64_t lddw, void* dbias,
                                   void* workspace, int64_t workspace_bytes, void* hip_stream);

/* bias_dtype and ldr are not read. */
jorge_status jorge_gated_linear_forward(const jorge_linear_shape* shape, const void* x, const void* gate,
                                        const void* up, void* y, void* workspace, int64_t workspace_bytes,
                                        void* hip_stream);

/* dgate, dup: outs x cols in the stride lddw; either both or neither. */
jorge_status jorge_gated_linear_backward(const jorge_linear_shape* shape, const void* dy, const void* x,
                                         const void* gate, const void* up, void* dx, int64_t lddx, void* dgate,
                                         void* dup, int64_t lddw, void* workspace, int64_t workspace_bytes,
                                         void* hip_stream);

/* ---------------------------------------------------------------- attention
 * Of queries q (batch x q_tokens x heads x dim) over k and v (batch x kv_tokens x kv_heads x dim), heads / kv_heads
 * consecutive heads to one of k and v, with z = scale q k^T over the keys that a query sees:
 *   lse = log sum exp z,  o = sum exp(z - lse) v.
 * A sequence b has q_lengths[b] queries and kv_lengths[b] keys (those of the whole batch where the pointer is NULL;
 * values outside 0 .. tokens count as the nearest of them), from its first row on. A query sees every key of its
 * sequence; with causal, query i stands at position kv length - q length + i and sees the keys up to its own position,
 * with a window of w > 0 the last w of those. A query that sees nothing, or that is past its sequence's length, has
 * o = 0, lse = minus infinity and no part in any gradient, whatever it holds; so has a key past its sequence's length,
 * whose rows of k and v may hold anything. What a key holds reaches no query that does not see it, and what a query or
 * its gradient holds no key that the query does not see, infinities and NaN among it.
 * Gradients, from the o and lse of the forward pass, with p = exp(z - lse):
 *   delta = do . o,  ds = scale p (do v^T - delta),  dq = ds k,  dk = ds^T q,  dv = p^T do,
 * dk and dv summed over the heads that share them. bfloat16: p and ds are rounded to bfloat16 for their products, all
 * else is fp32 (a gradient then errs by some 2.4e-3 of its size instead of the 1.7e-3 of its own rounding); where rows
 * see few keys, delta is the sum of p (do v^T), as o's rounding would not average out in it. fp32 is multiplied in
 * fp32, and summed over 32 rows at a time before the long sum. A p below 2^-126 (forward: of
 * the row's largest one) may count as 0. */

/* Largest dim, tokens, token stride, and rows: batch * heads * q_tokens of q, batch * kv_heads * kv_tokens of k. */
#define JORGE_ATTENTION_MAX_DIM    128
#define JORGE_ATTENTION_MAX_TOKENS (1 << 22)
#define JORGE_ATTENTION_MAX_STRIDE (1 << 22)
#define JORGE_ATTENTION_MAX_ROWS   (1 << 26)

/* A matrix of heads: element d of head h of token t of sequence b is data[b batch + t token + h head + d]. */
typedef struct jorge_heads {
    void*   data;
    int64_t batch, token, head;  /* strides in elements, >= 0 */
} jorge_heads;

typedef struct jorge_attention_shape {
    int64_t batch, q_tokens, kv_tokens; /* >= 0 */
    int32_t heads, kv_heads, dim;       /* heads a multiple of kv_heads */
    int32_t dtype;                      /* of q, k, v, out and their gradients */
    double  scale;                      /* > 0, below 1e30 */
    int32_t causal;                     /* 0 or 1 */
    int32_t reserved;                   /* 0 */
    int64_t window;                     /* 0 for none; needs causal */
    const int64_t *q_lengths, *kv_lengths; /* device: batch numbers each, or NULL */
    jorge_heads q, k, v;                /* their data is only read */
} jorge_attention_shape;

/* Bytes of workspace (host pointers; 0 where none is needed) of the forward pass (dout NULL) or the backward pass. It
 * depends on the matrices' addresses and strides too: those whose rows do not lie in whole 16 bytes are copied. */
jorge_status jorge_attention_workspace(const jorge_attention_shape* shape, const jorge_heads* dout, int64_t* bytes);

/* shape, out: host. lse: batch x heads x q_tokens floats. */
jorge_status jorge_attention_forward(const jorge_attention_shape* shape, const jorge_heads* out, float* lse,
                                     void* workspace, int64_t workspace_bytes, void* hip_stream);

/* dq like q, dk and dv like k: each written whole unless NULL. */
jorge_status jorge_attention_backward(const jorge_attention_shape* shape, const jorge_heads* dout,
                                      const jorge_heads* out, const float* lse, const jorge_heads* dq,
                                      const jorge_heads* dk, const jorge_heads* dv, void* workspace,
                                      int64_t workspace_bytes, void* hip_stream);

/* ---------------------------------------------------------------- AdamW
 * Step t of every element p of every tensor, with g its gradient times the clip factor:
 *   m <- m + (1 - beta1) (g - m),  v <- v + (1 - beta2) (g^2 - v),
 *   p <- p - (lr weight_decay p + lr / (1 - beta1^t) m / (sqrt(v) / sqrt(1 - beta2^t) + eps)).
 * The moments of all tensors lie in two flat buffers, in blocks of JORGE_ADAMW_BLOCK elements; a tensor
 * starts a block. With bits = 32 they are floats. With bits = 8 a block has one scale byte k in a buffer
 * of its own, 2^(k - 127) with k in 1 .. 253 the least that puts the block's largest magnitude at or below
 * 31/16 2^(k - 127), and a byte per element, y = x / 2^(k - 127) as a small float: the first moment with a
 * sign bit, three exponent bits E and four mantissa bits M, (1 + M/16) 2^(E - 7) or, at E = 0, (M/16) 2^-6;
 * the second without sign, four and four, (1 + M/16) 2^(E - 15) or (M/16) 2^-14. All zero bytes are zero
 * moments. y is rounded to one of its two neighbours by 16 random bits (made from seed, t and the element's
 * place in the buffers), so that slow averages move in the mean; a second moment above zero keeps at least
 * the smallest code. The step itself uses m and v before this rounding. A NaN or an infinity makes its
 * element's parameter NaN and, in 8 bits, its moments the largest code of their block, the rest of which
 * keeps its own scale. */
#define JORGE_ADAMW_BLOCK 256

typedef struct jorge_adamw_tensor {
    void*       param;  /* numel elements of dtype, updated in place; no two tensors' may overlap */
    const void* grad;   /* numel elements of dtype                   */
    int64_t     numel;  /* >= 0, at most 2^38                        */
    int64_t     block;  /* the tensor's first block in the moments' buffers; the tensors' blocks ascend
                           without overlap */
    int32_t     dtype;  /* JORGE_F32 or JORGE_BF16                   */
    int32_t     reserved; /* 0 */
} jorge_adamw_tensor;

typedef struct jorge_adamw_moments {
    void*    exp_avg;          /* blocks * 256 floats (bits = 32) or bytes (bits = 8), 16-byte aligned */
    void*    exp_avg_sq;
    uint8_t* exp_avg_scale;    /* blocks bytes each (bits = 8; NULL otherwise) */
    uint8_t* exp_avg_sq_scale;
    int64_t  blocks;           /* that the buffers hold */
    int32_t  bits;             /* 32 or 8 */
    uint32_t seed;             /* of the random bits (bits = 8) */
} jorge_adamw_moments;

/* Global norm of the gradients of n tensors (param and block are not read): out[0] = sqrt(sum g^2), out[1]
 * = the clip factor, min(1, max_norm / out[0]) for max_norm > 0 (finite), 1 for max_norm = 0; a norm that is
 * NaN makes the factor NaN, an infinite one 0. Squares are summed in fp32 by the lane and in fp64 beyond. tensors:
 * host, read before the call returns. out: two floats. */
jorge_status jorge_gradient_norm_workspace(const jorge_adamw_tensor* tensors, int32_t n, int64_t* bytes);
jorge_status jorge_gradient_norm(const jorge_adamw_tensor* tensors, int32_t n, double max_norm, float* out,
                                 void* workspace, int64_t workspace_bytes, void* hip_stream);

/* Step t >= 1 of n tensors: t counts a tensor's own steps, and tensors that have taken different numbers of them
 * go in calls of their own (with the same moments). tensors, moments: host, read before the call returns. clip: one
 * float, the factor of the gradients (out + 1 of jorge_gradient_norm), or NULL for 1. lr, eps, weight_decay >= 0,
 * 0 <= beta1, beta2 < 1, all finite. Scalars are formed in fp64 and enter the step as floats. A call captured into
 * a graph repeats its step t: replays have the bias corrections, rates and random bits of that one step, so they are
 * no sequence of steps, and 8-bit moments rounded by the same bits every time are not right in the mean. */
jorge_status jorge_adamw_step(const jorge_adamw_tensor* tensors, int32_t n, const jorge_adamw_moments* moments,
                              int64_t t, double lr, double beta1, double beta2, double eps, double weight_decay,
                              const float* clip, void* hip_stream);

/* The values that 8-bit moments stand for: count blocks from `first` on of one moment (second = 0: the first,
 * 1: the second) to out, count * 256 elements of dtype (both types hold them exactly, but that fp32's and
 * bfloat16's own range ends at 2^-126 (normal) and values below it keep what subnormals hold). And the
 * reverse, from floats, rounded to nearest (ties to the even code): how a state is loaded. */
jorge_status jorge_adamw_read(const jorge_adamw_moments* moments, int32_t second, int64_t first, int64_t count,
                              void* out, int32_t dtype, void* hip_stream);
jorge_status jorge_adamw_write(const jorge_adamw_moments* moments, int32_t second, int64_t first, int64_t count,
                               const float* values, void* hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* JORGE_LM_H */
