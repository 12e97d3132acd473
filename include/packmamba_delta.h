/*
 * packmamba_delta.h -- C ABI of the gated delta rule over packed rows, in chunks for training and
 * prompts and token by token for generation, and of the norms that a block around it takes: each
 * head's features divided by their length (queries and keys), and the layer norm before the block,
 * on AMD Instinct MI355X (gfx950).
 *
 * The conventions of packmamba.h hold: device pointers owned by the caller, 16-byte aligned,
 * contiguous, the sequence innermost; dtype codes PACKMAMBA_F32, PACKMAMBA_BF16 and
 * PACKMAMBA_BF16_F32OUT; status codes; nothing is allocated or synchronised; argument errors are
 * returned before anything is enqueued.  Outputs overlap neither inputs nor each other, except
 * where it is said.
 *
 * The rule, for every batch row b and head h, at token t:
 *   a_t = exp(decay_t), and 0 where position_indices[b,t] == 0 (a sequence starts)
 *   S'  = a_t S_{t-1}                    (dk x dv; S = initial_state before the row, or zeros)
 *   u_t = beta_t (v_t - S'^T k_t)
 *   S_t = S' + k_t u_t^T
 *   out_t = scale S_t^T q_t
 * What the state holds at k_t is replaced by v_t by the share beta_t.  The state stays bounded where
 * beta_t |k_t|^2 is between 0 and 2 (packmamba_head_l2norm_fwd, and beta in (0, 1) or (0, 2), see to that);
 * other values are taken as they are.
 * q and k belong to groups of heads: head h reads group h / (heads / groups).
 *   q, k      (batch, groups, dk, seqlen)  dtype
 *   v, out    (batch, heads, dv, seqlen)   dtype
 *   beta      (batch, heads, seqlen)       float
 *   decay     log decays, float: (batch, heads, seqlen) if decay_per_token, else (heads); NULL: 0.
 *             A value of -104 or less (exp of it is 0 in 32 bits; -infinity too) cuts as a start
 *             does.
 *             Values above 0 are taken as they are; where those of a sequence's tokens in a row sum to more
 *             than 88 over 64 tokens or fewer, their exponentials' products are infinite in 32 bits, and what
 *             they meet may become infinite or NaN though the state itself is not.
 *   states    (batch, heads, dk, dv) float
 * dk, dv in [1, 128]; heads a multiple of groups; seqlen at most 2^22 and batch * heads * ceil(seqlen / 64)
 * at most 2^20.
 * Arithmetic: products accumulate in 32 bits and the state is held in 32 bits.  All results have 32-bit accuracy, with
 * bf16 inputs too, and out, dq, dk and dv are rounded to a bf16 output once (a decay's gradient has the accuracy of the
 * sums of out . dout and v . dv that it is left of, over up to 64 tokens, or 256 in fp32).  The same call gives the same bits, and out the
 * same with a final state and without.
 * An infinity or NaN at token t reaches no other sequence and no other head (of q or k: no other group), and in
 * the forward no earlier token.  In the backward it may reach all gradients of its sequence and head (group).
 */
#ifndef PACKMAMBA_DELTA_H
#define PACKMAMBA_DELTA_H

#include "packmamba.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Largest dk and dv. */
#define PACKMAMBA_DELTA_MAX_HEAD 128

/* Bytes of workspace packmamba_delta_rule_fwd needs; 0 where the shape is invalid. */
size_t packmamba_delta_rule_fwd_workspace_size(int64_t batch, int64_t heads, int64_t groups, int64_t dk, int64_t dv,
                                               int64_t seqlen);

/*
 * Forward.  initial_state: NULL (zeros) or the state before each row, used where the row continues
 * a sequence (position_indices[b,0] != 0).  final_state: NULL, or receives the state after each row;
 * it may be initial_state's buffer.
 */
int packmamba_delta_rule_fwd(const void* q, const void* k, const void* v, const float* beta, const float* decay,
                             const int32_t* position_indices, const float* initial_state, float scale, void* out,
                             float* final_state, void* workspace, size_t workspace_bytes, int64_t batch, int64_t heads,
                             int64_t groups, int64_t dk, int64_t dv, int64_t seqlen, int32_t decay_per_token,
                             int32_t dtype, void* stream);

/* Bytes of workspace packmamba_delta_rule_bwd needs with inputs of the dtype. */
size_t packmamba_delta_rule_bwd_workspace_size(int64_t batch, int64_t heads, int64_t groups, int64_t dk, int64_t dv,
                                               int64_t seqlen, int32_t dtype);

/*
 * Backward: gradients of sum(dout * out) + sum(dfinal_state * final_state), from the inputs alone.
 *   dq, dk (batch, groups, dk, seqlen) and dv (batch, heads, dv, seqlen) in the dtype's output type; dq
 *   and dk are summed over the heads of a group in 32 bits, in an order that the call's sizes fix.
 *   dbeta (batch, heads, seqlen) float.
 *   ddecay: NULL, or decay's shape, float; 0 at a start (a cut multiplier is a constant).  It must
 *   be NULL where decay is.  dinitial_state: NULL iff initial_state is; it may be dfinal_state's
 *   buffer.  dfinal_state: NULL means 0.
 */
int packmamba_delta_rule_bwd(const void* q, const void* k, const void* v, const float* beta, const float* decay,
                             const int32_t* position_indices, const float* initial_state, float scale, const void* dout,
                             const float* dfinal_state, void* dq, void* dk, void* dv, float* dbeta, float* ddecay,
                             float* dinitial_state, void* workspace, size_t workspace_bytes, int64_t batch,
                             int64_t heads, int64_t groups, int64_t dk_size, int64_t dv_size, int64_t seqlen,
                             int32_t decay_per_token, int32_t dtype, void* stream);

/*
 * One token of each of `batch` sequences: q, k (batch, groups, dk), v, out (batch, heads, dv), beta (batch, heads),
 * decay (batch, heads) if decay_per_token, else (heads), or NULL; state (batch, heads, dk, dv) is read and
 * updated in place.  position_indices: NULL (every sequence goes on), or (batch): 0 starts a
 * sequence, whatever its state holds; a negative index marks an idle row, whose state is left as it is
 * and whose out is 0.  Arithmetic is in 32 bits throughout; out is rounded once.
 */
int packmamba_delta_rule_step(const void* q, const void* k, const void* v, const float* beta, const float* decay,
                              const int32_t* position_indices, float* state, float scale, void* out, int64_t batch,
                              int64_t heads, int64_t groups, int64_t dk, int64_t dv, int32_t decay_per_token,
                              int32_t dtype, void* stream);

/*
 * Each head's features divided by their length: the features of (batch, dim, seqlen) form `groups` groups of dim /
 * groups consecutive ones, and at every token out = x rnorm, rnorm = 1 / sqrt(sum over the group of x^2 + eps).
 *   x, out in dtype; rnorm (batch, groups, seqlen) float, written for the backward.
 *   dim a multiple of groups, at most 2^26 - 32; eps >= 0; batch * groups at most 2^20, batch * groups *
 *   ceil(seqlen / 16) below 2^22 and batch * dim * seqlen at most 2^33.
 */
int packmamba_head_l2norm_fwd(const void* x, float eps, void* out, float* rnorm, int64_t batch, int64_t dim,
                              int64_t seqlen, int64_t groups, int32_t dtype, void* stream);

/* Its backward: dx (the dtype's output type) from x, dout (dtype) and the forward's rnorm. */
int packmamba_head_l2norm_bwd(const void* x, const float* rnorm, const void* dout, void* dx, int64_t batch, int64_t dim,
                              int64_t seqlen, int64_t groups, int32_t dtype, void* stream);

/*
 * Layer norm over the features of (batch, dim, seqlen) activations, at every token:
 *   out = (x - mean) rstd weight + bias,   rstd = 1 / sqrt(mean of (x - mean)^2 + eps)
 *   x, out in dtype; weight, bias (dim) float, bias NULL for none; mean, rstd (batch, seqlen) float,
 *   written for the backward.  Limits as of packmamba_head_l2norm_fwd with one group.
 */
int packmamba_layernorm_fwd(const void* x, const float* weight, const float* bias, float eps, void* out, float* mean,
                            float* rstd, int64_t batch, int64_t dim, int64_t seqlen, int32_t dtype, void* stream);

/* Bytes of workspace packmamba_layernorm_bwd needs with inputs of the dtype. */
size_t packmamba_layernorm_bwd_workspace_size(int64_t batch, int64_t dim, int64_t seqlen, int32_t dtype);

/*
 * Its backward: dx (the dtype's output type), dweight (dim) and dbias (dim, or NULL), float, from x, dout (dtype)
 * and the forward's mean and rstd.  dresidual, if not NULL (dtype), is added to dx.  The sums over tokens are in a fixed
 * order.
 */
int packmamba_layernorm_bwd(const void* x, const float* weight, const float* mean, const float* rstd, const void* dout,
                            const void* dresidual, void* dx, float* dweight, float* dbias, void* workspace,
                            size_t workspace_bytes, int64_t batch, int64_t dim, int64_t seqlen, int32_t dtype,
                            void* stream);

#ifdef __cplusplus
}
#endif
#endif /* PACKMAMBA_DELTA_H */
