/*
 * packmamba_linear.h -- C ABI of the packed linear attention with a decay for each head, in
 * chunks for training and prompts and token by token for generation, and of the gated RMSNorm
 * that follows it in a block, on AMD Instinct MI355X (gfx950).
 *
 * The conventions of packmamba.h hold: device pointers owned by the caller, 16-byte aligned,
 * contiguous, the sequence innermost; dtype codes PACKMAMBA_F32, PACKMAMBA_BF16 and
 * PACKMAMBA_BF16_F32OUT; status codes; nothing is allocated or synchronised; argument errors are
 * returned before anything is enqueued.  Outputs overlap neither inputs nor each other, except
 * where it is said.
 *
 * The recurrence, for every batch row b and head h, at token t:
 *   a_t = exp(decay_t), and 0 where position_indices[b,t] == 0 (a sequence starts)
 *   S_t = a_t S_{t-1} + k_t v_t^T        (dk x dv; S = initial_state before the row, or zeros)
 *   out_t = scale S_t^T q_t
 * q and k belong to groups of heads: head h reads group h / (heads / groups).
 *   q, k      (batch, groups, dk, seqlen)  dtype
 *   v, out    (batch, heads, dv, seqlen)   dtype
 *   decay     log decays, float: (batch, heads, seqlen) if decay_per_token, else (heads); NULL: 0.
 *             A value of -104 or less (exp of it is 0 in 32 bits; -infinity too) cuts as a start
 *             does.  Values above 0 make the state grow and are taken as they are.
 *   states    (batch, heads, dk, dv) float
 * dk, dv in [1, 128]; heads a multiple of groups; seqlen at most 2^22, batch * heads at most 2^21, and
 * batch * heads * max(dk, dv) * seqlen at most 2^33.
 * Arithmetic: products accumulate in 32 bits and the state is held in 32 bits.  With bf16 inputs the
 * products inside a chunk of 64 tokens (q . k, weighted) and the copy of the state that q is
 * multiplied with are rounded to bf16 once, also where PACKMAMBA_BF16_F32OUT returns 32 bits: out
 * has bf16's accuracy in both.  Final states, the initial state's gradient and the decays' gradient
 * have 32-bit accuracy for all types.  The same call gives the same bits; with another choice of the
 * optional outputs (final states, ddecay) other kernels may run, and bf16 results may differ within
 * their accuracy.
 * An infinity or NaN at token t reaches no other sequence, and in its own only what the sums hold it in:
 *   q: out at t; dk, dv up to t          k: out, dq from t on; dv at t     v: out, dq from t on; dk at t
 *   dout: dq at t; dk, dv up to t        decay of t: out, dq from t on; dk, dv before t
 * and ddecay of the sequence's tokens (of the head, where it has one decay).
 */
#ifndef PACKMAMBA_LINEAR_H
#define PACKMAMBA_LINEAR_H

#include "packmamba.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Largest dk and dv. */
#define PACKMAMBA_LINEAR_MAX_HEAD 128

/* Bytes of workspace packmamba_linear_attention_fwd needs: nonzero only where few rows and heads
 * are cut into segments walked by separate blocks; 0 also where the shape is invalid. */
size_t packmamba_linear_attention_fwd_workspace_size(int64_t batch, int64_t heads, int64_t groups, int64_t dk,
                                                     int64_t dv, int64_t seqlen);

/*
 * Forward.  initial_state: NULL (zeros) or the state before each row, used where the row continues
 * a sequence (position_indices[b,0] != 0).  final_state: NULL, or receives the state after each row;
 * it may be initial_state's buffer.  workspace may be NULL where its size is 0.
 */
int packmamba_linear_attention_fwd(const void* q, const void* k, const void* v, const float* decay,
                                   const int32_t* position_indices, const float* initial_state, float scale,
                                   void* out, float* final_state, void* workspace, size_t workspace_bytes,
                                   int64_t batch, int64_t heads, int64_t groups, int64_t dk, int64_t dv,
                                   int64_t seqlen, int32_t decay_per_token, int32_t dtype, void* stream);

/* Bytes of workspace packmamba_linear_attention_bwd needs. */
size_t packmamba_linear_attention_bwd_workspace_size(int64_t batch, int64_t heads, int64_t groups, int64_t dk,
                                                     int64_t dv, int64_t seqlen);

/*
 * Backward: gradients of sum(dout * out) + sum(dfinal_state * final_state).
 *   dq, dk (batch, groups, dk, seqlen) and dv (batch, heads, dv, seqlen) in the dtype's output type; dq
 *   and dk are summed over the heads of a group in 32 bits, in the heads' order.
 *   ddecay: NULL, or decay's shape, float; 0 at a start (a cut multiplier is a constant).  It must
 *   be NULL where decay is.  dinitial_state: NULL iff initial_state is; it may be dfinal_state's
 *   buffer.  dfinal_state: NULL means 0.
 */
int packmamba_linear_attention_bwd(const void* q, const void* k, const void* v, const float* decay,
                                   const int32_t* position_indices, const float* initial_state, float scale,
                                   const void* dout, const float* dfinal_state, void* dq, void* dk, void* dv,
                                   float* ddecay, float* dinitial_state, void* workspace, size_t workspace_bytes,
                                   int64_t batch, int64_t heads, int64_t groups, int64_t dk_size, int64_t dv_size,
                                   int64_t seqlen, int32_t decay_per_token, int32_t dtype, void* stream);

/*
 * One token of each of `batch` sequences: q, k (batch, groups, dk), v, out (batch, heads, dv), decay
 * (batch, heads) if decay_per_token, else (heads), or NULL; state (batch, heads, dk, dv) is read and
 * updated in place.  position_indices: NULL (every sequence goes on), or (batch): 0 starts a
 * sequence, whatever its state holds; a negative index marks an idle row, whose state is left as it is
 * and whose out is 0.  Arithmetic is in 32 bits throughout; out is rounded once.
 */
int packmamba_linear_attention_step(const void* q, const void* k, const void* v, const float* decay,
                                    const int32_t* position_indices, float* state, float scale, void* out,
                                    int64_t batch, int64_t heads, int64_t groups, int64_t dk, int64_t dv,
                                    int32_t decay_per_token, int32_t dtype, void* stream);

/*
 * Gated RMSNorm of (batch, dim, seqlen) activations: the features form `groups` groups of dim / groups
 * consecutive ones, each normed by itself at every token.  With gate = z sigmoid(z):
 *   gate_first:  a = x gate,  out = a rstd weight          rstd = 1 / sqrt(mean over the group of a^2 + eps)
 *   otherwise:   a = x,       out = a rstd weight gate
 *   x, z, out in dtype; weight (dim) float; rstd (batch, groups, seqlen) float, written for the backward.
 *   dim a multiple of groups, at most 2^27 - 32; eps >= 0; batch * groups at most 2^20, batch * groups *
 *   ceil(seqlen / 32) below 2^22 and batch * dim * seqlen at most 2^33.
 */
int packmamba_gated_rmsnorm_fwd(const void* x, const void* z, const float* weight, float eps, void* out, float* rstd,
                                int64_t batch, int64_t dim, int64_t seqlen, int64_t groups, int32_t gate_first,
                                int32_t dtype, void* stream);

/* Bytes of workspace packmamba_gated_rmsnorm_bwd needs. */
size_t packmamba_gated_rmsnorm_bwd_workspace_size(int64_t batch, int64_t dim, int64_t seqlen, int64_t groups);

/*
 * Its backward: dx and dz (the dtype's output type) and dweight (dim, float), from x, z, dout (dtype) and
 * the forward's rstd.  dweight's sum is in a fixed order.
 */
int packmamba_gated_rmsnorm_bwd(const void* x, const void* z, const float* weight, const float* rstd,
                                const void* dout, void* dx, void* dz, float* dweight, void* workspace,
                                size_t workspace_bytes, int64_t batch, int64_t dim, int64_t seqlen, int64_t groups,
                                int32_t gate_first, int32_t dtype, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* PACKMAMBA_LINEAR_H */
