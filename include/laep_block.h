/*
 * laep_block.h -- what a pre-norm MoE block computes around the layer of
 * laep_moe.h in training and serving: layer norm, the router's balance loss,
 * and the expert FFN's pre-activations kept in 8 bits for the backward pass.
 *
 * The conventions of laep_moe.h hold: device pointers owned by the caller,
 * work enqueued on `stream` only, arguments checked on the host before any
 * HIP call, deterministic results, error codes and laep_last_error().
 * Activation buffers, logits and weights must be 16-byte aligned.
 */
#ifndef LAEP_BLOCK_H
#define LAEP_BLOCK_H

#include "laep_moe.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * moe_layer_norm -- the block's input rows: residual add and layer norm.
 *
 *   s    = residual ? round(x + residual) : x          (stored in sum_out)
 *   mu   = mean over c of s,  rstd = 1 / sqrt(mean over c of (s - mu)^2 + eps)
 *   y    = round((s - mu) * rstd * gamma + beta)
 *   Statistics and sums are float32; the norm is that of the rounded s, which
 *   the backward pass reads.
 *
 *   x, residual (or NULL), y  device [T, d_model] dtype
 *   gamma, beta (or NULL)     device [d_model] float32
 *   sum_out   device [T, d_model] dtype or NULL; needs a residual; may be x or
 *             residual (the residual stream updated in place)
 *   mean, rstd  device [T] float32 or NULL (the backward pass needs both)
 *   d_model % 8 == 0 and at most 2^28, T >= 0.  y must not overlap the inputs or sum_out.
 */
int moe_layer_norm(const void* x, const void* residual, const float* gamma,
                   const float* beta, int dtype, int T, int d_model, float eps,
                   void* sum_out, void* y, float* mean, float* rstd,
                   void* stream);

/*
 * moe_layer_norm_bwd -- backward of moe_layer_norm.  With
 * xh = (s - mean) * rstd and g = gamma * dy:
 *
 *   dx[t]  = round(rstd (g - mean_c(g) - xh mean_c(g xh)) + dres[t])
 *   dgamma = sum_t dy xh,   dbeta = sum_t dy      (float32, overwritten)
 *   dx is the gradient of s, hence of x and of the residual alike; dres (or
 *   NULL) is what reaches s past the norm (the residual path).
 *
 *   dy, s, dres, dx  device [T, d_model] dtype; s is moe_layer_norm's sum_out
 *   (x without a residual); mean, rstd as it wrote them; dx may be dy or dres.
 *   dgamma, dbeta    device [d_model] float32; either dbeta or both may be NULL.
 *   Workspace: moe_workspace_bytes(LAEP_CALL_LAYER_NORM_BWD, T, 1, 1, d_model, 0)
 *   (none without dgamma).  T = 0 zero-fills dgamma and dbeta.
 */
int moe_layer_norm_bwd(const void* dy, const void* s, const float* gamma,
                       const float* mean, const float* rstd, const void* dres,
                       int dtype, int T, int d_model, void* dx, float* dgamma,
                       float* dbeta, void* ws, size_t ws_bytes, void* stream);

/* Sequences of one balance loss. */
#define LAEP_MAX_SEQUENCES 1048576

/*
 * moe_balance_loss -- balance loss of one layer's router, over the batch or
 * per sequence, with the expert counts it uses.
 *
 *   p[t, e] = softmax over the alive experts of logits[t, :], 0 for dead ones
 *             (a token whose alive logits are all -inf has p = 0)
 *   sequence s holds the tokens [seq_offsets[s], seq_offsets[s + 1]), n_s of them
 *   counts[s, e]    = #{(t, j) : t in s, topk_idx[t, j] == e}
 *   prob_mean[s, e] = (1 / n_s) sum over t in s of p[t, e]
 *   f[s, e]         = N_alive * counts[s, e] / (k * n_s)
 *   loss            = coef * mean over the non-empty s of
 *                     sum_e f[s, e] * prob_mean[s, e]
 *   grad_coef[s, e] = coef * f[s, e] / (n_s * number of non-empty s)
 *   Evenly loaded experts give loss = coef.  Empty sequences get zeros.  The
 *   counts are piecewise constant, so grad_coef is dloss / dp[t, e], t in s.
 *
 *   logits    device [T, E] float32 (moe_route's); topk_idx device [T, k] int32
 *             (ids outside [0, E), such as -1, are not counted)
 *   alive     device [E] uint8 or NULL (all alive)
 *   seq_offsets device [n_seq + 1] int32, non-decreasing, in [0, T]; NULL with
 *             n_seq = 1: all T tokens.  Tokens of no sequence do not count.
 *   loss device [1] float32; counts device [n_seq, E] int32; prob_mean and
 *   grad_coef device [n_seq, E] float32.
 *   Workspace: moe_workspace_bytes(LAEP_CALL_BALANCE, T, n_seq, E, 0, 0).
 */
int moe_balance_loss(const float* logits, const int32_t* topk_idx,
                     const uint8_t* alive, const int32_t* seq_offsets, int T,
                     int E, int k, int n_seq, float coef, float* loss,
                     int32_t* counts, float* prob_mean, float* grad_coef,
                     void* ws, size_t ws_bytes, void* stream);

/*
 * moe_balance_loss_bwd -- gradient of the balance loss with respect to the
 * logits, the counts held fixed:
 *
 *   dlogits[t, e] (+)= dloss * p_e (c_e - sum_i p_i c_i),  c = grad_coef[s, :]
 *   of the token's sequence s; dead experts and tokens of no sequence get 0.
 *
 *   dloss device [1] float32 or NULL (1); dlogits device [T, E] float32,
 *   overwritten or (accumulate = 1) added to; it may be logits' buffer when not
 *   accumulating, and any other overlap with it is refused.  The other
 *   arguments as in moe_balance_loss.
 */
int moe_balance_loss_bwd(const float* logits, const float* grad_coef,
                         const uint8_t* alive, const int32_t* seq_offsets,
                         const float* dloss, int T, int E, int n_seq,
                         float* dlogits, int accumulate, void* stream);

/*
 * moe_route_bwd_balance -- moe_route_bwd of a router trained with a balance
 * loss: the loss's gradient is added to the gates' before the products.
 *
 *   dl[t, e] = moe_route_bwd's dl[t, e]
 *              + dloss * p_e (c_e - sum_i p_i c_i),  c = grad_coef[s, :]
 *   dlogits, dw_router, dbias, dx from that dl, as moe_route_bwd forms them.
 *   Every alive expert carries a gradient, so the products are dense for
 *   renormalised gates too, and offsets and row_src are not needed.
 *
 *   logits device [T, E] float32 (moe_route's output, both kinds of gates),
 *   which dlogits must not overlap;
 *   grad_coef, seq_offsets, n_seq, dloss as in moe_balance_loss_bwd; the other
 *   arguments, the workspace and T = 0 as in moe_route_bwd.
 */
int moe_route_bwd_balance(const float* dgate, const int32_t* topk_idx,
                          const float* topk_gate, const float* logits,
                          const uint8_t* alive, const void* x,
                          const void* w_router, const float* grad_coef,
                          const int32_t* seq_offsets, int n_seq,
                          const float* dloss, int dtype, int T, int d_model,
                          int E, int k, int renorm, float* dlogits,
                          float* dw_router, float* dbias, void* dx,
                          int accumulate_dx, void* ws, size_t ws_bytes,
                          void* stream);

/* Columns that share one scale of an 8-bit activation checkpoint. */
#define LAEP_ACT8_BLOCK 32

/*
 * moe_act8_save -- an activation matrix in 8 bits: every 32 consecutive
 * columns of a row share a power-of-two scale.
 *
 *   b = max(biased exponent of the block's largest magnitude - 6, 1)
 *   scale[r, c / 32] = b;  q[r, c] = clamp(round(act 2^(127 - b)), -127, 127)
 *   (ties to even); the value it stands for is q * 2^(b - 127).
 *   From 2^-120 up the largest magnitude takes 64 to 127 steps, so the error is
 *   at most half a step, 1/128 of it (float32 magnitudes that round past 127
 *   steps: under one step); below 2^-120 steps are 2^-126 and the error at most
 *   2^-127, however small the block.  Decoded values are exact in bf16.  A block
 *   that holds an infinity or a NaN gets b = 255 and decodes to NaNs.
 *
 *   act device [R, C] dtype; q device [R, C] int8; scale device [R, C / 32]
 *   uint8.  C % 32 == 0, 0 <= R < 2^31.
 */
int moe_act8_save(const void* act, int dtype, int64_t R, int C, int8_t* q,
                  uint8_t* scale, void* stream);

/*
 * moe_act8_load -- act[r, c] = q[r, c] * 2^(scale[r, c / 32] - 127), in dtype;
 * NaN where the scale is 255.  q and scale as moe_act8_save writes them
 * (scale 1 to 255).
 */
int moe_act8_load(const int8_t* q, const uint8_t* scale, int dtype, int64_t R,
                  int C, void* act, void* stream);

/*
 * moe_swiglu_bwd_act8 -- backward of the SwiGLU at pre-activations kept in 8
 * bits.  With (A_g, A_u) the decoded halves of a row and s = sigmoid(A_g):
 *
 *   da = round([dh * A_u * s * (1 + A_g (1 - s)),  dh * silu(A_g)])
 *   h  = round(silu(A_g) * A_u)      (the down projection's input, recomputed)
 *
 *   q device [R, 2*d_ff] int8, scale device [R, 2*d_ff / 32] uint8 (as
 *   moe_act8_save wrote them); dh device [R, d_ff] dtype; da device
 *   [R, 2*d_ff] dtype; h device [R, d_ff] dtype, may be dh.  d_ff % 32 == 0.
 */
int moe_swiglu_bwd_act8(const int8_t* q, const uint8_t* scale, const void* dh,
                        int dtype, int64_t R, int d_ff, void* da, void* h,
                        void* stream);

/*
 * moe_grouped_ffn_bwd_gather_act8 -- moe_grouped_ffn_bwd_gather at
 * pre-activations kept in 8 bits (moe_act8_save of act_save): the SwiGLU
 * backward decodes them, and dW_d takes the H recomputed there, so neither
 * act_save nor the forward's H is needed.  Results are bit-identical to
 * moe_grouped_ffn_bwd_gather with act_save = moe_act8_load(q, scale) and
 * h_fwd NULL.
 *
 *   act_q device [R, 2*d_ff] int8, act_scale device [R, 2*d_ff / 32] uint8;
 *   the other arguments and the workspace as in moe_grouped_ffn_bwd_gather.
 */
int moe_grouped_ffn_bwd_gather_act8(
    const void* dy_perm, const void* dout, const float* topk_gate,
    const void* x, const int32_t* row_src, int T, int k, const int8_t* act_q,
    const uint8_t* act_scale, const void* w_gate_up, const void* w_down,
    const int32_t* offsets, const int32_t* expert_map, int dtype, int E,
    int d_model, int d_ff, int64_t R, void* dx_perm, float* dw_gate_up,
    float* dw_down, int accumulate, void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LAEP_BLOCK_H */
