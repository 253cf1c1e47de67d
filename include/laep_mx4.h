/*
 * laep_mx4.h -- experts in microscaled 4 bits (MX4): quantisation, the grouped
 * product, and the SwiGLU expert FFN at 4-bit weights.
 *
 * The conventions of laep_moe.h hold: device pointers owned by the caller,
 * work enqueued on `stream` only, arguments checked on the host before any
 * HIP call, deterministic results, error codes and laep_last_error().
 * Every buffer must be 16-byte aligned (index arrays: 4).
 *
 * An MX4 matrix [R, C] (C % 32 == 0) is two arrays:
 *   codes  [R, C / 2] uint8: column c of a row in the low (c even) or high
 *          half of byte c / 2.  Bit 3 is the sign, bits 0..2 choose one of the
 *          steps 0, 1/2, 1, 3/2, 2, 3, 4, 6.
 *   scale  [ceil(C / 256), R, 8] uint8: the biased exponents b of the eight
 *          blocks of 32 columns in each 256; b = 0 for blocks past C.
 * The value is step * 2^(b - 127); every value of a block with b = 255 is NaN.
 * n matrices lie one after the other in both arrays.
 */
#ifndef LAEP_MX4_H
#define LAEP_MX4_H

#include "laep_moe.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Columns that share one scale, and columns whose scales lie together. */
#define LAEP_MX4_BLOCK 32
#define LAEP_MX4_GROUP 256

/*
 * moe_mx4_quantize -- n matrices [R, C] in MX4.
 *
 *   b = max(biased exponent of the block's largest magnitude - 2, 0)
 *   code = the step nearest to v 2^(127 - b) (ties to the even code; above 6,
 *   which b leaves room for up to 8, the step 6), with v's sign
 *   From 2^-125 up the largest magnitude takes the steps 4 and 6, and errors
 *   are at most 1 step unit (2^(b - 127)) up to 7 units, under 2 above.
 *   A block that holds an infinity or a NaN gets b = 255 and zero codes.
 *
 *   src device [n, R, C] dtype; codes device [n, R, C / 2] uint8; scale device
 *   [n, ceil(C / 256), R, 8] uint8, its blocks past C written as 0.
 *   C % 32 == 0, n >= 0, 0 <= R < 2^31.
 */
int moe_mx4_quantize(const void* src, int dtype, int n, int64_t R, int C,
                     uint8_t* codes, uint8_t* scale, void* stream);

/*
 * moe_mx4_dequantize -- the values codes and scales stand for, in dtype (exact
 * in bf16 and float32, but for scales that moe_mx4_quantize does not write: at
 * b = 253 the steps 4 and 6, at b = 254 those from 2 up are infinities); NaN where
 * the scale is 255.  Arrays as in moe_mx4_quantize.
 */
int moe_mx4_dequantize(const uint8_t* codes, const uint8_t* scale, int dtype,
                       int n, int64_t R, int C, void* out, void* stream);

/*
 * moe_mx4_grouped_product -- routed rows times their expert's MX4 matrix:
 *
 *   out[r, :] = round(X[src(r), :] W[slot(e), :, :]^T)
 *   for the rows r of expert e, offsets[e] <= r < offsets[e + 1]
 *   src(r) = row_src[r] / k, or r without row_src; sums are float32.
 *
 *   x        device [T, K]: MX4 codes with x_scale, or bf16 with x_scale NULL
 *   row_src  device [R] int32 (moe_expert_counts') or NULL (X's rows are
 *            already in the experts' order: T >= R, k unused)
 *   w, w_scale  device MX4 [slots, N, K]; beside bf16 activations their values are
 *            moe_mx4_dequantize's in bf16
 *   offsets  device [E + 1] int32; expert_map device [E] int32 or NULL (slot e);
 *            rows of experts with a negative slot, and rows outside every
 *            expert's range, are left as they were in out
 *   out      device [R, N] out_dtype
 *   K % 64 == 0, N % 64 == 0; x, one slot of w, and each scale array of x under
 *   2 GiB; out and ws must not overlap the inputs or each other (of w, a call with an
 *   expert_map checks the first slot only).
 *   Workspace: moe_workspace_bytes(LAEP_CALL_MX4_PRODUCT, T, k, E, K, N).
 */
int moe_mx4_grouped_product(const void* x, const uint8_t* x_scale,
                            const int32_t* row_src, int T, int k,
                            const uint8_t* w, const uint8_t* w_scale,
                            const int32_t* offsets, const int32_t* expert_map,
                            int out_dtype, int E, int N, int K, int64_t R,
                            void* out, void* ws, size_t ws_bytes, void* stream);

/*
 * moe_grouped_ffn_fwd_mx4 -- the grouped SwiGLU FFN at MX4 weights, dispatch
 * folded in (moe_grouped_ffn_fwd_gather's at 4-bit weights):
 *
 *   A = X[src(r), :] W_gu^T,  H = silu(A_gate) * A_up,  y_perm = round(H' W_d^T)
 *   act_bits 16: X and H' = round(H) are bf16;
 *   act_bits 4:  X and H' are moe_mx4_quantize's of x and of the float32 H.
 *
 *   x        device [T, d_model] bf16; row_src as in moe_mx4_grouped_product
 *   w_gate_up, w_down  device MX4 [slots, 2*d_ff, d_model], [slots, d_model, d_ff]
 *   y_perm   device [R, d_model] bf16
 *   act_save device [R, 2*d_ff] bf16 or NULL: the pre-activations A, as the
 *            backward calls take them (act_bits 16 only).  The gradients of
 *            quantisation-aware training are moe_grouped_ffn_bwd_gather's at
 *            this act_save and at the weights' values (moe_mx4_dequantize).
 *   d_model % 64 == 0, d_ff % 64 == 0; rows left as they were, and limits, as in
 *   moe_mx4_grouped_product.  y_perm, act_save and ws must not overlap the inputs or
 *   each other, likewise.
 *   Workspace: moe_workspace_bytes(LAEP_CALL_MX4_FFN, T, k, E, d_model, d_ff)
 *   (either act_bits; without row_src T and k as given).
 */
int moe_grouped_ffn_fwd_mx4(const void* x, const int32_t* row_src, int T, int k,
                            const uint8_t* w_gate_up,
                            const uint8_t* w_gate_up_scale,
                            const uint8_t* w_down, const uint8_t* w_down_scale,
                            const int32_t* offsets, const int32_t* expert_map,
                            int act_bits, int E, int d_model, int d_ff,
                            int64_t R, void* y_perm, void* act_save, void* ws,
                            size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* LAEP_MX4_H */
