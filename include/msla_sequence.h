/*
 * msla_sequence.h -- the library's operators over token sequences (same libmsla.so, same rules as msla.h).
 *
 *   msla_recurrence_*       the linear attention of Eq. (3) as a running state over a sequence: causal, with a forgetting
 *                           gate, forward (one scan over long sequences), backward, and one token a sequence
 *   msla_norm_*             root-mean-square norm with the addition of a residual, its gradient, and with rows of 8 bits out
 *   msla_quantize_rows      rows of 8 bits out of a map as it is (weights)
 *   msla_linear_quantized   the 1x1 projection of such rows
 *   msla_selective_scan_*   a scan whose states decay each at their own rate: forward, backward, and one token a sequence
 *   msla_causal_conv_*      the short causal convolution of each channel in front of it: forward, backward, and one token a sequence
 *   msla_layer_norm_*       layer norm with the addition of a residual, and its gradient
 *   msla_quantize_rows_integer, msla_linear_integer   rows in 8-bit integers and their projection
 *
 * General rules: those of msla.h.  Device pointers, 16-byte aligned unless a line below says otherwise; the caller owns every
 * buffer; nothing is allocated; work is enqueued on `stream` and the call returns; every argument is checked on the host before the
 * first launch, and a call that returns an error has enqueued nothing; outputs may not overlap inputs or the workspace unless a line
 * below says so; calls that overlap in time use workspaces of their own, and so do two captured graphs that may run at once.
 * What a workspace holds between calls means nothing.  Results do not depend on how work is spread over the GPU: the same call on
 * the same device gives the same bits.
 */
#ifndef MSLA_SEQUENCE_H_
#define MSLA_SEQUENCE_H_

#include <stddef.h>
#include <stdint.h>

#include "msla.h"

#ifdef __cplusplus
extern "C" {
#endif

/* [token, head, channel] in the storage type: channels next to each other, strides in elements (multiples of 16 bytes; not
 * negative; a token's below 16 MiB, a head's at most 512 MiB, else MSLA_ERR_UNSUPPORTED).  So heads may be part of a wider row: the
 * map that msla_linear projects with w_qkv's row order is q = {p, 3*Ct, 3*d}, k = {p + d, ...}, v = {p + 2*d, ...}.  An input's strides
 * may be 0 (one row for all tokens, or all heads); an output's rows must not overlap each other.
 * Where several query heads share a state and head_dim is 16 or 32, the forward and backward calls read n = 64 / head_dim states' rows (heads_kv
 * of them where those are fewer) of q and of out's gradient at one 32-bit offset: 63 token strides and (n - 1) * heads_q / heads_kv head strides and a
 * row make at most 2^32 - 16 bytes, else MSLA_ERR_UNSUPPORTED (token-major maps always do). */
typedef struct {
    void* data;                 /* read only where the operand is an input */
    int64_t token_stride;
    int64_t head_stride;
} msla_heads;

/* What the recurrence runs over.  Rows [0, tokens) of q, k, v, ... are the tokens of `sequences` sequences behind each other:
 * with offsets == NULL all of the same length (tokens a multiple of sequences), else sequence b is the rows
 * [offsets[b], offsets[b + 1]) -- a DEVICE array of sequences + 1 ints in [0, tokens] that does not fall; a sequence may be empty;
 * rows before offsets[0] and from offsets[sequences] on belong to none and are neither read nor written.  (The array is on the device,
 * so it is not checked: entries that fall or lie outside leave results undefined, but nothing outside of the buffers is touched.)
 * heads_q query heads share heads_kv states, heads_q / heads_kv (a whole number) neighbours each.
 * head_dim is 16, 32, 64 or 128, of keys and of values.  tokens below 2^31 - 64, sequences * heads_kv below 2^22, heads_q <= 32768. */
typedef struct {
    int sequences;
    int64_t tokens;
    const int32_t* offsets;
    int heads_q, heads_kv, head_dim;
    float scale;                /* of every product of a query and a key; finite */
    int rectify;                /* 1: q and k are taken as max(q, 0), max(k, 0), as in Eq. (2) (a NaN stays one); 0: as they are */
} msla_recurrence;

/* For every sequence, state head h and query head of it, with S_{-1} = initial_state (zero where that is NULL):
 *     S_i = exp(log_gate_i) S_{i-1} + k_i v_i^T        o_i = scale * q_i^T S_i
 * (the numerator of Eq. (3), over the tokens so far; without the division, whose gradient has no bound -- a norm over the head's
 * channels takes its place).
 *   q [tokens, heads_q, head_dim];  k, v [tokens, heads_kv, head_dim];  out like q
 *   log_gate [tokens, heads_kv] in the storage type (aligned to its element), rows gate_stride elements (below 16 MiB) apart, or NULL:
 *       nothing is forgotten.  At most 0 in earnest; -inf (and anything below -103) forgets all that was.
 *   initial_state, final_state [sequences, heads_kv, head_dim (of k), head_dim (of v)] fp32, either may be NULL; final_state may be
 *       initial_state itself.  A sequence without tokens hands its state on.
 * The state, the sums and the gates' running products are fp32 (or more), a state on the way with up to 2^16 times its value (in fp16 with
 * what takes v to fp16's range, as long as the state stays below 2^100 that way); an operand of a matrix instruction that is not an
 * input goes in as parts of the storage type, three in bf16 and two in fp16, which leave fp32's precision.  (fp16's range: a score is
 * held to 2^-39 of the largest that its head's q and k of a chunk of 64 tokens could make, an addend of the state to 2^-39 of the chunk's largest.)
 * The workspace hangs on the shape alone, offsets being NULL or not included.
 * A value that is not finite stays within its own sequence and head; there it reaches the tokens behind it and those of its own
 * chunk of 64 tokens before it. */
msla_status msla_recurrence_workspace_bytes(const msla_recurrence* shape, int backward, msla_dtype dt, size_t* bytes);
msla_status msla_recurrence_forward(const msla_recurrence* shape, msla_heads q, msla_heads k, msla_heads v,
                                    const void* log_gate, int64_t gate_stride, const float* initial_state,
                                    msla_heads out, float* final_state,
                                    void* workspace, size_t workspace_bytes, msla_dtype dt, void* stream);

/* The gradient of msla_recurrence_forward: from d_out (like out) and d_final_state (NULL: zero) to d_q, d_k, d_v (like q, k, v; sums
 * over the query heads of a state), d_log_gate [tokens, heads_kv] in the storage type (rows d_gate_stride apart; NULL: not wanted) and
 * d_initial_state (NULL: not wanted).  The rectifier's derivative is 0 at 0 and at a NaN.  Nothing of the forward call is needed but its inputs.
 * d_log_gate of a token is the sum of q . d_q - k . d_k from it to a later border of segments, and <d_state, state> there, in fp32 products: its error
 * goes by those terms' magnitudes, also where a gate that forgets everything makes the sum itself small.
 * d_initial_state may be neither d_final_state nor initial_state. */
msla_status msla_recurrence_backward(const msla_recurrence* shape, msla_heads q, msla_heads k, msla_heads v,
                                     const void* log_gate, int64_t gate_stride, const float* initial_state,
                                     msla_heads d_out, const float* d_final_state,
                                     msla_heads d_q, msla_heads d_k, msla_heads d_v,
                                     void* d_log_gate, int64_t d_gate_stride, float* d_initial_state,
                                     void* workspace, size_t workspace_bytes, msla_dtype dt, void* stream);

/* One token for each of shape->sequences sequences (shape->tokens equal to it, offsets NULL): what msla_recurrence_forward computes for
 * sequences of length one, without a workspace.  new_state may be state itself (in place); it may not overlap it otherwise. */
msla_status msla_recurrence_step(const msla_recurrence* shape, msla_heads q, msla_heads k, msla_heads v,
                                 const void* log_gate, int64_t gate_stride, const float* state,
                                 msla_heads out, float* new_state, msla_dtype dt, void* stream);

/* Root-mean-square norm of rows, with the residual's addition:
 *     r = x + residual        y = r / sqrt(mean(r^2) + eps) * weight
 *   x, residual, sum, y [rows, channels], contiguous, aligned to an element; weight [channels] in the storage type or NULL (ones);
 *   residual may be NULL (r = x); sum receives r (NULL: not wanted) and may be x or residual itself, y may be x itself where sum is not x.
 * r is fp32 on its way into y, and so are its squares (|r| below 1e18 in earnest; a row of zeros with eps = 0 is 0 / 0); sum is rounded.
 * channels <= 32768, rows below 2^31.
 * msla_norm_quantized writes y in 8 bits instead: y8 [rows, channels] in e4m3 (the finite form: largest value 448), scale [rows] fp32 with
 * y ~ y8 * scale, scale = max |y| of the row / 448 (a row of zeros: scale 0). */
msla_status msla_norm_forward(const void* x, const void* residual, const void* weight, void* y, void* sum,
                              int64_t rows, int channels, float eps, msla_dtype dt, void* stream);
msla_status msla_norm_quantized(const void* x, const void* residual, const void* weight, void* y8, float* scale, void* sum,
                                int64_t rows, int channels, float eps, msla_dtype dt, void* stream);

/* The gradient of the norm at r = `sum`: d_r (of x and of residual alike) = the norm's own + d_sum (what comes to r past the norm; NULL:
 * zero), and d_weight [channels] fp32 (NULL: not wanted), its sum over the rows in a fixed order.  d_r may be d_y or d_sum itself.
 * workspace: for d_weight alone. */
msla_status msla_norm_backward_workspace_bytes(int64_t rows, int channels, msla_dtype dt, size_t* bytes);
msla_status msla_norm_backward(const void* sum, const void* weight, const void* d_y, const void* d_sum, void* d_r, float* d_weight,
                               void* workspace, size_t workspace_bytes, int64_t rows, int channels, float eps, msla_dtype dt,
                               void* stream);

/* Rows of a map in 8 bits, as msla_norm_quantized writes them: x8 = x / scale, scale = max |x| / 448. */
msla_status msla_quantize_rows(const void* x, void* x8, float* scale, int64_t rows, int channels, msla_dtype dt, void* stream);

/* y[n, o] = x_scale[n] * w_scale[o] * sum_c x8[n, c] w8[o, c]   (msla_linear of rows that stand in 8 bits)
 *   x8 [rows, c_in], w8 [c_out, c_in] e4m3;  x_scale [rows], w_scale [c_out] fp32 (aligned to 4 bytes);  y [rows, c_out] in dt.
 * c_in, c_out multiples of 16 and at most 2^20, rows below 2^31.  Products are exact, sums fp32. */
msla_status msla_linear_quantized(const void* x8, const float* x_scale, const void* w8, const float* w_scale, void* y, int64_t rows, int c_in,
                                  int c_out, msla_dtype dt, void* stream);

/* ---- A selective state space layer: the scan, the convolution in front of it, layer norm, and the projection in 8-bit integers. ---- */

/* [token, channel] in the storage type: channels next to each other, rows token_stride elements apart (not negative), aligned to an element.  So
 * channels may be part of a wider row.  An input's stride may be 0 (one row for all tokens); an output's rows must not overlap each other. */
typedef struct {
    void* data;                 /* read only where the operand is an input */
    int64_t token_stride;
} msla_rows;

/* What the scan runs over: sequences, tokens and offsets as in msla_recurrence (tokens below 2^31 - 4096).  channels <= 2^20, in `groups` (a divisor) of
 * neighbours that share b and c; states of a channel: 8, 16, 32 or 64.
 * A launch has fewer than 2^23 workgroups, which takes what else there is of everything: (sequences + tokens / 64) * groups * (channels of a group / 32, rounded up), with
 * 8 states tokens / 32, below 2^23; sequences * (channels * states / 256, rounded up) below 2^23; in the gradient tokens * groups * states below 2^30; for single
 * tokens sequences * (channels / 64, rounded up) below 2^23 alone.  These are taken; what is beyond may be refused with MSLA_ERR_UNSUPPORTED. */
typedef struct {
    int sequences;
    int64_t tokens;
    const int32_t* offsets;
    int channels, groups, states;
    int softplus;               /* 1: a token's step is softplus(delta + delta_bias) = log(1 + exp(.)); 0: delta + delta_bias as it is */
} msla_selective_scan;

/* For every sequence, channel and state n of it, with t_i the step of token i and g the channel's group:
 *     h_i[n] = exp(t_i a[n]) h_{i-1}[n] + t_i x_i b_i[g, n]        y_i = sum_n c_i[g, n] h_i[n] + skip x_i        out_i = y_i silu(gate_i)
 *   x, delta, gate, out [tokens, channels], rows less than 16 MiB apart (else MSLA_ERR_UNSUPPORTED); gate.data may be NULL (out = y);  b, c [tokens, groups, states] (a row: groups * states next to each other)
 *   a [channels, states] fp32, negative in earnest (a decay exp(t a) below fp32's normal range is 0);  skip, delta_bias [channels] fp32 or NULL (0)
 *   initial_state, final_state [sequences, channels, states] fp32, either may be NULL; final_state may be initial_state itself.  A sequence without tokens
 *       hands its state on.
 * States, steps and sums are fp32; a, skip, delta_bias and states are aligned to 4 bytes.  The workspace hangs on the shape alone, offsets being NULL
 * or not included.  A value that is not finite stays within its sequence and channel (one in b or c: its group), and reaches no token before its own. */
msla_status msla_selective_scan_workspace_bytes(const msla_selective_scan* shape, int backward, msla_dtype dt, size_t* bytes);
msla_status msla_selective_scan_forward(const msla_selective_scan* shape, msla_rows x, msla_rows delta, const float* a, msla_rows b, msla_rows c,
                                        const float* skip, const float* delta_bias, msla_rows gate, const float* initial_state, msla_rows out,
                                        float* final_state, void* workspace, size_t workspace_bytes, msla_dtype dt, void* stream);

/* The gradient of msla_selective_scan_forward: from d_out (like out) and d_final_state (NULL: zero) to d_x, d_delta, d_gate (like x; d_gate where there is a
 * gate, and only there), d_b, d_c (like b; sums over a group's channels), and in fp32 d_a [channels, states], d_skip, d_delta_bias [channels] (sums over all
 * tokens; each may be NULL: not wanted) and d_initial_state (NULL: not wanted).  Sums over tokens and channels are taken in a fixed order.  Nothing of
 * the forward call is needed but its inputs.  d_initial_state may be neither d_final_state nor initial_state. */
msla_status msla_selective_scan_backward(const msla_selective_scan* shape, msla_rows x, msla_rows delta, const float* a, msla_rows b, msla_rows c,
                                         const float* skip, const float* delta_bias, msla_rows gate, const float* initial_state, msla_rows d_out,
                                         const float* d_final_state, msla_rows d_x, msla_rows d_delta, float* d_a, msla_rows d_b, msla_rows d_c,
                                         float* d_skip, float* d_delta_bias, msla_rows d_gate, float* d_initial_state, void* workspace,
                                         size_t workspace_bytes, msla_dtype dt, void* stream);

/* One token for each of shape->sequences sequences (shape->tokens equal to it, offsets NULL), without a workspace.  new_state may be state itself (in
 * place); it may not overlap it otherwise. */
msla_status msla_selective_scan_step(const msla_selective_scan* shape, msla_rows x, msla_rows delta, const float* a, msla_rows b, msla_rows c,
                                     const float* skip, const float* delta_bias, msla_rows gate, const float* state, msla_rows out, float* new_state,
                                     msla_dtype dt, void* stream);

/* What the convolution runs over: sequences, tokens and offsets as in msla_recurrence (tokens below 2^31 - 4096).  channels <= 2^20; width 2, 3 or 4.
 * (sequences + tokens / 32) * (bytes of a row / 1024 + 2) below 2^23 is taken; what is beyond may be refused with MSLA_ERR_UNSUPPORTED (a launch's workgroups). */
typedef struct {
    int sequences;
    int64_t tokens;
    const int32_t* offsets;
    int channels, width;
    int silu;                   /* 1: out = pre sigmoid(pre); 0: out = pre */
} msla_causal_conv;

/* For every sequence and channel: pre_i = bias + sum_k weight[k] x_{i - width + 1 + k}, k = 0 .. width - 1
 *   x, out [tokens, channels];  weight [channels, width], bias [channels] or NULL (0) in the storage type
 *   initial_state [sequences, width - 1, channels] in the storage type: the rows in front of each sequence's first, oldest first (NULL: zeros);
 *   final_state the same behind its last (NULL: not wanted; not initial_state itself).  A sequence without tokens hands its state on.
 * Sums are fp32; states, weight and bias are aligned to an element. */
msla_status msla_causal_conv_forward(const msla_causal_conv* shape, msla_rows x, const void* weight, const void* bias, const void* initial_state,
                                     msla_rows out, void* final_state, msla_dtype dt, void* stream);

/* Its gradient: from d_out and d_final_state (NULL: zero) to d_x, d_initial_state (in the storage type; NULL: not wanted), and d_weight [channels, width]
 * and d_bias [channels] fp32 (either NULL: not wanted), sums over all tokens in a fixed order; workspace: for these two alone.  d_initial_state may be neither
 * d_final_state nor initial_state. */
msla_status msla_causal_conv_backward_workspace_bytes(const msla_causal_conv* shape, msla_dtype dt, size_t* bytes);
msla_status msla_causal_conv_backward(const msla_causal_conv* shape, msla_rows x, const void* weight, const void* bias, const void* initial_state,
                                      msla_rows d_out, const void* d_final_state, msla_rows d_x, float* d_weight, float* d_bias,
                                      void* d_initial_state, void* workspace, size_t workspace_bytes, msla_dtype dt, void* stream);

/* One token for each of shape->sequences sequences (shape->tokens equal to it, offsets NULL).  new_state may be state itself (in place). */
msla_status msla_causal_conv_step(const msla_causal_conv* shape, msla_rows x, const void* weight, const void* bias, const void* state, msla_rows out,
                                  void* new_state, msla_dtype dt, void* stream);

/* Layer norm of rows, with the residual's addition:
 *     r = x + residual        y = (r - mean(r)) / sqrt(mean((r - mean(r))^2) + eps) * weight + bias
 * Operands, overlaps and limits as of msla_norm_forward; weight and bias [channels] in the storage type, either may be NULL (ones; zeros). */
msla_status msla_layer_norm_forward(const void* x, const void* residual, const void* weight, const void* bias, void* y, void* sum, int64_t rows,
                                    int channels, float eps, msla_dtype dt, void* stream);

/* Its gradient at r = `sum`, as msla_norm_backward's, with d_bias [channels] fp32 (NULL: not wanted).  workspace: for d_weight and d_bias alone. */
msla_status msla_layer_norm_backward_workspace_bytes(int64_t rows, int channels, msla_dtype dt, size_t* bytes);
msla_status msla_layer_norm_backward(const void* sum, const void* weight, const void* d_y, const void* d_sum, void* d_r, float* d_weight, float* d_bias,
                                     void* workspace, size_t workspace_bytes, int64_t rows, int channels, float eps, msla_dtype dt, void* stream);

/* Rows in 8-bit integers: scale [rows] fp32 = max |x| * (1 / 127 in fp32), x8 [rows, channels] = x / scale to the nearest whole number, ties to even
 * (product and quotient as IEEE rounds them; a row whose scale is 0 or not finite: zeros).  channels <= 32768, rows below 2^31; x is aligned to an element. */
msla_status msla_quantize_rows_integer(const void* x, void* x8, float* scale, int64_t rows, int channels, msla_dtype dt, void* stream);

/* y[n, o] = x_scale[n] * w_scale[o] * sum_c x8[n, c] w8[o, c]: msla_linear_quantized of 8-bit integers (-128 to 127).  Sums are exact.  c_in, c_out
 * multiples of 16, c_in below 131072, c_out at most 2^20, rows below 2^31. */
msla_status msla_linear_integer(const void* x8, const float* x_scale, const void* w8, const float* w_scale, void* y, int64_t rows, int c_in, int c_out,
                                msla_dtype dt, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MSLA_SEQUENCE_H_ */
