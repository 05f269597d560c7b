/*
 * ttc_block.h -- C ABI of the operators that stand around the Test-Time Control layer in a block of a language model,
 * NVIDIA B200 (sm_100a) only; part of the same library as ttc_lqr.h, with its status codes and error texts
 * (ttc_lqr_status_string, ttc_lqr_last_error).
 *
 *   ttc_linear                  y = act(x W' + b) + r: the projections that give the layer its initial state and its
 *                               coefficient vectors (ttc_layer_inputs), and take its output back to the residual stream
 *   ttc_causal_conv             short depthwise causal convolution of token rows
 *   ttc_selective_scan          state space recurrence with a diagonal, token-dependent transition: the memory layer that a
 *                               hybrid model runs beside the control layer
 *   ttc_decay_attention         linear attention with a decay for each head: the same with a matrix for a state, in chunks
 *   ttc_block_norm              the norms behind and in front of a block, with its gate, residual scale and residual
 * each with its gradients (.._grad) and, for decoding, a form for single tokens (.._step; ttc_linear and ttc_block_norm take few rows themselves).
 *
 * TOKEN ROWS.  A ttc_rows names a matrix of token rows: channel c of token t of sequence b is element
 * b * bstride + t * tstride + c, so that slices of wider rows (a projection that gives several operands at once) are
 * passed as they are.  Strides count elements and are >= 0; a null ptr is a missing operand.  Sequences come in one of two forms:
 *   equal:   seq_offsets NULL, `batch` sequences of `tokens` tokens;
 *   packed:  seq_offsets [batch + 1] (device, int32, not decreasing): sequence b is rows seq_offsets[b] up to
 *            seq_offsets[b + 1] of ONE matrix of `tokens` rows (bstride is ignored).  Sequences may be empty.  Rows outside
 *            every sequence are neither used nor written.  Offsets are clamped to [0, tokens] on the device, so wrong
 *            ones give wrong results but no access out of range.
 * Element types: TTC_F32, TTC_BF16, TTC_F16; all row operands of a call have the same one (ttc_linear, ttc_decay_attention: see there).
 * Arithmetic, sums and states are float32.  Parameter vectors (A, D, bias, convolution taps) and their gradients are float32.
 *
 * CALLS.  Every pointer is device memory of `device` and owned by the caller, aligned to its element.  A call is
 * asynchronous on cuda_stream, allocates nothing and keeps no state between calls; the calling thread's current device
 * is put back.  What scratch it needs the caller hands over, aligned to 256 bytes: ttc_.._workspace returns the bytes for the
 * same arguments (0: none is needed; pointers are not followed), or a negative status; its contents are undefined before and after.  Two
 * calls that may run at the same time need a workspace each, and a captured call keeps using the one it was captured with.
 * Gradients are sums in a fixed order: the same call gives the same bits.  They overwrite their outputs; every output of a
 * gradient call may be missing.  Outputs must overlap neither inputs, unless it is said, nor one another; they may lie in the same
 * storage, in other columns, tokens or sequences.
 */
#ifndef TTC_BLOCK_H_
#define TTC_BLOCK_H_

#include "ttc_lqr.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TTC_F16  2          /* element type of row operands, beside TTC_F32 and TTC_BF16 */

/* activations */
#define TTC_ACT_NONE      0
#define TTC_ACT_RELU      1
#define TTC_ACT_SILU      2   /* z / (1 + exp(-z))                    */
#define TTC_ACT_GELU      3   /* z Phi(z), the error-function form    */
#define TTC_ACT_SOFTPLUS  4   /* log(1 + exp(z))                      */

typedef struct ttc_rows {
    void*   ptr;
    int64_t bstride;
    int64_t tstride;
} ttc_rows;

/*
 * Depthwise causal convolution with `taps` (2 .. 4) taps:
 *     z_t = bias + sum_j w[:, j] * x_{t - (taps - 1) + j},    y_t = act(z_t)      (act: TTC_ACT_NONE or TTC_ACT_SILU)
 * Inputs in front of a sequence come from state [batch][taps - 1][d] (rows' type, oldest first; NULL: zeros), and
 * state_out receives the last taps - 1 inputs of every sequence (those of `state` where it is shorter), for the next call.
 * state_out may be state itself.  w is [d][taps], bias [d] (NULL: none).
 */
typedef struct ttc_conv_args {
    int64_t batch, tokens;
    const int32_t* seq_offsets;
    int32_t d, taps, act, dtype;
    ttc_rows x, y;
    const float *w, *bias;
    const void* state;
    void* state_out;
} ttc_conv_args;

int ttc_causal_conv(int32_t device, const ttc_conv_args* a, void* cuda_stream);

/*
 * One token of each of `batch` sequences (tokens and seq_offsets are ignored; row b of x and y is element b * bstride):
 * y as above, and the window in `state_out` moves on by one token in place.  state is not used.
 */
int ttc_causal_conv_step(int32_t device, const ttc_conv_args* a, void* cuda_stream);

/*
 * Gradients of ttc_causal_conv given dy and, optionally, the gradient dstate_out of the last windows (NULL: zero).
 * `a` as in the forward call (y and state_out are ignored).  dw [d][taps], dbias [d]; dstate [batch][taps - 1][d] in the rows' type.
 */
typedef struct ttc_conv_grads {
    ttc_rows dy, dx;
    const void* dstate_out;
    float *dw, *dbias;
    void* dstate;
} ttc_conv_grads;

int64_t ttc_causal_conv_grad_workspace(int32_t device, const ttc_conv_args* a, const ttc_conv_grads* g);
int ttc_causal_conv_grad(int32_t device, const ttc_conv_args* a, const ttc_conv_grads* g, void* workspace,
                         int64_t workspace_bytes, void* cuda_stream);

/*
 * Selective state space scan.  Per channel c of d, with n states (1 .. 128) and the group g(c) = c / (d / groups):
 *     D_t = delta_t + delta_bias;  with softplus: D_t = log(1 + exp(delta_t + delta_bias))
 *     h_t = exp(D_t A) h_{t-1} + D_t x_t B_t[g]            (element by element over the n states)
 *     y_t = (C_t[g] . h_t + D x_t) silu(z_t)
 * A [d][n], D [d] (NULL: 0), delta_bias [d] (NULL: 0); z missing: no gate.  B and C rows hold groups * n elements.
 * state [batch][d][n] float32 is h in front of every sequence (NULL: zero), state_out receives the last one; it may be
 * state itself.  y may be x or z (the same pointer and strides).  Exponents D_t A are expected to be <= 0.
 */
typedef struct ttc_scan_args {
    int64_t batch, tokens;
    const int32_t* seq_offsets;
    int32_t d, n, groups, dtype, softplus, reserved;
    ttc_rows x, delta, B, C, z, y;
    const float *A, *D, *delta_bias;
    const float* state;
    float* state_out;
} ttc_scan_args;

int64_t ttc_selective_scan_workspace(int32_t device, const ttc_scan_args* a);
int ttc_selective_scan(int32_t device, const ttc_scan_args* a, void* workspace, int64_t workspace_bytes, void* cuda_stream);

/* One token of each of `batch` sequences (as ttc_causal_conv_step): h in `state_out` is moved on in place, `state` is not used. */
int ttc_selective_scan_step(int32_t device, const ttc_scan_args* a, void* cuda_stream);

/*
 * Gradients of ttc_selective_scan given dy and, optionally, the gradient dstate_out of the last states (NULL: zero).  `a` as in
 * the forward call (y and state_out are ignored).  With the co-states q_t = C_t dy_t silu(z_t) + exp(D_{t+1} A) q_{t+1}:
 *     dC_t = sum_c h_t dy_t silu(z_t)    dB_t = sum_c q_t D_t x_t    dx_t = D_t (q_t . B_t) + D dy_t silu(z_t)
 *     dA = sum_t D_t q_t exp(D_t A) h_{t-1}          dD_t = x_t (q_t . B_t) + A . (q_t exp(D_t A) h_{t-1})
 * (sums over the channels of a group), ddelta from dD_t through the softplus, dz, and the sums dD, ddelta_bias over all tokens.
 * dA [d][n], dD, ddelta_bias [d], dstate [batch][d][n] float32; the row gradients in the rows' type.  Scratch: two floats for each state of
 * every 16 tokens, and with dB or dC two for each state (n rounded up to a power of two, 8 at least) of each token and block of
 * channels; a block holds 1024 over that n of them: 8192 tokens of 4096 channels take 0.38 GB with 16 states, 0.88 with 32, 2.3 with 64 and 6.7 with 128.
 */
typedef struct ttc_scan_grads {
    ttc_rows dy, dx, ddelta, dB, dC, dz;
    const float* dstate_out;
    float *dA, *dD, *ddelta_bias, *dstate;
} ttc_scan_grads;

int64_t ttc_selective_scan_grad_workspace(int32_t device, const ttc_scan_args* a, const ttc_scan_grads* g);
int ttc_selective_scan_grad(int32_t device, const ttc_scan_args* a, const ttc_scan_grads* g, void* workspace,
                            int64_t workspace_bytes, void* cuda_stream);

/*
 * Linear attention with a decay for each head.  Per head h of `heads`, with the group g(h) = h / (heads / groups) of its queries and keys:
 *     D_t = delta_t + delta_bias;  with softplus: D_t = log(1 + exp(delta_t + delta_bias));  delta missing: D_t = 1
 *     S_t = exp(A D_t) S_{t-1} + k_t[g] v_t'              [dk][dv]
 *     y_t = scale q_t[g] S_t
 * q and k rows hold groups * dk elements, v and y rows heads * dv, delta rows `heads`; dk, dv 1 .. 128.  Rows are bfloat16 or float16.
 * A [heads], delta_bias [heads] (NULL: 0; not used without delta).  state [batch][heads][dk][dv] float32 is S in front of every sequence
 * (NULL: zero), state_out receives the last one; it may be state itself.  y may be v (the same pointer and strides).
 * Exponents A D_t are expected to be <= 0; minus infinity forgets everything.  Tokens go through the tensor cores in chunks of 128, counted from their
 * sequence's begin: an infinity or NaN reaches the results of the whole chunk that it stands in, earlier tokens' too, and of those behind it.  Scratch: none where sequences, heads and columns fill the SMs; else sequences are walked along in pieces, with
 * 512 bytes for each value channel (dv rounded up to 64 or 128) of a piece and head, of which there are as many as SMs, and one more for each packed sequence.  Rows of q, k, v (and
 * dy of the gradients) that do not begin on 16 bytes, whose heads do not (dk, dv not a multiple of 8) or that are one row for many tokens are copied there too, 2 bytes for each channel.
 */
typedef struct ttc_decay_args {
    int64_t batch, tokens;
    const int32_t* seq_offsets;
    int32_t heads, groups, dk, dv, dtype, softplus;
    float scale;
    int32_t reserved;
    ttc_rows q, k, v, delta, y;
    const float *A, *delta_bias;
    const float* state;
    float* state_out;
} ttc_decay_args;

int64_t ttc_decay_attention_workspace(int32_t device, const ttc_decay_args* a);
int ttc_decay_attention(int32_t device, const ttc_decay_args* a, void* workspace, int64_t workspace_bytes, void* cuda_stream);

/* One token of each of `batch` sequences (as ttc_causal_conv_step): S in `state_out` is moved on in place, `state` is not used. */
int ttc_decay_attention_step(int32_t device, const ttc_decay_args* a, void* cuda_stream);

/*
 * Gradients of ttc_decay_attention given dy and, optionally, the gradient dstate_out of the last states (NULL: zero).  `a` as in
 * the forward call (y and state_out are ignored).  With Z_t = scale q_t dy_t' + exp(A D_{t+1}) Z_{t+1}:
 *     dq_t = scale S_t dy_t    dk_t = Z_t v_t    dv_t = Z_t' k_t    (dq, dk summed over the heads of a group)
 *     dD_t = A exp(A D_t) <Z_t, S_{t-1}>         dA = sum_t D_t exp(A D_t) <Z_t, S_{t-1}>
 * ddelta from dD_t through the softplus, ddelta_bias its sum over all tokens; dA, ddelta_bias [heads], dstate [batch][heads][dk][dv] float32; the row
 * gradients in the rows' type.  Scratch: for each element of a state (dk, dv rounded up to 64 or 128) of every chunk of 128 tokens 8 bytes, or 12 of bfloat16 rows where ddelta, dA
 * or ddelta_bias are wanted; with these 20 bytes for every token and head; where heads share queries and keys, 8 dk for every token and head; and twice the forward call's.
 */
typedef struct ttc_decay_grads {
    ttc_rows dy, dq, dk, dv, ddelta;
    const float* dstate_out;
    float *dA, *ddelta_bias, *dstate;
} ttc_decay_grads;

int64_t ttc_decay_attention_grad_workspace(int32_t device, const ttc_decay_args* a, const ttc_decay_grads* g);
int ttc_decay_attention_grad(int32_t device, const ttc_decay_args* a, const ttc_decay_grads* g, void* workspace,
                             int64_t workspace_bytes, void* cuda_stream);

/*
 * Projection of `rows` token rows:  z = x W' + bias,  y = act(z) + r.
 * x [rows][k] and W [m][k] are bfloat16 or float16 (`dtype`), row strides ldx, ldw; bias [m] float32 (NULL: none); residual r
 * [rows][m] (NULL: none) and y have the type `out_dtype`: dtype, or TTC_F32; pre (NULL: not wanted) receives z in `dtype`, which
 * the gradients want.  Products are accumulated in float32, by the tensor cores, which cut sums off where they would have to be rounded:
 * 1e-9 of the result for every contraction index, which float32 results of more than 1024 indices are spared by sums in segments.
 * y may be r (the same pointer and stride).
 */
typedef struct ttc_linear_args {
    int64_t rows;
    int32_t k, m, dtype, out_dtype, act, reserved;
    const void *x, *w;
    const float* bias;
    const void* residual;
    void *y, *pre;
    int64_t ldx, ldw, ldr, ldy, ldp;
} ttc_linear_args;

int64_t ttc_linear_workspace(int32_t device, const ttc_linear_args* a);
int ttc_linear(int32_t device, const ttc_linear_args* a, void* workspace, int64_t workspace_bytes, void* cuda_stream);

/*
 * Gradients of ttc_linear given dy [rows][m] (type `out_dtype`, row stride lddy; the gradient of the residual is dy itself):
 *     dZ = dy act'(pre);   dx = dZ W [rows][k],   dw = dZ' x [m][k],   dbias = sum over the rows of dZ [m] (float32).
 * pre is what the forward call wrote (needed unless act is TTC_ACT_NONE).  dZ is rounded to `dtype` for the products
 * (their operands; a relative 2^-9 for bfloat16, as the rounding of dx and dw themselves), not for dbias.  dx and dw are of
 * type `dtype`, with row strides lddx, lddw.
 */
typedef struct ttc_linear_grads {
    const void* dy;
    void *dx, *dw;
    float* dbias;
    int64_t lddy, lddx, lddw;
} ttc_linear_grads;

int64_t ttc_linear_grad_workspace(int32_t device, const ttc_linear_args* a, const ttc_linear_grads* g);
int ttc_linear_grad(int32_t device, const ttc_linear_args* a, const ttc_linear_grads* g, void* workspace,
                    int64_t workspace_bytes, void* cuda_stream);

/*
 * Norms behind and in front of a block, with its gate, residual scale and residual:
 *     u = x rms_g(x) w_post      (w_post [d]; NULL: u = x)             rms_g(v) = 1 / sqrt(mean of v^2 over the channels of a group + eps)
 *     u = u silu(z)              (z missing: no gate)
 *     h = residual + scale u     (scale [d], NULL: 1; residual missing: 0)
 *     y = h rms(h) w_pre         (w_pre [d]; the mean over all channels)
 * Rows [rows][d] of one type (1 .. 16384 channels), each with its row stride; w_post, scale, w_pre float32.  `groups` equal groups of neighbouring
 * channels (a head's, say) for w_post.  y is given with w_pre and only then; h may be missing.  h and y may each be x, z or residual (the same pointer and stride).
 * y is taken from h before that is rounded.
 */
typedef struct ttc_norm_args {
    int64_t rows;
    int32_t d, groups, dtype;
    float eps;
    const void *x, *z, *residual;
    void *h, *y;
    int64_t ldx, ldz, ldr, ldh, ldy;
    const float *w_post, *scale, *w_pre;
} ttc_norm_args;

int ttc_block_norm(int32_t device, const ttc_norm_args* a, void* cuda_stream);

/*
 * Gradients of ttc_block_norm given dy (with w_pre) and dh (the gradient of h by what else reads it; NULL: zero).  `a` as in the forward call, but h is an input, as
 * the forward call wrote it (needed with w_pre; NULL where nothing changes x, no residual either: h is x then), and y is not used, nor what residual points to.  dresidual receives the whole gradient of h, and may be dh;
 * dx, dz in the rows' type, dw_post, dscale, dw_pre [d] float32.
 */
typedef struct ttc_norm_grads {
    const void *dy, *dh;
    void *dx, *dz, *dresidual;
    int64_t lddy, lddh, lddx, lddz, lddr;
    float *dw_post, *dscale, *dw_pre;
} ttc_norm_grads;

int64_t ttc_block_norm_grad_workspace(int32_t device, const ttc_norm_args* a, const ttc_norm_grads* g);
int ttc_block_norm_grad(int32_t device, const ttc_norm_args* a, const ttc_norm_grads* g, void* workspace,
                        int64_t workspace_bytes, void* cuda_stream);

/*
 * Every wait inside the kernels on the tensor cores is bounded.  *value receives 1 if one of them has given up on `device` since
 * the library was loaded (the results of that call are not valid), else 0.  Synchronous.
 */
int ttc_block_device_error(int32_t device, int32_t* value);

#ifdef __cplusplus
}
#endif
#endif /* TTC_BLOCK_H_ */
