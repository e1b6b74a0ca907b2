/*
 * wm_seq.h -- C ABI of the sequence operators: what a gated recurrent block over
 * recorded episodes, its training step and its single-token form need around the
 * matrix products.
 *
 *   wm_seq_embed, _backward        rows of a table by token, scaled; the table's gradient
 *   wm_seq_layer_norm, _backward   layer norm; input, weight and bias gradients
 *   wm_seq_gated_scan, _backward   a gated linear recurrence over time
 *   wm_seq_clip                    the global norm of many gradients, and clipping by it
 *
 * The LSTM of wm.h multiplies its state by W_h at every step, so its steps run one
 * after the other.  The recurrence here is linear in the state, with gates that depend
 * on the input alone: the steps of a sequence can be joined in any grouping, and a long
 * recording fills the GPU even when there is only one.
 *
 * Types: `dtype` is WM_FP32 or WM_BF16 and holds for the arrays declared `void *`;
 * arithmetic, states, statistics and sums are fp32 (or wider), rounded once when an
 * output is written.
 *
 * Sizes: D, H, T and the tokens of a gradient are at most 2^31 - 65536; what a declaration
 * gives as long long may be larger.
 *
 * Memory: every array is device or managed memory of the handle's device; host memory
 * is an argument error (nothing is staged).  Outputs must not overlap inputs or each
 * other except where a declaration says so.  Arrays of zero elements may be NULL.
 * Scratch is a workspace of the handle, grown when a call needs more than any before it
 * (that synchronises the device; under stream capture it is an error: make a call of
 * the same size first).  Graphs captured earlier stay valid when it grows.
 *
 * Streams: calls are asynchronous on cuda_stream (a cudaStream_t; NULL = the legacy
 * default stream).  Calls on one handle share the workspace: issue them on one stream,
 * or order them between streams.  Calls of several threads on one handle take turns; its
 * message and launch count are those of the last.
 *
 * Errors: argument errors are returned at once and leave outputs untouched.  What only
 * the device can see (a token outside the table, a length outside [0, T]) is recorded in
 * a status word that wm_seq_sync returns and clears; the kernels then go on as each
 * declaration says.  wm_seq_last_error gives the message of the last failing call.
 *
 * Results are deterministic: the same call on the same device gives the same bits.
 */
#ifndef WM_SEQ_H
#define WM_SEQ_H

#include <stddef.h>
#include <stdint.h>

#include "wm.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct wm_seq wm_seq;

/* A handle on the current CUDA device: workspace, status word, messages. */
wm_status wm_seq_create(wm_seq **out);

/* Synchronises the device and returns the first device-side error since the last call
 * (WM_ERR_INVALID_ARG: a token or length out of range; WM_ERR_TIMEOUT: a bounded wait
 * gave up), then clears it. */
wm_status wm_seq_sync(wm_seq *h);

/* Message of the last failing call on h (never NULL; "" if none). */
const char *wm_seq_last_error(const wm_seq *h);

/* Kernels that the last call launched (memory sets not counted). */
int wm_seq_last_launches(const wm_seq *h);

/* Failure injection for tests of the timeout path: every wait inside a kernel is bounded.
 * With polls > 0 the next call whose CTAs wait for one another (a scan of few channels and
 * many steps, or wm_seq_clip of up to 30 MB) makes its first CTA poll, at most that often,
 * for something that nothing sets; it records WM_ERR_TIMEOUT, as a real bounded wait does,
 * and goes on.  One shot.  After WM_ERR_TIMEOUT outputs are undefined until wm_seq_sync has
 * returned it. */
wm_status wm_seq_inject_wait_timeout(wm_seq *h, unsigned int polls);

/* Frees what the handle owns (after the device has finished); graphs that hold its calls
 * must not be launched any more.  NULL is a no-op. */
void wm_seq_destroy(wm_seq *h);

/* Embedding lookup: out[i, :] = scale * table[tokens[i], :].
 *   table  [V, D] dtype, dense;  tokens [n] int32;  out [n, D] dtype, dense
 * A negative token takes no row (as an action < 0 in wm_mdn_nll): its output row is 0.
 * A token >= V is recorded as WM_ERR_INVALID_ARG and treated the same. */
wm_status wm_seq_embed(wm_seq *h, int dtype, long long n, int V, int D, const void *table, const int32_t *tokens,
                       float scale, void *out, void *cuda_stream);

/* Its gradient: dtable[v, :] = scale * sum over i with tokens[i] = v of dout[i, :].
 *   tokens [n] int32;  dout [n, D] dtype, dense;  dtable [V, D] dtype, dense, overwritten
 * The tokens are sorted stably, so that the sums run in a fixed order; rows that no token took
 * are 0, whatever the scale.  Tokens outside [0, V) as above. */
wm_status wm_seq_embed_backward(wm_seq *h, int dtype, long long n, int V, int D, const int32_t *tokens, const void *dout,
                                float scale, void *dtable, void *cuda_stream);

/* Layer norm over the last axis: y = (x - mean) * rstd * weight + bias,
 * rstd = 1 / sqrt(mean((x - mean)^2) + eps).
 *   x [rows, D] dtype, row stride ldx elements;  y [rows, D] dtype, row stride ldy
 *   weight, bias [D] fp32, either may be NULL (1 and 0)
 *   mean, rstd [rows] fp32, optional (both or neither): what the backward takes
 * y may be x with the same stride (in place).  eps >= 0. */
wm_status wm_seq_layer_norm(wm_seq *h, int dtype, long long rows, int D, const void *x, long long ldx,
                            const float *weight, const float *bias, float eps, void *y, long long ldy, float *mean,
                            float *rstd, void *cuda_stream);

/* Its gradients: with xhat = (x - mean) rstd and g = dy * weight,
 *   dx = rstd (g - mean(g) - xhat mean(g xhat)),  dweight = sum over rows of dy xhat,
 *   dbias = sum over rows of dy.
 *   x, dy, dx [rows, D] dtype with row strides;  mean, rstd [rows] fp32 from the forward
 *   weight [D] fp32 or NULL (1);  dweight, dbias [D] fp32, optional
 * dx may be dy with the same stride (in place). */
wm_status wm_seq_layer_norm_backward(wm_seq *h, int dtype, long long rows, int D, const void *x, long long ldx,
                                     const float *weight, const float *mean, const float *rstd, const void *dy,
                                     long long lddy, void *dx, long long lddx, float *dweight, float *dbias,
                                     void *cuda_stream);

/* An array [T, N, H] of the call's dtype whose last axis is dense: element (t, n, j) is
 * data[t * stride_t + n * stride_n + j].  Column slices of a wider array and batch-major
 * arrays are such views.  Inputs may have any strides >= 0; an output's elements must be
 * apart: stride_t >= (N-1) stride_n + H or stride_n >= (T-1) stride_t + H, the smaller
 * of the two (of axes longer than 1) at least H. */
typedef struct {
    void *data;
    long long stride_t, stride_n;
} wm_seq_view;

/* Gated linear recurrence over time:
 *   keep_t = sigmoid(gate_t),  write_t = 1 - keep_t
 *   h_t = keep_t * h_{t-1} + write_t * x_t
 * for N sequences of H channels each, all independent.
 *   gate, x  [T, N, H] dtype: pre-activations of the gate, and values
 *   h0       [N, H] fp32 dense or NULL = zeros: the state entering the call
 *   reset    [T, N] uint8 dense or NULL: nonzero = step t starts a new episode, its
 *            h_{t-1} is 0 whatever came before (also when that holds inf or NaN)
 *   lengths  [N] int32 or NULL = T: steps t >= lengths[n] are padding: gate, x and reset
 *            are not read there, the outputs h are 0 and the state is carried on.  A
 *            length outside [0, T] is recorded as WM_ERR_INVALID_ARG and clamped.
 *   h        [T, N, H] dtype, out
 *   h_last   [N, H] fp32 dense, optional out: the state after the last step; may be h0
 * T = 1 is the single-token form.  A call of T steps and calls on its parts (each
 * entering with the h_last before it) agree to rounding. */
wm_status wm_seq_gated_scan(wm_seq *h, int dtype, long long T, int N, int H, const wm_seq_view *gate,
                            const wm_seq_view *x, const float *h0, const uint8_t *reset, const int32_t *lengths,
                            const wm_seq_view *out, float *h_last, void *cuda_stream);

/* Its gradients.  gate, x, h0, reset, lengths as in the forward call and
 *   h        [T, N, H] dtype: the forward's output (its rounding is taken as given)
 *   dh       [T, N, H] dtype: the gradient with respect to h, not read in padding
 *   dh_last  [N, H] fp32 dense or NULL: the gradient with respect to h_last
 *   dgate, dx [T, N, H] dtype, out (0 in padding)
 *   dh0      [N, H] fp32 dense, optional out; may be dh_last
 * with L_t = dh_t + keep_{t+1} L_{t+1} (no second term into a reset step; dh_last enters
 * after the last step): dx_t = L_t write_t, dgate_t = L_t (h_{t-1} - x_t) keep_t write_t,
 * dh0 = keep_0 L_0. */
wm_status wm_seq_gated_scan_backward(wm_seq *h, int dtype, long long T, int N, int H, const wm_seq_view *gate,
                                     const wm_seq_view *x, const float *h0, const uint8_t *reset,
                                     const int32_t *lengths, const wm_seq_view *h_seq, const wm_seq_view *dh,
                                     const float *dh_last, const wm_seq_view *dgate, const wm_seq_view *dx, float *dh0,
                                     void *cuda_stream);

/* One gradient of a clipping call: n values at src, written (scaled) to dst, which may
 * be src.  Gradients must not overlap one another. */
typedef struct {
    const void *src;
    void *dst;
    long long n;
    int dtype;
} wm_seq_grad;

/* Clipping by the global norm: norm = sqrt(sum of g^2 over all values of all gradients),
 * every gradient times min(1, max_norm / norm).
 *   grads [count] host array;  max_norm >= 0 (+inf: only the norm, and copies where dst
 *   is not src);  norm [1] fp32 device, out
 * Gradients that are within the bound are not changed (dst != src: copied).  A norm that
 * is inf or NaN leaves them unchanged too: the caller reads `norm` and skips the update.
 * Squares are summed in fp32 within 16 bytes of values, in a pair of fp32 (a sum and its
 * error) over a thread's and a warp's, in fp64 over all; values whose squares leave fp32's
 * range are squared in fp64: the norm of finite gradients is finite unless it passes fp32's
 * range itself.  A factor below fp32's normal range is applied as two.  Empty gradients are
 * allowed; count = 0 gives norm 0.
 * count <= 65536. */
wm_status wm_seq_clip(wm_seq *h, int count, const wm_seq_grad *grads, float max_norm, float *norm, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* WM_SEQ_H */
