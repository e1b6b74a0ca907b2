/*
 * wm_seq.h -- C ABI of the sequence operators: what a gated recurrent block over
 * recorded episodes, its training step and its single-token form need around the
 * matrix products.
 *
 *   wm_seq_embed, _backward        rows of a table by token, scaled; the table's gradient
 *   wm_seq_layer_norm, _backward   layer norm; input, weight and bias gradients
 *   wm_seq_gated_scan, _backward   a gated linear recurrence over time
 *   wm_seq_head_norm, _backward    the norm of queries' and keys' heads, and their rotation by position
 *   wm_seq_decay_attention, _backward  linear attention whose weights decay with the distance
 *   wm_seq_clip                    the global norm of many gradients, and clipping by it
 *
 * The LSTM of wm.h multiplies its state by W_h at every step, so its steps run one
 * after the other.  The recurrence here is linear in the state, with gates that depend
 * on the input alone: the steps of a sequence can be joined in any grouping, and a long
 * recording fills the GPU even when there is only one.
 *
 * Types: `dtype` is WM_FP32 or WM_BF16 and holds for the arrays declared `void *`;
 * arithmetic, states, statistics and sums are fp32 (or wider), rounded once when an
 * output is written.  The decayed attention rounds factors of the tensor cores to bf16
 * besides, as its declaration says.
 *
 * Sizes: D, H, T and the tokens of a gradient are at most 2^31 - 65536; what a declaration
 * gives as long long may be larger.
 *
 * Memory: every array is device or managed memory of the handle's device; host memory
 * is an argument error (nothing is staged).  Outputs must not overlap inputs or each
 * other except where a declaration says so (the head norm and the decayed attention refuse
 * an output that begins where another array of the call does).  Arrays of zero elements may be NULL.
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
 * With polls > 0 the next call whose CTAs or warps wait for one another (a scan of few channels
 * and many steps, wm_seq_clip of up to 30 MB, or a decayed attention on the tensor cores) makes its
 * first CTA poll, at most that often, for something that nothing sets; it records WM_ERR_TIMEOUT,
 * as a real bounded wait does, and goes on.  One shot.  After WM_ERR_TIMEOUT outputs are undefined until wm_seq_sync has
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

/* An array [T, N, heads, D] of the call's dtype whose last axis is dense: element (t, n, h, j) is
 * data[t * stride_t + n * stride_n + h * stride_h + j].  Inputs may have any strides >= 0 (0: an axis
 * that is broadcast; gradients come for each of its places, and their sum is the caller's); an
 * output's elements must be apart: of the axes longer than 1, in some order, each stride is at least
 * the extent of the axes inside it. */
typedef struct {
    void *data;
    long long stride_t, stride_n, stride_h;
} wm_seq_heads;

/* The norm of each head's vector and its rotation by position, of queries and keys in one pass:
 *   y = x / sqrt(mean(x^2) + eps) * weight over the D values of a head, then of the first `rotary`
 *   values the pairs (y_i, y_{i + rotary/2}), or with `interleaved` (y_{2i}, y_{2i+1}), turn by
 *   positions[t, n] * freqs[i]:  (a, b) -> (a cos - b sin, b cos + a sin).
 *   q [T, N, q_heads, D], k [T, N, k_heads, D] dtype (k_heads 0: no keys);  q_out, k_out alike; an
 *   output may be its input with the same strides (in place)
 *   q_weight, k_weight [D] fp32, either may be NULL (1)
 *   positions [T, N] int32 dense;  freqs [rotary / 2] fp32: radians a position
 * rotary is even, 0 <= rotary <= D <= 1024; with 0 positions and freqs are not read.  Positions may be
 * negative.  An angle is taken as a fraction of a turn in 64-bit integers, so that it is as good at far
 * positions as at near ones; its frequency is the fp32 value as it is.  eps >= 0.  Squares are summed in fp32: a row
 * whose sum of squares leaves fp32's range (values of 10^18 and more) gives zeros. */
wm_status wm_seq_head_norm(wm_seq *h, int dtype, long long T, int N, int D, int rotary, int interleaved, int q_heads,
                           const wm_seq_heads *q, const float *q_weight, int k_heads, const wm_seq_heads *k,
                           const float *k_weight, float eps, const int32_t *positions, const float *freqs,
                           const wm_seq_heads *q_out, const wm_seq_heads *k_out, void *cuda_stream);

/* Its gradients.  q, k, weights, eps, positions and freqs as in the forward call (the norms are taken again
 * from q and k) and
 *   dq_out, dk_out  the gradients with respect to q_out and k_out
 *   dq, dk  out; each may be its dq_out or dk_out with the same strides (in place)
 *   dq_weight, dk_weight [D] fp32, optional out
 * with g = weight * (dy turned back), r = 1 / sqrt(mean(x^2) + eps), xhat = x r:
 *   dx = r (g - xhat mean(g xhat)),  dweight = sum over all heads of (dy turned back) xhat. */
wm_status wm_seq_head_norm_backward(wm_seq *h, int dtype, long long T, int N, int D, int rotary, int interleaved,
                                    int q_heads, const wm_seq_heads *q, const float *q_weight, const wm_seq_heads *dq_out,
                                    int k_heads, const wm_seq_heads *k, const float *k_weight, const wm_seq_heads *dk_out,
                                    float eps, const int32_t *positions, const float *freqs, const wm_seq_heads *dq,
                                    const wm_seq_heads *dk, float *dq_weight, float *dk_weight, void *cuda_stream);

/* Linear attention whose weights decay with the distance, for N sequences of `heads` heads, all independent:
 *   S_t = lambda S_{t-1} + k_t v_t^T,  o_t = scale * S_t^T q_t,  lambda = exp(log_decay[head])
 * that is o_t = scale * sum over s <= t of lambda^(t-s) (q_t . k_s) v_s.
 *   q, k     [T, N, heads, Dk] dtype;  v [T, N, heads, Dv] dtype;  1 <= Dk, Dv <= 256
 *   log_decay [heads] fp32, <= 0 (-inf: only the token itself; 0: no decay).  A constant of the model:
 *            it has no gradient here
 *   s0       [N, heads, Dk, Dv] fp32 dense or NULL = zeros: the state entering the call
 *   reset    [T, N] uint8 dense or NULL: nonzero = step t starts a new episode, nothing before it is seen
 *            (also when that holds inf or NaN)
 *   lengths  [N] int32 or NULL = T: steps t >= lengths[n] are padding: whatever their inputs and reset hold, their
 *            outputs are 0 and the state is carried on.  A length outside [0, T] is recorded as
 *            WM_ERR_INVALID_ARG and clamped.
 *   out      [T, N, heads, Dv] dtype, out
 *   s_last   [N, heads, Dk, Dv] fp32 dense, optional out: the state after the last step; may be s0
 * What is not finite reaches the outputs that see it, and no others (a sequence that holds such values is taken again
 * in fp32, which takes longer): with a finite log_decay every later token sees it, however far, with -inf none does.
 * A log_decay of NaN makes NaN of what it weighs.  T = 1 is the single-token form.  A call of T steps and calls on its parts (each
 * entering with the s_last before it) agree to rounding.
 * In bf16 the products of queries and keys, and the state as the queries read it, are rounded to bf16 as factors of
 * the tensor cores (heads of up to 128 values and more than 12 tokens); sums stay fp32, and s_last is as good as in fp32.
 * Wider heads take the fp32 kernel, at its speed; rows that are not whole 16 bytes, or not aligned to them, are read value
 * by value. */
wm_status wm_seq_decay_attention(wm_seq *h, int dtype, long long T, int N, int heads, int Dk, int Dv, const wm_seq_heads *q,
                                 const wm_seq_heads *k, const wm_seq_heads *v, const float *log_decay, float scale,
                                 const float *s0, const uint8_t *reset, const int32_t *lengths, const wm_seq_heads *out,
                                 float *s_last, void *cuda_stream);

/* Its gradients.  q, k, v, log_decay, scale, s0, reset, lengths as in the forward call and
 *   dout     [T, N, heads, Dv] dtype: the gradient with respect to out; padding may hold anything
 *   ds_last  [N, heads, Dk, Dv] fp32 dense or NULL: the gradient with respect to s_last
 *   dq, dk, dv  like q, k, v, out (0 in padding)
 *   ds0      [N, heads, Dk, Dv] fp32 dense, optional out; may be ds_last
 * with G_t = scale q_t dout_t^T + lambda G_{t+1} (no second term into a reset step; ds_last enters after the last
 * step): dq_t = scale * S_t dout_t, dk_t = G_t v_t, dv_t = G_t^T k_t, ds0 = lambda G_0. */
wm_status wm_seq_decay_attention_backward(wm_seq *h, int dtype, long long T, int N, int heads, int Dk, int Dv,
                                          const wm_seq_heads *q, const wm_seq_heads *k, const wm_seq_heads *v,
                                          const float *log_decay, float scale, const float *s0, const uint8_t *reset,
                                          const int32_t *lengths, const wm_seq_heads *dout, const float *ds_last,
                                          const wm_seq_heads *dq, const wm_seq_heads *dk, const wm_seq_heads *dv,
                                          float *ds0, void *cuda_stream);

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
