/*
 * lstm_approx_ops.h -- operators of a gated-linear-recurrence block on sm_103a
 * (GB300), in liblstm_approx.so beside the approximate LSTM.
 *
 * A recurrent language model whose gates do not see h_{t-1} is built of
 * blocks: norm -> projections -> recurrence -> projection.  Such a model is
 * trained on whole sequences (the recurrence is a scan over T) and serves
 * single tokens of many streams from a pool of states.  The operators:
 *
 *   lstm_approx_rms_norm           root-mean-square norm with the residual's
 *                                  addition; output in the input's type, or as
 *                                  8-bit floats with a scale per column group
 *   lstm_approx_rms_norm_backward  its gradients
 *   lstm_approx_gated_scan         the recurrence over a sequence
 *   lstm_approx_gated_scan_backward  its gradients
 *   lstm_approx_gated_step         one timestep of it on a pool of states
 *   lstm_approx_w4_quantize        a matrix to 4 bits per value
 *   lstm_approx_w4_matvec          matrix-vector products with such a matrix
 *
 * Conventions for every entry point, beside those of lstm_approx.h (an
 * lstm_approx_status is returned; nothing aborts, throws or prints; arguments
 * are checked before anything is launched; no CPU fallback):
 *   - every tensor is a caller-owned DEVICE pointer on the current device;
 *     the arrays of strides are HOST arrays, read before the call returns;
 *   - calls are asynchronous on cuda_stream (cudaStream_t, NULL = the legacy
 *     default stream), allocate nothing and may be captured into a graph; a
 *     kernel may be launched while the one ahead of it in the stream still
 *     runs, and waits for its end before it touches memory;
 *   - msg is an optional host buffer of msg_len bytes for an error text;
 *   - strides and pitches count elements unless stated; the last axis of every
 *     tensor is contiguous; strides are not negative;
 *   - the same call on the same inputs gives the same bits;
 *   - no output overlaps an input or another output unless stated;
 *   - sizes of zero are valid (nothing is read; sums over nothing are zero).
 * Errors: EINVAL (NULL, sizes, types, alignment), ECUDA (no sm_103a device, a
 * launch failed).
 */
#ifndef LSTM_APPROX_OPS_H
#define LSTM_APPROX_OPS_H

#include "lstm_approx.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of the operators' tensors: 32-bit, bfloat16 and 16-bit floats, and
 * 8-bit floats with 4 exponent and 3 mantissa bits (largest value 448, no
 * infinities).  Pointers are aligned to their type's size.  Sums, norms,
 * states and statistics are held in 32 bits whatever the type. */
enum lstm_approx_op_dtype {
  LSTM_APPROX_OP_FP32 = 0,
  LSTM_APPROX_OP_BF16 = 1,
  LSTM_APPROX_OP_FP16 = 2,
  LSTM_APPROX_OP_E4M3 = 3
};

/*
 * Root-mean-square norm of each row, after the residual's addition:
 *
 *     s = x + residual;  rstd = 1 / sqrt(mean(s^2) + eps);  y = s rstd weight
 *
 * s stays in 32 bits for the norm; sum_out receives it rounded to dtype.
 *
 *   dtype     FP32, BF16 or FP16: x, residual, sum_out, and out when group = 0
 *   group     0: out is dtype.  Otherwise out is E4M3, with one scale for each
 *             `group` columns of a row (the last group may be short): group is
 *             32, 64, 128, 256 or >= D (one scale per row).  scale = the
 *             group's largest |y| / 448 (1 for a group of zeros, at least
 *             2^-126), out = y / scale, the quotient to a few units in
 *             32 bits' last place, rounded to nearest even.  A group that
 *             holds an infinity or NaN gets a scale that is not finite, so that
 *             out * scale is NaN throughout it.
 *   x         [rows][D], row pitch x_pitch;  residual likewise, or NULL (s = x)
 *   weight    [D] fp32;  eps >= 0
 *   rows >= 0, 1 <= D <= 32768
 *   out       [rows][D] contiguous
 *   scales    [rows][ceil(D / group)] fp32 when group > 0, else NULL
 *   sum_out   [rows][D] contiguous, or NULL; may be x or residual itself where
 *             that is contiguous (the residual stream updated in place)
 *   sum_low   [rows][D] contiguous, or NULL; 16-bit types without 8-bit output
 *             only: what sum_out's rounding took off s, for the backward pass
 *             (without it dweight is off by that rounding)
 *   rstd      [rows] fp32, or NULL: kept for the backward pass
 */
int lstm_approx_rms_norm(int dtype, int group, const void *x, long long x_pitch, const void *residual,
                         long long residual_pitch, const float *weight, float eps, long long rows,
                         int D, void *out, float *scales, void *sum_out, short *sum_low, float *rstd,
                         void *cuda_stream, char *msg, int msg_len);

/*
 * Gradients of the norm with output in dtype:
 *
 *     ds = rstd (weight dy - s rstd^2 mean(weight dy s)) + dsum
 *     dweight = sum over rows of dy s rstd
 *
 *   dy        [rows][D], pitch dy_pitch: gradient of out
 *   s         [rows][D], pitch s_pitch: sum_out of the forward call (x itself
 *             where there was no residual);  rstd [rows] of that call
 *   s_low     [rows][D] contiguous: sum_low of that call, or NULL
 *   dsum      [rows][D], pitch dsum_pitch: gradient that reaches sum_out by
 *             another way (the residual stream), or NULL
 *   dx        [rows][D] contiguous: ds, the gradient of x and of residual
 *             alike; may be dy or dsum itself where that is contiguous
 *   dweight   [D] fp32, or NULL
 *   workspace at least lstm_approx_rms_norm_workspace_bytes(rows, D) bytes,
 *             16-byte aligned, not shared by calls in flight; NULL when
 *             dweight is NULL
 */
int lstm_approx_rms_norm_backward(int dtype, const void *dy, long long dy_pitch, const void *s,
                                  long long s_pitch, const short *s_low, const float *weight, const float *rstd,
                                  const void *dsum, long long dsum_pitch, long long rows, int D,
                                  void *dx, float *dweight, void *workspace, size_t workspace_bytes,
                                  void *cuda_stream, char *msg, int msg_len);
/* Workspace bytes of the call above; 0 for invalid sizes. */
size_t lstm_approx_rms_norm_workspace_bytes(long long rows, int D);

/*
 * The gated linear recurrence over a sequence, for every stream b and channel:
 *
 *     log a_t = -c softplus(decay) sigma(r_t)
 *     h_t = a_t h_{t-1} + sqrt(1 - a_t^2) sigma(i_t) x_t;   y_t = h_t
 *
 * (sigma: logistic function.)  h is held in 32 bits.
 *
 *   dtype     FP32, BF16 or FP16: x, r, i, y
 *   x, r, i, y  [T][B][D]; r and i are the gates before their sigmoids
 *   strides   HOST [8]: the t and b strides of x, r, i and y in this order
 *             (slices of one projection's output, or batch-major tensors, need
 *             no copy); NULL: all contiguous
 *   decay     [D] fp32;  c > 0 (8 is usual)
 *   h0        [B][D] fp32, or NULL (zeros)
 *   lengths   [B] int32, or NULL (all T): stream b has min(max(lengths[b], 0),
 *             T) timesteps.  Nothing from later ones enters any result, whatever
 *             they hold; their y is zero.
 *   reset     [T][B] bytes, contiguous, or NULL: where not zero, h_{t-1} counts as zero
 *             (the first token of a packed document), whatever it holds; the
 *             input is scaled by sqrt(1 - a_t^2) there as elsewhere
 *   h_last    [B][D] fp32: the state after the stream's last timestep (h0
 *             where it has none); may be h0 itself
 *   states    [ceil(T / LSTM_APPROX_SCAN_CHUNK)][B][D] fp32, or NULL: the state
 *             before every chunk's first timestep, kept for the backward pass
 *   workspace at least lstm_approx_gated_scan_workspace_bytes(T, B, D) bytes,
 *             16-byte aligned, not shared by calls in flight
 *
 * A sequence longer than a chunk is split over blocks that run at once and pass
 * its state on through the workspace (a cooperative launch: ECUDA where the
 * device cannot hold it).  Should a wait for another block's part run out (2 s;
 * on a device that works, none does), what depends on that part is NaN.
 */
#define LSTM_APPROX_SCAN_CHUNK 64
int lstm_approx_gated_scan(int dtype, const void *x, const void *r, const void *i, const float *decay,
                           float c, const float *h0, const int32_t *lengths,
                           const unsigned char *reset, int T, int B, int D, void *y,
                           const long long *strides, float *h_last, float *states, void *workspace,
                           size_t workspace_bytes, void *cuda_stream, char *msg, int msg_len);
/* Workspace bytes of the call above and of the next; 0 for invalid sizes. */
size_t lstm_approx_gated_scan_workspace_bytes(int T, int B, int D);

/*
 * Gradients of the recurrence.  With g_t the gradient of h_t (dy_t and what
 * comes back from t + 1):
 *
 *   dy        [T][B][D] dtype;  dh_last [B][D] fp32 or NULL (zeros)
 *   x, r, i, decay, c, lengths, reset: as in the forward call; states its output
 *   dx, dr, di  [T][B][D] dtype (zero past a stream's length)
 *   ddecay    [D] fp32: summed over t and b;  dh0 [B][D] fp32
 *   strides   HOST [14]: the t and b strides of dy, x, r, i, dx, dr and di in
 *             this order; NULL: all contiguous
 *   workspace at least lstm_approx_gated_scan_workspace_bytes(T, B, D) bytes,
 *             16-byte aligned, not shared by calls in flight
 *
 * Where sigma(r_t) is too small for a_t to differ from 1 (r_t below about
 * -80), the gradients are the limits: zero.
 */
int lstm_approx_gated_scan_backward(int dtype, const void *dy, const float *dh_last, const void *x,
                                    const void *r, const void *i, const float *decay, float c,
                                    const float *states, const int32_t *lengths,
                                    const unsigned char *reset, int T, int B, int D, void *dx,
                                    void *dr, void *di, const long long *strides, float *ddecay,
                                    float *dh0, void *workspace, size_t workspace_bytes,
                                    void *cuda_stream, char *msg, int msg_len);

/*
 * One timestep of the recurrence for B streams, states updated in place:
 *
 *   x, r, i   [B][D] dtype, row pitches x_pitch, r_pitch, i_pitch
 *   state     [n_slots][D] fp32, contiguous
 *   slots     [B] int32, or NULL (stream b owns row b; then B <= n_slots): the
 *             row of state that holds stream b.  A stream whose slot lies
 *             outside [0, n_slots) is idle: no state changes, its y is zero.
 *             Slots in range are distinct.
 *   reset     [B] bytes, or NULL: where not zero the state counts as zero
 *   y         [B][D] dtype, contiguous
 */
int lstm_approx_gated_step(int dtype, const void *x, long long x_pitch, const void *r,
                           long long r_pitch, const void *i, long long i_pitch, const float *decay,
                           float c, float *state, int n_slots, const int32_t *slots,
                           const unsigned char *reset, int B, int D, void *y, void *cuda_stream,
                           char *msg, int msg_len);

/*
 * 4-bit matrices.  W [N][K] has, in each row, one scale and one zero point
 * for each `group` columns (32, 64 or 128; the last group may be short):
 *
 *     W[n][k] = (q[n][k] - zero[n][k / group]) scale[n][k / group]
 *
 *   q      [N][q_pitch] bytes: column k in the low (k even) or high (k odd)
 *          half of byte k / 2; 16-byte aligned, q_pitch a multiple of 16 and at
 *          least ceil(K / 2).  What lies beyond column K is read, not used.
 *          1 <= K <= 32768.
 *   scale  [N][ceil(K / group)] scale_dtype (FP32, BF16 or FP16)
 *   zero   [N][ceil(K / group)] bytes, each 0..15 (only the low 4 bits are
 *          read), or NULL (8 throughout)
 *
 * lstm_approx_w4_quantize fills them from w [N][K] (dtype, pitch w_pitch).
 * Per group, over the values and zero: lo <= 0 <= hi; scale = (hi - lo) / 15
 * rounded to scale_dtype (1 where that is zero), zero = round(-lo / scale),
 * q = round(w / scale) + zero, each clamped to [0, 15], ties to even; values
 * are to be finite and inside scale_dtype's range.  Bytes of q beyond column
 * K are set to zero.
 */
int lstm_approx_w4_quantize(int dtype, const void *w, long long w_pitch, int N, int K, int group,
                            unsigned char *q, long long q_pitch, void *scale, int scale_dtype,
                            unsigned char *zero, void *cuda_stream, char *msg, int msg_len);

/*
 * y[m][n] = sum_k x[m][k] W[n][k] (+ bias[n]) for a few rows m (the streams
 * that are served together; up to 65535 are right).  W is read once for as many
 * rows as lie in a block's shared memory over all of K: 16-bit rows up to 32 at
 * K = 2048 and 12 at 8192, a 32-bit row counting as three; more rows read it
 * again.
 *
 *   x_dtype   FP32, BF16, FP16, or E4M3 with scales
 *   x         [M][K], row pitch x_pitch
 *   x_scale   E4M3: [M][ceil(K / x_group)] fp32, x_group 128 or >= K (the
 *             outputs of lstm_approx_rms_norm); else NULL (x_group is ignored)
 *   bias      [N] fp32, or NULL
 *   y         [M][N] y_dtype (FP32, BF16 or FP16), contiguous
 *   workspace at least lstm_approx_w4_workspace_bytes(x_dtype, M, K) bytes,
 *             16-byte aligned, not shared by calls in flight; NULL where that
 *             is 0
 * Products are exact; sums are held in 32 bits.
 */
int lstm_approx_w4_matvec(int x_dtype, const void *x, long long x_pitch, const float *x_scale,
                          int x_group, const unsigned char *q, long long q_pitch, const void *scale,
                          int scale_dtype, const unsigned char *zero, const float *bias, int M, int N,
                          int K, int group, void *y, int y_dtype, void *workspace,
                          size_t workspace_bytes, void *cuda_stream, char *msg, int msg_len);
/* Workspace bytes of the call above (0: none, or invalid sizes). */
size_t lstm_approx_w4_workspace_bytes(int x_dtype, int M, int K);

#ifdef __cplusplus
}
#endif
#endif /* LSTM_APPROX_OPS_H */
