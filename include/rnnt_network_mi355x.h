/*
 * rnnt_network_mi355x.h -- the operators between an encoder and the transducer
 * loss of rnnt_mi355x.h, for AMD Instinct MI355X (gfx950): label embedding and
 * gated recurrence (a prediction network over the units), dropout, and the
 * joint's hidden layer, which adds every frame to every unit's state and whose
 * projection to the vocabulary gives the logits that rnnt_loss takes.
 *
 * Conventions are those of rnnt_mi355x.h: device pointers unless a comment says
 * otherwise, work queued on `stream`, no synchronisation, no state kept between
 * calls, host-visible errors return a status and launch nothing.  In addition
 *   - tensors need the alignment of their elements only; accesses are as wide at
 *     any address, and fastest where rows and pointers are multiples of 16 bytes.
 *   - outputs share no memory with inputs or with one another, unless a call says so.
 *   - lengths are (B) int32; rows behind a length are never used (they may hold
 *     anything, NaN included) and are exactly 0 in every output.  A length
 *     outside its range, seen on the device, gives NaN in that utterance's
 *     outputs and zeros in its gradients; other utterances are unaffected.
 *   - arithmetic, sums and states are float32; an output of 16 bits is rounded
 *     once, to nearest even.
 *   - a workspace is device memory of at least the stated size, 256-byte
 *     aligned, not shared by calls that overlap in time, or NULL: the library
 *     then takes one with hipMallocAsync / hipFreeAsync on `stream`, or returns
 *     RNNT_ERR_WORKSPACE where `stream` is being captured (a captured call
 *     brings a workspace that lives as long as the graph).
 */
#ifndef RNNT_NETWORK_MI355X_H
#define RNNT_NETWORK_MI355X_H

#include "rnnt_mi355x.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------------------
 * Label embedding.
 *
 *   out[b, i, :] = scale * weight[token(b, i), :]
 * over labels (B, N) int32.  With start >= 0 every utterance is preceded by that
 * row (the prediction network's state before the first unit, usually the blank's):
 * the output has N + 1 rows, token(b, 0) = start, token(b, i) = labels[b, i-1],
 * valid for i <= lens[b]; with start = -1 it has N rows, token(b, i) =
 * labels[b, i], valid for i < lens[b].  lens NULL: every row is valid.
 * A valid label outside [0, V) gives a row of NaN and no gradient.
 *
 * The gradient sums the rows of every token in one order, so equal inputs give equal
 * bits (by position (b, i) in stretches of up to 32 rows, then the stretches' sums):
 *   dweight[v, :] = scale * sum over valid (b, i) with token(b, i) = v of dout[b, i, :].
 * Every element of dweight (V, D) is written.
 *
 * RNNT_ERR_BAD_SHAPE: B < 1, N < 0, V < 1, D < 1 or start outside [-1, V).
 * RNNT_ERR_UNSUPPORTED: more than 2^31 - 2^16 - 1 rows in the output, or D > 2^30; in the
 * gradient, (rows + 2 V) times the KB of a row, rounded up, of about 2^28 or more.  The
 * workspace's size is 0 for a shape that the gradient refuses.
 */
typedef struct {
  int32_t B, N, V, D;
  int32_t start; /* weight row put before every utterance, or -1 */
  rnnt_dtype_t dtype;
} rnnt_embedding_shape_t;

rnnt_status_t rnnt_label_embedding(const int32_t* labels, const int32_t* lens, rnnt_embedding_shape_t shape,
                                   const void* weight, float scale, void* out, hipStream_t stream);

size_t rnnt_label_embedding_grad_workspace_bytes(rnnt_embedding_shape_t shape);
rnnt_status_t rnnt_label_embedding_grad(const int32_t* labels, const int32_t* lens, rnnt_embedding_shape_t shape,
                                        const void* dout, float scale, void* dweight, void* workspace,
                                        size_t workspace_bytes, hipStream_t stream);

/* ---------------------------------------------------------------------------
 * Gated linear recurrence.
 *
 *   a_t = sigmoid(z_t),   h_t = a_t h_{t-1} + (1 - a_t) x_t,   t < lens[b],
 * channel by channel over x, z (B, L, D); h_{-1} = h0 (B, D) float32 or zero
 * (h0 NULL).  h_out (B, L, D), last_out (B, D) float32: the state after the last
 * valid step (h0 where lens[b] = 0).  One step of a streaming decoder is L = 1.
 * Roundings have the size of a h and of (1 - a) x, so what a shut gate lets in keeps
 * its digits whatever the state that it drops.  An infinite x or state makes the states
 * behind it infinite, or NaN where it meets the other infinity or a gate that is 0 in
 * float32 (|z| of 88 and more).
 *
 * x and z may be views with contiguous channels: *_stride_b and *_stride_t are
 * in elements (halves of one projection, for instance); outputs are dense.
 *
 * For a backward pass the forward one stores float32 states in states_out (NULL: none),
 * rnnt_recurrence_states_bytes(shape) bytes, 16-byte aligned: the state before
 * every RNNT_RECURRENCE_STATE_STEPS-th step, from which rnnt_recurrence_grad
 * forms the ones between again.  With dh (B, L, D) or NULL (zero) and dlast
 * (B, D) float32 or NULL (zero), the gradients of h_out and last_out,
 *   s_t = dh_t + a_{t+1} s_{t+1}  (+ dlast at the last valid step),
 *   dx_t = (1 - a_t) s_t,  dz_t = s_t (h_{t-1} - x_t) a_t (1 - a_t),  dh0 = a_0 s_0
 * (dlast where lens[b] = 0).  dx, dz (B, L, D); dh0 (B, D) float32 or NULL.
 *
 * Only long sequences that are few need a workspace (0 bytes: none).
 *
 * RNNT_ERR_BAD_SHAPE: B < 1, L < 0, D < 1, or a stride below 0.
 * RNNT_ERR_UNSUPPORTED: L > 2^30, D > 2^21, or B * ceil(D / 64) of 2^21 or more; h0 and
 * last_out, or dlast and dh0, that share memory (a streaming caller keeps two states in turn).
 */
#define RNNT_RECURRENCE_STATE_STEPS 8

typedef struct {
  int32_t B, L, D;
  rnnt_dtype_t dtype;
  int64_t x_stride_b, x_stride_t, z_stride_b, z_stride_t;
} rnnt_recurrence_shape_t;

size_t rnnt_recurrence_states_bytes(rnnt_recurrence_shape_t shape);
size_t rnnt_recurrence_workspace_bytes(rnnt_recurrence_shape_t shape);
rnnt_status_t rnnt_recurrence(const void* x, const void* z, rnnt_recurrence_shape_t shape, const int32_t* lens,
                              const float* h0, void* h_out, float* last_out, void* states_out, void* workspace,
                              size_t workspace_bytes, hipStream_t stream);
rnnt_status_t rnnt_recurrence_grad(const void* x, const void* z, rnnt_recurrence_shape_t shape, const int32_t* lens,
                                   const void* states, const void* dh, const float* dlast, void* dx, void* dz,
                                   float* dh0, void* workspace, size_t workspace_bytes, hipStream_t stream);

/* ---------------------------------------------------------------------------
 * Dropout from a counter-based generator; the mask is never stored.
 *
 * rng: two int64 on the device, {seed, offset}, read by the kernel, so that a
 * captured graph takes new numbers when the program changes them.  Element n of
 * the flat tensor takes 16 bits of block n / 8 of Philox4x32 with 7 rounds
 * (Salmon et al., "Parallel random numbers: as easy as 1, 2, 3", SC 2011):
 * counter {n/8 low, n/8 high, offset low, offset high}, key {seed low, seed high};
 * n % 8 picks a half of the four words, low halves first.  With
 * q = min(round(65536 p), 65535), the element is kept when its number is at least
 * q, and y = x * 65536 / (65536 - q); otherwise y is exactly 0.
 *
 * rng_out (two int64, or NULL) receives the numbers used.  The gradient is the
 * same call on dy with those numbers.  In place (y = x) is allowed.
 * RNNT_ERR_BAD_SHAPE: n < 0.  RNNT_ERR_BAD_VARIANT: p outside [0, 1).
 * RNNT_ERR_UNSUPPORTED: n of 2^34 - 2^12 or more.
 */
rnnt_status_t rnnt_dropout(const void* x, int64_t n, rnnt_dtype_t dtype, double p, const int64_t* rng,
                           int64_t* rng_out, void* y, hipStream_t stream);

/* ---------------------------------------------------------------------------
 * Hidden layer of the joint.
 *
 *   h[b, t, u, :] = drop(act(enc[b, t, :] + pred[b, u, :])),  t < logit_lens[b], u <= label_lens[b],
 * over enc (B, T_max, H) and pred (B, U_max+1, H); h (B, T_max, U_max+1, H).
 * drop is the dropout above on the flat index in h (p = 0: none, rng may be NULL).
 * One step of a streaming decoder is T_max = 1, U_max = 0.
 *
 * The gradient reads dh once and forms both sums,
 *   denc[b, t, :] = sum_u w dh,   dpred[b, u, :] = sum_t w dh,   w = drop' act'(enc + pred),
 * in a fixed order.
 *
 * logit_lens outside [0, T_max] or label_lens outside [0, U_max] is a bad length.
 * RNNT_ERR_BAD_SHAPE: B < 1, T_max < 1, U_max < 0, H outside [1, 2^20], 2^31 or more
 * rows (t, u) of an utterance, or more than 2^40 rows.  RNNT_ERR_BAD_VARIANT: unknown
 * activation, p outside [0, 1).
 * RNNT_ERR_UNSUPPORTED, forward: B * T_max or B * (U_max+1) of 2^31 or more,
 * B * ceil(T_max / 4) of 2^23 or more, or an utterance's pred of about 2^30 elements or
 * more.  Gradient: B * ceil(T_max / 16) (8 in float32) times ceil(H / 120) of 2^23 or
 * more, B * (U_max+1) * H of about 2^33 or more (2^31, H < 8), or an utterance's pred of
 * 2^29 elements or more; its workspace's size is 0 for such a shape.
 */
typedef enum { RNNT_ACT_RELU = 0, RNNT_ACT_TANH = 1 } rnnt_activation_t;

typedef struct {
  int32_t B, T_max, U_max, H;
  rnnt_dtype_t dtype;
} rnnt_joint_shape_t;

rnnt_status_t rnnt_joint_hidden(const void* enc, const void* pred, rnnt_joint_shape_t shape,
                                const int32_t* logit_lens, const int32_t* label_lens, rnnt_activation_t act, double p,
                                const int64_t* rng, int64_t* rng_out, void* h_out, hipStream_t stream);

size_t rnnt_joint_hidden_grad_workspace_bytes(rnnt_joint_shape_t shape);
rnnt_status_t rnnt_joint_hidden_grad(const void* enc, const void* pred, rnnt_joint_shape_t shape,
                                     const int32_t* logit_lens, const int32_t* label_lens, rnnt_activation_t act,
                                     double p, const int64_t* rng, const void* dh, void* denc, void* dpred,
                                     void* workspace, size_t workspace_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* RNNT_NETWORK_MI355X_H */
