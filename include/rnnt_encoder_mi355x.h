/*
 * rnnt_encoder_mi355x.h -- the operators of an encoder's layers that have no
 * library product, in training and in streaming service, for AMD Instinct MI355X
 * (gfx950): the root-mean-square norm, rotary positions, the product in 8-bit
 * integers, and the attention of a chunk of new tokens over a paged cache.  What
 * they bring are the states that the joint of rnnt_network_mi355x.h adds up, and
 * the product in 8 bits also the logits that rnnt_viterbi takes.
 *
 * Conventions are those of rnnt_network_mi355x.h: device pointers, work queued on
 * `stream`, no synchronisation, no state between calls; tensors need the alignment
 * of their elements only, unless a call says more; outputs share no memory with
 * inputs or with one another; lens is (B) int32 or NULL (every row is valid), rows
 * behind a length are never used and are exactly 0 in every output, and a length
 * outside its range gives NaN in that utterance's outputs and zeros in its gradients;
 * arithmetic and sums are float32, rounded once to nearest even, but for the attention's weights (below);
 * workspaces as there.
 */
#ifndef RNNT_ENCODER_MI355X_H
#define RNNT_ENCODER_MI355X_H

#include "rnnt_network_mi355x.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---------------------------------------------------------------------------
 * Root-mean-square norm, with the addition of a residual.
 *
 *   t = x + residual (x where residual is NULL),   y = t / sqrt(mean(t^2) + eps) * weight
 * over the rows of x (B, L, D); weight (D) of the same type.  sum_out receives t, rounded
 * (where residual is NULL it is not written, and may be NULL); y is formed from t before that
 * rounding.
 * Squares are summed in float32: a row whose squares pass its range (values of about 1e18)
 * gives 0 where the values are finite, as one that holds an infinity does; with eps 0 one whose
 * squares fall below it (values of about 1e-19) can give infinities, and one of zeros NaN.
 *
 * The gradient forms t again from x and residual, without the rounding of sum_out, and takes
 * the gradients dy and dsum (NULL: zero) of y and of sum_out:
 *   r = 1 / sqrt(mean(t^2) + eps),  g = dy * weight,
 *   dx = r (g - t r^2 mean(g t)) + dsum,   dweight = sum over valid rows of dy t r;
 * dx is the gradient of x and of residual alike.  dweight's sums have one order, so equal
 * inputs give equal bits.
 *
 * RNNT_ERR_BAD_SHAPE: B < 1, L < 0, D < 1.  RNNT_ERR_BAD_VARIANT: eps below 0 or not finite.
 * RNNT_ERR_UNSUPPORTED: D > 32768 (16384 in float32), or B * L of 2^31 / 128 or more.
 */
typedef struct {
  int32_t B, L, D;
  rnnt_dtype_t dtype;
} rnnt_norm_shape_t;

rnnt_status_t rnnt_rms_norm(const void* x, const void* residual, rnnt_norm_shape_t shape, const int32_t* lens,
                            const void* weight, float eps, void* y, void* sum_out, hipStream_t stream);

size_t rnnt_rms_norm_grad_workspace_bytes(rnnt_norm_shape_t shape);
rnnt_status_t rnnt_rms_norm_grad(const void* x, const void* residual, rnnt_norm_shape_t shape, const int32_t* lens,
                                 const void* weight, float eps, const void* dy, const void* dsum, void* dx,
                                 void* dweight, void* workspace, size_t workspace_bytes, hipStream_t stream);

/* ---------------------------------------------------------------------------
 * Rows in 8 bits: signed integers and one float32 scale a row,
 *   scale = max |v| / 127,   q = v / scale to the nearest integer, ties to even,
 * so |q| <= 127 and the value is q * scale.  A row of zeros, or one whose largest value (in
 * rnnt_rms_norm8 the largest t * weight) is below 2^-100, has q = 0 and scale 0; one that holds an infinity
 * or NaN has q = 0 and scale NaN.  Row i begins at q + i * pitch (bytes, a multiple of 16 and at least D; q is
 * 16-byte aligned); the bytes behind the D first are not written.
 *
 * rnnt_quantize_rows: v = x, `rows` rows of D elements.  rnnt_rms_norm8: v = the norm's y
 * before it is rounded; rows behind a length have q = 0 and scale 0.
 * Statuses as above, and RNNT_ERR_ALIGNMENT for q or pitch; rows < 0 is RNNT_ERR_BAD_SHAPE.
 */
rnnt_status_t rnnt_quantize_rows(const void* x, int64_t rows, int32_t D, rnnt_dtype_t dtype, int8_t* q, int64_t pitch,
                                 float* scale, hipStream_t stream);

rnnt_status_t rnnt_rms_norm8(const void* x, const void* residual, rnnt_norm_shape_t shape, const int32_t* lens,
                             const void* weight, float eps, int8_t* q, int64_t pitch, float* scale, void* sum_out,
                             hipStream_t stream);

/* ---------------------------------------------------------------------------
 * Product in 8-bit integers.
 *
 *   y[m, n] = (sum_k x[m, k] w[n, k]) x_scale[m] w_scale[n] + bias[n]
 * with x (M, K) and w (N, K) rows in 8 bits, as above (any values of -128 .. 127; x_pitch and
 * w_pitch in bytes), the sum exact in 32 bits, bias (N) of y's type or NULL, y (M, N) dense.
 * The bytes between K and a row's pitch are read and not used.
 *
 * rnnt_linear8_dynamic: x holds rows of `dtype` (dense, x_pitch is not used), taken to 8 bits
 * as rnnt_quantize_rows does within the call.
 *
 * RNNT_ERR_BAD_SHAPE: M < 0, N < 1, K < 1, a pitch below K.  RNNT_ERR_ALIGNMENT: x or w in 8 bits not
 * 16-byte aligned, or a pitch that is no multiple of 16.  RNNT_ERR_UNSUPPORTED: K of 2^17 or more
 * (the sum could pass 32 bits), rnnt_linear8_dynamic with K > 32768 (16384 in float32), M of
 * 2^31 / 128 or more, N > 2^21, 2^23 or more tiles of 128 x 128 results, or a pitch of 2^20 or more.
 */
typedef struct {
  int32_t M, N, K;
  rnnt_dtype_t dtype; /* of y and bias, and of x in rnnt_linear8_dynamic */
  int64_t x_pitch, w_pitch;
} rnnt_linear8_shape_t;

rnnt_status_t rnnt_linear8(const int8_t* x, const float* x_scale, const int8_t* w, const float* w_scale,
                           rnnt_linear8_shape_t shape, const void* bias, void* y, hipStream_t stream);

size_t rnnt_linear8_dynamic_workspace_bytes(rnnt_linear8_shape_t shape);
rnnt_status_t rnnt_linear8_dynamic(const void* x, const int8_t* w, const float* w_scale, rnnt_linear8_shape_t shape,
                                   const void* bias, void* y, void* workspace, size_t workspace_bytes,
                                   hipStream_t stream);

/* ---------------------------------------------------------------------------
 * Rotary positions.
 *
 *   (a, b) -> (a cos - b sin, a sin + b cos) at the angle (start[b] + t) * freq[i]
 * for the R / 2 pairs of the first R channels of each head of x (B, L, H, D): channels 2i and
 * 2i + 1 (interleaved), or i and R/2 + i; channels from R on are copied.  start (B) int32 is
 * the position of an utterance's first token, or NULL (0); freq (R / 2) float64, radians a
 * position, 8-byte aligned: angles are formed and reduced in float64, so far positions keep
 * their digits.  inverse != 0 turns the other way, which is the gradient: a length outside its range gives 0 there.
 * x may be a view with contiguous channels (strides in elements); y (B, L, H, D) is dense.
 *
 * RNNT_ERR_BAD_SHAPE: B < 1, L < 0, H < 1, D < 1, R odd or outside [2, D], or a stride below 0.
 * RNNT_ERR_UNSUPPORTED: H * D > 2^16, R > 1024, or B * L of 2^31 / 128 or more.
 */
typedef struct {
  int32_t B, L, H, D, R, interleaved;
  rnnt_dtype_t dtype;
  int64_t stride_b, stride_t, stride_h;
} rnnt_rotary_shape_t;

rnnt_status_t rnnt_rotary(const void* x, rnnt_rotary_shape_t shape, const double* freq, const int32_t* start,
                          const int32_t* lens, int32_t inverse, void* y, hipStream_t stream);

/* ---------------------------------------------------------------------------
 * Attention of a chunk of new tokens over a paged cache.
 *
 * Utterance b has cached[b] tokens in the cache and brings lens[b] <= L new ones, whose
 * positions follow: the call writes their keys and values into the cache and attends,
 *   out[b, t, h] = sum_j p_j v_j,   p = softmax over the visible j of scale q[b, t, h] . k_j,
 * with head h / (Hq / Hkv) of k and v.  Query t, at position i = cached[b] + t, sees position j
 * when  j <= i (causal), or j < cached[b] + lens[b] (else: the chunk's tokens see one another),
 * and, with left >= 0, j >= i - left.  The caller then adds lens to cached.  One step of a
 * decoder is L = 1.
 *
 * q (B, L, Hq, D), k and v (B, L, Hkv, D): views with contiguous channels, strides in elements.
 * k_cache, v_cache (num_pages, Hkv, page, D) dense, 16-byte aligned; pages (B, table) int32: position j
 * of utterance b is row j % page of page pages[b, j / page].  Entries of pages that no query of the
 * call sees (behind the new tokens, or further back than left) are not used, and may be
 * anything.  A page that the call writes to belongs to one utterance of the call; pages that it
 * only reads may be shared.  out (B, L, Hq, D) is dense.
 * A key on a page outside [0, num_pages) gives NaN to the queries that see it, and is not
 * written.  lens[b] outside [0, L], or cached[b] outside [0, table * page - lens[b]], gives NaN in
 * that utterance's outputs, and nothing of it is written.
 * Keys and values that a query does not see do not reach it, whatever they hold.
 * In the 16-bit types the weights p_j, before they are divided by their sum, are rounded to that type for their
 * product with the values (in float16 scaled, so that one of 2^-26 of the row's largest keeps 2^-10 of itself); scores,
 * maxima and sums are float32 in every type.
 *
 * RNNT_ERR_BAD_SHAPE: B, Hq, Hkv, D, page, table or num_pages < 1, L < 0, Hq no multiple of Hkv, a
 * stride below 0.  RNNT_ERR_BAD_VARIANT: scale times log2 e no finite float32.  RNNT_ERR_ALIGNMENT: q, k or v not 16-byte
 * aligned, or a stride that is no multiple of 16 bytes.  RNNT_ERR_UNSUPPORTED: D no multiple of 8 or above 256, page
 * no power of two or above 1024, a stride of k's or v's tokens of 2^31 or more, num_pages * Hkv * page or L * Hq of 2^31 or more, table * page + L of 2^30 or more,
 * or B * Hkv times the tiles of an utterance's L * (Hq / Hkv) rows (16 rows, or 128 where they are many) of 2^23 or
 * more.
 */
typedef struct {
  int32_t B, L, Hq, Hkv, D, page, table, num_pages, causal, left;
  rnnt_dtype_t dtype;
  int64_t q_stride_b, q_stride_t, q_stride_h;
  int64_t k_stride_b, k_stride_t, k_stride_h;
  int64_t v_stride_b, v_stride_t, v_stride_h;
} rnnt_attention_shape_t;

size_t rnnt_cached_attention_workspace_bytes(rnnt_attention_shape_t shape);
rnnt_status_t rnnt_cached_attention(const void* q, const void* k, const void* v, rnnt_attention_shape_t shape,
                                    const int32_t* lens, const int32_t* cached, const int32_t* pages, void* k_cache,
                                    void* v_cache, float scale, void* out, void* workspace, size_t workspace_bytes,
                                    hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* RNNT_ENCODER_MI355X_H */
