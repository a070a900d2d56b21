/*
 * pnerf_layers.h -- C ABI of the layer operators of libpnerf: what a network
 * that proposes or refines pose hypotheses is made of when its queries (the
 * hypotheses) read an encoder's states of the observed image.
 *
 *   pnerf_cross_attention   attention to states of another length, its gradient,
 *                           and the form for one or few query rows
 *   pnerf_norm_rotate       the norm of every query and key head and the
 *                           position rotation in one pass, and its gradient
 *   pnerf_linear            matrix product with bias, activation and residual,
 *                           and its gradient
 *   pnerf_layer_norm        the norm of whole rows, with mean and bias, and its
 *                           gradient
 *   pnerf_rotate_axes       the position rotation where positions have several axes
 *                           (a patch's row, column and frame), with or without the
 *                           norm, and its gradient
 *   pnerf_clip_gradients    the norm over all gradients of a step, and their scaling
 *   pnerf_quantize_states   keys and values in 8 bits, a scale for each block of rows
 *   pnerf_cross_attention_q8  attention to such states
 *
 * The conventions of pnerf.h hold: arguments are validated on the host before
 * anything is enqueued (PNERF_ERR_INVALID_ARG or PNERF_ERR_NOT_SUPPORTED, the
 * message from pnerf_last_error), `stream` is a hipStream_t (NULL = the default
 * stream), device pointers stay valid until the queued work has finished.
 * Further, for every call here:
 *  - It only enqueues kernels on `stream`: no synchronisation, no allocation (but for
 *    host memory that pnerf_clip_gradients takes for its list and gives back), no
 *    state kept between calls, so it can be captured into a HIP graph, and calls
 *    on different streams or threads may overlap.
 *  - The workspace is the caller's: at least the bytes that the operator's
 *    *_workspace function (host only, no device call) gives for the same params,
 *    16-byte aligned, its contents irrelevant before and undefined after the
 *    call, not shared by calls that may overlap.  NULL where 0 bytes are needed.
 *  - dtype is the element type of every data tensor: PNERF_F32, PNERF_F16,
 *    PNERF_BF16.  Sums, softmax statistics and norms are held in float32; what a
 *    call rounds on the way is named with it.
 *  - Strides are in elements, >= 0, and the last dimension is contiguous.  A
 *    stride of an input may be 0 or overlap; an output may not overlap itself or
 *    an input, save where stated.  Any stride and any pointer aligned to its
 *    elements will do; the fast kernels want every row to start on 16 bytes
 *    (pointers and strides), as contiguous tensors with rows of a multiple of 8
 *    16-bit elements do, and of 16 bytes for 8-bit states.  (Linear layers copy large operands of other sizes and
 *    strides to such rows in the workspace.  The workspace follows from sizes and
 *    strides alone: where those are of whole 16-byte chunks and only a pointer is off 16
 *    bytes nothing is copied, and a large product runs element by element, an order
 *    of magnitude slower.)
 *  - The same inputs give the same bits on every call (no atomics on results).
 */
#ifndef PNERF_LAYERS_H
#define PNERF_LAYERS_H
#include "pnerf.h"

#ifdef __cplusplus
extern "C" {
#endif

#define PNERF_F32 0
#define PNERF_F16 1
#define PNERF_BF16 2

/* Cross attention.  For batch entry b, query row i < q_len[b], query head h and
 * kv head g = h / (q_heads / kv_heads), over the allowed keys j (j < kv_len[b] and
 * kv_mask[b][j] != 0):
 *   a_ij = scale q_i . k_j,  lse_i = log sum_j exp(a_ij),
 *   o_i = sum_j exp(a_ij - lse_i) v_j
 * A row without an allowed key, or with i >= q_len[b], has o_i = 0 and
 * lse_i = -inf.  What keys, values and mask hold at j >= kv_len[b], keys and
 * values where the mask is 0, and queries at i >= q_len[b] has no influence,
 * infinities and NaN among them.  exp(a - m), m at most 8 ln 2 below the row's
 * running maximum, is rounded to the data type before it meets the values.
 * Backward, given do = dL/do:
 *   p_ij = exp(a_ij - lse_i),  delta_i = do_i . o_i,
 *   ds_ij = p_ij (do_i . v_j - delta_i),  dv_j = sum p_ij do_i,
 *   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum ds_ij q_i
 * (dk, dv: summed over the rows and the query heads that share the kv head; 0
 * where the key is not allowed).  p and ds are rounded to the data type.  In float16
 * they are kept times powers of two on the way: p times 2^14, ds times one that a row
 * (dq) or a key (dk) takes from the norms of do and v, such that no ds overflows and
 * one is a normal number down to 2^-28 of 2 max |do| max |v|.  A batch entry's dk and
 * dv are its own also where k and v are one tensor broadcast over the batch.
 *
 * Requires 0 <= batch <= 65535, q_rows, kv_rows >= 0, kv_heads >= 1, q_heads a
 * multiple of kv_heads (at most 65535), 1 <= head_dim <= 128, finite scale > 0,
 * batch * kv_heads at most 2^22, batch * q_heads * q_rows and batch * kv_heads *
 * kv_rows at most 2^27 (PNERF_ERR_CAPACITY); dtype PNERF_F16 or PNERF_BF16. */
typedef struct {
  int32_t dtype;
  int32_t batch, q_rows, kv_rows, q_heads, kv_heads, head_dim;
  float scale;
  /* (batch, row, head) strides; those of the gradients are read by the backward only */
  int64_t q_stride[3], k_stride[3], v_stride[3], o_stride[3];
  int64_t do_stride[3], dq_stride[3], dk_stride[3], dv_stride[3];
  const int32_t* q_len;    /* (device) [batch], clamped to 0..q_rows, or NULL: all q_rows */
  const int32_t* kv_len;   /* (device) [batch], clamped to 0..kv_rows, or NULL: all kv_rows */
  const uint8_t* kv_mask;  /* (device) [batch][kv_rows], nonzero = allowed, or NULL */
  int64_t kv_mask_stride;  /* between batch entries */
} pnerf_attention_params;

pnerf_status pnerf_cross_attention_workspace(const pnerf_attention_params* params,
                                             int32_t backward, int64_t* bytes);
/* lse (device): float32 [batch][q_heads][q_rows], or NULL when no backward follows. */
pnerf_status pnerf_cross_attention(const pnerf_attention_params* params, const void* q,
                                   const void* k, const void* v, void* o, float* lse,
                                   void* workspace, int64_t workspace_bytes, void* stream);
/* o and lse as pnerf_cross_attention left them. */
pnerf_status pnerf_cross_attention_backward(const pnerf_attention_params* params, const void* q,
                                            const void* k, const void* v, const void* o,
                                            const float* lse, const void* dout, void* dq, void* dk,
                                            void* dv, void* workspace, int64_t workspace_bytes,
                                            void* stream);

/* Norm and rotation of the heads of queries and keys, both in one launch.  For
 * every head x of head_dim D components at position t:
 *   n_d = x_d w_d / sqrt(mean_d x_d^2 + eps)
 *   y_a = n_a c_j - n_b s_j,  y_b = n_a s_j + n_b c_j      (pair j < rotary_dim / 2)
 *   y_d = n_d                                              (d >= rotary_dim)
 * with c_j = table[t][0][j], s_j = table[t][1][j] and (a, b) = (j, j + rotary_dim / 2),
 * or (2j, 2j + 1) when interleaved = 1.  A position outside [0, n_positions)
 * gives NaN in that row's rotated components.  The outputs may be the inputs
 * themselves (same pointer and strides).
 * Backward, given dy: with g the gradient turned back (the rotation transposed)
 * and r = 1 / sqrt(mean x^2 + eps),
 *   dx_d = r (g_d w_d - x_d r^2 mean_e(g_e w_e x_e)),  dw_d = sum_rows g_d x_d r
 * dx may be dy itself.  dq_weight / dk_weight may be NULL (not wanted).
 *
 * Requires q_rows, k_rows >= 0 (0: no such operand, its pointers are not read),
 * heads >= 1 where rows > 0, 1 <= head_dim <= 256, rotary_dim even in
 * 0..head_dim, n_positions >= 1 when rotary_dim > 0, rows * heads at most 2^26, finite
 * eps >= 0; any dtype. */
typedef struct {
  int32_t dtype;
  int32_t q_rows, k_rows, q_heads, k_heads, head_dim, rotary_dim, interleaved, n_positions;
  float eps;
  /* (row, head) strides of the inputs, the outputs and, for the backward, dL/d output and dL/d input */
  int64_t q_stride[2], k_stride[2], q_out_stride[2], k_out_stride[2];
  int64_t dq_out_stride[2], dk_out_stride[2], dq_stride[2], dk_stride[2];
  const void* q_weight; /* (device) [head_dim], or NULL: ones */
  const void* k_weight;
  const float* table;   /* (device) float32 [n_positions][2][rotary_dim / 2]: cosines, sines */
  const int32_t* q_pos; /* (device) [q_rows] */
  const int32_t* k_pos; /* (device) [k_rows] */
} pnerf_norm_rotate_params;

pnerf_status pnerf_norm_rotate(const pnerf_norm_rotate_params* params, const void* q, const void* k,
                               void* q_out, void* k_out, void* stream);
pnerf_status pnerf_norm_rotate_workspace(const pnerf_norm_rotate_params* params, int64_t* bytes);
pnerf_status pnerf_norm_rotate_backward(const pnerf_norm_rotate_params* params, const void* q,
                                        const void* k, const void* dq_out, const void* dk_out,
                                        void* dq, void* dk, void* dq_weight, void* dk_weight,
                                        void* workspace, int64_t workspace_bytes, void* stream);

/* Linear layer, weights [in][out] as the field's networks keep them:
 *   z = x W + bias,  y = act(z) + residual
 * x [m][k], W [k][n], bias [n], residual, y, z [m][n]; bias, residual and z may be
 * NULL.  z is act's argument, kept for the backward, which takes act' at it as it
 * was rounded to the data type.  y may be the residual itself (same pointer and
 * stride).
 * Backward, given dy:  dz = dy act'(z),  dx = dz W^T,  dW = x^T dz,  db = sum_m dz;
 * dz is rounded to the data type before the products.  The gradient of the
 * residual is dy.  z may be NULL when activation is 0; dx, dw and db may each be
 * NULL (not wanted).
 *
 * Requires 0 <= m, 1 <= n, k, each at most 2^27, and m * n, m * k, k * n at most 2^34;
 * dtype PNERF_F16 or PNERF_BF16. */
#define PNERF_ACT_NONE 0
#define PNERF_ACT_RELU 1 /* derivative 0 at 0 */
#define PNERF_ACT_GELU 2 /* z Phi(z), Phi the normal distribution function */
#define PNERF_ACT_SILU 3 /* z / (1 + exp(-z)) */
typedef struct {
  int32_t dtype, activation;
  int32_t m, n, k;
  /* row strides; the last three are read by the backward only */
  int64_t x_stride, w_stride, residual_stride, y_stride, z_stride, dy_stride, dx_stride, dw_stride;
} pnerf_linear_params;

pnerf_status pnerf_linear_workspace(const pnerf_linear_params* params, int32_t backward,
                                    int64_t* bytes);
pnerf_status pnerf_linear(const pnerf_linear_params* params, const void* x, const void* w,
                          const void* bias, const void* residual, void* y, void* z, void* workspace,
                          int64_t workspace_bytes, void* stream);
pnerf_status pnerf_linear_backward(const pnerf_linear_params* params, const void* x, const void* w,
                                   const void* z, const void* dy, void* dx, void* dw, void* db,
                                   void* workspace, int64_t workspace_bytes, void* stream);

/* Layer norm of every row x of `width` W elements:
 *   y_d = (x_d - mean) r w_d + b_d,  r = 1 / sqrt(mean_d (x_d - mean)^2 + eps)
 * y may be x itself (same pointer and stride).
 * Backward, given dy and, if not NULL, dres (the gradient that reaches x past the
 * norm, of a residual connection), with g_d = dy_d w_d, n_d = (x_d - mean) r:
 *   dx_d = r (g_d - mean g - n_d mean(g n)) + dres_d
 *   dweight_d = sum_rows dy_d n_d,  dbias_d = sum_rows dy_d
 * dx may be dy, dres or x itself.  weight (ones) and bias (zeros) may be NULL, dweight
 * and dbias too (not wanted).  A row is what its elements were rounded to: the mean is
 * taken in two steps, so that a mean large beside the spread costs nothing more.  A row
 * of equal elements has n = 0 exactly where eps > 0; where eps = 0 its n is NaN.  Where
 * the sum of a row's squared differences passes float32's range (differences of some
 * 10^19 / sqrt(W)) r and n are 0.  An infinity or NaN makes n NaN in all of its row.
 * Squared differences are 32-bit numbers too: with eps = 0, r is as exact as their mean is
 * where that is below 2^-126, and infinite where they are all below 2^-150.
 * Rows of up to 16384 elements, 8192 in the gradient, are read once, whatever their width
 * and alignment (fastest where they start on 16 bytes and have a multiple of 8 elements).
 * Wider ones are read again for each step, and the gradient of rows wider than 16384 adds
 * to the weights' sums in memory, row by row.
 *
 * Requires rows >= 0, 1 <= width <= 2^20, rows * width at most 2^40, finite eps >= 0;
 * any dtype. */
typedef struct {
  int32_t dtype, rows, width;
  float eps;
  /* row strides; the last three are read by the backward only */
  int64_t x_stride, y_stride, dy_stride, dres_stride, dx_stride;
} pnerf_layer_norm_params;

pnerf_status pnerf_layer_norm(const pnerf_layer_norm_params* params, const void* x,
                              const void* weight, const void* bias, void* y, void* stream);
pnerf_status pnerf_layer_norm_workspace(const pnerf_layer_norm_params* params, int64_t* bytes);
pnerf_status pnerf_layer_norm_backward(const pnerf_layer_norm_params* params, const void* x,
                                       const void* weight, const void* dy, const void* dres,
                                       void* dx, void* dweight, void* dbias, void* workspace,
                                       int64_t workspace_bytes, void* stream);

/* Rotation at positions of several axes: as pnerf_norm_rotate with
 *   c_j = table[t_a][0][j], s_j = table[t_a][1][j],  a = pair_axis[j],
 * t_a the row's position along axis a: base.q_pos is [q_rows][axes], base.k_pos
 * [k_rows][axes].  Every frequency an axis may want is in the columns of its pairs.
 * A position outside [0, n_positions) gives NaN in the pairs of its axis.
 * Pairs that share an axis in runs of 8 (of 4 where interleaved = 1) are the fastest.
 * norm = 1: the heads are normed first, as there; norm = 0: n = x, the weights are not
 * read, the gradient is the rotation back alone (q and k are not read and may be NULL,
 * no weight has a gradient, no workspace is needed).
 *
 * Requires what pnerf_norm_rotate does, norm 0 or 1, 1 <= axes <= 4 and
 * pair_axis[j] < axes for the rotary_dim / 2 pairs. */
typedef struct {
  pnerf_norm_rotate_params base;
  int32_t norm, axes;
  uint8_t pair_axis[128];
} pnerf_rotate_axes_params;

pnerf_status pnerf_rotate_axes(const pnerf_rotate_axes_params* params, const void* q, const void* k,
                               void* q_out, void* k_out, void* stream);
pnerf_status pnerf_rotate_axes_workspace(const pnerf_rotate_axes_params* params, int64_t* bytes);
pnerf_status pnerf_rotate_axes_backward(const pnerf_rotate_axes_params* params, const void* q,
                                        const void* k, const void* dq_out, const void* dk_out,
                                        void* dq, void* dk, void* dq_weight, void* dk_weight,
                                        void* workspace, int64_t workspace_bytes, void* stream);

/* The norm over all elements of `count` gradients and their scaling by it:
 *   norm = sqrt(sum g^2),  out = c g,  c = min(1, max_norm / (norm + eps))
 * Squares and their sum are float64; norm (device) is the result in float32, c is
 * rounded to float32, c g to the output's type.  An output may be its gradient (same
 * pointer and dtype; where c = 1 it is not touched), and overlaps no other gradient or
 * output.  max_norm may be infinite: c = 1.  A NaN among the gradients makes the norm
 * and every output NaN (max_norm infinite: the norm alone); an infinity makes the norm
 * infinite and c = 0.
 * `gradients` (host) is read before the call returns.
 *
 * Requires 0 <= count <= 65536, n >= 0, all n together at most 2^42, out_dtype the
 * gradient's or PNERF_F32, max_norm > 0, finite eps >= 0. */
typedef struct {
  const void* grad; /* (device) [n] */
  void* out;        /* (device) [n] */
  int64_t n;
  int32_t dtype, out_dtype;
} pnerf_gradient;

pnerf_status pnerf_clip_gradients_workspace(int32_t count, int64_t* bytes);
pnerf_status pnerf_clip_gradients(const pnerf_gradient* gradients, int32_t count, double max_norm,
                                  double eps, float* norm, void* workspace,
                                  int64_t workspace_bytes, void* stream);

/* Keys and values in 8 bits.  For each block of PNERF_STATE_BLOCK rows of a head,
 * over its allowed rows (as for pnerf_cross_attention):
 *   scale = the least power of two, at least 2^-126, with max |x| <= 448 scale
 *           (1 where all x are 0 or no row is allowed)
 *   x8 = x / scale to the nearest e4m3 number (ties to the even one; no infinities:
 *        those of x become NaN, which like NaN do not count for the scale)
 * x8 is 0 in rows that are not allowed; what x holds there has no influence.
 * k8, v8 are bytes [batch][kv_rows][kv_heads][head_dim], the scales float32
 * [batch][blocks][kv_heads], blocks = kv_rows / PNERF_STATE_BLOCK rounded up.
 *
 * Requires of the sizes what pnerf_cross_attention does; dtype PNERF_F16 or PNERF_BF16. */
#define PNERF_STATE_BLOCK 64
typedef struct {
  int32_t dtype, batch, kv_rows, kv_heads, head_dim;
  int64_t k_stride[3], v_stride[3], k8_stride[3], v8_stride[3]; /* (batch, row, head) */
  int64_t k_scale_stride[2], v_scale_stride[2];                 /* (batch, block) */
  const int32_t* kv_len;   /* (device) [batch], clamped to 0..kv_rows, or NULL: all kv_rows */
  const uint8_t* kv_mask;  /* (device) [batch][kv_rows], nonzero = allowed, or NULL */
  int64_t kv_mask_stride;  /* between batch entries */
} pnerf_states_params;

pnerf_status pnerf_quantize_states(const pnerf_states_params* params, const void* k, const void* v,
                                   void* k8, void* v8, float* k_scale, float* v_scale, void* stream);

/* Cross attention to 8-bit states: pnerf_cross_attention with
 *   k_j = k_scale[j / PNERF_STATE_BLOCK] k8_j,  v_j = v_scale[j / PNERF_STATE_BLOCK] v8_j
 * as pnerf_quantize_states leaves them (attention.k_stride and v_stride are those of k8
 * and v8; attention.dtype is that of q and o).  The scales are any positive normal
 * numbers, not only powers of two.  exp(a - m) times the value scale, in a unit that
 * follows it, is rounded to the data type before it meets the values.  What a block adds
 * is lost beside a row's result 2^50 times as large, and where its exp(a - lse) is below
 * 2^-118.  Keys, values and masks in places that are not allowed, and the scales of blocks
 * without an allowed key, have no influence.  A query with an infinity or NaN has NaN for
 * o and lse where a key is allowed, 0 and -inf where none is.  No gradient: states are
 * kept in 8 bits for proposals, not for training.
 * States in 8 bits take half the memory of those in 16.  With heads of 128 the attention
 * takes 0.55 to 0.6 of the other one's time at up to 32 rows of a kv head (q_rows q_heads
 * / kv_heads), 0.8 at 64 and 1 to 1.1 beyond; with heads of 64, whose states are fewer
 * bytes, 0.8 to 1.25.  The fast kernels want a head_dim of a multiple of 16 and rows of k8
 * and v8 on 16 bytes; others take 4 to 8 times as long, where the attention to 16-bit
 * states is fast at multiples of 8. */
typedef struct {
  pnerf_attention_params attention;
  int64_t k_scale_stride[2], v_scale_stride[2]; /* (batch, block) */
} pnerf_attention_q8_params;

pnerf_status pnerf_cross_attention_q8_workspace(const pnerf_attention_q8_params* params, int64_t* bytes);
/* lse (device): float32 [batch][q_heads][q_rows], or NULL. */
pnerf_status pnerf_cross_attention_q8(const pnerf_attention_q8_params* params, const void* q,
                                      const void* k8, const void* v8, const float* k_scale,
                                      const float* v_scale, void* o, float* lse, void* workspace,
                                      int64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif
