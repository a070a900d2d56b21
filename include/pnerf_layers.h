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
 *
 * The conventions of pnerf.h hold: arguments are validated on the host before
 * anything is enqueued (PNERF_ERR_INVALID_ARG or PNERF_ERR_NOT_SUPPORTED, the
 * message from pnerf_last_error), `stream` is a hipStream_t (NULL = the default
 * stream), device pointers stay valid until the queued work has finished.
 * Further, for every call here:
 *  - It only enqueues kernels on `stream`: no synchronisation, no allocation, no
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
 *    16-bit elements do.  (Linear layers copy large operands of other sizes and
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

#ifdef __cplusplus
}
#endif
#endif
