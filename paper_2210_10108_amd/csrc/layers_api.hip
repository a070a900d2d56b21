// C ABI of the layer operators (include/pnerf_layers.h): argument checks and the
// kernels' arguments.  Nothing here allocates or synchronises.
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <utility>

#include "../../include/pnerf_layers.h"
#include "layers_internal.h"
#include "pnerf_internal.h"

using namespace pnerf;

namespace {

// Head rows of a call: no launch reaches 2^32 threads (attention: up to 16 a row
// and 512 a batch entry and kv head; norm: up to 32 a row).
constexpr int64_t kMaxAttnRows = (int64_t)1 << 27, kMaxAttnHeads = (int64_t)1 << 22,
                  kMaxNormRows = (int64_t)1 << 26;

pnerf_status fail(pnerf_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  set_last_error(buf);
  return st;
}

pnerf_status launched(hipError_t e, const char* what) {
  return e == hipSuccess ? PNERF_OK : fail(PNERF_ERR_DEVICE, "%s launch: %s", what, hipGetErrorString(e));
}

pnerf_status check_workspace(const void* ws, int64_t have, int64_t need) {
  if (need == 0) return PNERF_OK;
  if (!ws) return fail(PNERF_ERR_INVALID_ARG, "NULL workspace, %lld bytes needed", (long long)need);
  if (have < need)
    return fail(PNERF_ERR_CAPACITY, "workspace of %lld bytes, %lld needed", (long long)have, (long long)need);
  if ((uintptr_t)ws % 16) return fail(PNERF_ERR_INVALID_ARG, "the workspace is not 16-byte aligned");
  return PNERF_OK;
}

bool aligned(const void* p, size_t n) { return (uintptr_t)p % n == 0; }

// A tensor of n dimensions, the last contiguous: pointer, sizes, strides.
struct View {
  const char* name;
  const void* p;
  int n;
  int64_t size[4], stride[4];
};

bool empty(const View& v) {
  for (int i = 0; i < v.n; ++i)
    if (v.size[i] == 0) return true;
  return false;
}

// Strides at least 0; an element's alignment; no overflow of a 64-bit byte offset.
pnerf_status check_view(const View& v, int elem, bool out) {
  if (empty(v)) return PNERF_OK;
  if (!v.p) return fail(PNERF_ERR_INVALID_ARG, "%s is NULL", v.name);
  if (!aligned(v.p, elem)) return fail(PNERF_ERR_INVALID_ARG, "%s is not aligned to its elements", v.name);
  std::pair<int64_t, int64_t> dim[4];  // (stride, size), to be sorted
  for (int i = 0; i < v.n; ++i) {
    if (v.stride[i] < 0 || v.stride[i] > ((int64_t)1 << 46))
      return fail(PNERF_ERR_INVALID_ARG, "%s has stride %lld", v.name, (long long)v.stride[i]);
    if (v.size[i] > 1 && v.stride[i] > ((int64_t)1 << 58) / v.size[i])
      return fail(PNERF_ERR_INVALID_ARG, "%s spans too much memory", v.name);
    dim[i] = {v.stride[i], v.size[i]};
  }
  if (!out) return PNERF_OK;
  std::sort(dim, dim + v.n);
  int64_t span = 1;  // elements the smaller dimensions cover
  for (int i = 0; i < v.n; ++i) {
    if (dim[i].second == 1) continue;
    if (dim[i].first < span) return fail(PNERF_ERR_INVALID_ARG, "%s overlaps itself", v.name);
    span = dim[i].first * (dim[i].second - 1) + span;
  }
  return PNERF_OK;
}

// Every row of v starts on 16 bytes.
bool rows_aligned(const View& v, int elem) {
  if (empty(v) || !v.p) return true;
  if (!aligned(v.p, 16)) return false;
  for (int i = 0; i + 1 < v.n; ++i)
    if (v.size[i] > 1 && v.stride[i] * elem % 16) return false;
  return true;
}

#define TRY(expr)                          \
  do {                                     \
    pnerf_status st_ = (expr);             \
    if (st_ != PNERF_OK) return st_;       \
  } while (0)

// ---------------------------------------------------------------- attention
pnerf_status attention_args(const pnerf_attention_params* p, AttnArgs* out, bool backward) {
  if (!p) return fail(PNERF_ERR_INVALID_ARG, "NULL params");
  if (p->dtype < PNERF_F32 || p->dtype > PNERF_BF16) return fail(PNERF_ERR_INVALID_ARG, "dtype=%d", p->dtype);
  if (p->dtype == PNERF_F32) return fail(PNERF_ERR_NOT_SUPPORTED, "dtype=0 (supported: 1 float16, 2 bfloat16)");
  if (p->batch < 0 || p->batch > 65535) return fail(PNERF_ERR_INVALID_ARG, "batch=%d outside 0..65535", p->batch);
  if (p->q_rows < 0 || p->kv_rows < 0)
    return fail(PNERF_ERR_INVALID_ARG, "q_rows=%d and kv_rows=%d must be >= 0", p->q_rows, p->kv_rows);
  if (p->kv_heads < 1 || p->q_heads < 1 || p->q_heads > 65535 || p->q_heads % p->kv_heads)
    return fail(PNERF_ERR_INVALID_ARG, "q_heads=%d must be a multiple of kv_heads=%d, at most 65535",
                p->q_heads, p->kv_heads);
  if (p->head_dim < 1) return fail(PNERF_ERR_INVALID_ARG, "head_dim=%d", p->head_dim);
  if (p->head_dim > 128) return fail(PNERF_ERR_NOT_SUPPORTED, "head_dim=%d (supported: 1..128)", p->head_dim);
  if (!(std::isfinite(p->scale) && p->scale > 0.0f)) return fail(PNERF_ERR_INVALID_ARG, "scale must be finite and > 0");
  const int64_t bq = (int64_t)p->batch * p->q_heads, bk = (int64_t)p->batch * p->kv_heads;
  if (bk > kMaxAttnHeads) return fail(PNERF_ERR_CAPACITY, "batch * kv_heads exceeds 2^22");
  if ((bq && p->q_rows > kMaxAttnRows / bq) || (bk && p->kv_rows > kMaxAttnRows / bk))
    return fail(PNERF_ERR_CAPACITY, "batch * heads * rows exceeds 2^27");
  if ((int64_t)p->q_rows * (p->q_heads / p->kv_heads) > kMaxAttnRows)
    return fail(PNERF_ERR_CAPACITY, "q_rows * q_heads / kv_heads exceeds 2^27");
  AttnArgs a = {};
  a.dtype = p->dtype;
  a.B = p->batch, a.Sq = p->q_rows, a.Sk = p->kv_rows, a.Hq = p->q_heads, a.Hkv = p->kv_heads;
  a.G = a.Hq / a.Hkv, a.D = p->head_dim, a.M = a.Sq * a.G;
  a.scale = p->scale;
  a.c = (float)((double)p->scale * 1.4426950408889634);
  for (int i = 0; i < 3; ++i) {
    a.qs[i] = p->q_stride[i], a.ks[i] = p->k_stride[i], a.vs[i] = p->v_stride[i], a.os[i] = p->o_stride[i];
    a.dos[i] = p->do_stride[i], a.dqs[i] = p->dq_stride[i], a.dks[i] = p->dk_stride[i], a.dvs[i] = p->dv_stride[i];
  }
  // the stride of a single row is not what the caller's may be: the tiles' loads
  // want one that keeps the rows after it apart
  const int64_t apart = (p->head_dim + 7) / 8 * 8;
  if (a.Sq == 1) a.qs[1] = a.os[1] = a.dos[1] = a.dqs[1] = apart;
  if (a.Sk == 1) a.ks[1] = a.vs[1] = a.dks[1] = a.dvs[1] = apart;
  a.q_len = p->q_len, a.kv_len = p->kv_len, a.mask = p->kv_mask, a.mask_stride = p->kv_mask_stride;
  if (a.mask && (a.mask_stride < 0 || a.mask_stride > ((int64_t)1 << 40)))
    return fail(PNERF_ERR_INVALID_ARG, "kv_mask has stride %lld", (long long)a.mask_stride);
  if ((a.q_len && !aligned(a.q_len, 4)) || (a.kv_len && !aligned(a.kv_len, 4)))
    return fail(PNERF_ERR_INVALID_ARG, "q_len and kv_len must be aligned to 4 bytes");
  a.splits = backward ? 1 : attn_fwd_splits(a);
  *out = a;
  return PNERF_OK;
}

// ---------------------------------------------------------------- norm and rotation
pnerf_status norm_args(const pnerf_norm_rotate_params* p, NormArgs* out) {
  if (!p) return fail(PNERF_ERR_INVALID_ARG, "NULL params");
  if (p->dtype < PNERF_F32 || p->dtype > PNERF_BF16) return fail(PNERF_ERR_INVALID_ARG, "dtype=%d", p->dtype);
  if (p->q_rows < 0 || p->k_rows < 0)
    return fail(PNERF_ERR_INVALID_ARG, "q_rows=%d and k_rows=%d must be >= 0", p->q_rows, p->k_rows);
  if ((p->q_rows && p->q_heads < 1) || (p->k_rows && p->k_heads < 1))
    return fail(PNERF_ERR_INVALID_ARG, "q_heads=%d and k_heads=%d must be >= 1", p->q_heads, p->k_heads);
  if (p->head_dim < 1) return fail(PNERF_ERR_INVALID_ARG, "head_dim=%d", p->head_dim);
  if (p->head_dim > 256) return fail(PNERF_ERR_NOT_SUPPORTED, "head_dim=%d (supported: 1..256)", p->head_dim);
  if (p->rotary_dim < 0 || p->rotary_dim > p->head_dim || p->rotary_dim % 2)
    return fail(PNERF_ERR_INVALID_ARG, "rotary_dim=%d must be even, 0..head_dim", p->rotary_dim);
  if (p->interleaved != 0 && p->interleaved != 1) return fail(PNERF_ERR_INVALID_ARG, "interleaved=%d", p->interleaved);
  if (p->rotary_dim && p->n_positions < 1) return fail(PNERF_ERR_INVALID_ARG, "n_positions=%d", p->n_positions);
  if (!(std::isfinite(p->eps) && p->eps >= 0.0f)) return fail(PNERF_ERR_INVALID_ARG, "eps must be finite and >= 0");
  if ((p->q_rows && (int64_t)p->q_rows * p->q_heads > kMaxNormRows) ||
      (p->k_rows && (int64_t)p->k_rows * p->k_heads > kMaxNormRows))
    return fail(PNERF_ERR_CAPACITY, "rows * heads exceeds 2^26");
  NormArgs a = {};
  a.dtype = p->dtype, a.D = p->head_dim, a.R = p->rotary_dim, a.interleaved = p->interleaved;
  a.n_pos = p->n_positions, a.eps = p->eps, a.table = p->table;
  NormSide &q = a.side[0], &k = a.side[1];
  q.rows = p->q_rows, q.heads = p->q_rows ? p->q_heads : 1, q.w = p->q_weight, q.pos = p->q_pos;
  k.rows = p->k_rows, k.heads = p->k_rows ? p->k_heads : 1, k.w = p->k_weight, k.pos = p->k_pos;
  for (int i = 0; i < 2; ++i) {
    q.xs[i] = p->q_stride[i], q.ys[i] = p->q_out_stride[i], q.dys[i] = p->dq_out_stride[i], q.dxs[i] = p->dq_stride[i];
    k.xs[i] = p->k_stride[i], k.ys[i] = p->k_out_stride[i], k.dys[i] = p->dk_out_stride[i], k.dxs[i] = p->dk_stride[i];
  }
  *out = a;
  return PNERF_OK;
}

pnerf_status norm_tensors(NormArgs* a, bool backward) {
  const int elem = a->dtype == kF32 ? 4 : 2;
  const char* names[2][4] = {{"q", "q_out", "dq_out", "dq"}, {"k", "k_out", "dk_out", "dk"}};
  bool vec = a->D % 8 == 0 && a->R % (a->interleaved ? 8 : 16) == 0 && aligned(a->table, 16);
  if (a->R && (a->side[0].rows || a->side[1].rows)) {
    if (!a->table) return fail(PNERF_ERR_INVALID_ARG, "table is NULL");
    if (!aligned(a->table, 4)) return fail(PNERF_ERR_INVALID_ARG, "table is not aligned to its elements");
  }
  for (int i = 0; i < 2; ++i) {
    const NormSide& x = a->side[i];
    if (!x.rows) continue;
    if (a->R && !x.pos) return fail(PNERF_ERR_INVALID_ARG, "%s_pos is NULL", i ? "k" : "q");
    if (x.pos && !aligned(x.pos, 4)) return fail(PNERF_ERR_INVALID_ARG, "%s_pos is not aligned to 4 bytes", i ? "k" : "q");
    if (x.w && !aligned(x.w, elem)) return fail(PNERF_ERR_INVALID_ARG, "%s_weight is not aligned to its elements", i ? "k" : "q");
    auto view = [&](int n, const void* p, const int64_t s[2]) {
      return View{names[i][n], p, 3, {x.rows, x.heads, a->D}, {s[0], s[1], 1}};
    };
    View v[3] = {view(0, x.x, x.xs), view(1, x.y, x.ys), {}};
    int n = 2;
    if (backward) v[1] = view(2, x.dy, x.dys), v[2] = view(3, x.dx, x.dxs), n = 3;
    for (int j = 0; j < n; ++j) {
      TRY(check_view(v[j], elem, j == n - 1));
      vec = vec && rows_aligned(v[j], elem);
    }
    if (x.dw && !aligned(x.dw, elem)) return fail(PNERF_ERR_INVALID_ARG, "d%s_weight is not aligned to its elements", i ? "k" : "q");
    vec = vec && (!x.w || aligned(x.w, 16));
  }
  a->vec = vec;
  return PNERF_OK;
}

// ---------------------------------------------------------------- linear
pnerf_status linear_args(const pnerf_linear_params* p, LinearArgs* out) {
  if (!p) return fail(PNERF_ERR_INVALID_ARG, "NULL params");
  if (p->dtype < PNERF_F32 || p->dtype > PNERF_BF16) return fail(PNERF_ERR_INVALID_ARG, "dtype=%d", p->dtype);
  if (p->dtype == PNERF_F32) return fail(PNERF_ERR_NOT_SUPPORTED, "dtype=0 (supported: 1 float16, 2 bfloat16)");
  if (p->activation < PNERF_ACT_NONE || p->activation > PNERF_ACT_SILU)
    return fail(PNERF_ERR_INVALID_ARG, "activation=%d outside 0..3", p->activation);
  if (p->m < 0 || p->n < 1 || p->k < 1)
    return fail(PNERF_ERR_INVALID_ARG, "m=%d must be >= 0, n=%d and k=%d >= 1", p->m, p->n, p->k);
  const int64_t m = p->m, n = p->n, k = p->k, most = (int64_t)1 << 34;
  if (std::max({m, n, k}) > (1 << 27) || m * n > most || m * k > most || k * n > most)
    return fail(PNERF_ERR_CAPACITY, "m=%d n=%d k=%d: a size exceeds 2^27 or a product of two 2^34", p->m, p->n, p->k);
  LinearArgs a = {};
  a.dtype = p->dtype, a.act = p->activation, a.M = p->m, a.N = p->n, a.K = p->k;
  a.xs = p->x_stride, a.ws = p->w_stride, a.rs = p->residual_stride, a.ys = p->y_stride, a.zs = p->z_stride;
  a.dys = p->dy_stride, a.dxs = p->dx_stride, a.dws = p->dw_stride;
  *out = a;
  return PNERF_OK;
}

}  // namespace

extern "C" {

pnerf_status pnerf_cross_attention_workspace(const pnerf_attention_params* p, int32_t backward,
                                             int64_t* bytes) {
  AttnArgs a;
  if (!bytes) return fail(PNERF_ERR_INVALID_ARG, "NULL bytes");
  TRY(attention_args(p, &a, backward != 0));
  *bytes = backward ? attn_bwd_bytes(a) : attn_fwd_bytes(a);
  return PNERF_OK;
}

pnerf_status pnerf_cross_attention(const pnerf_attention_params* p, const void* q, const void* k,
                                   const void* v, void* o, float* lse, void* workspace,
                                   int64_t workspace_bytes, void* stream) {
  AttnArgs a;
  TRY(attention_args(p, &a, false));
  auto view = [&](const char* name, const void* ptr, int64_t rows, int64_t heads, const int64_t* s) {
    return View{name, ptr, 4, {a.B, rows, heads, a.D}, {s[0], s[1], s[2], 1}};
  };
  const View t[4] = {view("q", q, a.Sq, a.Hq, a.qs), view("k", k, a.Sk, a.Hkv, a.ks),
                     view("v", v, a.Sk, a.Hkv, a.vs), view("o", o, a.Sq, a.Hq, a.os)};
  a.vec = a.D % 8 == 0;
  for (int i = 0; i < 4; ++i) {
    TRY(check_view(t[i], 2, i == 3));
    a.vec = a.vec && rows_aligned(t[i], 2);
  }
  if (!aligned(lse, 4)) return fail(PNERF_ERR_INVALID_ARG, "lse is not aligned to its elements");
  TRY(check_workspace(workspace, workspace_bytes, attn_fwd_bytes(a)));
  a.q = q, a.k = k, a.v = v, a.o = o, a.lse = lse;
  return launched(launch_attn_fwd(a, workspace, (hipStream_t)stream), "cross attention");
}

pnerf_status pnerf_cross_attention_backward(const pnerf_attention_params* p, const void* q,
                                            const void* k, const void* v, const void* o,
                                            const float* lse, const void* dout, void* dq, void* dk,
                                            void* dv, void* workspace, int64_t workspace_bytes,
                                            void* stream) {
  AttnArgs a;
  TRY(attention_args(p, &a, true));
  auto view = [&](const char* name, const void* ptr, int64_t rows, int64_t heads, const int64_t* s) {
    return View{name, ptr, 4, {a.B, rows, heads, a.D}, {s[0], s[1], s[2], 1}};
  };
  const View t[8] = {view("q", q, a.Sq, a.Hq, a.qs),       view("k", k, a.Sk, a.Hkv, a.ks),
                     view("v", v, a.Sk, a.Hkv, a.vs),      view("o", o, a.Sq, a.Hq, a.os),
                     view("dout", dout, a.Sq, a.Hq, a.dos), view("dq", dq, a.Sq, a.Hq, a.dqs),
                     view("dk", dk, a.Sk, a.Hkv, a.dks),   view("dv", dv, a.Sk, a.Hkv, a.dvs)};
  a.vec = a.D % 8 == 0;
  for (int i = 0; i < 8; ++i) {
    TRY(check_view(t[i], 2, i >= 5));
    a.vec = a.vec && rows_aligned(t[i], 2);
  }
  if (a.B && a.Sq && !lse) return fail(PNERF_ERR_INVALID_ARG, "lse is NULL");
  if (!aligned(lse, 4)) return fail(PNERF_ERR_INVALID_ARG, "lse is not aligned to its elements");
  TRY(check_workspace(workspace, workspace_bytes, attn_bwd_bytes(a)));
  a.q = q, a.k = k, a.v = v, a.o = (void*)o, a.lse = (float*)lse, a.dout = dout;
  a.dq = dq, a.dk = dk, a.dv = dv;
  return launched(launch_attn_bwd(a, workspace, (hipStream_t)stream), "cross attention backward");
}

pnerf_status pnerf_norm_rotate(const pnerf_norm_rotate_params* p, const void* q, const void* k,
                               void* q_out, void* k_out, void* stream) {
  NormArgs a;
  TRY(norm_args(p, &a));
  a.side[0].x = q, a.side[0].y = q_out;
  a.side[1].x = k, a.side[1].y = k_out;
  TRY(norm_tensors(&a, false));
  return launched(launch_norm_fwd(a, (hipStream_t)stream), "norm and rotation");
}

pnerf_status pnerf_norm_rotate_workspace(const pnerf_norm_rotate_params* p, int64_t* bytes) {
  NormArgs a;
  if (!bytes) return fail(PNERF_ERR_INVALID_ARG, "NULL bytes");
  TRY(norm_args(p, &a));
  *bytes = norm_bwd_bytes(a);
  return PNERF_OK;
}

pnerf_status pnerf_norm_rotate_backward(const pnerf_norm_rotate_params* p, const void* q,
                                        const void* k, const void* dq_out, const void* dk_out,
                                        void* dq, void* dk, void* dq_weight, void* dk_weight,
                                        void* workspace, int64_t workspace_bytes, void* stream) {
  NormArgs a;
  TRY(norm_args(p, &a));
  a.side[0].x = q, a.side[0].dy = dq_out, a.side[0].dx = dq, a.side[0].dw = dq_weight;
  a.side[1].x = k, a.side[1].dy = dk_out, a.side[1].dx = dk, a.side[1].dw = dk_weight;
  TRY(norm_tensors(&a, true));
  TRY(check_workspace(workspace, workspace_bytes, norm_bwd_bytes(a)));
  return launched(launch_norm_bwd(a, workspace, (hipStream_t)stream), "norm and rotation backward");
}

pnerf_status pnerf_linear_workspace(const pnerf_linear_params* p, int32_t backward, int64_t* bytes) {
  LinearArgs a;
  if (!bytes) return fail(PNERF_ERR_INVALID_ARG, "NULL bytes");
  TRY(linear_args(p, &a));
  *bytes = backward ? linear_bwd_bytes(a) : linear_fwd_bytes(a);
  return PNERF_OK;
}

pnerf_status pnerf_linear(const pnerf_linear_params* p, const void* x, const void* w,
                          const void* bias, const void* residual, void* y, void* z, void* workspace,
                          int64_t workspace_bytes, void* stream) {
  LinearArgs a;
  TRY(linear_args(p, &a));
  const View t[5] = {{"x", x, 2, {a.M, a.K}, {a.xs, 1}},
                     {"w", w, 2, {a.K, a.N}, {a.ws, 1}},
                     {"residual", residual, 2, {a.M, a.N}, {a.rs, 1}},
                     {"y", y, 2, {a.M, a.N}, {a.ys, 1}},
                     {"z", z, 2, {a.M, a.N}, {a.zs, 1}}};
  for (int i = 0; i < 5; ++i) {
    if ((i == 2 || i == 4) && !t[i].p) continue;
    TRY(check_view(t[i], 2, i >= 3));
  }
  if (!aligned(bias, 2)) return fail(PNERF_ERR_INVALID_ARG, "bias is not aligned to its elements");
  TRY(check_workspace(workspace, workspace_bytes, linear_fwd_bytes(a)));
  a.x = x, a.w = w, a.bias = bias, a.res = residual, a.y = y, a.z = z;
  return launched(launch_linear_fwd(a, workspace, (hipStream_t)stream), "linear");
}

pnerf_status pnerf_linear_backward(const pnerf_linear_params* p, const void* x, const void* w,
                                   const void* z, const void* dy, void* dx, void* dw, void* db,
                                   void* workspace, int64_t workspace_bytes, void* stream) {
  LinearArgs a;
  TRY(linear_args(p, &a));
  const View t[6] = {{"x", x, 2, {a.M, a.K}, {a.xs, 1}},   {"w", w, 2, {a.K, a.N}, {a.ws, 1}},
                     {"z", z, 2, {a.M, a.N}, {a.zs, 1}},   {"dy", dy, 2, {a.M, a.N}, {a.dys, 1}},
                     {"dx", dx, 2, {a.M, a.K}, {a.dxs, 1}}, {"dw", dw, 2, {a.K, a.N}, {a.dws, 1}}};
  for (int i = 0; i < 6; ++i) {
    if (i == 0 && !dw) continue;  // x is read for dw alone, w for dx alone
    if (i == 1 && !dx) continue;
    if (i == 2 && a.act == PNERF_ACT_NONE) continue;
    if (i >= 4 && !t[i].p) continue;
    TRY(check_view(t[i], 2, i >= 4));
  }
  if (!aligned(db, 2)) return fail(PNERF_ERR_INVALID_ARG, "db is not aligned to its elements");
  a.x = x, a.w = w, a.z = (void*)z, a.dy = dy, a.dx = dx, a.dw = dw, a.db = db;
  TRY(check_workspace(workspace, workspace_bytes, linear_bwd_bytes(a)));
  return launched(launch_linear_bwd(a, workspace, (hipStream_t)stream), "linear backward");
}

}  // extern "C"
