// Layer norm of rows: y = (x - mean) / sqrt(var + eps) w + b, and its gradient
//   dx = r (g - mean g - n mean(g n)) + dres,  dw = sum_rows dy n,  db = sum_rows dy
// with g = dy w, n = (x - mean) r, r = 1 / sqrt(var + eps).
//
// Sums are float32.  A row's mean is taken in two steps, m = mean x and then c =
// mean(x - m), and var = mean (x - m)^2 - c^2: rows whose mean is large beside their
// spread lose nothing but what x itself was rounded to, and the gradient makes its
// statistics again from the row that it reads anyway.
#define PNERF_LAYERS_DEVICE
#include <algorithm>

#include "rows_common.h"

namespace pnerf {
namespace {

constexpr int kBlock = 256;

// A row of W elements is TPR threads, NV groups of 8 consecutive elements (16-byte
// accesses) each: part of a wavefront, a wavefront, or a workgroup of up to 1024
// threads.  The row stays in registers, its reductions are exchanges within the
// wavefront and, past one, a value a wavefront through LDS; the next row's loads are on
// their way meanwhile.
template <int TPR>
struct Shape {
  static constexpr int kThreads = TPR < kBlock ? kBlock : TPR;
  static constexpr int kRows = kThreads / TPR;  // of a workgroup
};

// Sums of N values over the threads of a row, in all of them.  (Two sets of places in
// turn: the next sum's writes need not wait for this one's reads.)
template <int TPR>
struct RowSums {
  static constexpr int kWaves = TPR / 64;
  float* red;
  int set;
  __device__ __forceinline__ explicit RowSums(float* lds) : red(lds), set(0) {}
  template <int N>
  __device__ __forceinline__ void sum(float (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = row_sum<(TPR < 64 ? TPR : 64)>(v[i]);
    if constexpr (TPR > 64) {
      float* r = red + set * kWaves * 4;
      set ^= 1;
      if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) r[(threadIdx.x >> 6) * 4 + i] = v[i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = 0.0f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += r[w * 4 + i];
    }
  }
};

// NV groups of 8 elements of a row as they are loaded.
template <class E, int TPR, int NV>
struct Group {
  typename Elem<E>::Raw raw[NV];
  __device__ __forceinline__ void load(const void* p, int64_t at, int W) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int d = 8 * ((int)(threadIdx.x % TPR) + v * TPR);
      if (d < W) raw[v] = Elem<E>::raw((const E*)p + at + d);
    }
  }
};

template <class E, int TPR, int NV>
__global__ __launch_bounds__(Shape<TPR>::kThreads) void k_layer_norm(const LayerNormArgs a) {
  constexpr int kRows = Shape<TPR>::kRows;
  __shared__ float lds[TPR > 64 ? TPR / 8 : 1];
  RowSums<TPR> sums(lds);
  const int group = threadIdx.x / TPR;
  const float inv = 1.0f / a.W;
  Group<E, TPR, NV> x = {}, w = {}, b = {};
  if (a.w) w.load(a.w, 0, a.W);
  if (a.b) b.load(a.b, 0, a.W);
  int64_t row = (int64_t)blockIdx.x * kRows + group;
  const int64_t step = (int64_t)gridDim.x * kRows;
  if (row < a.rows) x.load(a.x, row * a.xs, a.W);
  for (; row - group < a.rows; row += step) {
    float v[NV][8], t[1] = {0.0f}, u[2] = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      Elem<E>::unpack(x.raw[k], v[k]);
#pragma unroll
      for (int j = 0; j < 8; ++j) t[0] += 8 * ((int)(threadIdx.x % TPR) + k * TPR) < a.W ? v[k][j] : 0.0f;
    }
    if (row + step < a.rows) x.load(a.x, (row + step) * a.xs, a.W);
    sums.sum(t);
    const float m = t[0] * inv;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const bool on = 8 * ((int)(threadIdx.x % TPR) + k * TPR) < a.W;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[k][j] = on ? v[k][j] - m : 0.0f;
        u[0] += v[k][j], u[1] += v[k][j] * v[k][j];
      }
    }
    sums.sum(u);
    const float c = u[0] * inv, r = inv_rms(fmaxf(u[1] * inv - c * c, 0.0f), a.eps);
    if (row >= a.rows) continue;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int d = 8 * ((int)(threadIdx.x % TPR) + k * TPR);
      if (d >= a.W) continue;
      float wk[8], bk[8];
      Elem<E>::unpack(w.raw[k], wk);
      Elem<E>::unpack(b.raw[k], bk);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float n = (v[k][j] - c) * r;
        v[k][j] = (a.w ? n * wk[j] : n) + (a.b ? bk[j] : 0.0f);
      }
      Elem<E>::store((E*)a.y + row * a.ys + d, v[k]);
    }
  }
}

// Each workgroup leaves its sums of dw and db, [workgroup][2][W].
template <class E, int TPR, int NV>
__global__ __launch_bounds__(Shape<TPR>::kThreads) void k_layer_norm_bwd(const LayerNormArgs a, float* part) {
  constexpr int kRows = Shape<TPR>::kRows;
  __shared__ float lds[TPR > 64 ? TPR / 8 : 1];
  RowSums<TPR> sums(lds);
  const int group = threadIdx.x / TPR;
  const float inv = 1.0f / a.W;
  Group<E, TPR, NV> x = {}, dy = {}, res = {}, w = {};
  if (a.w) w.load(a.w, 0, a.W);
  int64_t row = (int64_t)blockIdx.x * kRows + group;
  const int64_t step = (int64_t)gridDim.x * kRows;
  auto fetch = [&](int64_t at) {
    if (at >= a.rows) return;
    x.load(a.x, at * a.xs, a.W);
    dy.load(a.dy, at * a.dys, a.W);
  };
  fetch(row);
  float dw[NV][8] = {}, db[NV][8] = {};
  for (; row - group < a.rows; row += step) {
    float v[NV][8], g[NV][8], t[1] = {0.0f}, u[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const bool in = row < a.rows;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const bool on = in && 8 * ((int)(threadIdx.x % TPR) + k * TPR) < a.W;
      Elem<E>::unpack(x.raw[k], v[k]);
      Elem<E>::unpack(dy.raw[k], g[k]);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        t[0] += on ? v[k][j] : 0.0f;
        g[k][j] = on ? g[k][j] : 0.0f;
      }
    }
    if (a.dres && in) res.load(a.dres, row * a.drs, a.W);
    fetch(row + step);
    sums.sum(t);
    const float m = t[0] * inv;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const bool on = in && 8 * ((int)(threadIdx.x % TPR) + k * TPR) < a.W;
      float wk[8];
      Elem<E>::unpack(w.raw[k], wk);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[k][j] = on ? v[k][j] - m : 0.0f;
        const float gw = a.w ? g[k][j] * wk[j] : g[k][j];
        u[0] += v[k][j], u[1] += v[k][j] * v[k][j];
        u[2] += gw, u[3] += gw * v[k][j];
      }
    }
    sums.sum(u);
    const float c = u[0] * inv, r = inv_rms(fmaxf(u[1] * inv - c * c, 0.0f), a.eps);
    const float s1 = u[2] * inv, s2 = r * (u[3] * inv - c * s1);
    if (!in) continue;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int d = 8 * ((int)(threadIdx.x % TPR) + k * TPR);
      if (d >= a.W) continue;
      float wk[8], rk[8];
      Elem<E>::unpack(w.raw[k], wk);
      Elem<E>::unpack(res.raw[k], rk);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float n = (v[k][j] - c) * r;
        dw[k][j] += g[k][j] * n;
        db[k][j] += g[k][j];
        v[k][j] = r * ((a.w ? g[k][j] * wk[j] : g[k][j]) - s1 - n * s2) + (a.dres ? rk[j] : 0.0f);
      }
      Elem<E>::store((E*)a.dx + row * a.dxs + d, v[k]);
    }
  }
  if (!a.dw && !a.db) return;
  part += (int64_t)blockIdx.x * 2 * a.W;
  if constexpr (kRows == 1) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int d = 8 * ((int)threadIdx.x + k * TPR);
      if (d >= a.W) continue;
      Elem<float>::store(part + d, dw[k]);
      Elem<float>::store(part + a.W + d, db[k]);
    }
  } else {  // the rows' sums meet in LDS, those of dw and then those of db
    __shared__ float all[kRows][TPR * NV * 8];
    for (int side = 0; side < 2; ++side) {
      __syncthreads();
#pragma unroll
      for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int j = 0; j < 8; ++j)
          all[group][8 * ((int)(threadIdx.x % TPR) + k * TPR) + j] = side ? db[k][j] : dw[k][j];
      __syncthreads();
      for (int d = threadIdx.x; d < a.W; d += Shape<TPR>::kThreads) {
        float t = 0.0f;
        for (int i = 0; i < kRows; ++i) t += all[i][d];
        part[side * a.W + d] = t;
      }
    }
  }
}

// N values of a row from element d on, as numbers: one load of 8, or one element.
template <class E, int N>
__device__ __forceinline__ void values(const void* p, int64_t at, float (&v)[N]) {
  if constexpr (N == 8)
    load<E>((const E*)p + at, v);
  else
    v[0] = (float)((const E*)p)[at];
}
template <class E, int N>
__device__ __forceinline__ void put(void* p, int64_t at, const float (&v)[N]) {
  if constexpr (N == 8)
    Elem<E>::store((E*)p + at, v);
  else
    ((E*)p)[at] = (E)v[0];
}

// Any width: a workgroup a row, read again for each step.  N = 8: rows wider than the
// registers hold, by 16-byte accesses; N = 1: any stride and alignment, element by element.
template <class E, int N>
__global__ __launch_bounds__(kBlock) void k_layer_norm_any(const LayerNormArgs a) {
  __shared__ float lds[kBlock / 8];
  RowSums<kBlock> sums(lds);
  const float inv = 1.0f / a.W;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const int64_t x = row * a.xs;
    float t[1] = {0.0f}, u[2] = {0.0f, 0.0f}, v[N];
    for (int d = N * threadIdx.x; d < a.W; d += N * kBlock) {
      values<E, N>(a.x, x + d, v);
#pragma unroll
      for (int j = 0; j < N; ++j) t[0] += v[j];
    }
    sums.sum(t);
    const float m = t[0] * inv;
    for (int d = N * threadIdx.x; d < a.W; d += N * kBlock) {
      values<E, N>(a.x, x + d, v);
#pragma unroll
      for (int j = 0; j < N; ++j) u[0] += v[j] - m, u[1] += (v[j] - m) * (v[j] - m);
    }
    sums.sum(u);
    const float c = u[0] * inv, r = inv_rms(fmaxf(u[1] * inv - c * c, 0.0f), a.eps);
    for (int d = N * threadIdx.x; d < a.W; d += N * kBlock) {
      float w[N], b[N];
      values<E, N>(a.x, x + d, v);
      if (a.w) values<E, N>(a.w, d, w);
      if (a.b) values<E, N>(a.b, d, b);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float n = (v[j] - m - c) * r;
        v[j] = (a.w ? n * w[j] : n) + (a.b ? b[j] : 0.0f);
      }
      put<E, N>(a.y, row * a.ys + d, v);
    }
  }
}

// Each workgroup leaves its sums of dw and db, [workgroup][2][W].
template <class E, int N>
__global__ __launch_bounds__(kBlock) void k_layer_norm_bwd_any(const LayerNormArgs a, float* part) {
  __shared__ float lds[kBlock / 8];
  RowSums<kBlock> sums(lds);
  const float inv = 1.0f / a.W;
  const bool wanted = a.dw || a.db;
  float* mine = part + (int64_t)blockIdx.x * 2 * a.W;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const int64_t x = row * a.xs, dy = row * a.dys;
    float t[1] = {0.0f}, u[4] = {0.0f, 0.0f, 0.0f, 0.0f}, v[N], g[N], w[N];
    for (int d = N * threadIdx.x; d < a.W; d += N * kBlock) {
      values<E, N>(a.x, x + d, v);
#pragma unroll
      for (int j = 0; j < N; ++j) t[0] += v[j];
    }
    sums.sum(t);
    const float m = t[0] * inv;
    for (int d = N * threadIdx.x; d < a.W; d += N * kBlock) {
      values<E, N>(a.x, x + d, v);
      values<E, N>(a.dy, dy + d, g);
      if (a.w) values<E, N>(a.w, d, w);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float e = v[j] - m, gw = a.w ? g[j] * w[j] : g[j];
        u[0] += e, u[1] += e * e, u[2] += gw, u[3] += gw * e;
      }
    }
    sums.sum(u);
    const float c = u[0] * inv, r = inv_rms(fmaxf(u[1] * inv - c * c, 0.0f), a.eps);
    const float s1 = u[2] * inv, s2 = r * (u[3] * inv - c * s1);
    const bool first = row == (int)blockIdx.x;
    for (int d = N * threadIdx.x; d < a.W; d += N * kBlock) {
      float rd[N], dw[N] = {}, db[N] = {};
      values<E, N>(a.x, x + d, v);
      values<E, N>(a.dy, dy + d, g);
      if (a.w) values<E, N>(a.w, d, w);
      if (a.dres) values<E, N>(a.dres, row * a.drs + d, rd);
      if (wanted && !first) values<float, N>(mine, d, dw), values<float, N>(mine, a.W + d, db);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float n = (v[j] - m - c) * r;
        dw[j] += g[j] * n, db[j] += g[j];
        v[j] = r * ((a.w ? g[j] * w[j] : g[j]) - s1 - n * s2) + (a.dres ? rd[j] : 0.0f);
      }
      put<E, N>(a.dx, row * a.dxs + d, v);
      if (wanted) put<float, N>(mine, d, dw), put<float, N>(mine, a.W + d, db);
    }
  }
}

// dw and db: the workgroups' sums added up in order, 16 columns a workgroup, 64 sums at a time.
template <class E>
__global__ __launch_bounds__(1024) void k_layer_norm_dw(const LayerNormArgs a, int n, const float* part) {
  __shared__ float red[64][17];
  const int col = blockIdx.x * 16 + threadIdx.x % 16, r = threadIdx.x / 16;  // of dw, then of db
  float t = 0.0f;
  if (col < 2 * a.W)
#pragma unroll 4
    for (int i = r; i < n; i += 64) t += part[(int64_t)i * 2 * a.W + col];
  red[r][threadIdx.x % 16] = t;
  __syncthreads();
  if (r != 0 || col >= 2 * a.W) return;
  E* out = (E*)(col < a.W ? a.dw : a.db);
  if (!out) return;
  t = 0.0f;
  for (int i = 0; i < 64; ++i) t += red[i][threadIdx.x];
  out[col < a.W ? col : col - a.W] = (E)t;
}

// Workgroups of the gradient: each leaves its sums, so they are bounded.
int bwd_blocks(const LayerNormArgs& a, int rows_wg) {
  const int64_t most = std::max<int64_t>(kCUs, std::min<int64_t>(4 * kCUs, ((int64_t)1 << 21) / a.W));
  return (int)std::min<int64_t>(((int64_t)a.rows + rows_wg - 1) / rows_wg, most);
}

template <class E, int TPR, int NV>
void forward(const LayerNormArgs& a, hipStream_t s) {
  constexpr int kRows = Shape<TPR>::kRows;
  const int n = (int)std::min<int64_t>(((int64_t)a.rows + kRows - 1) / kRows, 16 * kCUs);
  k_layer_norm<E, TPR, NV><<<n, Shape<TPR>::kThreads, 0, s>>>(a);
}
template <class E>
void forward(const LayerNormArgs& a, hipStream_t s) {
  const int W = a.W;
  if (!a.vec || W > 16384)
    (a.vec ? k_layer_norm_any<E, 8> : k_layer_norm_any<E, 1>)<<<std::min(a.rows, 16 * kCUs), kBlock, 0, s>>>(a);
  else if (W <= 32)
    forward<E, 4, 1>(a, s);
  else if (W <= 64)
    forward<E, 8, 1>(a, s);
  else if (W <= 128)
    forward<E, 16, 1>(a, s);
  else if (W <= 256)
    forward<E, 32, 1>(a, s);
  else if (W <= 512)
    forward<E, 64, 1>(a, s);
  else if (W <= 1024)
    forward<E, 64, 2>(a, s);
  else if (W <= 2048)
    forward<E, 256, 1>(a, s);
  else if (W <= 4096)
    forward<E, 256, 2>(a, s);
  else if (W <= 8192)
    forward<E, 256, 4>(a, s);
  else
    forward<E, 1024, 2>(a, s);
}

template <class E, int TPR, int NV>
int backward(const LayerNormArgs& a, float* part, hipStream_t s) {
  const int n = bwd_blocks(a, Shape<TPR>::kRows);
  if (n) k_layer_norm_bwd<E, TPR, NV><<<n, Shape<TPR>::kThreads, 0, s>>>(a, part);
  return n;
}
template <class E>
void backward(const LayerNormArgs& a, float* part, hipStream_t s) {
  const int W = a.W;
  int n;
  if (!a.vec || W > 8192) {
    n = bwd_blocks(a, 1);
    if (n) (a.vec ? k_layer_norm_bwd_any<E, 8> : k_layer_norm_bwd_any<E, 1>)<<<n, kBlock, 0, s>>>(a, part);
  } else if (W <= 32)
    n = backward<E, 4, 1>(a, part, s);
  else if (W <= 64)
    n = backward<E, 8, 1>(a, part, s);
  else if (W <= 128)
    n = backward<E, 16, 1>(a, part, s);
  else if (W <= 256)
    n = backward<E, 32, 1>(a, part, s);
  else if (W <= 512)
    n = backward<E, 64, 1>(a, part, s);
  else if (W <= 1024)
    n = backward<E, 64, 2>(a, part, s);
  else if (W <= 2048)
    n = backward<E, 256, 1>(a, part, s);
  else if (W <= 4096)
    n = backward<E, 256, 2>(a, part, s);
  else
    n = backward<E, 512, 2>(a, part, s);
  if (a.dw || a.db) k_layer_norm_dw<E><<<(2 * W + 15) / 16, 1024, 0, s>>>(a, n, part);
}

}  // namespace

hipError_t launch_layer_norm_fwd(const LayerNormArgs& a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  if (a.dtype == kF32) forward<float>(a, s);
  if (a.dtype == kF16) forward<_Float16>(a, s);
  if (a.dtype == kBF16) forward<__bf16>(a, s);
  return hipGetLastError();
}

// (From the sizes alone: no call has more workgroups than one with a row each.)
int64_t layer_norm_bwd_bytes(const LayerNormArgs& a) { return (int64_t)bwd_blocks(a, 1) * 2 * a.W * 4; }

hipError_t launch_layer_norm_bwd(const LayerNormArgs& a, void* ws, hipStream_t s) {
  if (a.dtype == kF32) backward<float>(a, (float*)ws, s);
  if (a.dtype == kF16) backward<_Float16>(a, (float*)ws, s);
  if (a.dtype == kBF16) backward<__bf16>(a, (float*)ws, s);
  return hipGetLastError();
}

}  // namespace pnerf
