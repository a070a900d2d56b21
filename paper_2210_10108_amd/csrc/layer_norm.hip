// Layer norm of rows: y = (x - mean) / sqrt(var + eps) w + b, and its gradient
//   dx = r (g - mean g - n mean(g n)) + dres,  dw = sum_rows dy n,  db = sum_rows dy
// with g = dy w, n = (x - mean) r, r = 1 / sqrt(var + eps).
//
// A stream, bound by memory: x in and y out, x, dy (and dres) in and dx out (16384 x 1024
// bf16: 13.9 us or 4.8 TB/s forward, 24.7 us or 4.1 TB/s backward with its sums; 8192 x 3000
// f32: 5.1 and 5.1 TB/s; a copy reaches 5.2).
//
// Sums are float32.  A row's mean is taken in two steps, m = x_0 + mean(x - x_0) and then
// c = mean(x - m), and var = mean (x - m)^2 - c^2: rows whose mean is large beside their
// spread lose nothing but what x itself was rounded to, equal elements give 0 exactly at
// any size, and the gradient makes its statistics again from the row that it reads anyway.
// Where the sum of squares passes float32's range, r and n are 0.
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

// Eight elements from or to an address that is aligned to its elements alone (the
// hardware takes it in one access as well), and n < 8 of them.
template <class E>
struct Odd {
  struct __attribute__((packed, aligned(sizeof(E)))) Eight {
    uint32_t w[2 * sizeof(E)];
  };
  static __device__ __forceinline__ typename Elem<E>::Raw raw(const E* p, int n) {
    typename Elem<E>::Raw r;
    if (n >= 8) {
      const Eight x = *reinterpret_cast<const Eight*>(p);
      __builtin_memcpy(&r, &x, sizeof(r));
      return r;
    }
    alignas(16) E e[8] = {};
#pragma unroll
    for (int j = 0; j < 7; ++j)
      if (j < n) e[j] = p[j];
    __builtin_memcpy(&r, e, sizeof(r));
    return r;
  }
  static __device__ __forceinline__ void store(E* p, const float (&v)[8], int n) {
    if (n >= 8) {
      alignas(16) E e[8];
      Elem<E>::store(e, v);
      Eight x;
      __builtin_memcpy(&x, e, sizeof(x));
      *reinterpret_cast<Eight*>(p) = x;
      return;
    }
#pragma unroll
    for (int j = 0; j < 7; ++j)
      if (j < n) p[j] = (E)v[j];
  }
};
// The n (1 or more) elements of a row from p on, at most 8.  ODD: any width and
// alignment; otherwise n >= 8 and p is on 16 bytes.
template <class E, bool ODD>
__device__ __forceinline__ typename Elem<E>::Raw raw8(const void* p, int64_t at, int n) {
  if (ODD) return Odd<E>::raw((const E*)p + at, n);
  return Elem<E>::raw((const E*)p + at);
}
template <class E, bool ODD>
__device__ __forceinline__ void store8(void* p, int64_t at, const float (&v)[8], int n) {
  if (ODD)
    Odd<E>::store((E*)p + at, v, n);
  else
    Elem<E>::store((E*)p + at, v);
}

// Statistics of a row: c = mean d and r, from the sums of d = x - m and d^2.  Where those
// pass float32's range (far) c and r are 0, and n is the sum of 0 x in all places: 0, or
// NaN where the row itself holds one or an infinity.
struct Stats {
  float c, r;
  bool far;
  __device__ __forceinline__ Stats(float sum, float squares, float inv, float eps)
      : c(sum * inv), far(!(squares < INFINITY)) {
    r = inv_rms(fmaxf(squares * inv - c * c, 0.0f), eps);
    if (far) c = r = 0.0f;
  }
};

// The sum of 0 x over a row (NULL: 0), which is read again for it.
template <class E, int TPR>
__device__ __forceinline__ float zeros_of(RowSums<TPR>& sums, const E* row, int W) {
  float z[1] = {0.0f};
  if (row)
#pragma unroll 1
    for (int d = threadIdx.x % TPR; d < W; d += TPR) z[0] += 0.0f * (float)row[d];
  sums.sum(z);
  return z[0];
}

// NV groups of 8 elements of a row as they are loaded; zeros past its end.
template <class E, int TPR, int NV, bool ODD>
struct Group {
  typename Elem<E>::Raw raw[NV];
  E head;  // the row's first element, where other wavefronts have it
  __device__ __forceinline__ void load_row(const void* p, int64_t at, int W) {
    load(p, at, W);
    if (TPR > 64) head = ((const E*)p)[at];
  }
  // The first element; v: of this thread's first group.
  __device__ __forceinline__ float first(float v) const {
    if (TPR > 64) return (float)head;
    if (TPR == 64) return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v)));
    return __shfl(v, (int)(threadIdx.x & 63) / TPR * TPR);
  }
  __device__ __forceinline__ void load(const void* p, int64_t at, int W) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int d = 8 * ((int)(threadIdx.x % TPR) + v * TPR);
      if (d < W) raw[v] = raw8<E, ODD>(p, at + d, W - d);
    }
  }
};

template <int NV>
__device__ __forceinline__ void fill(float (&v)[NV][8], float x) {
#pragma unroll
  for (int k = 0; k < NV; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) v[k][j] = x;
}

template <class E, int TPR, int NV, bool ODD>
__global__ __launch_bounds__(Shape<TPR>::kThreads) void k_layer_norm(const LayerNormArgs a) {
  constexpr int kRows = Shape<TPR>::kRows;
  __shared__ float lds[TPR > 64 ? TPR / 8 : 1];
  RowSums<TPR> sums(lds);
  const int group = threadIdx.x / TPR;
  const float inv = 1.0f / a.W;
  // x where the row has an element j of group k, 0 past its end (groups are whole but for ODD)
  auto here = [&](int k, int j, float x) { return 8 * ((int)(threadIdx.x % TPR) + k * TPR) + (ODD ? j : 0) < a.W ? x : 0.0f; };
  Group<E, TPR, NV, ODD> x = {}, w = {}, b = {};
  if (a.w) w.load(a.w, 0, a.W);
  if (a.b) b.load(a.b, 0, a.W);
  int64_t row = (int64_t)blockIdx.x * kRows + group;
  const int64_t step = (int64_t)gridDim.x * kRows;
  if (row < a.rows) x.load_row(a.x, row * a.xs, a.W);
  for (; row - group < a.rows; row += step) {
    float v[NV][8], t[1] = {0.0f}, u[2] = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < NV; ++k) Elem<E>::unpack(x.raw[k], v[k]);
    const float x0 = x.first(v[0][0]);
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int j = 0; j < 8; ++j) t[0] += v[k][j] - here(k, j, x0);
    if (row + step < a.rows) x.load_row(a.x, (row + step) * a.xs, a.W);
    sums.sum(t);
    const float m = x0 + t[0] * inv;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[k][j] -= here(k, j, m);
        u[0] += v[k][j], u[1] += v[k][j] * v[k][j];
      }
    }
    sums.sum(u);
    const Stats st(u[0], u[1], inv, a.eps);
    if (__any(st.far)) {
      const float n = zeros_of(sums, row < a.rows ? (const E*)a.x + row * a.xs : nullptr, a.W);
      if (st.far) fill(v, n);
    }
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
        const float n = (v[k][j] - st.c) * st.r;
        v[k][j] = (a.w ? n * wk[j] : n) + (a.b ? bk[j] : 0.0f);
      }
      store8<E, ODD>(a.y, row * a.ys + d, v[k], a.W - d);
    }
  }
}

// Each workgroup leaves its sums of dw and db, [workgroup][2][W].
template <class E, int TPR, int NV, bool ODD>
__global__ __launch_bounds__(Shape<TPR>::kThreads) void k_layer_norm_bwd(const LayerNormArgs a, float* part) {
  constexpr int kRows = Shape<TPR>::kRows;
  __shared__ float lds[TPR > 64 ? TPR / 8 : 1];
  RowSums<TPR> sums(lds);
  const int group = threadIdx.x / TPR;
  const float inv = 1.0f / a.W;
  auto here = [&](int k, int j, float x) { return 8 * ((int)(threadIdx.x % TPR) + k * TPR) + (ODD ? j : 0) < a.W ? x : 0.0f; };
  Group<E, TPR, NV, ODD> x = {}, dy = {}, res = {}, w = {};
  if (a.w) w.load(a.w, 0, a.W);
  int64_t row = (int64_t)blockIdx.x * kRows + group;
  const int64_t step = (int64_t)gridDim.x * kRows;
  auto fetch = [&](int64_t at) {
    if (at >= a.rows) return;
    x.load_row(a.x, at * a.xs, a.W);
    dy.load(a.dy, at * a.dys, a.W);
  };
  fetch(row);
  float dw[NV][8] = {}, db[NV][8] = {};
  for (; row - group < a.rows; row += step) {
    float v[NV][8], g[NV][8], t[1] = {0.0f}, u[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const bool in = row < a.rows;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      Elem<E>::unpack(x.raw[k], v[k]);
      Elem<E>::unpack(dy.raw[k], g[k]);
    }
    const float x0 = x.first(v[0][0]);
#pragma unroll
    for (int k = 0; k < NV; ++k) {
#pragma unroll
      for (int j = 0; j < 8; ++j) t[0] += v[k][j] - here(k, j, x0);
    }
    if (a.dres && in) res.load(a.dres, row * a.drs, a.W);
    fetch(row + step);
    sums.sum(t);
    const float m = x0 + t[0] * inv;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      float wk[8];
      Elem<E>::unpack(w.raw[k], wk);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[k][j] -= here(k, j, m);
        const float gw = a.w ? g[k][j] * wk[j] : g[k][j];
        u[0] += v[k][j], u[1] += v[k][j] * v[k][j];
        u[2] += gw, u[3] += gw * v[k][j];
      }
    }
    sums.sum(u);
    const Stats st(u[0], u[1], inv, a.eps);
    const float c = st.c, r = st.r, s1 = u[2] * inv, s2 = st.far ? 0.0f : r * (u[3] * inv - c * s1);
    if (__any(st.far)) {
      const float n = zeros_of(sums, in ? (const E*)a.x + row * a.xs : nullptr, a.W);
      if (st.far) fill(v, n);
    }
    if (!in) continue;  // (what the sums of such a row are does not matter)
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
      store8<E, ODD>(a.dx, row * a.dxs + d, v[k], a.W - d);
    }
  }
  if (!a.dw && !a.db) return;
  part += (int64_t)blockIdx.x * 2 * a.W;
  if constexpr (kRows == 1) {
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int d = 8 * ((int)threadIdx.x + k * TPR);
      if (d >= a.W) continue;
      store8<float, ODD>(part, d, dw[k], a.W - d);
      store8<float, ODD>(part, a.W + d, db[k], a.W - d);
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

// Rows wider than the registers hold: a workgroup a row, which is read again for each
// step (from a cache, mostly).
template <class E>
__global__ __launch_bounds__(kBlock) void k_layer_norm_wide(const LayerNormArgs a) {
  __shared__ float lds[kBlock / 8];
  RowSums<kBlock> sums(lds);
  const float inv = 1.0f / a.W;
  auto values = [&](const void* p, int64_t at, int d, float (&v)[8]) {
    Elem<E>::unpack(raw8<E, true>(p, at + d, a.W - d), v);
  };
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const int64_t x = row * a.xs;
    const float x0 = (float)((const E*)a.x)[x];
    float t[2] = {0.0f, 0.0f}, u[2] = {0.0f, 0.0f}, v[8];
    for (int d = 8 * threadIdx.x; d < a.W; d += 8 * kBlock) {
      values(a.x, x, d, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) t[0] += d + j < a.W ? v[j] - x0 : 0.0f, t[1] += 0.0f * v[j];
    }
    sums.sum(t);
    const float m = x0 + t[0] * inv;
    for (int d = 8 * threadIdx.x; d < a.W; d += 8 * kBlock) {
      values(a.x, x, d, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float e = d + j < a.W ? v[j] - m : 0.0f;
        u[0] += e, u[1] += e * e;
      }
    }
    sums.sum(u);
    const Stats st(u[0], u[1], inv, a.eps);
    for (int d = 8 * threadIdx.x; d < a.W; d += 8 * kBlock) {
      float w[8], b[8];
      values(a.x, x, d, v);
      if (a.w) values(a.w, 0, d, w);
      if (a.b) values(a.b, 0, d, b);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float n = st.far ? t[1] : (v[j] - m - st.c) * st.r;
        v[j] = (a.w ? n * w[j] : n) + (a.b ? b[j] : 0.0f);
      }
      store8<E, true>(a.y, row * a.ys + d, v, a.W - d);
    }
  }
}

// The same for the gradient.  The sums of dw and db are in registers, NV groups of 8
// columns a thread, where those hold them; NV = 0: in the workgroup's place in memory,
// where every row adds to them.
template <class E, int NV>
__global__ __launch_bounds__(1024) void k_layer_norm_bwd_wide(const LayerNormArgs a, float* part) {
  constexpr int T = 1024;
  __shared__ float lds[T / 8];
  RowSums<T> sums(lds);
  const float inv = 1.0f / a.W;
  float* mine = part + (int64_t)blockIdx.x * 2 * a.W;
  float dw[NV ? NV : 1][8] = {}, db[NV ? NV : 1][8] = {};
  auto values = [&](const void* p, int64_t at, int d, float (&v)[8]) {
    Elem<E>::unpack(raw8<E, true>(p, at + d, a.W - d), v);
  };
  auto groups = [&](auto f) {  // f(d, k) for this thread's groups
    if constexpr (NV > 0) {
#pragma unroll
      for (int k = 0; k < NV; ++k)
        if (const int d = 8 * ((int)threadIdx.x + k * T); d < a.W) f(d, k);
    } else {
      for (int d = 8 * threadIdx.x; d < a.W; d += 8 * T) f(d, 0);
    }
  };
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const int64_t x = row * a.xs, dy = row * a.dys;
    const float x0 = (float)((const E*)a.x)[x];
    float t[2] = {0.0f, 0.0f}, u[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    groups([&](int d, int) {
      float v[8];
      values(a.x, x, d, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) t[0] += d + j < a.W ? v[j] - x0 : 0.0f, t[1] += 0.0f * v[j];
    });
    sums.sum(t);
    const float m = x0 + t[0] * inv;
    groups([&](int d, int) {
      float v[8], g[8], w[8];
      values(a.x, x, d, v);
      values(a.dy, dy, d, g);
      if (a.w) values(a.w, 0, d, w);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float e = d + j < a.W ? v[j] - m : 0.0f, gw = a.w ? g[j] * w[j] : g[j];
        u[0] += e, u[1] += e * e, u[2] += gw, u[3] += gw * e;
      }
    });
    sums.sum(u);
    const Stats st(u[0], u[1], inv, a.eps);
    const float c = st.c, r = st.r, s1 = u[2] * inv, s2 = st.far ? 0.0f : r * (u[3] * inv - c * s1);
    groups([&](int d, int k) {
      float v[8], g[8], w[8], rd[8];
      values(a.x, x, d, v);
      values(a.dy, dy, d, g);
      if (a.w) values(a.w, 0, d, w);
      if (a.dres) values(a.dres, row * a.drs, d, rd);
      if (NV == 0) {
        const bool first = row == (int)blockIdx.x;
#pragma unroll
        for (int j = 0; j < 8; ++j) dw[0][j] = db[0][j] = 0.0f;
        if (!first) {
          Elem<float>::unpack(raw8<float, true>(mine, d, a.W - d), dw[0]);
          Elem<float>::unpack(raw8<float, true>(mine, a.W + d, a.W - d), db[0]);
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float n = st.far ? t[1] : (v[j] - m - c) * r;
        dw[k][j] += g[j] * n, db[k][j] += g[j];
        v[j] = r * ((a.w ? g[j] * w[j] : g[j]) - s1 - n * s2) + (a.dres ? rd[j] : 0.0f);
      }
      store8<E, true>(a.dx, row * a.dxs + d, v, a.W - d);
      if (NV == 0) {
        store8<float, true>(mine, d, dw[0], a.W - d);
        store8<float, true>(mine, a.W + d, db[0], a.W - d);
      }
    });
  }
  if (NV > 0 && (a.dw || a.db))
    groups([&](int d, int k) {
      store8<float, true>(mine, d, dw[k], a.W - d);
      store8<float, true>(mine, a.W + d, db[k], a.W - d);
    });
}

// dw and db: the workgroups' sums added up in order, kCols columns a workgroup, kSums sums
// at a time.
constexpr int kCols = 32, kSums = 32;
template <class E>
__global__ __launch_bounds__(kCols * kSums) void k_layer_norm_dw(const LayerNormArgs a, int n, const float* part) {
  __shared__ float red[kSums][kCols + 1];
  const int c = threadIdx.x % kCols, r = threadIdx.x / kCols;
  const int64_t col = (int64_t)blockIdx.x * kCols + c;  // of dw, then of db
  float t = 0.0f;
  if (col < 2 * a.W)
#pragma unroll 8
    for (int i = r; i < n; i += kSums) t += part[(int64_t)i * 2 * a.W + col];
  red[r][c] = t;
  __syncthreads();
  if (r != 0 || col >= 2 * a.W) return;
  E* out = (E*)(col < a.W ? a.dw : a.db);
  if (!out) return;
  t = 0.0f;
#pragma unroll
  for (int i = 0; i < kSums; ++i) t += red[i][c];
  out[col < a.W ? col : col - a.W] = (E)t;
}

// Workgroups of the gradient: each leaves its sums, so they are bounded; and no more
// than run at once, `per_cu` a compute unit by their registers (16384 x 1024, bf16: 25 us
// with 2 or 3, 28 with 4; 8192 x 3000, f32: 57 with 2, 69 with the 699 that the sums allow.
// 16381 x 2048, bf16, forward and backward: 82 us with 4, 87 with 2).
int bwd_blocks(const LayerNormArgs& a, int rows_wg, int per_cu) {
  const int64_t most = std::max<int64_t>(kCUs, std::min<int64_t>(per_cu * kCUs, ((int64_t)1 << 21) / a.W));
  return (int)std::min<int64_t>(((int64_t)a.rows + rows_wg - 1) / rows_wg, most);
}

// Threads of a row: the fewest that hold it in one group each up to a wavefront, two
// groups of a wavefront up to 1024 (16384 x 1024, bf16: 13.5 us, backward 25; a workgroup
// of 256 with barriers, half of it idle: 17.4 and 35), then a workgroup, with few groups a
// thread rather than many threads (8192 x 3000, bf16: two groups of 256 threads 19 and 40
// us, one of 512 21 and 48; 8192 x 8192: four groups of 256 42 us, one of 1024 68).
template <class E, int TPR, int NV>
void forward(const LayerNormArgs& a, hipStream_t s) {
  constexpr int kRows = Shape<TPR>::kRows;
  const int n = (int)std::min<int64_t>(((int64_t)a.rows + kRows - 1) / kRows, 16 * kCUs);
  (a.vec ? k_layer_norm<E, TPR, NV, false> : k_layer_norm<E, TPR, NV, true>)<<<n, Shape<TPR>::kThreads, 0, s>>>(a);
}
template <class E>
void forward(const LayerNormArgs& a, hipStream_t s) {
  const int W = a.W;
  if (W <= 32) return forward<E, 4, 1>(a, s);
  if (W <= 64) return forward<E, 8, 1>(a, s);
  if (W <= 128) return forward<E, 16, 1>(a, s);
  if (W <= 256) return forward<E, 32, 1>(a, s);
  if (W <= 512) return forward<E, 64, 1>(a, s);
  if (W <= 1024) return forward<E, 64, 2>(a, s);
  if (W <= 2048) return forward<E, 256, 1>(a, s);
  if (W <= 4096) return forward<E, 256, 2>(a, s);
  if (W <= 8192) return forward<E, 256, 4>(a, s);
  if (W <= 16384) return forward<E, 1024, 2>(a, s);
  k_layer_norm_wide<E><<<std::min(a.rows, 16 * kCUs), kBlock, 0, s>>>(a);
}

template <class E, int TPR, int NV>
int backward(const LayerNormArgs& a, float* part, hipStream_t s) {
  constexpr int kPerCu = NV == 2 ? (sizeof(E) == 4 ? 2 : 3) : 4;
  const int n = bwd_blocks(a, Shape<TPR>::kRows, kPerCu);
  if (n) (a.vec ? k_layer_norm_bwd<E, TPR, NV, false> : k_layer_norm_bwd<E, TPR, NV, true>)<<<n, Shape<TPR>::kThreads, 0, s>>>(a, part);
  return n;
}
template <class E, int NV>
int backward_wide(const LayerNormArgs& a, float* part, hipStream_t s) {
  const int n = bwd_blocks(a, 1, 1);
  if (n) k_layer_norm_bwd_wide<E, NV><<<n, 1024, 0, s>>>(a, part);
  return n;
}
// Workgroups that ran, each with its sums.
template <class E>
int backward_rows(const LayerNormArgs& a, float* part, hipStream_t s) {
  const int W = a.W;
  if (W <= 32) return backward<E, 4, 1>(a, part, s);
  if (W <= 64) return backward<E, 8, 1>(a, part, s);
  if (W <= 128) return backward<E, 16, 1>(a, part, s);
  if (W <= 256) return backward<E, 32, 1>(a, part, s);
  if (W <= 512) return backward<E, 64, 1>(a, part, s);
  if (W <= 1024) return backward<E, 64, 2>(a, part, s);
  if (W <= 2048) return backward<E, 256, 1>(a, part, s);
  if (W <= 4096) return backward<E, 256, 2>(a, part, s);
  if (W <= 8192) return backward<E, 512, 2>(a, part, s);
  if (W <= 16384) return backward_wide<E, 2>(a, part, s);
  return backward_wide<E, 0>(a, part, s);
}
template <class E>
void backward(const LayerNormArgs& a, float* part, hipStream_t s) {
  const int n = backward_rows<E>(a, part, s);
  if (a.dw || a.db) k_layer_norm_dw<E><<<(2 * a.W + kCols - 1) / kCols, kCols * kSums, 0, s>>>(a, n, part);
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
int64_t layer_norm_bwd_bytes(const LayerNormArgs& a) { return (int64_t)bwd_blocks(a, 1, 4) * 2 * a.W * 4; }

hipError_t launch_layer_norm_bwd(const LayerNormArgs& a, void* ws, hipStream_t s) {
  if (a.dtype == kF32) backward<float>(a, (float*)ws, s);
  if (a.dtype == kF16) backward<_Float16>(a, (float*)ws, s);
  if (a.dtype == kBF16) backward<__bf16>(a, (float*)ws, s);
  return hipGetLastError();
}

}  // namespace pnerf
