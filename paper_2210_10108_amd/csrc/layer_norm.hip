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

// Sums of N values over the workgroup's NW wavefronts, in all threads.
template <int N, int NW>
__device__ __forceinline__ void block_sum(float (&v)[N], float* red) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = row_sum<64>(v[i]);
  if (NW == 1) return;
  __syncthreads();
  if (lane == 0)
#pragma unroll
    for (int i = 0; i < N; ++i) red[wave * N + i] = v[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    v[i] = 0.0f;
#pragma unroll
    for (int w = 0; w < NW; ++w) v[i] += red[w * N + i];
  }
}

// Any width, stride and alignment: a workgroup a row, element by element, the row
// read again for each step.
template <class E>
__global__ __launch_bounds__(kBlock) void k_layer_norm_any(const LayerNormArgs a) {
  __shared__ float red[8];
  const float inv = 1.0f / a.W;
  for (int row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const E* x = (const E*)a.x + row * a.xs;
    float t[2] = {0.0f, 0.0f};
    for (int d = threadIdx.x; d < a.W; d += kBlock) t[0] += (float)x[d];
    block_sum<2, 4>(t, red);
    const float m = t[0] * inv;
    t[0] = t[1] = 0.0f;
    for (int d = threadIdx.x; d < a.W; d += kBlock) {
      const float v = (float)x[d] - m;
      t[0] += v, t[1] += v * v;
    }
    block_sum<2, 4>(t, red);
    const float c = t[0] * inv, r = inv_rms(fmaxf(t[1] * inv - c * c, 0.0f), a.eps);
    E* y = (E*)a.y + row * a.ys;
    for (int d = threadIdx.x; d < a.W; d += kBlock) {
      const float w = a.w ? (float)((const E*)a.w)[d] : 1.0f, b = a.b ? (float)((const E*)a.b)[d] : 0.0f;
      y[d] = (E)(((float)x[d] - m - c) * r * w + b);
    }
  }
}

// Each workgroup leaves its sums of dw and db, [workgroup][2][W].
template <class E>
__global__ __launch_bounds__(kBlock) void k_layer_norm_bwd_any(const LayerNormArgs a, float* part) {
  __shared__ float red[16];
  const float inv = 1.0f / a.W;
  const bool sums = a.dw || a.db;
  float* mine = part + (int64_t)blockIdx.x * 2 * a.W;
  for (int row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const E *x = (const E*)a.x + row * a.xs, *dy = (const E*)a.dy + row * a.dys;
    const E* res = a.dres ? (const E*)a.dres + row * a.drs : nullptr;
    float t[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int d = threadIdx.x; d < a.W; d += kBlock) t[0] += (float)x[d];
    block_sum<4, 4>(t, red);
    const float m = t[0] * inv;
    t[0] = t[1] = t[2] = t[3] = 0.0f;
    for (int d = threadIdx.x; d < a.W; d += kBlock) {
      const float v = (float)x[d] - m, g = (float)dy[d] * (a.w ? (float)((const E*)a.w)[d] : 1.0f);
      t[0] += v, t[1] += v * v, t[2] += g, t[3] += g * v;
    }
    block_sum<4, 4>(t, red);
    const float c = t[0] * inv, r = inv_rms(fmaxf(t[1] * inv - c * c, 0.0f), a.eps);
    const float s1 = t[2] * inv, s2 = r * (t[3] * inv - c * s1);
    E* dx = (E*)a.dx + row * a.dxs;
    for (int d = threadIdx.x; d < a.W; d += kBlock) {
      const float dyd = (float)dy[d], n = ((float)x[d] - m - c) * r;
      const float g = dyd * (a.w ? (float)((const E*)a.w)[d] : 1.0f);
      const float rd = res ? (float)res[d] : 0.0f;
      dx[d] = (E)(r * (g - s1 - n * s2) + rd);
      if (sums) {
        const bool first = row == (int)blockIdx.x;
        mine[d] = (first ? 0.0f : mine[d]) + dyd * n;
        mine[a.W + d] = (first ? 0.0f : mine[a.W + d]) + dyd;
      }
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
int bwd_blocks(const LayerNormArgs& a) {
  const int64_t most = std::max<int64_t>(kCUs, std::min<int64_t>(4 * kCUs, ((int64_t)1 << 21) / a.W));
  return (int)std::min<int64_t>(a.rows, most);
}

template <class E>
void forward(const LayerNormArgs& a, hipStream_t s) {
  k_layer_norm_any<E><<<std::min(a.rows, 16 * kCUs), kBlock, 0, s>>>(a);
}
template <class E>
void backward(const LayerNormArgs& a, float* part, hipStream_t s) {
  const int n = bwd_blocks(a);
  if (n) k_layer_norm_bwd_any<E><<<n, kBlock, 0, s>>>(a, part);
  if (a.dw || a.db) k_layer_norm_dw<E><<<(2 * a.W + 15) / 16, 1024, 0, s>>>(a, n, part);
}

}  // namespace

hipError_t launch_layer_norm_fwd(const LayerNormArgs& a, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  if (a.dtype == kF32) forward<float>(a, s);
  if (a.dtype == kF16) forward<_Float16>(a, s);
  if (a.dtype == kBF16) forward<__bf16>(a, s);
  return hipGetLastError();
}

int64_t layer_norm_bwd_bytes(const LayerNormArgs& a) { return (int64_t)bwd_blocks(a) * 2 * a.W * 4; }

hipError_t launch_layer_norm_bwd(const LayerNormArgs& a, void* ws, hipStream_t s) {
  if (a.dtype == kF32) backward<float>(a, (float*)ws, s);
  if (a.dtype == kF16) backward<_Float16>(a, (float*)ws, s);
  if (a.dtype == kBF16) backward<__bf16>(a, (float*)ws, s);
  return hipGetLastError();
}

}  // namespace pnerf
