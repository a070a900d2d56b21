// The norm of every query and key head and its position rotation in one pass:
//   n = x w / sqrt(mean x^2 + eps),  y = n with its pairs turned by the position's angle
// and its gradient.  A pure stream: every element is read once and written
// once, so memory bounds it; sums and the rotation are float32, rounded once.
//
// A head of D elements is a row of LR lanes, 8 consecutive elements each
// (16-byte accesses), LR the power of two that holds D / 8: the sum of squares
// is log2 LR exchanges, and a rotation partner at distance R / 2 is the same
// element of another lane of the row.  A group of LR lanes takes one position
// and some of its heads, with the position's cosines and sines in registers;
// neighbouring groups take neighbouring heads.
#define PNERF_LAYERS_DEVICE
#include "norm_common.h"

namespace pnerf {
namespace {

template <class E, int LR, Pairs P>
__global__ __launch_bounds__(kBlock) void k_norm_fwd(const NormArgs a, int blocks0, int blocks1) {
  constexpr int NG = kBlock / LR;
  const bool second = (int)blockIdx.x >= blocks0;
  const NormSide& x = second ? a.side[1] : a.side[0];
  const int blk = second ? blockIdx.x - blocks0 : blockIdx.x, blocks = second ? blocks1 : blocks0;
  const int d = 8 * (threadIdx.x % LR);
  // what lies past the rotated part passes as it is (see rotate_axes.hip)
  const bool col = d < a.D, turned = P == kHalf || d < a.R;
  float w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = 1.0f;
  if (col && x.w) load<E>((const E*)x.w + d, w);
  const float inv_d = 1.0f / a.D;
  Walk at(x, (int64_t)blk * NG + threadIdx.x / LR, (int64_t)blocks * NG);
  typename Elem<E>::Raw raw = {};
  int pos = 0;
  auto fetch = [&] {
    if (!at.on() || !col) return;
    raw = Elem<E>::raw((const E*)x.x + at.row * x.xs[0] + at.head * x.xs[1] + d);
    if (a.R) pos = x.pos[at.row];
  };
  fetch();
  // every lane of a wavefront makes the same number of rounds: the exchanges need them all
  while (__any(at.on())) {
    float v[8], p[8], c[8], s[8];
    const bool here = at.on() && col;
    Elem<E>::unpack(raw, v);
    angles<P>(a, pos, here ? d : a.R, c, s);
    E* y = (E*)x.y + at.row * x.ys[0] + at.head * x.ys[1] + d;
    at.next();
    fetch();
    float q = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) q += here ? v[j] * v[j] : 0.0f;
    const float r = inv_rms(row_sum<LR>(q) * inv_d, a.eps);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= r * w[j];
    partners<P, LR>(a, d, v, p);
    if (turned)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = v[j] * c[j] + p[j] * s[j];
    if (here) Elem<E>::store(y, v);
  }
}

// Each workgroup leaves its sum of dw.
template <class E, int LR, Pairs P>
__global__ __launch_bounds__(kBlock) void k_norm_bwd(const NormArgs a, int blocks0, int blocks1, float* part) {
  constexpr int NG = kBlock / LR;
  __shared__ float red[NG][8 * LR];
  const bool second = (int)blockIdx.x >= blocks0;
  const NormSide& x = second ? a.side[1] : a.side[0];
  const int blk = second ? blockIdx.x - blocks0 : blockIdx.x, blocks = second ? blocks1 : blocks0;
  const int grp = threadIdx.x / LR, d = 8 * (threadIdx.x % LR);
  const bool col = d < a.D, turned = P == kHalf || d < a.R;
  float w[8], dw[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = 1.0f, dw[i] = 0.0f;
  if (col && x.w) load<E>((const E*)x.w + d, w);
  const float inv_d = 1.0f / a.D;
  Walk at(x, (int64_t)blk * NG + grp, (int64_t)blocks * NG);
  typename Elem<E>::Raw raw_x = {}, raw_g = {};
  int pos = 0;
  auto fetch = [&] {
    if (!at.on() || !col) return;
    raw_x = Elem<E>::raw((const E*)x.x + at.row * x.xs[0] + at.head * x.xs[1] + d);
    raw_g = Elem<E>::raw((const E*)x.dy + at.row * x.dys[0] + at.head * x.dys[1] + d);
    if (a.R) pos = x.pos[at.row];
  };
  fetch();
  while (__any(at.on())) {
    float v[8], g[8], p[8], c[8], s[8];
    const bool here = at.on() && col;
    Elem<E>::unpack(raw_x, v);
    Elem<E>::unpack(raw_g, g);
    angles<P>(a, pos, here ? d : a.R, c, s);
    E* dx = (E*)x.dx + at.row * x.dxs[0] + at.head * x.dxs[1] + d;
    at.next();
    fetch();
    partners<P, LR>(a, d, g, p);
    float q = 0.0f, dot = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      g[j] = !here ? 0.0f : turned ? g[j] * c[j] - p[j] * s[j] : g[j];  // turned back
      v[j] = here ? v[j] : 0.0f;
      q += v[j] * v[j];
      dot += g[j] * w[j] * v[j];
    }
    const float r = inv_rms(row_sum<LR>(q) * inv_d, a.eps);
    const float k = row_sum<LR>(dot) * inv_d * r * r;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (here) dw[j] += g[j] * v[j] * r;
      g[j] = r * (g[j] * w[j] - v[j] * k);
    }
    if (here) Elem<E>::store(dx, g);
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) red[grp][d + j] = dw[j];
  __syncthreads();
  for (int e = threadIdx.x; e < a.D; e += kBlock) {
    float t = 0.0f;
    for (int i = 0; i < NG; ++i) t += red[i][e];
    part[(int64_t)blockIdx.x * a.D + e] = t;
  }
}

// Any head width, stride and alignment: a wavefront a head, element by element,
// the partners by way of LDS.
template <class E, bool BWD>
__global__ __launch_bounds__(kBlock) void k_norm_any(const NormArgs a, int blocks0, int blocks1,
                                                     float* part) {
  __shared__ float buf[4][256];
  const bool second = (int)blockIdx.x >= blocks0;
  const NormSide& x = second ? a.side[1] : a.side[0];
  const int blk = second ? blockIdx.x - blocks0 : blockIdx.x, blocks = second ? blocks1 : blocks0;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = a.R / 2;
  const int64_t heads = (int64_t)x.rows * x.heads;
  const float inv_d = 1.0f / a.D;
  float dw[4] = {};
  for (int64_t i0 = (int64_t)blk * 4; i0 < heads; i0 += (int64_t)blocks * 4) {
    const bool on = i0 + wave < heads;
    const int row = on ? (int)((i0 + wave) / x.heads) : 0, h = on ? (int)((i0 + wave) % x.heads) : 0;
    const E* xp = (const E*)x.x + row * x.xs[0] + h * x.xs[1];
    const E* gp = BWD ? (const E*)x.dy + row * x.dys[0] + h * x.dys[1] : nullptr;
    const int pos = on && a.R ? x.pos[row] : 0;
    const bool in = pos >= 0 && pos < a.n_pos;
    const float* t = a.table + (int64_t)(in ? pos : 0) * a.R;
    float v[4] = {}, w[4] = {}, q = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = lane + 64 * i;
      if (!on || d >= a.D) continue;
      v[i] = (float)xp[d];
      w[i] = x.w ? (float)((const E*)x.w)[d] : 1.0f;
      q += v[i] * v[i];
    }
    const float r = inv_rms(row_sum<64>(q) * inv_d, a.eps);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = lane + 64 * i;
      if (on && d < a.D) buf[wave][d] = BWD ? (float)gp[d] : v[i] * r * w[i];
    }
    __syncthreads();
    float y[4], dot = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = lane + 64 * i;
      y[i] = 0.0f;
      if (!on || d >= a.D) continue;
      y[i] = buf[wave][d];
      if (d < a.R) {
        const int j = a.interleaved ? d / 2 : d < half ? d : d - half;
        const bool first = a.interleaved ? !(d & 1) : d < half;
        const int e = a.interleaved ? d ^ 1 : first ? d + half : d - half;
        const float s = first ? -t[half + j] : t[half + j];
        y[i] = in ? y[i] * t[j] + buf[wave][e] * (BWD ? -s : s) : __builtin_nanf("");
      }
      if (BWD) dot += y[i] * w[i] * v[i];
    }
    const float k = BWD ? row_sum<64>(dot) * inv_d * r * r : 0.0f;
    E* op = BWD ? (E*)x.dx + row * x.dxs[0] + h * x.dxs[1] : (E*)x.y + row * x.ys[0] + h * x.ys[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = lane + 64 * i;
      if (!on || d >= a.D) continue;
      if (BWD) {
        dw[i] += y[i] * v[i] * r;
        y[i] = r * (y[i] * w[i] - v[i] * k);
      }
      op[d] = (E)y[i];
    }
  }
  if (!BWD) return;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) buf[wave][lane + 64 * i] = dw[i];
  __syncthreads();
  for (int e = threadIdx.x; e < a.D; e += kBlock)
    part[(int64_t)blockIdx.x * a.D + e] = buf[0][e] + buf[1][e] + buf[2][e] + buf[3][e];
}

template <class E, int LR, Pairs P>
void launch_vec(const NormArgs& a, bool bwd, float* part, hipStream_t s) {
  int b[2];
  blocks_of(a, bwd ? kBwdBlocks : kFwdBlocks, b);
  if (bwd)
    k_norm_bwd<E, LR, P><<<b[0] + b[1], kBlock, 0, s>>>(a, b[0], b[1], part);
  else
    k_norm_fwd<E, LR, P><<<b[0] + b[1], kBlock, 0, s>>>(a, b[0], b[1]);
}
template <class E, int LR>
void launch_lr(const NormArgs& a, bool bwd, float* part, hipStream_t s) {
  if (a.interleaved)
    launch_vec<E, LR, kInside>(a, bwd, part, s);
  else if (a.R == 8 * LR)
    launch_vec<E, LR, kHalf>(a, bwd, part, s);
  else
    launch_vec<E, LR, kAway>(a, bwd, part, s);
}

template <class E>
void launch_e(const NormArgs& a, bool bwd, float* part, hipStream_t s) {
  int b[2];
  blocks_of(a, bwd ? kBwdBlocks : kFwdBlocks, b);
  if (b[0] + b[1] == 0) return;
  if (!a.vec) {
    if (bwd)
      k_norm_any<E, true><<<b[0] + b[1], kBlock, 0, s>>>(a, b[0], b[1], part);
    else
      k_norm_any<E, false><<<b[0] + b[1], kBlock, 0, s>>>(a, b[0], b[1], part);
    return;
  }
  switch (lanes(a.D)) {
    case 4: launch_lr<E, 4>(a, bwd, part, s); break;
    case 8: launch_lr<E, 8>(a, bwd, part, s); break;
    case 16: launch_lr<E, 16>(a, bwd, part, s); break;
    default: launch_lr<E, 32>(a, bwd, part, s); break;
  }
}

}  // namespace

hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t s) {
  if (a.dtype == kF32) launch_e<float>(a, false, nullptr, s);
  if (a.dtype == kF16) launch_e<_Float16>(a, false, nullptr, s);
  if (a.dtype == kBF16) launch_e<__bf16>(a, false, nullptr, s);
  return hipGetLastError();
}

// The workspace follows from the sizes alone: whatever the tensors' alignment, no
// call has more workgroups than one whose heads go 4 to a workgroup.
int64_t norm_bwd_bytes(const NormArgs& a) {
  NormArgs any = a;
  any.vec = 0;
  int b[2];
  blocks_of(any, kBwdBlocks, b);
  return (int64_t)(b[0] + b[1]) * a.D * 4;
}

hipError_t launch_norm_bwd(const NormArgs& a, void* ws, hipStream_t s) {
  float* part = (float*)ws;
  if (a.dtype == kF32) launch_e<float>(a, true, part, s), launch_dw<float>(a, part, s);
  if (a.dtype == kF16) launch_e<_Float16>(a, true, part, s), launch_dw<_Float16>(a, part, s);
  if (a.dtype == kBF16) launch_e<__bf16>(a, true, part, s), launch_dw<__bf16>(a, part, s);
  return hipGetLastError();
}

}  // namespace pnerf
