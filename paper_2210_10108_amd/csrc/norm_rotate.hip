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
#include <algorithm>

#include "layers_internal.h"

namespace pnerf {
namespace {

constexpr int kBlock = 256;
constexpr int kMaxPart = 512;  // workgroups of a side of the backward, each with one partial dw

template <class E>
struct Elem;
template <>
struct Elem<float> {
  static __device__ __forceinline__ void load(const void* p, float v[8]) {
    const floatx4 a = reinterpret_cast<const floatx4*>(p)[0], b = reinterpret_cast<const floatx4*>(p)[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
  }
  static __device__ __forceinline__ void store(void* p, const float v[8]) {
    reinterpret_cast<floatx4*>(p)[0] = floatx4{v[0], v[1], v[2], v[3]};
    reinterpret_cast<floatx4*>(p)[1] = floatx4{v[4], v[5], v[6], v[7]};
  }
};
template <class T>
struct Elem16 {
  static __device__ __forceinline__ void load(const void* p, float v[8]) {
    const uint4 w = *reinterpret_cast<const uint4*>(p);
    v[0] = T::lo(w.x), v[1] = T::hi(w.x), v[2] = T::lo(w.y), v[3] = T::hi(w.y);
    v[4] = T::lo(w.z), v[5] = T::hi(w.z), v[6] = T::lo(w.w), v[7] = T::hi(w.w);
  }
  static __device__ __forceinline__ void store(void* p, const float v[8]) {
    *reinterpret_cast<uint4*>(p) = make_uint4(T::pack(v[0], v[1]), T::pack(v[2], v[3]),
                                              T::pack(v[4], v[5]), T::pack(v[6], v[7]));
  }
};
template <>
struct Elem<_Float16> : Elem16<F16> {};
template <>
struct Elem<__bf16> : Elem16<BF16> {};

// Cosines and sines of a lane's 8 elements at position pos: element i turns
// with its partner by (c[i], s[i]), s negated for the first of a pair; (1, 0)
// past the rotated part, NaN for a position that is not in the table.
template <bool INTER>
__device__ __forceinline__ void angles(const NormArgs& a, int pos, int d, float c[8], float s[8]) {
  const int half = a.R / 2;
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = 1.0f, s[i] = 0.0f;
  if (d >= a.R) return;
  const bool in = pos >= 0 && pos < a.n_pos;
  const float* t = a.table + (int64_t)(in ? pos : 0) * a.R;
  if (INTER) {
    const floatx4 cc = *reinterpret_cast<const floatx4*>(t + d / 2);
    const floatx4 ss = *reinterpret_cast<const floatx4*>(t + half + d / 2);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      c[2 * i] = c[2 * i + 1] = cc[i];
      s[2 * i] = -ss[i], s[2 * i + 1] = ss[i];
    }
  } else {
    const int j = d < half ? d : d - half;
    float v[8];
    Elem<float>::load(t + j, c);
    Elem<float>::load(t + half + j, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = d < half ? -v[i] : v[i];
  }
  if (!in)
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = s[i] = __builtin_nanf("");
}

// The rotation partners of a lane's 8 elements.
template <bool INTER, int LR>
__device__ __forceinline__ void partners(const NormArgs& a, int d, const float v[8], float p[8]) {
  if (INTER) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) p[i] = v[i + 1], p[i + 1] = v[i];
  } else {
    const int step = a.R / 16;  // lanes of half the rotated part
    const int lane = threadIdx.x & 63;
    const int from = d >= a.R ? lane : d < a.R / 2 ? lane + step : lane - step;
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = __shfl(v[i], from);
  }
}

template <int LR>
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
  for (int m = LR / 2; m; m >>= 1) x += __shfl_xor(x, m);
  return x;
}

// Groups of the grid: of the queries first, then of the keys.
struct Split {
  int hpg[2];        // heads a group takes
  int nhg[2];        // groups of a position
  int64_t groups[2];
};

template <class E, int LR, bool INTER>
__global__ __launch_bounds__(kBlock) void k_norm_fwd(const NormArgs a, const Split sp) {
  int64_t gid = (int64_t)blockIdx.x * (kBlock / LR) + threadIdx.x / LR;
  const int d = 8 * (threadIdx.x % LR);
  const bool second = gid >= sp.groups[0];
  if (second) gid -= sp.groups[0];
  const NormSide& x = second ? a.side[1] : a.side[0];
  const int nhg = second ? sp.nhg[1] : sp.nhg[0];
  const bool on = gid < (second ? sp.groups[1] : sp.groups[0]);
  const int row = on ? (int)(gid / nhg) : 0, h0 = (int)(gid % nhg);
  const bool mine = on && d < a.D;
  float w[8], c[8], s[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = 1.0f;
  if (mine && x.w) Elem<E>::load((const E*)x.w + d, w);
  angles<INTER>(a, mine && a.R ? x.pos[row] : 0, mine ? d : a.R, c, s);
  const E* xp = (const E*)x.x + row * x.xs[0] + d;
  E* yp = (E*)x.y + row * x.ys[0] + d;
  const float inv_d = 1.0f / a.D;
  // every lane of a wavefront makes the same number of rounds: the exchanges need them all
  const int rounds = max(sp.hpg[0], sp.hpg[1]);
  for (int i = 0; i < rounds; ++i) {
    const int h = h0 + i * nhg;
    const bool here = mine && h < x.heads;
    float v[8] = {}, p[8];
    if (here) Elem<E>::load(xp + h * x.xs[1], v);
    float q = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) q += v[j] * v[j];
    const float r = 1.0f / sqrtf(row_sum<LR>(q) * inv_d + a.eps);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= r * w[j];
    partners<INTER, LR>(a, d, v, p);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = v[j] * c[j] + p[j] * s[j];
    if (here) Elem<E>::store(yp + h * x.ys[1], v);
  }
}

// Workgroups of a side walk its groups in strides; each leaves its sum of dw.
template <class E, int LR, bool INTER>
__global__ __launch_bounds__(kBlock) void k_norm_bwd(const NormArgs a, const Split sp, int blocks0,
                                                     int blocks1, float* part) {
  constexpr int NG = kBlock / LR;
  __shared__ float red[NG][8 * LR];
  const bool second = (int)blockIdx.x >= blocks0;
  const NormSide& x = second ? a.side[1] : a.side[0];
  const int nhg = second ? sp.nhg[1] : sp.nhg[0], hpg = second ? sp.hpg[1] : sp.hpg[0];
  const int64_t groups = second ? sp.groups[1] : sp.groups[0];
  const int blk = second ? blockIdx.x - blocks0 : blockIdx.x, blocks = second ? blocks1 : blocks0;
  const int grp = threadIdx.x / LR, d = 8 * (threadIdx.x % LR);
  float w[8], dw[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = 1.0f, dw[i] = 0.0f;
  if (d < a.D && x.w) Elem<E>::load((const E*)x.w + d, w);
  const float inv_d = 1.0f / a.D;
  for (int64_t g0 = (int64_t)blk * NG; g0 < groups; g0 += (int64_t)blocks * NG) {
    const int64_t gid = g0 + grp;
    const int row = gid < groups ? (int)(gid / nhg) : 0, h0 = (int)(gid % nhg);
    const bool mine = gid < groups && d < a.D;
    float c[8], s[8];
    angles<INTER>(a, mine && a.R ? x.pos[row] : 0, mine ? d : a.R, c, s);
    for (int i = 0; i < hpg; ++i) {
      const int h = h0 + i * nhg;
      const bool here = mine && h < x.heads;
      float v[8] = {}, g[8] = {}, p[8];
      if (here) {
        Elem<E>::load((const E*)x.x + row * x.xs[0] + h * x.xs[1] + d, v);
        Elem<E>::load((const E*)x.dy + row * x.dys[0] + h * x.dys[1] + d, g);
      }
      partners<INTER, LR>(a, d, g, p);
      float q = 0.0f, dot = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        g[j] = g[j] * c[j] - p[j] * s[j];  // turned back
        q += v[j] * v[j];
        dot += g[j] * w[j] * v[j];
      }
      const float r = 1.0f / sqrtf(row_sum<LR>(q) * inv_d + a.eps);
      const float k = row_sum<LR>(dot) * inv_d * r * r;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (here) dw[j] += g[j] * v[j] * r;
        g[j] = r * (g[j] * w[j] - v[j] * k);
      }
      if (here) Elem<E>::store((E*)x.dx + row * x.dxs[0] + h * x.dxs[1] + d, g);
    }
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
    const float r = 1.0f / sqrtf(row_sum<64>(q) * inv_d + a.eps);
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

// dw: the workgroups' sums added up in order, 16 columns a workgroup, 16 rows at a time.
template <class E>
__global__ __launch_bounds__(256) void k_norm_dw(const NormArgs a, int blocks0, int blocks1,
                                                 const float* part) {
  __shared__ float red[16][17];
  const int tiles = (a.D + 15) / 16, side = blockIdx.x / tiles;
  const int col = (blockIdx.x % tiles) * 16 + threadIdx.x % 16, r = threadIdx.x / 16;
  const int first = side ? blocks0 : 0, n = side ? blocks1 : blocks0;
  E* out = (E*)(side ? a.side[1].dw : a.side[0].dw);
  float t = 0.0f;
  if (col < a.D)
    for (int i = r; i < n; i += 16) t += part[(int64_t)(first + i) * a.D + col];
  red[r][threadIdx.x % 16] = t;
  __syncthreads();
  if (r == 0 && col < a.D && out) {
    t = 0.0f;
    for (int i = 0; i < 16; ++i) t += red[i][threadIdx.x];
    out[col] = (E)t;
  }
}

int lanes(int D) {
  int l = 4;
  while (8 * l < D) l *= 2;
  return l;
}

// Heads a group takes: as many as leave the chip 16 wavefronts a compute unit.
Split split_of(const NormArgs& a) {
  Split sp;
  for (int i = 0; i < 2; ++i) {
    const NormSide& x = a.side[i];
    const int64_t want = (int64_t)kCUs * 16 * 64 / lanes(a.D);  // groups
    const int64_t all = (int64_t)x.rows * x.heads;
    sp.hpg[i] = (int)std::max<int64_t>(1, std::min<int64_t>({x.heads, all / want, 8}));
    sp.nhg[i] = std::max(1, (x.heads + sp.hpg[i] - 1) / sp.hpg[i]);
    sp.groups[i] = (int64_t)x.rows * sp.nhg[i];
  }
  return sp;
}

void blocks_of(const NormArgs& a, int b[2]) {
  for (int i = 0; i < 2; ++i) {
    const int64_t n = (int64_t)a.side[i].rows * a.side[i].heads;
    const int64_t per = a.vec ? kBlock / lanes(a.D) : 4;
    b[i] = (int)std::min<int64_t>(kMaxPart, (n + per - 1) / per);
  }
}

template <class E, int LR, bool INTER>
void launch_vec(const NormArgs& a, bool bwd, float* part, hipStream_t s) {
  const Split sp = split_of(a);
  constexpr int per = kBlock / LR;
  if (!bwd) {
    k_norm_fwd<E, LR, INTER><<<(unsigned)((sp.groups[0] + sp.groups[1] + per - 1) / per), kBlock, 0, s>>>(a, sp);
  } else {
    int b[2];
    blocks_of(a, b);
    k_norm_bwd<E, LR, INTER><<<b[0] + b[1], kBlock, 0, s>>>(a, sp, b[0], b[1], part);
  }
}

template <class E>
void launch_e(const NormArgs& a, bool bwd, float* part, hipStream_t s) {
  int b[2];
  blocks_of(a, b);
  if (b[0] + b[1] == 0) return;
  if (!a.vec) {
    if (bwd)
      k_norm_any<E, true><<<b[0] + b[1], kBlock, 0, s>>>(a, b[0], b[1], part);
    else
      k_norm_any<E, false><<<b[0] + b[1], kBlock, 0, s>>>(a, b[0], b[1], part);
  } else {
    const int l = lanes(a.D);
    if (a.interleaved) {
      if (l == 4) launch_vec<E, 4, true>(a, bwd, part, s);
      if (l == 8) launch_vec<E, 8, true>(a, bwd, part, s);
      if (l == 16) launch_vec<E, 16, true>(a, bwd, part, s);
      if (l == 32) launch_vec<E, 32, true>(a, bwd, part, s);
    } else {
      if (l == 4) launch_vec<E, 4, false>(a, bwd, part, s);
      if (l == 8) launch_vec<E, 8, false>(a, bwd, part, s);
      if (l == 16) launch_vec<E, 16, false>(a, bwd, part, s);
      if (l == 32) launch_vec<E, 32, false>(a, bwd, part, s);
    }
  }
}

template <class E>
void launch_dw(const NormArgs& a, float* part, hipStream_t s) {
  int b[2];
  blocks_of(a, b);
  if (a.side[0].dw || a.side[1].dw)
    k_norm_dw<E><<<2 * ((a.D + 15) / 16), 256, 0, s>>>(a, b[0], b[1], part);
}

}  // namespace

hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t s) {
  if (a.dtype == kF32) launch_e<float>(a, false, nullptr, s);
  if (a.dtype == kF16) launch_e<_Float16>(a, false, nullptr, s);
  if (a.dtype == kBF16) launch_e<__bf16>(a, false, nullptr, s);
  return hipGetLastError();
}

int64_t norm_bwd_bytes(const NormArgs& a) {
  int b[2];
  blocks_of(a, b);
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
