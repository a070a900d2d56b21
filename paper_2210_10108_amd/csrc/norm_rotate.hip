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
// Workgroups, at most.  The gradient's each leave a sum for dw, so they are fewer, but
// enough for their loads to cover each other (8192 x 32 and 8192 x 8 heads of 128,
// bf16: 79 us with 2 a compute unit, 54 with 4 or 8).
constexpr int kFwdBlocks = 16 * kCUs, kBwdBlocks = 4 * kCUs;

// 8 consecutive elements: as they are loaded, and as numbers.
template <class E>
struct Elem;
template <>
struct Elem<float> {
  struct Raw {
    floatx4 a, b;
  };
  static __device__ __forceinline__ Raw raw(const void* p) {
    return {reinterpret_cast<const floatx4*>(p)[0], reinterpret_cast<const floatx4*>(p)[1]};
  }
  static __device__ __forceinline__ void unpack(const Raw& r, float v[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = r.a[i], v[4 + i] = r.b[i];
  }
  static __device__ __forceinline__ void store(void* p, const float v[8]) {
    reinterpret_cast<floatx4*>(p)[0] = floatx4{v[0], v[1], v[2], v[3]};
    reinterpret_cast<floatx4*>(p)[1] = floatx4{v[4], v[5], v[6], v[7]};
  }
};
template <class T>
struct Elem16 {
  using Raw = uint4;
  static __device__ __forceinline__ Raw raw(const void* p) { return *reinterpret_cast<const uint4*>(p); }
  static __device__ __forceinline__ void unpack(const Raw& w, float v[8]) {
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
template <class E>
__device__ __forceinline__ void load(const void* p, float v[8]) {
  Elem<E>::unpack(Elem<E>::raw(p), v);
}

template <int CTRL>
__device__ __forceinline__ float dpp(float x) {  // a move within rows of 16 lanes, all lanes active
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xF, 0xF, true));
}

// Sum over a row of LR lanes, in all of them.
template <int LR>
__device__ __forceinline__ float row_sum(float x) {
  x += dpp<0xB1>(x);                       // quad_perm [1, 0, 3, 2]
  x += dpp<0x4E>(x);                       // quad_perm [2, 3, 0, 1]
  if (LR >= 8) x += dpp<0x141>(x);         // row_half_mirror
  if (LR >= 16) x += dpp<0x140>(x);        // row_mirror
  if (LR >= 32) x += __shfl_xor(x, 16);
  if (LR >= 64) x += __shfl_xor(x, 32);
  return x;
}

// Where the rotation partner of a lane's 8 elements is.
enum Pairs {
  kInside,  // interleaved: in the lane itself
  kHalf,    // in the lane half a row away (the whole head turns and fills its LR lanes)
  kAway     // in the lane R / 16 away
};
template <Pairs P, int LR>
__device__ __forceinline__ void partners(const NormArgs& a, int d, const float v[8], float p[8]) {
  if (P == kInside) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) p[i] = v[i + 1], p[i + 1] = v[i];
  } else if (P == kHalf && LR <= 16) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (LR == 4) p[i] = dpp<0x4E>(v[i]);
      if (LR == 8) p[i] = dpp<0x1B>(dpp<0x141>(v[i]));  // row_half_mirror, quad_perm [3, 2, 1, 0]
      if (LR == 16) p[i] = dpp<0x128>(v[i]);            // row_ror 8
    }
  } else {
    const int step = a.R / 16;  // lanes of half the rotated part
    const int lane = threadIdx.x & 63;
    const int from = d >= a.R ? lane : d < a.R / 2 ? lane + step : lane - step;
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = __shfl(v[i], from);
  }
}

// (The instruction takes a subnormal number for zero.)
__device__ __forceinline__ float inv_rms(float mean, float eps) {
  const float x = mean + eps;
  const bool small = x < 0x1p-126f;
  return __builtin_amdgcn_rsqf(small ? x * 0x1p64f : x) * (small ? 0x1p32f : 1.0f);
}

// Cosines and sines of a lane's 8 elements at position pos: element i turns
// with its partner by (c[i], s[i]), s negated for the first of a pair; (1, 0)
// past the rotated part, NaN for a position that is not in the table.
template <Pairs P>
__device__ __forceinline__ void angles(const NormArgs& a, int pos, int d, float c[8], float s[8]) {
  const int half = a.R / 2;
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = 1.0f, s[i] = 0.0f;
  if (d >= a.R) return;
  const bool in = pos >= 0 && pos < a.n_pos;
  const float* t = a.table + (int64_t)(in ? pos : 0) * a.R;
  if (P == kInside) {
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
    load<float>(t + j, c);
    load<float>(t + half + j, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i] = d < half ? -v[i] : v[i];
  }
  if (!in)
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = s[i] = __builtin_nanf("");
}

// The workgroups of the queries come first, then those of the keys.  Each side's
// walk its heads in memory order, all of them together through one moving window
// (walking each position's heads in one wavefront, which keeps the cosines in
// registers, sends the wavefronts to addresses a position apart, and those to few
// memory channels at a time: 58 us where this takes 45 for the 203 MB of 8192 x 32
// and 16382 x 8 heads of 128).  A lane's row and head of the next step, by steps:
struct Walk {
  int row, head;        // current
  int d_row, d_head, heads;
  int64_t left;         // heads from the current one to the end
  int64_t step;
  __device__ __forceinline__ Walk(const NormSide& x, int64_t first, int64_t step_)
      : heads(x.heads), left((int64_t)x.rows * x.heads - first), step(step_) {
    row = (int)(first / heads), head = (int)(first - (int64_t)row * heads);
    d_row = (int)(step / heads), d_head = (int)(step - (int64_t)d_row * heads);
  }
  __device__ __forceinline__ bool on() const { return left > 0; }
  __device__ __forceinline__ void next() {
    left -= step;
    row += d_row, head += d_head;
    if (head >= heads) head -= heads, ++row;
  }
};

template <class E, int LR, Pairs P>
__global__ __launch_bounds__(kBlock) void k_norm_fwd(const NormArgs a, int blocks0, int blocks1) {
  constexpr int NG = kBlock / LR;
  const bool second = (int)blockIdx.x >= blocks0;
  const NormSide& x = second ? a.side[1] : a.side[0];
  const int blk = second ? blockIdx.x - blocks0 : blockIdx.x, blocks = second ? blocks1 : blocks0;
  const int d = 8 * (threadIdx.x % LR);
  const bool col = d < a.D;
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
  const bool col = d < a.D;
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
      g[j] = here ? g[j] * c[j] - p[j] * s[j] : 0.0f;  // turned back
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

// dw: the workgroups' sums added up in order, 16 columns a workgroup, 64 rows at a time.
template <class E>
__global__ __launch_bounds__(1024) void k_norm_dw(const NormArgs a, int blocks0, int blocks1,
                                                  const float* part) {
  __shared__ float red[64][17];
  const int tiles = (a.D + 15) / 16, side = blockIdx.x / tiles;
  const int col = (blockIdx.x % tiles) * 16 + threadIdx.x % 16, r = threadIdx.x / 16;
  const int first = side ? blocks0 : 0, n = side ? blocks1 : blocks0;
  E* out = (E*)(side ? a.side[1].dw : a.side[0].dw);
  float t = 0.0f;
  if (col < a.D)
#pragma unroll 4
    for (int i = r; i < n; i += 64) t += part[(int64_t)(first + i) * a.D + col];
  red[r][threadIdx.x % 16] = t;
  __syncthreads();
  if (r == 0 && col < a.D && out) {
    t = 0.0f;
    for (int i = 0; i < 64; ++i) t += red[i][threadIdx.x];
    out[col] = (E)t;
  }
}

int lanes(int D) {
  int l = 4;
  while (8 * l < D) l *= 2;
  return l;
}

// Workgroups of both sides, in proportion to their heads: at most `most` in all
// (the forward: what the chip holds; the backward, whose partial sums of dw each
// cost a read: fewer), and at least one where there are heads.
void blocks_of(const NormArgs& a, int64_t most, int b[2]) {
  const int64_t per = a.vec ? kBlock / lanes(a.D) : 4;
  int64_t want[2];
  for (int i = 0; i < 2; ++i) want[i] = ((int64_t)a.side[i].rows * a.side[i].heads + per - 1) / per;
  const int64_t all = want[0] + want[1];
  if (all > most && want[0] && want[1]) {
    want[0] = std::min(std::max<int64_t>(want[0] * most / all, 1), most - 1);
    want[1] = most - want[0];
  }
  for (int i = 0; i < 2; ++i) b[i] = (int)std::min(want[i], most);
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

template <class E>
void launch_dw(const NormArgs& a, float* part, hipStream_t s) {
  int b[2];
  blocks_of(a, kBwdBlocks, b);
  if (a.side[0].dw || a.side[1].dw)
    k_norm_dw<E><<<2 * ((a.D + 15) / 16), 1024, 0, s>>>(a, b[0], b[1], part);
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
