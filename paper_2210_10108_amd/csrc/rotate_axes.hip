// The rotation of query and key heads at positions of several axes (a patch's row,
// column and frame), with or without the norm, and its gradient: norm_rotate.hip's
// formulas and walk over the heads, but every pair turns by the position along its own
// axis.  The gradient of a rotation alone is the rotation back, the forward kernel with
// the sines negated.
//
// A stream, bound by memory (16382 rows of 16 and of 8 bf16 heads of 128: 45 us or 4.5
// TB/s).  Where the pairs of a lane's 8 elements share an axis
// (kWhole: runs of pairs in multiples of 8, of 4 where pairs lie side by side) its
// cosines and sines are four 16-byte loads from one row of the table, as with a single
// axis.  Otherwise (kMixed: axes in turn) a workgroup looks its rows' up together.
#define PNERF_LAYERS_DEVICE
#include "norm_common.h"

namespace pnerf {
namespace {

// Workgroups that look angles up in advance: no more than run at once (31 us with twice as
// many, 29 with half, where these take 28).
constexpr int kMixedBlocks = 8 * kCUs;

// Which positions a lane's pairs turn by.
enum Axes {
  kWhole,  // that of one axis, which the lane's pairs share
  kMixed   // each pair its own
};

// The cosines and sines of a lane's pairs, where they share an axis: one row of the table.
template <Axes X, Pairs P, int LR>
struct Angles {
  int axis, pos;
  __device__ __forceinline__ Angles(const NormArgs& a, const NormSide& x, int blk, int blocks, float*) : axis(0), pos(0) {
    const int d = 8 * (threadIdx.x % LR);
    if (d >= a.R) return;
    const int j = P == kInside ? d / 2 : d < a.R / 2 ? d : d - a.R / 2;
    axis = a.pair_axis[j / 16] >> (2 * (j % 16)) & 3;
  }
  __device__ __forceinline__ void start(const NormArgs&) {}
  // Called where the row's data are requested.
  __device__ __forceinline__ void fetch(const NormArgs& a, const NormSide& x, int row) {
    pos = x.pos[(int64_t)row * a.axes + axis];
  }
  __device__ __forceinline__ void of(const NormArgs& a, int, int d, float c[8], float s[8]) { angles<P>(a, pos, d, c, s); }
};

// Where each pair has its own, a workgroup's heads are neighbours, mostly of one row: the
// angles of its rows are looked up once a pair and shared through LDS.  (A lane that
// looks up its own, 16 four-byte loads: 67 us where this takes 28, and shared axes 21, for
// 8192 rows of 16 and of 8 bfloat16 heads of 128.)  They are requested one step ahead of
// their use, the positions two.
template <Pairs P, int LR>
struct Angles<kMixed, P, LR> {
  static constexpr int kGroups = kBlock / LR, kPairs = 4 * LR, kLoads = 4;  // rows of a load: kGroups / 4
  const NormSide& x;
  float* stage;  // [2][kGroups][R]
  Walk now, next, later;  // the workgroup's first head: of this step, the next two
  int j, axis, first, buf;
  bool mine;
  int pos[kLoads];
  float c[kLoads], s[kLoads];
  __device__ __forceinline__ Angles(const NormArgs& a, const NormSide& x_, int blk, int blocks, float* lds)
      : x(x_), stage(lds), now(x_, (int64_t)blk * kGroups, (int64_t)blocks * kGroups), next(now), later(now),
        j(threadIdx.x % kPairs), axis(0), first(threadIdx.x / kPairs), buf(1), mine(j < a.R / 2) {
    if (mine) axis = a.pair_axis[j / 16] >> (2 * (j % 16)) & 3;
    next.next();
    later.next(), later.next();
  }
  // Rows of a step.
  __device__ __forceinline__ static int rows(const Walk& w) {
    return w.on() ? (w.head + (int)min(w.left, (int64_t)kGroups) - 1) / w.heads + 1 : 0;
  }
  __device__ __forceinline__ void positions(const NormArgs& a, const Walk& w) {
    const int n = rows(w);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = first + i * (kGroups / 4);
      if (mine && r < n) pos[i] = x.pos[(int64_t)(w.row + r) * a.axes + axis];
    }
  }
  __device__ __forceinline__ void look_up(const NormArgs& a, const Walk& w) {
    const int n = rows(w);
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      if (!mine || first + i * (kGroups / 4) >= n) continue;
      const bool in = pos[i] >= 0 && pos[i] < a.n_pos;
      const float* t = a.table + (int64_t)(in ? pos[i] : 0) * a.R + j;
      c[i] = in ? t[0] : __builtin_nanf("");
      s[i] = in ? t[a.R / 2] : __builtin_nanf("");
    }
  }
  __device__ __forceinline__ void start(const NormArgs& a) {
    positions(a, now);
    look_up(a, now);
    positions(a, next);
  }
  __device__ __forceinline__ void fetch(const NormArgs&, const NormSide&, int) {}
  // For this step, which every wavefront of the workgroup makes; row: the lane's.
  __device__ __forceinline__ void of(const NormArgs& a, int row, int d, float cs[8], float sn[8]) {
    buf ^= 1;
    float* to = stage + buf * kGroups * a.R;
    const int n = rows(now), row0 = now.row;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = first + i * (kGroups / 4);
      if (mine && r < n) to[r * a.R + j] = c[i], to[r * a.R + a.R / 2 + j] = s[i];
    }
    look_up(a, next);
    positions(a, later);
    now = next, next = later;
    later.next();
    __syncthreads();
    const int half = a.R / 2;
#pragma unroll
    for (int i = 0; i < 8; ++i) cs[i] = 1.0f, sn[i] = 0.0f;
    if (d >= a.R) return;
    const float* t = to + (row - row0) * a.R;
    if (P == kInside) {
      const floatx4 cc = *reinterpret_cast<const floatx4*>(t + d / 2), ss = *reinterpret_cast<const floatx4*>(t + half + d / 2);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        cs[2 * i] = cs[2 * i + 1] = cc[i];
        sn[2 * i] = -ss[i], sn[2 * i + 1] = ss[i];
      }
    } else {
      const int k = d < half ? d : d - half;
      float v[8];
      load<float>(t + k, cs);
      load<float>(t + half + k, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) sn[i] = d < half ? -v[i] : v[i];
    }
  }
};
template <Axes X>
constexpr int kStage = X == kMixed ? 2 * 8 * kBlock : 1;  // floats: 8 a lane, twice

// Holds the compiler to have these values here: waited for after the next step's loads
// were issued, they would be waited for together with those.
__device__ __forceinline__ void arrived(float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(v[i]));
}

template <class E, int LR, Pairs P, Axes X>
__global__ __launch_bounds__(kBlock) void k_axes_fwd(const NormArgs a, int blocks0, int blocks1) {
  constexpr int NG = kBlock / LR;
  __shared__ __attribute__((aligned(16))) float stage[kStage<X>];
  const bool second = (int)blockIdx.x >= blocks0;
  const NormSide& x = second ? a.side[1] : a.side[0];
  const int blk = second ? blockIdx.x - blocks0 : blockIdx.x, blocks = second ? blocks1 : blocks0;
  const int d = 8 * (threadIdx.x % LR);
  // what lies past the rotated part passes as it is: times 1 and plus 0 times its
  // neighbour, an infinity or NaN there would become or reach another number
  const bool col = d < a.D, turned = P == kHalf || d < a.R;
  float w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = 1.0f;
  if (col && x.w) load<E>((const E*)x.w + d, w);
  const float inv_d = 1.0f / a.D;
  Walk at(x, (int64_t)blk * NG + threadIdx.x / LR, (int64_t)blocks * NG);
  int64_t left = (int64_t)x.rows * x.heads - (int64_t)blk * NG;  // of the workgroup's first head
  Angles<X, P, LR> angle(a, x, blk, blocks, stage);
  if (a.R) angle.start(a);
  typename Elem<E>::Raw raw = {};
  auto fetch = [&] {
    if (!at.on() || !col) return;
    raw = Elem<E>::raw((const E*)x.x + at.row * x.xs[0] + at.head * x.xs[1] + d);
    if (a.R) angle.fetch(a, x, at.row);
  };
  fetch();
  // every wavefront makes the same number of rounds: the exchanges and barriers need them all
  for (; left > 0; left -= (int64_t)blocks * NG) {
    float v[8], p[8], c[8], s[8];
    const bool here = at.on() && col;
    Elem<E>::unpack(raw, v);
    arrived(v);
    if (a.R) {
      angle.of(a, at.row, here ? d : a.R, c, s);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) c[j] = 1.0f, s[j] = 0.0f;
    }
    E* y = (E*)x.y + at.row * x.ys[0] + at.head * x.ys[1] + d;
    at.next();
    fetch();
    if (a.norm) {
      float q = 0.0f;
#pragma unroll
      for (int j = 0; j < 8; ++j) q += here ? v[j] * v[j] : 0.0f;
      const float r = inv_rms(row_sum<LR>(q) * inv_d, a.eps);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= r * w[j];
    }
    partners<P, LR>(a, d, v, p);
    if (turned)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = v[j] * c[j] + p[j] * (a.sign * s[j]);
    if (here) Elem<E>::store(y, v);
  }
}

// Each workgroup leaves its sum of dw.
template <class E, int LR, Pairs P, Axes X>
__global__ __launch_bounds__(kBlock) void k_axes_bwd(const NormArgs a, int blocks0, int blocks1, float* part) {
  constexpr int NG = kBlock / LR;
  __shared__ float red[NG][8 * LR];
  __shared__ __attribute__((aligned(16))) float stage[kStage<X>];
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
  int64_t left = (int64_t)x.rows * x.heads - (int64_t)blk * NG;
  Angles<X, P, LR> angle(a, x, blk, blocks, stage);
  if (a.R) angle.start(a);
  typename Elem<E>::Raw raw_x = {}, raw_g = {};
  auto fetch = [&] {
    if (!at.on() || !col) return;
    raw_x = Elem<E>::raw((const E*)x.x + at.row * x.xs[0] + at.head * x.xs[1] + d);
    raw_g = Elem<E>::raw((const E*)x.dy + at.row * x.dys[0] + at.head * x.dys[1] + d);
    if (a.R) angle.fetch(a, x, at.row);
  };
  fetch();
  for (; left > 0; left -= (int64_t)blocks * NG) {
    float v[8], g[8], p[8], c[8], s[8];
    const bool here = at.on() && col;
    Elem<E>::unpack(raw_x, v);
    Elem<E>::unpack(raw_g, g);
    arrived(v);
    arrived(g);
    if (a.R) {
      angle.of(a, at.row, here ? d : a.R, c, s);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) c[j] = 1.0f, s[j] = 0.0f;
    }
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
__global__ __launch_bounds__(kBlock) void k_axes_any(const NormArgs a, int blocks0, int blocks1,
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
    float v[4] = {}, w[4] = {}, q = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = lane + 64 * i;
      if (!on || d >= a.D) continue;
      v[i] = (float)xp[d];
      w[i] = x.w ? (float)((const E*)x.w)[d] : 1.0f;
      q += v[i] * v[i];
    }
    const float r = !a.norm ? 1.0f : inv_rms(row_sum<64>(q) * inv_d, a.eps);
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
        const int pos = x.pos[(int64_t)row * a.axes + (a.pair_axis[j / 16] >> (2 * (j % 16)) & 3)];
        const bool in = pos >= 0 && pos < a.n_pos;
        const float* t = a.table + (int64_t)(in ? pos : 0) * a.R;
        const float s = a.sign * (first ? -t[half + j] : t[half + j]);
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
void launch_vec(const NormArgs& a, bool bwd, float* part, int n, const int b[2], hipStream_t s) {
  if (bwd)
    (a.whole ? k_axes_bwd<E, LR, P, kWhole> : k_axes_bwd<E, LR, P, kMixed>)<<<n, kBlock, 0, s>>>(a, b[0], b[1], part);
  else
    (a.whole ? k_axes_fwd<E, LR, P, kWhole> : k_axes_fwd<E, LR, P, kMixed>)<<<n, kBlock, 0, s>>>(a, b[0], b[1]);
}
template <class E, int LR>
void launch_lr(const NormArgs& a, bool bwd, float* part, int n, const int b[2], hipStream_t s) {
  if (a.interleaved)
    launch_vec<E, LR, kInside>(a, bwd, part, n, b, s);
  else if (a.R == 8 * LR)
    launch_vec<E, LR, kHalf>(a, bwd, part, n, b, s);
  else
    launch_vec<E, LR, kAway>(a, bwd, part, n, b, s);
}
template <class E>
void launch_e(const NormArgs& a, bool bwd, float* part, hipStream_t s) {
  int b[2];
  blocks_of(a, bwd ? kBwdBlocks : a.whole || !a.vec ? kFwdBlocks : kMixedBlocks, b);
  const int n = b[0] + b[1];
  if (n == 0) return;
  if (!a.vec) {
    (bwd ? k_axes_any<E, true> : k_axes_any<E, false>)<<<n, kBlock, 0, s>>>(a, b[0], b[1], part);
    return;
  }
  switch (lanes(a.D)) {
    case 4: launch_lr<E, 4>(a, bwd, part, n, b, s); break;
    case 8: launch_lr<E, 8>(a, bwd, part, n, b, s); break;
    case 16: launch_lr<E, 16>(a, bwd, part, n, b, s); break;
    default: launch_lr<E, 32>(a, bwd, part, n, b, s); break;
  }
}

}  // namespace

hipError_t launch_axes_fwd(const NormArgs& a, hipStream_t s) {
  if (a.dtype == kF32) launch_e<float>(a, false, nullptr, s);
  if (a.dtype == kF16) launch_e<_Float16>(a, false, nullptr, s);
  if (a.dtype == kBF16) launch_e<__bf16>(a, false, nullptr, s);
  return hipGetLastError();
}

hipError_t launch_axes_bwd(const NormArgs& a, void* ws, hipStream_t s) {
  float* part = (float*)ws;
  if (a.dtype == kF32) launch_e<float>(a, true, part, s), launch_dw<float>(a, part, s);
  if (a.dtype == kF16) launch_e<_Float16>(a, true, part, s), launch_dw<_Float16>(a, part, s);
  if (a.dtype == kBF16) launch_e<__bf16>(a, true, part, s), launch_dw<__bf16>(a, part, s);
  return hipGetLastError();
}

}  // namespace pnerf
