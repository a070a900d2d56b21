// What norm_rotate.hip and rotate_axes.hip share: rotation pairs, the walk over the
// heads of queries and keys, workgroups, and the weights' gradient.
#pragma once
#include <algorithm>

#include "rows_common.h"

namespace pnerf {
namespace {

constexpr int kBlock = 256;
// Workgroups, at most.  The gradient's each leave a sum for dw, so they are fewer, but
// enough for their loads to cover each other (8192 x 32 and 8192 x 8 heads of 128,
// bf16: 79 us with 2 a compute unit, 54 with 4 or 8).
constexpr int kFwdBlocks = 16 * kCUs, kBwdBlocks = 4 * kCUs;

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

template <class E>
void launch_dw(const NormArgs& a, float* part, hipStream_t s) {
  int b[2];
  blocks_of(a, kBwdBlocks, b);
  if (a.side[0].dw || a.side[1].dw)
    k_norm_dw<E><<<2 * ((a.D + 15) / 16), 1024, 0, s>>>(a, b[0], b[1], part);
}

}  // namespace
}  // namespace pnerf
