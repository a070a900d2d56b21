// What the forward passes of attention share: the softmax state and sums of a
// lane's row, a workgroup's place, and the join of the parts of the key axis.
#pragma once
#include "attention_common.h"

#if defined(__HIP_DEVICE_COMPILE__) || defined(PNERF_LAYERS_DEVICE)
namespace pnerf {
namespace {

// The softmax state and sums of a lane's row.
template <class T, int DP>
struct Rows {
  uint4 qf[DP / 16];
  floatx16 o[DP / 32], s[2];
  float m, l, top;

  template <bool VEC>
  __device__ __forceinline__ void init(const uint16_t* q, bool ok, int D, int h) {
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
      const int d = 16 * s + 8 * h;
      qf[s] = load8<VEC>(q + d, ok ? min(D - d, 8) : 0);
    }
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) o[i] = floatx16{};
    m = -INFINITY, l = 0.0f;
  }

  // The scores of one tile, in units of 1 / c; vm: its keys that may be read.  Sets
  // `top`, the maximum with them.
  __device__ __forceinline__ void scores(const uint4* sk, uint64_t vm, float c, int lane) {
    constexpr int CH = DP / 8;
    const int r = lane & 31, h = lane >> 5;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      s[n] = floatx16{};
#pragma unroll
      for (int i = 0; i < DP / 16; ++i) s[n] = T::mma(sk[swz<CH>(32 * n + r, 2 * i + h)], qf[i], s[n]);
    }
    if (vm != ~0ull) {
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const uint32_t w = (uint32_t)(vm >> (32 * n)) >> (4 * h);
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (!((w >> (8 * (i / 4) + i % 4)) & 1)) s[n][i] = -INFINITY;
      }
    }
    raise(c);
  }
  // `top` of the scores that are there.
  __device__ __forceinline__ void raise(float c) {
    float mx = -INFINITY;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[n][i]);
    float m0, m1;
    halves(mx, m0, m1);
    top = fmaxf(m, c * fmaxf(m0, m1));
  }
  // m may lag behind the maximum by 8 (p is then up to 2^8, and as exact as with
  // it): the sums are rescaled a few times a pass, not in most tiles.
  __device__ __forceinline__ bool grown() const { return __any(top > m + 8.0f); }
  __device__ __forceinline__ void rescale() {
    const float alpha = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.0f : top));
    m = top;
    l *= alpha;
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) o[i] *= alpha;
  }
  // The scores' exponentials, and their sum.
  __device__ __forceinline__ void weights(float c) {
    const float base = m == -INFINITY ? 0.0f : m;  // no allowed key yet
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[n][i] = __builtin_amdgcn_exp2f(fmaf(s[n][i], c, -base));
        l += s[n][i];
      }
  }
  // Adds the tile whose scores are there.
  __device__ __forceinline__ void add(const uint4* sv, float c, int lane) {
    constexpr int CH = DP / 8;
    weights(c);
#pragma unroll
    for (int n = 0; n < 4; ++n) {  // 16 keys each
      const uint4 pf = pack8<T>(s[n / 2], 8 * (n % 2));
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) o[d] = T::mma(tr_frag<CH>(sv, 16 * n, 32 * d, lane), pf, o[d]);
    }
  }
  // All tiles: next() makes the following one's scores, false where there is none;
  // values() is where its values are.  (The rescaling stands outside the inner
  // loop: in a branch of it the sums, tuples of registers, would be copied on the
  // path that does not take it.)
  template <class N, class V>
  __device__ __forceinline__ void run(float c, int lane, N next, V values) {
    bool more = next();
    while (more) {
      rescale();
      do {
        add(values(), c, lane);
        more = next();
      } while (more && !grown());
    }
  }

  // The row's sum of both halves; nothing where the row is not to be computed.
  __device__ __forceinline__ void close(bool ok) {
    float l0, l1;
    halves(l, l0, l1);
    l = l0 + l1;
    if (!ok) {  // past q_len, beside rows that are not
      m = -INFINITY, l = 0.0f;
#pragma unroll
      for (int i = 0; i < DP / 32; ++i) o[i] = floatx16{};
    }
  }

  __device__ __forceinline__ void store_partial(const AttnArgs& a, int sp, int64_t at, int h, bool some) const {
    const int64_t rows = (int64_t)a.B * a.Hkv * a.M;
    if (h == 0)
      reinterpret_cast<floatx2*>(a.part + (int64_t)a.splits * rows * DP)[sp * rows + at] = floatx2{m, l};
    if (some) store_part<DP>(o, a.part + (sp * rows + at) * DP, h);  // the join reads no empty part's sums
  }
  template <bool VEC>
  __device__ __forceinline__ void store(const AttnArgs& a, int b, int qi, int head, int h) const {
    uint16_t* op = (uint16_t*)a.o + b * a.os[0] + (int64_t)qi * a.os[1] + head * a.os[2];
    store_cols<T, DP, VEC>(o, op, l == 0.0f ? 0.0f : 1.0f / l, a.D, h);
    if (a.lse && h == 0) a.lse[((int64_t)b * a.Hq + head) * a.Sq + qi] = log_sum(m, l);
  }
};

// Which part of the keys, rows and heads a workgroup takes, and a lane's row.
struct Place {
  int b, g, sp, t0, t1, row, qi, head, nk;
  bool ok;
  const uint16_t* q;
  const uint8_t* mask;
  __device__ __forceinline__ Place(const AttnArgs& a, const Order& order, int rows_wg, int row_in)
      : Place(a, Item(order, a.splits, a.Hkv, a.B), rows_wg, row_in) {}
  __device__ __forceinline__ Place(const AttnArgs& a, const Item& item, int rows_wg, int row_in) {
    const int mt = item.tile;  // past the last: every row is, too
    sp = item.sp, g = item.g, b = item.b;
    row = mt * rows_wg + row_in;
    qi = row / a.G, head = g * a.G + row % a.G;
    const int nq = clamp_len(a.q_len, b, a.Sq);
    nk = clamp_len(a.kv_len, b, a.Sk);
    ok = row < a.M && qi < nq;
    const int all = (nk + kBN - 1) / kBN, per = (all + a.splits - 1) / a.splits;
    t0 = min(sp * per, all);
    t1 = min(t0 + per, all);
    if ((mt * rows_wg) / a.G >= nq) t1 = t0;  // no row of this workgroup is valid
    q = (const uint16_t*)a.q + b * a.qs[0] + (int64_t)qi * a.qs[1] + head * a.qs[2];
    mask = a.mask ? a.mask + b * a.mask_stride : nullptr;
  }
  __device__ __forceinline__ bool allowed(int j) const { return j < nk && (!mask || mask[j]); }
  // The same in two steps: what the mask says, which may still be on its way (nothing
  // looks at it here), and the answer.
  __device__ __forceinline__ uint32_t mask_at(int j) const { return mask && j < nk ? mask[j] : 1u; }
  __device__ __forceinline__ uint64_t allowed_of(uint32_t m, int j) const { return __ballot(j < nk && m != 0); }
};

// Two groups of four wavefronts with the same rows: adds the second group's sums to
// the first's, by way of LDS that all have done with; false in the second.
template <int DP>
constexpr int kGroupsLds = 4 * 64 * (DP / 8 * 16 + 8);
template <class T, int DP>
__device__ __forceinline__ bool join_groups(Rows<T, DP>& x, void* lds, int wave, int grp, int lane) {
  floatx4* red = reinterpret_cast<floatx4*>(lds) + wave * (DP / 8) * 64 + lane;
  floatx2* red_ml = reinterpret_cast<floatx2*>(reinterpret_cast<floatx4*>(lds) + 4 * (DP / 8) * 64) + wave * 64 + lane;
  wait_reads();
  __syncthreads();
  if (grp == 1) {
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        red[(4 * d + i) * 64] = floatx4{x.o[d][4 * i], x.o[d][4 * i + 1], x.o[d][4 * i + 2], x.o[d][4 * i + 3]};
    *red_ml = floatx2{x.m, x.l};
  }
  __syncthreads();
  if (grp == 1) return false;
  const floatx2 ml = *red_ml;
  const float m = fmaxf(x.m, ml[0]), base = m == -INFINITY ? 0.0f : m;
  const float f0 = __builtin_amdgcn_exp2f(x.m - base), f1 = __builtin_amdgcn_exp2f(ml[0] - base);
  x.m = m;
  x.l = x.l * f0 + ml[1] * f1;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const floatx4 o = red[(4 * d + i) * 64];
#pragma unroll
      for (int j = 0; j < 4; ++j) x.o[d][4 * i + j] = x.o[d][4 * i + j] * f0 + o[j] * f1;
    }
  return true;
}

// NW wavefronts with the same rows: their sums meet in LDS, and the result (or the
// part's) goes to memory.
template <int DP, int NW = 4>
constexpr int kFewLds = NW * 32 * (DP + 4) * 4 + NW * 64 * 4;
template <class T, int DP, int NW = 4>
__device__ __forceinline__ void finish_few(const AttnArgs& a, const Place& at, Rows<T, DP>& x, void* lds, int wave, int lane, int h) {
  // the wavefronts' sums at the largest of their maxima
  __syncthreads();
  float* red = reinterpret_cast<float*>(lds);
  floatx2* red_ml = reinterpret_cast<floatx2*>(red + NW * 32 * (DP + 4));
  x.close(at.ok);
  if (h == 0) red_ml[wave * 32 + lane] = floatx2{x.m, x.l};
  store_part<DP>(x.o, red + (wave * 32 + (lane & 31)) * (DP + 4), h);
  __syncthreads();
  constexpr int kLanes = DP / 4;  // of a row, 4 elements each
  for (int r = threadIdx.x / kLanes; r < min(a.M, 32); r += 64 * NW / kLanes) {
    const int d = 4 * (threadIdx.x % kLanes);
    float m = -INFINITY, l = 0.0f;
    floatx4 o = {};
#pragma unroll
    for (int w = 0; w < NW; ++w) m = fmaxf(m, red_ml[w * 32 + r][0]);
    const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const floatx2 v = red_ml[w * 32 + r];
      const float f = __builtin_amdgcn_exp2f(v[0] - base);
      l += f * v[1];
      o += f * *reinterpret_cast<const floatx4*>(red + (w * 32 + r) * (DP + 4) + d);
    }
    const int64_t rows = (int64_t)a.B * a.Hkv * a.M, row = ((int64_t)at.b * a.Hkv + at.g) * a.M + r;
    if (a.splits > 1) {
      if (d == 0)
        reinterpret_cast<floatx2*>(a.part + (int64_t)a.splits * rows * DP)[at.sp * rows + row] = floatx2{m, l};
      *reinterpret_cast<floatx4*>(a.part + (at.sp * rows + row) * DP + d) = o;
    } else {
      const int qi = r / a.G, head = at.g * a.G + r % a.G;
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;
      store4<true>((uint16_t*)a.o + at.b * a.os[0] + (int64_t)qi * a.os[1] + head * a.os[2] + d,
                   make_uint2(T::pack(o[0] * inv, o[1] * inv), T::pack(o[2] * inv, o[3] * inv)), a.D - d);
      if (a.lse && d == 0) a.lse[((int64_t)at.b * a.Hq + head) * a.Sq + qi] = log_sum(m, l);
    }
  }
}

// Joins the parts of the key axis, in a fixed order: the parts' sums meet at the
// largest of their maxima.  A row is NG groups of DP / 4 lanes, each with every
// NG-th part: one group where rows are many and parts fewer than a workgroup's
// groups (16384 rows of two parts, heads of 64: 4.5 us, 20.6 with a workgroup each), a
// whole workgroup elsewhere (128 rows of 8 parts: 3.3 us, 6.4 with a group each).
template <class T, int DP, int NG>
__global__ __launch_bounds__(256) void k_attn_join(const AttnArgs a) {
  constexpr int kLanes = DP / 4, kRowsWg = 256 / (kLanes * NG);
  const int64_t rows = (int64_t)a.B * a.Hkv * a.M;
  const int64_t at = (int64_t)blockIdx.x * kRowsWg + threadIdx.x / (kLanes * NG);
  const bool ok = at < rows;
  const floatx2* ml = reinterpret_cast<const floatx2*>(a.part + (int64_t)a.splits * rows * DP);
  float m = -INFINITY;
  if constexpr (NG == 1) {
    if (ok)
#pragma unroll 4
      for (int s = 0; s < a.splits; ++s) m = fmaxf(m, ml[s * rows + at][0]);
  } else {
    for (int s = threadIdx.x & 63; s < a.splits; s += 64) m = fmaxf(m, ml[s * rows + at][0]);
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  }
  const int grp = threadIdx.x / kLanes % NG, d4 = 4 * (threadIdx.x % kLanes);
  floatx4 acc = {};
  float l = 0.0f;
  if (ok)
#pragma unroll 2
    for (int s = grp; s < a.splits; s += NG) {
      const floatx2 v = ml[s * rows + at];
      // a part without an allowed key has no sums (NaN scores: the sum is NaN)
      if (v[0] == -INFINITY && v[1] == 0.0f) continue;
      const float w = __builtin_amdgcn_exp2f(v[0] - (m == -INFINITY ? 0.0f : m));
      l += w * v[1];
      acc += w * *reinterpret_cast<const floatx4*>(a.part + (s * rows + at) * DP + d4);
    }
  if constexpr (NG > 1) {  // one row: the groups' sums
    __shared__ floatx4 red[NG][kLanes];
    __shared__ float red_l[NG];
    red[grp][d4 / 4] = acc;
    if (d4 == 0) red_l[grp] = l;
    __syncthreads();
    if (grp > 0) return;
    acc = floatx4{};
    l = 0.0f;
    for (int i = 0; i < NG; ++i) acc += red[i][d4 / 4], l += red_l[i];
  }
  if (!ok) return;
  const uint32_t bg = (uint32_t)at / a.M, row = (uint32_t)at % a.M;
  const int g = bg % a.Hkv, b = bg / a.Hkv, qi = row / a.G, head = g * a.G + row % a.G;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  uint16_t* op = (uint16_t*)a.o + b * a.os[0] + (int64_t)qi * a.os[1] + head * a.os[2] + d4;
  const uint2 x = make_uint2(T::pack(acc[0] * inv, acc[1] * inv), T::pack(acc[2] * inv, acc[3] * inv));
  if (a.vec)
    store4<true>(op, x, min(a.D - d4, 4));
  else
    store4<false>(op, x, min(a.D - d4, 4));
  if (a.lse && d4 == 0) a.lse[((int64_t)b * a.Hq + head) * a.Sq + qi] = log_sum(m, l);
}

template <class T, int DP>
void join(const AttnArgs& a, hipStream_t s) {
  if (a.splits == 1) return;
  constexpr int kGroups = 256 / (DP / 4);
  const int64_t all = (int64_t)a.B * a.Hkv * a.M;
  if (a.splits < kGroups && all > 2 * kCUs)
    k_attn_join<T, DP, 1><<<(unsigned)((all + kGroups - 1) / kGroups), 256, 0, s>>>(a);
  else
    k_attn_join<T, DP, kGroups><<<(unsigned)all, 256, 0, s>>>(a);
}

}  // namespace
}  // namespace pnerf
#endif
