// Cross attention, forward: o_i = sum_j exp(a_ij - lse_i) v_j over the allowed
// keys j, a_ij = scale q_i . k_j, for queries and keys of different lengths.
//
// The query heads that share a kv head are rows of one product: row r of kv head
// g is query row r / G, head g G + r % G.  A wavefront holds 32 rows and passes
// over tiles of 64 keys with the running maximum m and sum l of each row's
// softmax:
//   S^T = K Q^T     (A = keys from LDS, B = the rows' queries, in registers)
//   P = exp2(c S - m), l += sum P
//   O^T += V^T P^T  (A = values by transposed LDS reads, B = P)
// Both products have the row as their column, so that all of a row's scores are
// in two lanes (l and l + 32): the softmax needs one exchange a tile, and P is
// the second product's B operand as it stands -- lane half h holds keys
// 8 i + 4 h + 0..3, an order of the contraction that the value reads follow.
//
// Keys and values go from memory to LDS by loads that write LDS themselves.  A
// key that may not be read (past its length, masked) and the elements past the
// head's width are zeros there: its lanes take an offset beyond the descriptor's
// bound, so that what such a place holds never enters a product.
#define PNERF_LAYERS_DEVICE
#include <algorithm>

#include "attention_common.h"

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
  // Adds the tile whose scores are there.
  __device__ __forceinline__ void add(const uint4* sv, float c, int lane) {
    constexpr int CH = DP / 8;
    const float base = m == -INFINITY ? 0.0f : m;  // no allowed key yet
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[n][i] = __builtin_amdgcn_exp2f(fmaf(s[n][i], c, -base));
        l += s[n][i];
      }
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
  __device__ __forceinline__ Place(const AttnArgs& a, const Order& order, int rows_wg, int row_in) {
    const Item item(order, a.splits, a.Hkv, a.B);
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
};

// Many rows: four wavefronts of 32 rows share the tiles, two of them in LDS: the
// loads of the next run while the products of one do.  One barrier a tile.
// KS = 2: two such groups with the same rows take the tiles in turn, each with its
// own LDS, and join at the end: where workgroups are few (two_groups) that puts a
// second wavefront on every SIMD (1024 rows, 1200 keys, 2 x 16 heads of 64, one
// workgroup a CU: 33 us with one group, 22 with two; 2048 rows, 4096 keys, 16 heads
// of 128: 0.84 PFLOP/s with two, 0.54 with one on 17 heads).
template <class T, int DP, int KS>
__global__ __launch_bounds__(256 * KS, 3 - KS) void k_attn_fwd(const AttnArgs a, const Order order) {
  using Tile = RowTile<DP, 4>;
  __shared__ uint4 lds[KS][2][2 * Tile::kPieces];  // keys, then values
  const int lane = threadIdx.x & 63, all_waves = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int wave = all_waves & 3, grp = all_waves >> 2;
  const Place at(a, order, 128, wave * 32 + (lane & 31));
  const Tile kt(a.k, at.b * a.ks[0] + at.g * a.ks[2], a.ks[1], a.D, wave, lane);
  const Tile vt(a.v, at.b * a.vs[0] + at.g * a.vs[2], a.vs[1], a.D, wave, lane);
  Rows<T, DP> x;
  x.template init<true>(at.q, at.ok, a.D, h);
  const uint32_t to[2] = {lds_address(lds[grp][0]), lds_address(lds[grp][1])};
  auto load = [&](int buf, int t, uint64_t vm) {
    kt.load(to[buf], t, at.nk, vm, lane);
    vt.load(to[buf] + 16 * Tile::kPieces, t, at.nk, vm, lane);
  };
  uint64_t vm = 0, vm_next = 0;
  bool allowed = false;  // key `lane` of the tile after the next
  int t = at.t0 + grp;
  if (t < at.t1) {
    vm_next = __ballot(at.allowed(t * kBN + lane));
    load(0, t, vm_next);
    allowed = at.allowed((t + KS) * kBN + lane);
  }
  const int rounds = (at.t1 - at.t0 + KS - 1) / KS;  // the same for both groups: they share the barrier
  int round = 0;
  x.run(
      a.c, lane,
      [&] {
        if (round == rounds) return false;
        const int buf = round & 1;
        wait_loads();
        __builtin_amdgcn_s_barrier();  // this tile is there, and the one before has been read
        vm = vm_next;
        vm_next = __ballot(allowed);
        const bool here = t < at.t1;  // the last round may have no tile for the second group
        t += KS;
        if (t < at.t1) {
          load(buf ^ 1, t, vm_next);
          allowed = at.allowed((t + KS) * kBN + lane);
        }
        if (!here) return false;
        x.scores(lds[grp][buf], vm, a.c, lane);
        ++round;
        return true;
      },
      [&] { return lds[grp][(round - 1) & 1] + Tile::kPieces; });
  if constexpr (KS == 2) {
    static_assert(4 * 64 * (DP / 8 * 16 + 8) <= sizeof(lds), "a group's sums fit LDS");
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
    if (grp == 1) return;
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
  }
  x.close(at.ok);
  if (at.row >= a.M) return;
  if (a.splits > 1)
    x.store_partial(a, at.sp, ((int64_t)at.b * a.Hkv + at.g) * a.M + at.row, h, at.t0 < at.t1);
  else
    x.template store<true>(a, at.b, at.qi, at.head, h);
}

// At most 32 rows of a kv head (single tokens): the bytes of the states are the
// time.  Four wavefronts with the same rows take the tiles in turn, each with its
// own keys and values in LDS and no barrier; keys are loaded again as soon as the
// scores are there, values as soon as they have been used.  At the end the
// wavefronts' sums meet in LDS.
template <class T, int DP>
__global__ __launch_bounds__(256) void k_attn_few(const AttnArgs a, const Order order) {
  using Tile = RowTile<DP, 1>;
  __shared__ uint4 lds[4][2 * Tile::kPieces];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const Place at(a, order, 32, lane & 31);
  const Tile kt(a.k, at.b * a.ks[0] + at.g * a.ks[2], a.ks[1], a.D, 0, lane);
  const Tile vt(a.v, at.b * a.vs[0] + at.g * a.vs[2], a.vs[1], a.D, 0, lane);
  Rows<T, DP> x;
  x.template init<true>(at.q, at.ok, a.D, h);
  uint4 *sk = lds[wave], *sv = sk + Tile::kPieces;
  const uint32_t to_k = lds_address(sk), to_v = lds_address(sv);
  int t = at.t0 + wave;    // of the next scores
  uint64_t vm_next = 0;    // its keys that may be read
  bool allowed = false, first = true;
  if (t < at.t1) {
    vm_next = __ballot(at.allowed(t * kBN + lane));
    kt.load(to_k, t, at.nk, vm_next, lane);
    vt.load(to_v, t, at.nk, vm_next, lane);
    allowed = at.allowed((t + 4) * kBN + lane);
  }
  x.run(
      a.c, lane,
      [&] {
        if (!first) {
          wait_reads();  // the values before have been used
          if (t < at.t1) vt.load(to_v, t, at.nk, vm_next, lane);
        }
        if (t >= at.t1) return false;
        first = false;
        wait_loads();
        const uint64_t vm = vm_next;
        vm_next = __ballot(allowed);
        x.scores(sk, vm, a.c, lane);
        wait_reads();
        t += 4;
        if (t < at.t1) {
          kt.load(to_k, t, at.nk, vm_next, lane);
          allowed = at.allowed((t + 4) * kBN + lane);
        }
        return true;
      },
      [&] { return sv; });

  // the wavefronts' sums at the largest of their maxima
  __syncthreads();
  float* red = reinterpret_cast<float*>(lds);
  static_assert(4 * 32 * (DP + 4) * 4 + 4 * 64 * 4 <= sizeof(lds), "the sums fit the tiles' LDS");
  floatx2* red_ml = reinterpret_cast<floatx2*>(red + 4 * 32 * (DP + 4));
  x.close(at.ok);
  if (h == 0) red_ml[wave * 32 + lane] = floatx2{x.m, x.l};
  store_part<DP>(x.o, red + (wave * 32 + (lane & 31)) * (DP + 4), h);
  __syncthreads();
  constexpr int kLanes = DP / 4;  // of a row, 4 elements each
  for (int r = threadIdx.x / kLanes; r < min(a.M, 32); r += 256 / kLanes) {
    const int d = 4 * (threadIdx.x % kLanes);
    float m = -INFINITY, l = 0.0f;
    floatx4 o = {};
#pragma unroll
    for (int w = 0; w < 4; ++w) m = fmaxf(m, red_ml[w * 32 + r][0]);
    const float base = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
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

// Any strides, alignment and head width: as k_attn_fwd, the tiles by way of
// registers, element by element.
template <class T, int DP>
__global__ __launch_bounds__(256) void k_attn_any(const AttnArgs a, const Order order) {
  __shared__ uint4 sk[kBN * DP / 8], sv[kBN * DP / 8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
  const Place at(a, order, 128, wave * 32 + (lane & 31));
  Rows<T, DP> x;
  x.template init<false>(at.q, at.ok, a.D, h);
  int t = at.t0;
  x.run(
      a.c, lane,
      [&] {
        if (t >= at.t1) return false;
        const uint64_t vm = __ballot(at.allowed(t * kBN + lane));
        __syncthreads();
        copy_tile<DP>(sk, a.k, a.ks, at.b, at.g, a.D, t, vm);
        copy_tile<DP>(sv, a.v, a.vs, at.b, at.g, a.D, t, vm);
        __syncthreads();
        x.scores(sk, vm, a.c, lane);
        ++t;
        return true;
      },
      [&] { return sv; });
  x.close(at.ok);
  if (at.row >= a.M) return;
  if (a.splits > 1)
    x.store_partial(a, at.sp, ((int64_t)at.b * a.Hkv + at.g) * a.M + at.row, h, at.t0 < at.t1);
  else
    x.template store<false>(a, at.b, at.qi, at.head, h);
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
void launch(const AttnArgs& a, hipStream_t s) {
  const bool few = a.M <= 32;
  const int rows = few ? 32 : 128;
  const Order o = order_of(((int64_t)a.M + rows - 1) / rows, a.Hkv);
  const unsigned n = (unsigned)workgroups(o, a.splits, a);
  if (!fast_loads(a))
    k_attn_any<T, DP><<<n, 256, 0, s>>>(a, o);
  else if (few)
    k_attn_few<T, DP><<<n, 256, 0, s>>>(a, o);
  else if (two_groups(n, a))
    k_attn_fwd<T, DP, 2><<<n, 512, 0, s>>>(a, o);
  else
    k_attn_fwd<T, DP, 1><<<n, 256, 0, s>>>(a, o);
  if (a.splits == 1) return;
  constexpr int kGroups = 256 / (DP / 4);
  const int64_t all = (int64_t)a.B * a.Hkv * a.M;
  if (a.splits < kGroups && all > 2 * kCUs)
    k_attn_join<T, DP, 1><<<(unsigned)((all + kGroups - 1) / kGroups), 256, 0, s>>>(a);
  else
    k_attn_join<T, DP, kGroups><<<(unsigned)all, 256, 0, s>>>(a);
}

}  // namespace

// Few workgroups leave compute units idle: where there are not enough for half of
// them, the keys are cut into parts, of at least 4 tiles (16 for few rows, where
// 4 wavefronts share a part) each.
int attn_fwd_splits(const AttnArgs& a) {
  const bool few = a.M <= 32;
  const int rows = few ? 32 : 128;
  const int64_t wgs = (int64_t)((a.M + rows - 1) / rows) * a.Hkv * a.B;
  const int64_t tiles = (a.Sk + kBN - 1) / kBN;
  if (wgs == 0) return 1;
  return (int)std::max<int64_t>(1, std::min(kCUs / wgs, tiles / (few ? 16 : 4)));
}

int64_t attn_fwd_bytes(const AttnArgs& a) {
  if (a.splits <= 1) return 0;
  return (int64_t)a.splits * a.B * a.Hkv * a.M * (padded(a.D) + 2) * 4;
}

hipError_t launch_attn_fwd(const AttnArgs& a0, void* ws, hipStream_t s) {
  AttnArgs a = a0;
  a.part = (float*)ws;
  if (a.B == 0 || a.M == 0) return hipSuccess;
  const bool wide = padded(a.D) == 128;
  if (a.dtype == kF16)
    wide ? launch<F16, 128>(a, s) : launch<F16, 64>(a, s);
  else
    wide ? launch<BF16, 128>(a, s) : launch<BF16, 64>(a, s);
  return hipGetLastError();
}

}  // namespace pnerf
