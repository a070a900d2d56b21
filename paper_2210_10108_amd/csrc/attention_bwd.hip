// Cross attention, backward.  With p_ij = exp(a_ij - lse_i) recomputed from the
// row's log-sum, delta_i = do_i . o_i and ds_ij = p_ij (do_i . v_j - delta_i):
//   dv_j = sum_i p_ij do_i,  dk_j = scale sum_i ds_ij q_i,  dq_i = scale sum_j ds_ij k_j
// Three kernels, no atomics: the rows' (lse, delta); dq by workgroups that own
// rows and pass over the keys; dk and dv by workgroups that own keys and pass
// over the rows of all the query heads that share their kv head, so that the
// sum over those heads never leaves the registers.  s and dp are computed twice (7
// products where 5 would do): dq from the second kernel would have to be added up
// in memory, by atomics, whose order changes the result, or from as many partial
// sums as there are tiles of keys.
//
// Fragments as in the forward kernel: what the second products contract over is
// in the registers of the first ones' results, as their B operand.
//
// Float16 and its range: p and ds are rounded to 16 bits as operands, and float16
// has normal numbers from 2^-14 to 2^16 alone.  p is at most 1 and is kept times
// 2^14.  ds may be anything: |ds_ij| <= |do_i| |v_j| + |delta_i|, and |delta_i| <= |do_i|
// max |v|.  Both kernels hold a row (dq) or a key (dk) a lane and contract over the
// other, so each lane keeps its ds times a power of two of its own, by which that
// bound lies in [2^14, 2^15), and divides its sums by it: no ds overflows, and one
// is a normal number down to 2^-28 of the bound.  The norms are made with the rows'
// statistics and a workgroup takes the largest of its part at its start (the whole
// gradient with it and without: 333 and 326 us for 2 x 2011 rows, 2500 keys, 16 heads of
// 128; 70 and 63 for 2 x 1024 rows, 1200 keys, 16 heads of 64).
#define PNERF_LAYERS_DEVICE
#include <algorithm>
#include <type_traits>

#include "attention_common.h"

namespace pnerf {
namespace {

constexpr int kKeys = 128;  // keys of a workgroup of the dk, dv pass: 32 a wavefront
// Rows of one of its tiles.
constexpr int dkv_rows(int width, bool fast) { return fast && width == 128 ? 32 : 64; }

template <class T>
constexpr bool kNarrow = std::is_same_v<T, F16>;  // p and ds are kept times powers of two
template <class T>
constexpr int kBitsP = kNarrow<T> ? 14 : 0;       // ... p times 2^kBitsP

// The power of two by which a number of at most `bound` stays below 2^15.  (A delta
// may be as small as p is, and with it the bound: the power has an end.)
__device__ __forceinline__ int bits_within(float bound) {
  return bound > 0.0f ? 15 - max(__builtin_amdgcn_frexp_expf(bound), -80) : 0;
}
// The maximum of x over the NW wavefronts of a workgroup, by way of red.
template <int NW>
__device__ __forceinline__ float max_of_all(float x, float* red) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x = fmaxf(x, __shfl_xor(x, d));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
  __syncthreads();
  x = red[0];
#pragma unroll
  for (int i = 1; i < NW; ++i) x = fmaxf(x, red[i]);
  return x;
}
// The sum of squares of 8 elements.
template <class T>
__device__ __forceinline__ float squares(uint4 x) {
  return T::lo(x.x) * T::lo(x.x) + T::hi(x.x) * T::hi(x.x) + T::lo(x.y) * T::lo(x.y) + T::hi(x.y) * T::hi(x.y) +
         T::lo(x.z) * T::lo(x.z) + T::hi(x.z) * T::hi(x.z) + T::lo(x.w) * T::lo(x.w) + T::hi(x.w) * T::hi(x.w);
}

// |v| of key `at` in memory order, DP / 8 lanes a key with 8 elements each from d.
template <class T, int DP, bool VEC>
__device__ __forceinline__ void v_norm(const AttnArgs& a, int64_t at, int d) {
  const int g = (int)(at % a.Hkv), bj = (int)(at / a.Hkv), j = bj % a.Sk, b = bj / a.Sk;
  const bool ok = j < clamp_len(a.kv_len, b, a.Sk) && (!a.mask || a.mask[b * a.mask_stride + j]);
  float sq = squares<T>(load8<VEC>((const uint16_t*)a.v + b * a.vs[0] + (int64_t)j * a.vs[1] + g * a.vs[2] + d,
                                   ok ? min(a.D - d, 8) : 0));
#pragma unroll
  for (int m = DP / 16; m; m >>= 1) sq += __shfl_xor(sq, m);
  if (d == 0) a.v_norm[((int64_t)b * a.Hkv + g) * a.Sk + j] = sqrtf(sq);
}

// (lse / ln 2 - kBitsP, delta) of every row; (+inf, 0) where the row has no
// allowed key or is past q_len, which makes all of its p zero.  Float16: |do| too,
// and in the grid's second row |v| of every key (0 where it may not be read).
template <class T, int DP, bool VEC>
__global__ __launch_bounds__(256) void k_attn_stat(const AttnArgs a) {
  constexpr int LR = DP / 8;  // lanes of a row
  const int64_t rows = (int64_t)a.B * a.Hq * a.Sq;
  const int64_t at = (int64_t)blockIdx.x * (256 / LR) + threadIdx.x / LR;
  const int d = 8 * (threadIdx.x % LR);
  if constexpr (kNarrow<T>) {
    if (blockIdx.y == 1) {
      if (at < (int64_t)a.B * a.Hkv * a.Sk) v_norm<T, DP, VEC>(a, at, d);
      return;
    }
  }
  float sum = 0.0f;
  if (at < rows) {
    // neighbours are the heads of one row, as they are in memory
    const int head = (int)(at % a.Hq), bq = (int)(at / a.Hq), qi = bq % a.Sq, b = bq / a.Sq;
    const int64_t out = ((int64_t)b * a.Hq + head) * a.Sq + qi;
    const float lse = a.lse[out];
    const bool ok = qi < clamp_len(a.q_len, b, a.Sq) && lse != -INFINITY;
    const int n = ok ? min(a.D - d, 8) : 0;
    const uint4 x = load8<VEC>((const uint16_t*)a.o + b * a.os[0] + (int64_t)qi * a.os[1] +
                                   head * a.os[2] + d, n);
    const uint4 y = load8<VEC>((const uint16_t*)a.dout + b * a.dos[0] + (int64_t)qi * a.dos[1] +
                                   head * a.dos[2] + d, n);
    sum = T::lo(x.x) * T::lo(y.x) + T::hi(x.x) * T::hi(y.x) + T::lo(x.y) * T::lo(y.y) +
          T::hi(x.y) * T::hi(y.y) + T::lo(x.z) * T::lo(y.z) + T::hi(x.z) * T::hi(y.z) +
          T::lo(x.w) * T::lo(y.w) + T::hi(x.w) * T::hi(y.w);
#pragma unroll
    for (int m = LR / 2; m; m >>= 1) sum += __shfl_xor(sum, m);
    if (d == 0)
      reinterpret_cast<floatx2*>(a.delta)[out] =
          ok ? floatx2{lse * 1.4426950408889634f - (float)kBitsP<T>, sum} : floatx2{INFINITY, 0.0f};
    if constexpr (kNarrow<T>) {
      float sq = squares<T>(y);
#pragma unroll
      for (int m = LR / 2; m; m >>= 1) sq += __shfl_xor(sq, m);
      if (d == 0) a.do_norm[out] = sqrtf(sq);
    }
  }
}


// dq: four wavefronts of 32 rows share the tiles of keys and values, two of them
// in LDS (FAST; else one, by way of registers).  As in the forward kernel the row
// is the column of every product: its lse and delta are a lane's own; and KS = 2
// groups of wavefronts take the tiles in turn where workgroups are few.
template <class T, int DP, bool FAST, int KS>
__global__ __launch_bounds__(256 * KS, 3 - KS) void k_attn_dq(const AttnArgs a, const Order order, int splits, float* part) {
  constexpr int CH = DP / 8, NS = DP / 16, ND = DP / 32;
  using Tile = RowTile<DP, 4>;
  __shared__ uint4 lds[KS][FAST ? 2 : 1][2 * Tile::kPieces];  // keys, then values

  const Item item(order, splits, a.Hkv, a.B);
  const int mt = item.tile, sp = item.sp, g = item.g, b = item.b;  // past the last tile every row is past the last
  const int lane = threadIdx.x & 63, all_waves = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave = all_waves & 3, grp = all_waves >> 2;
  const int r = lane & 31, h = lane >> 5;
  const int row = mt * 128 + wave * 32 + r;
  const int qi = row / a.G, head = g * a.G + row % a.G;
  const int nq = clamp_len(a.q_len, b, a.Sq), nk = clamp_len(a.kv_len, b, a.Sk);
  int t1 = (nk + kBN - 1) / kBN;
  const int per = (t1 + splits - 1) / splits, t0 = min(sp * per, t1);
  t1 = min(t0 + per, t1);
  if ((mt * 128) / a.G >= nq) t1 = t0;

  const int64_t rows = (int64_t)a.B * a.Hkv * a.M;
  const int64_t at = ((int64_t)b * a.Hkv + g) * a.M + row;
  floatx2* stat = reinterpret_cast<floatx2*>(a.delta) + ((int64_t)b * a.Hq + head) * a.Sq + qi;
  floatx2 st = floatx2{INFINITY, 0.0f};
  if (row < a.M) st = *stat;
  const bool ok = st[0] != INFINITY;

  const uint16_t* qp = (const uint16_t*)a.q + b * a.qs[0] + (int64_t)qi * a.qs[1] + head * a.qs[2];
  const uint16_t* gp = (const uint16_t*)a.dout + b * a.dos[0] + (int64_t)qi * a.dos[1] + head * a.dos[2];
  const uint8_t* mp = a.mask ? a.mask + b * a.mask_stride : nullptr;
  auto may_read = [&](int j) { return j < nk && (!mp || mp[j]); };
  uint4 qf[NS], gf[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const int d = 16 * s + 8 * h, n = ok ? min(a.D - d, 8) : 0;
    qf[s] = load8<FAST>(qp + d, n);
    gf[s] = load8<FAST>(gp + d, n);
  }
  floatx16 acc[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i) acc[i] = floatx16{};

  const Tile kt(a.k, b * a.ks[0] + g * a.ks[2], a.ks[1], a.D, wave, lane);
  const Tile vt(a.v, b * a.vs[0] + g * a.vs[2], a.vs[1], a.D, wave, lane);
  const uint32_t to[2] = {lds_address(lds[grp][0]), lds_address(lds[grp][FAST])};
  auto load = [&](int buf, int t, uint64_t vm) {
    kt.load(to[buf], t, nk, vm, lane);
    vt.load(to[buf] + 16 * Tile::kPieces, t, nk, vm, lane);
  };
  uint64_t vm_next = 0;
  bool allowed = false;  // key `lane` of the tile after the next
  int t = t0 + grp;
  if (FAST && t < t1) {
    vm_next = __ballot(may_read(t * kBN + lane));
    load(0, t, vm_next);
    allowed = may_read((t + KS) * kBN + lane);
  }
  int bits = 0;  // of this row's ds
  if constexpr (kNarrow<T>) {
    __shared__ float red[4 * KS];
    const float* norms = a.v_norm + ((int64_t)b * a.Hkv + g) * a.Sk;
    float v = 0.0f;
#pragma unroll 4
    for (int j = t0 * kBN + threadIdx.x; j < min(t1 * kBN, nk); j += 256 * KS) v = fmaxf(v, norms[j]);
    v = max_of_all<4 * KS>(v, red);
    if (ok) bits = bits_within(2.0f * v * a.do_norm[((int64_t)b * a.Hq + head) * a.Sq + qi]);
    st[0] += (float)(kBitsP<T> - bits);  // p of this kernel is kept times 2^bits
  }
  const int rounds = (t1 - t0 + KS - 1) / KS;  // the same for both groups: they share the barrier
  for (int round = 0; round < rounds; ++round, t += KS) {
    const int buf = FAST ? round & 1 : 0;
    const uint4 *sk = lds[grp][buf], *sv = sk + Tile::kPieces;
    uint64_t vm;
    if (FAST) {
      wait_loads();
      __builtin_amdgcn_s_barrier();  // this tile is there, and the one before has been read
      vm = vm_next;
      vm_next = __ballot(allowed);
      if (t + KS < t1) {
        load(buf ^ 1, t + KS, vm_next);
        allowed = may_read((t + 2 * KS) * kBN + lane);
      }
      if (t >= t1) break;  // the last round has no tile for this group
    } else {
      vm = __ballot(may_read(t * kBN + lane));
      __syncthreads();
      copy_tile<DP>(lds[0][0], a.k, a.ks, b, g, a.D, t, vm);
      copy_tile<DP>(lds[0][0] + Tile::kPieces, a.v, a.vs, b, g, a.D, t, vm);
      __syncthreads();
    }
    auto first = [&](int n, floatx16& s, floatx16& dp) {
      s = dp = floatx16{};
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        const int p = swz<CH>(32 * n + r, 2 * i + h);
        s = T::mma(sk[p], qf[i], s);
        dp = T::mma(sv[p], gf[i], dp);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], a.c, -st[0]));
    };
    if (nk <= kBN) {
      // few keys: o's rounding weighs on do . o, so delta is taken as sum_j p dp,
      // which this one tile holds, for the dk, dv pass as well
      float sum = 0.0f;
#pragma unroll 1
      for (int n = 0; n < 2; ++n) {
        floatx16 s, dp;
        first(n, s, dp);
        const uint32_t w = (uint32_t)(vm >> (32 * n)) >> (4 * h);
#pragma unroll
        for (int i = 0; i < 16; ++i) sum += (w >> (8 * (i / 4) + i % 4)) & 1 ? s[i] * dp[i] : 0.0f;
      }
      float s0, s1;
      halves(sum, s0, s1);
      st[1] = ldexpf(s0 + s1, -bits);
      if (h == 0 && ok) (*stat)[1] = st[1];
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      floatx16 s, dp;
      first(n, s, dp);
      const uint32_t valid = (uint32_t)(vm >> (32 * n));
      if (valid == ~0u) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] *= dp[i] - st[1];
      } else {
        const uint32_t w = valid >> (4 * h);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = (w >> (8 * (i / 4) + i % 4)) & 1 ? s[i] * (dp[i] - st[1]) : 0.0f;
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint4 f = pack8<T>(s, 8 * k);
#pragma unroll
        for (int d = 0; d < ND; ++d)
          acc[d] = T::mma(tr_frag<CH>(sk, 32 * n + 16 * k, 32 * d, lane), f, acc[d]);
      }
    }
  }
  if constexpr (KS == 2) {
    static_assert(4 * 64 * (DP / 8) * 16 <= sizeof(lds), "a group's sums fit LDS");
    floatx4* red = reinterpret_cast<floatx4*>(lds) + wave * (DP / 8) * 64 + lane;
    wait_reads();
    __syncthreads();
    if (grp == 1)
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          red[(4 * d + i) * 64] = floatx4{acc[d][4 * i], acc[d][4 * i + 1], acc[d][4 * i + 2], acc[d][4 * i + 3]};
    __syncthreads();
    if (grp == 1) return;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const floatx4 o = red[(4 * d + i) * 64];
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[d][4 * i + j] += o[j];
      }
  }
  if (row >= a.M) return;
  const float back = ldexpf(1.0f, -bits);
  if (splits > 1) {
    if (t0 < t1) store_part<DP>(acc, part + (sp * rows + at) * DP, h, back);
  } else {
    uint16_t* out = (uint16_t*)a.dq + b * a.dqs[0] + (int64_t)qi * a.dqs[1] + head * a.dqs[2];
    store_cols<T, DP, FAST>(acc, out, a.scale * back, a.D, h);
  }
}

// dk and dv: a wavefront holds 32 keys and values, as columns, and passes over
// the query heads of its kv head and their rows, in tiles of one head's rows
// (whose addresses are a plain progression) that the workgroup's wavefronts share.
// At the wide head the sums take 128 registers and the keys 32; the values, each
// lane's its own, wait in LDS, which leaves registers for two wavefronts a SIMD
// (4 x 4096 rows and keys, 16 heads of 128, bf16: 1.00 to 1.05 PFLOP/s; with the values in
// registers and one wavefront a SIMD 0.70).  The tiles are then of 32 rows.
template <class T, int DP, bool FAST>
__global__ __launch_bounds__(256, FAST ? 2 : 1) void k_attn_dkv(const AttnArgs a, const Order order, int splits, float* part) {
  constexpr bool kStash = FAST && DP == 128;
  constexpr int CH = DP / 8, NS = DP / 16, ND = DP / 32, kR = dkv_rows(DP, FAST), kPieces = kR * CH;
  __shared__ uint4 lds[FAST ? 2 : 1][2 * kPieces + 64];  // queries, their gradients, (lse, delta) of each row
  __shared__ uint4 stash[kStash ? 4 : 1][kStash ? NS : 1][64];

  const Item item(order, splits, a.Hkv, a.B);
  const int kt = item.tile, sp = item.sp, g = item.g, b = item.b;  // past the last tile every key is past the last
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & 31, h = lane >> 5;
  const int key = kt * kKeys + wave * 32 + r;
  const int nq = clamp_len(a.q_len, b, a.Sq), nk = clamp_len(a.kv_len, b, a.Sk);
  const bool ok = key < nk && (!a.mask || a.mask[b * a.mask_stride + key]);
  const int tiles_q = (nq + kR - 1) / kR;  // of a head
  int t1 = tiles_q * a.G;
  const int per = (t1 + splits - 1) / splits, t0 = min(sp * per, t1);
  t1 = min(t0 + per, t1);
  if (kt * kKeys >= nk) t1 = t0;

  const uint16_t* kp = (const uint16_t*)a.k + b * a.ks[0] + (int64_t)key * a.ks[1] + g * a.ks[2];
  const uint16_t* vp = (const uint16_t*)a.v + b * a.vs[0] + (int64_t)key * a.vs[1] + g * a.vs[2];
  uint4 kf[NS], vf[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const int d = 16 * s + 8 * h, n = ok ? min(a.D - d, 8) : 0;
    kf[s] = load8<FAST>(kp + d, n);
    vf[s] = load8<FAST>(vp + d, n);
    if (kStash) stash[wave][s][lane] = vf[s];
  }
  floatx16 dk[ND], dv[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i) dk[i] = dv[i] = floatx16{};

  const float* stat = a.delta + 2 * ((int64_t)b * a.Hq + g * a.G) * a.Sq;
  RowTile<DP, 4, kR> qt(a.q, b * a.qs[0] + (int64_t)g * a.G * a.qs[2], a.qs[1], a.D, wave, lane);
  RowTile<DP, 4, kR> gt(a.dout, b * a.dos[0] + (int64_t)g * a.G * a.dos[2], a.dos[1], a.D, wave, lane);
  const uint32_t to[2] = {lds_address(lds[0]), lds_address(lds[FAST])};
  int head = 0, tile = t0;  // of the next tile: its head and its number there
  if (t0 < t1) {
    head = t0 / tiles_q, tile = t0 - head * tiles_q;
    qt.base += 2 * head * a.qs[2], gt.base += 2 * head * a.dos[2];
    stat += 2 * (int64_t)head * a.Sq;
  }
  auto next = [&] {
    if (++tile < tiles_q) return;
    tile = 0;
    ++head;
    qt.base += 2 * a.qs[2], gt.base += 2 * a.dos[2];
    stat += 2 * a.Sq;
  };
  auto load = [&](int buf) {  // the next tile; past the last row all is zeros
    qt.load(to[buf], tile, nq, ~0ull, lane);
    gt.load(to[buf] + 16 * kPieces, tile, nq, ~0ull, lane);
    if (wave == 0)
      load_to_lds(to[buf] + 32 * kPieces, lane < kR / 2 ? 16 * lane : kOutside,
                  descriptor(stat + 2 * tile * kR, (int64_t)(nq - tile * kR) * 8));
    next();
  };
  auto copy = [&] {
    __syncthreads();
    for (int e = tid; e < kPieces; e += 256) {
      const int qi = tile * kR + e / CH, d = 8 * (e % CH);
      const int n = qi < nq ? min(a.D - d, 8) : 0, p = swz<CH>(e / CH, e % CH);
      lds[0][p] = load8<false>((const uint16_t*)qt.base + qi * a.qs[1] + d, n);
      lds[0][kPieces + p] = load8<false>((const uint16_t*)gt.base + qi * a.dos[1] + d, n);
    }
    if (tid < 2 * kR)
      reinterpret_cast<float*>(lds[0] + 2 * kPieces)[tid] = tile * kR + tid / 2 < nq ? stat[2 * tile * kR + tid] : 0.0f;
    __syncthreads();
    next();
  };
  if (FAST && t0 < t1) load(t0 & 1);
  int bits = 0;  // of this key's ds
  if constexpr (kNarrow<T>)
    if (t0 < t1) {
      // the largest |do| and |delta| of this part's rows, from its first to its last
      __shared__ float red[2][4];
      const int64_t head0 = ((int64_t)b * a.Hq + g * a.G) * a.Sq;
      const int h0 = t0 / tiles_q, h1 = (t1 - 1) / tiles_q;
      const int i0 = h0 * a.Sq + (t0 - h0 * tiles_q) * kR, i1 = h1 * a.Sq + min((t1 - h1 * tiles_q) * kR, nq);
      float x = 0.0f, y = 0.0f;
#pragma unroll 4
      for (int i = i0 + tid; i < i1; i += 256) {
        x = fmaxf(x, a.do_norm[head0 + i]);
        y = fmaxf(y, fabsf(a.delta[2 * (head0 + i) + 1]));
      }
      x = max_of_all<4>(x, red[0]);
      y = max_of_all<4>(y, red[1]);
      if (ok) bits = bits_within(fmaf(x, a.v_norm[((int64_t)b * a.Hkv + g) * a.Sk + key], y));
    }
  const float up = ldexpf(1.0f, bits - kBitsP<T>);  // ds comes out times 2^kBitsP, as p does
  for (int t = t0; t < t1; ++t) {
    if (FAST) {
      wait_loads();
      __builtin_amdgcn_s_barrier();  // this tile is there, and the one before has been read
      if (t + 1 < t1) load((t + 1) & 1);
    } else {
      copy();
    }
    const uint4 *sq = lds[FAST ? t & 1 : 0], *sg = sq + kPieces;
    const floatx4* sst = reinterpret_cast<const floatx4*>(sg + kPieces);
#pragma unroll
    for (int n = 0; n < kR / 32; ++n) {
      floatx16 s = {}, dp = {};
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        const int p = swz<CH>(32 * n + r, 2 * i + h);
        s = T::mma(sq[p], kf[i], s);
        dp = T::mma(sg[p], kStash ? stash[wave][i][lane] : vf[i], dp);
      }
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const floatx4 st = sst[16 * n + 4 * (i / 4) + 2 * h + i % 4 / 2];  // two rows
        s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], a.c, -st[0]));
        s[i + 1] = __builtin_amdgcn_exp2f(fmaf(s[i + 1], a.c, -st[2]));
        dp[i] = s[i] * (dp[i] - st[1]);
        dp[i + 1] = s[i + 1] * (dp[i + 1] - st[3]);
        if (kNarrow<T>) dp[i] *= up, dp[i + 1] *= up;
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint4 pf = pack8<T>(s, 8 * k), df = pack8<T>(dp, 8 * k);
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          dv[d] = T::mma(tr_frag<CH>(sg, 32 * n + 16 * k, 32 * d, lane), pf, dv[d]);
          dk[d] = T::mma(tr_frag<CH>(sq, 32 * n + 16 * k, 32 * d, lane), df, dk[d]);
        }
      }
    }
  }
  if (key >= a.Sk) return;
  // a masked key's column has gathered exp(0 - lse) and the like: it is 0
  if (!ok)
#pragma unroll
    for (int i = 0; i < ND; ++i) dk[i] = dv[i] = floatx16{};
  const float back_k = ldexpf(1.0f, -bits), back_v = ldexpf(1.0f, -kBitsP<T>);
  if (splits > 1) {
    if (t0 >= t1) return;  // the sum reads no empty part
    const int64_t keys = (int64_t)a.B * a.Hkv * a.Sk, at = ((int64_t)b * a.Hkv + g) * a.Sk + key;
    float* p = part + 2 * (sp * keys + at) * DP;
    store_part<DP>(dk, p, h, back_k);
    store_part<DP>(dv, p + DP, h, back_v);
  } else {
    store_cols<T, DP, FAST>(dk, (uint16_t*)a.dk + b * a.dks[0] + (int64_t)key * a.dks[1] + g * a.dks[2],
                            a.scale * back_k, a.D, h);
    store_cols<T, DP, FAST>(dv, (uint16_t*)a.dv + b * a.dvs[0] + (int64_t)key * a.dvs[1] + g * a.dvs[2],
                            back_v, a.D, h);
  }
}

// Adds the parts up in order, 4 elements a thread: dq (KV = false), dk and dv.  Of a
// batch entry's parts the first ones have tiles, the others were not written, and
// nothing was for rows and keys past its lengths.
template <class T, int DP, bool KV, bool VEC>
__global__ __launch_bounds__(256) void k_attn_sum(const AttnArgs a, int splits, const float* part) {
  const int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
  const int len = KV ? a.Sk : a.M;
  const int64_t n = (int64_t)a.B * a.Hkv * len * (KV ? 2 : 1) * DP;
  const int d = (int)(e % DP);
  if (e >= n || d >= a.D) return;
  uint32_t i = (uint32_t)(e / DP);
  const bool val = KV && (i & 1);
  if (KV) i >>= 1;
  const int at = (int)(i % len), bg = (int)(i / len), g = bg % a.Hkv, b = bg / a.Hkv;
  const int nq = clamp_len(a.q_len, b, a.Sq), nk = clamp_len(a.kv_len, b, a.Sk);
  const int tiles = KV ? (nq + dkv_rows(DP, VEC) - 1) / dkv_rows(DP, VEC) * a.G : (nk + kBN - 1) / kBN;
  const int per = (tiles + splits - 1) / splits;
  int parts = tiles ? (tiles + per - 1) / per : 0;
  if (KV ? at >= nk : at / a.G >= nq) parts = 0;
  floatx4 x = {};
#pragma unroll 4
  for (int s = 0; s < parts; ++s) x += *reinterpret_cast<const floatx4*>(part + s * n + e);
  const float f = val ? 1.0f : a.scale;
  uint16_t* out;
  if (!KV)
    out = (uint16_t*)a.dq + b * a.dqs[0] + (int64_t)(at / a.G) * a.dqs[1] + (g * a.G + at % a.G) * a.dqs[2];
  else if (val)
    out = (uint16_t*)a.dv + b * a.dvs[0] + at * a.dvs[1] + g * a.dvs[2];
  else
    out = (uint16_t*)a.dk + b * a.dks[0] + at * a.dks[1] + g * a.dks[2];
  store4<VEC>(out + d, make_uint2(T::pack(x[0] * f, x[1] * f), T::pack(x[2] * f, x[3] * f)), a.D - d);
}

// Parts of the contracted axis, so that the chip is busy also where the other is
// short: of at least 4 tiles each.
int dq_splits(const AttnArgs& a) {
  const int64_t wgs = (((int64_t)a.M + 127) / 128) * a.Hkv * a.B, tiles = (a.Sk + kBN - 1) / kBN;
  return wgs ? (int)std::max<int64_t>(1, std::min(kCUs / wgs, tiles / 4)) : 1;
}
int dkv_splits(const AttnArgs& a) {
  const int64_t wgs = (int64_t)((a.Sk + kKeys - 1) / kKeys) * a.Hkv * a.B;
  const int rows = dkv_rows(padded(a.D), true);
  const int64_t tiles = (int64_t)((a.Sq + rows - 1) / rows) * a.G;
  return wgs ? (int)std::max<int64_t>(1, std::min<int64_t>(2 * kCUs / wgs, tiles / 4)) : 1;
}
// Whether tiles of rows can go to LDS by 16-byte loads with 32-bit offsets, the
// rows past the last beyond the descriptor's bound.
bool fast_rows(const AttnArgs& a) {
  auto fits = [&](int64_t stride) { return stride >= a.D && stride <= kMaxTileStride; };
  return fits(a.qs[1]) && fits(a.dos[1]);
}
int64_t stat_floats(const AttnArgs& a) { return ((int64_t)2 * a.B * a.Hkv * a.M + 3) / 4 * 4; }
int64_t norm_floats(const AttnArgs& a) {
  return a.dtype == kF16 ? ((int64_t)a.B * a.Hkv * ((int64_t)a.M + a.Sk) + 3) / 4 * 4 : 0;
}
int64_t dq_floats(const AttnArgs& a) {
  const int s = dq_splits(a);
  return s > 1 ? (int64_t)s * a.B * a.Hkv * a.M * padded(a.D) : 0;
}
int64_t dkv_floats(const AttnArgs& a) {
  const int s = dkv_splits(a);
  return s > 1 ? (int64_t)s * a.B * a.Hkv * a.Sk * 2 * padded(a.D) : 0;
}

template <class T, int DP, bool FAST>
void launch(const AttnArgs& a, float* part_q, float* part_kv, hipStream_t s) {
  const int64_t rows = (int64_t)a.B * a.Hkv * a.M, keys = (int64_t)a.B * a.Hkv * a.Sk;
  if (rows) {
    const int per = 256 / (DP / 8);
    const int64_t most = kNarrow<T> ? std::max(rows, keys) : rows;
    k_attn_stat<T, DP, FAST><<<dim3((unsigned)((most + per - 1) / per), kNarrow<T> ? 2 : 1), 256, 0, s>>>(a);
    const int ns = dq_splits(a);
    const Order o = order_of(((int64_t)a.M + 127) / 128, a.Hkv);
    const int64_t n = workgroups(o, ns, a);
    if constexpr (FAST) {
      if (two_groups(n, a))
        k_attn_dq<T, DP, true, 2><<<(unsigned)n, 512, 0, s>>>(a, o, ns, part_q);
      else
        k_attn_dq<T, DP, true, 1><<<(unsigned)n, 256, 0, s>>>(a, o, ns, part_q);
    } else {
      k_attn_dq<T, DP, false, 1><<<(unsigned)n, 256, 0, s>>>(a, o, ns, part_q);
    }
    if (ns > 1) k_attn_sum<T, DP, false, FAST><<<(unsigned)((rows * DP / 4 + 255) / 256), 256, 0, s>>>(a, ns, part_q);
  }
  if (keys) {
    const int ns = dkv_splits(a);
    const Order o = order_of(((int64_t)a.Sk + kKeys - 1) / kKeys, a.Hkv);
    const int64_t n = workgroups(o, ns, a);
    k_attn_dkv<T, DP, FAST><<<(unsigned)n, 256, 0, s>>>(a, o, ns, part_kv);
    if (ns > 1)
      k_attn_sum<T, DP, true, FAST><<<(unsigned)((keys * 2 * DP / 4 + 255) / 256), 256, 0, s>>>(a, ns, part_kv);
  }
}

template <class T>
void launch_t(const AttnArgs& a, float* pq, float* pk, hipStream_t s) {
  const bool fast = fast_loads(a) && fast_rows(a);
  if (padded(a.D) == 128)
    fast ? launch<T, 128, true>(a, pq, pk, s) : launch<T, 128, false>(a, pq, pk, s);
  else
    fast ? launch<T, 64, true>(a, pq, pk, s) : launch<T, 64, false>(a, pq, pk, s);
}

}  // namespace

int64_t attn_bwd_bytes(const AttnArgs& a) {
  return 4 * (stat_floats(a) + norm_floats(a) + dq_floats(a) + dkv_floats(a));
}

hipError_t launch_attn_bwd(const AttnArgs& a0, void* ws, hipStream_t s) {
  AttnArgs a = a0;
  a.delta = (float*)ws;
  a.do_norm = a.delta + stat_floats(a);
  a.v_norm = a.do_norm + (int64_t)a.B * a.Hkv * a.M;
  float* pq = a.do_norm + norm_floats(a);
  float* pk = pq + dq_floats(a);
  if (a.B == 0) return hipSuccess;
  a.dtype == kF16 ? launch_t<F16>(a, pq, pk, s) : launch_t<BF16>(a, pq, pk, s);
  return hipGetLastError();
}

}  // namespace pnerf
