// Cross attention, backward.  With p_ij = exp(a_ij - lse_i) recomputed from the
// row's log-sum, delta_i = do_i . o_i and ds_ij = p_ij (do_i . v_j - delta_i):
//   dv_j = sum_i p_ij do_i,  dk_j = scale sum_i ds_ij q_i,  dq_i = scale sum_j ds_ij k_j
// Three kernels, no atomics: the rows' (lse, delta); dq by workgroups that own
// rows and pass over the keys; dk and dv by workgroups that own keys and pass
// over the rows of all the query heads that share their kv head, so that the
// sum over those heads never leaves the registers.  s and dp are computed twice
// (7 products where 5 would do), which costs less than adding dq up in memory.
//
// Fragments as in the forward kernel: what the second products contract over is
// in the registers of the first ones' results, as their B operand.
#define PNERF_LAYERS_DEVICE
#include <algorithm>

#include "attention_common.h"

namespace pnerf {
namespace {

constexpr int kKeys = 128;   // keys of a workgroup of the dk, dv pass: 32 a wavefront

// (lse / ln 2 - shift, delta) of every row; (+inf, 0) where the row has no
// allowed key or is past q_len, which makes all of its p zero.
template <class T, int DP, bool VEC>
__global__ __launch_bounds__(256) void k_attn_stat(const AttnArgs a) {
  constexpr int LR = DP / 8;  // lanes of a row
  const int64_t rows = (int64_t)a.B * a.Hkv * a.M;
  const int64_t at = (int64_t)blockIdx.x * (256 / LR) + threadIdx.x / LR;
  const int d = 8 * (threadIdx.x % LR);
  float sum = 0.0f;
  if (at < rows) {
    const int row = (int)(at % a.M), bg = (int)(at / a.M), g = bg % a.Hkv, b = bg / a.Hkv;
    const int qi = row / a.G, head = g * a.G + row % a.G;
    const float lse = a.lse[((int64_t)b * a.Hq + head) * a.Sq + qi];
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
      reinterpret_cast<floatx2*>(a.delta)[at] =
          ok ? floatx2{lse * 1.4426950408889634f - (float)a.shift, sum} : floatx2{INFINITY, 0.0f};
  }
}

template <class T, int DP, int NW, bool VEC>
__global__ __launch_bounds__(NW * 64) void k_attn_dq(const AttnArgs a, int splits, float* part) {
  constexpr int CH = DP / 8, NT = NW * 64, NS = DP / 16, ND = DP / 32;
  constexpr int NL = kBN * CH / NT;
  __shared__ uint4 sk[kBN * CH], sv[kBN * CH];

  const int tiles_m = (a.M + NW * 32 - 1) / (NW * 32);
  int id = xcd_order(blockIdx.x, gridDim.x);
  const int mt = id % tiles_m;
  id /= tiles_m;
  const int sp = id % splits;
  id /= splits;
  const int g = id % a.Hkv, b = id / a.Hkv;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r = lane & 31, h = lane >> 5;
  const int row = mt * NW * 32 + wave * 32 + r;
  const int qi = row / a.G, head = g * a.G + row % a.G;
  const int nq = clamp_len(a.q_len, b, a.Sq), nk = clamp_len(a.kv_len, b, a.Sk);
  int t1 = (nk + kBN - 1) / kBN;
  const int per = (t1 + splits - 1) / splits, t0 = min(sp * per, t1);
  t1 = min(t0 + per, t1);
  if ((mt * NW * 32) / a.G >= nq) t1 = t0;

  const int64_t rows = (int64_t)a.B * a.Hkv * a.M;
  const int64_t at = ((int64_t)b * a.Hkv + g) * a.M + row;
  floatx2 st = floatx2{INFINITY, 0.0f};
  if (row < a.M) st = reinterpret_cast<const floatx2*>(a.delta)[at];
  const bool ok = st[0] != INFINITY;

  const uint16_t* qp = (const uint16_t*)a.q + b * a.qs[0] + (int64_t)qi * a.qs[1] + head * a.qs[2];
  const uint16_t* gp = (const uint16_t*)a.dout + b * a.dos[0] + (int64_t)qi * a.dos[1] + head * a.dos[2];
  const uint16_t* kp = (const uint16_t*)a.k + b * a.ks[0] + g * a.ks[2];
  const uint16_t* vp = (const uint16_t*)a.v + b * a.vs[0] + g * a.vs[2];
  const uint8_t* mp = a.mask ? a.mask + b * a.mask_stride : nullptr;

  uint4 qf[NS], gf[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const int d = 16 * s + 8 * h, n = ok ? min(a.D - d, 8) : 0;
    qf[s] = load8<VEC>(qp + d, n);
    gf[s] = load8<VEC>(gp + d, n);
  }
  floatx16 acc[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i) acc[i] = floatx16{};

  uint4 rk[NL], rv[NL];
  bool allowed = false;
  auto fetch = [&](int t) {
    const int j = t * kBN + lane;
    allowed = j < nk && (!mp || mp[j]);
#pragma unroll
    for (int n = 0; n < NL; ++n) {
      const int e = tid + n * NT, jr = t * kBN + e / CH, d = 8 * (e % CH);
      const int cnt = jr < nk ? min(a.D - d, 8) : 0;
      rk[n] = load8<VEC>(kp + (int64_t)jr * a.ks[1] + d, cnt);
      rv[n] = load8<VEC>(vp + (int64_t)jr * a.vs[1] + d, cnt);
    }
  };
  if (t0 < t1) fetch(t0);
  for (int t = t0; t < t1; ++t) {
    const uint64_t vm = __ballot(allowed);
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NL; ++n) {
      const int e = tid + n * NT, kr = e / CH, p = swz<CH>(kr, e % CH);
      const bool on = (vm >> kr) & 1;
      sk[p] = on ? rk[n] : make_uint4(0, 0, 0, 0);
      sv[p] = on ? rv[n] : make_uint4(0, 0, 0, 0);
    }
    __syncthreads();
    if (t + 1 < t1) fetch(t + 1);
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
      st[1] = ldexpf(s0 + s1, -a.shift);
      if (h == 0 && ok) reinterpret_cast<floatx2*>(a.delta)[at] = st;
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      floatx16 s, dp;
      first(n, s, dp);
      const uint32_t w = (uint32_t)(vm >> (32 * n)) >> (4 * h);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[i] = (w >> (8 * (i / 4) + i % 4)) & 1 ? s[i] * (dp[i] - st[1]) : 0.0f;
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
  if (row >= a.M) return;
  if (splits > 1) {
    store_part<DP>(acc, part + (sp * rows + at) * DP, h);
  } else {
    uint16_t* out = (uint16_t*)a.dq + b * a.dqs[0] + (int64_t)qi * a.dqs[1] + head * a.dqs[2];
    store_cols<T, DP, VEC>(acc, out, ldexpf(a.scale, -a.shift), a.D, h);
  }
}

template <class T, int DP, bool VEC>
__global__ __launch_bounds__(256) void k_attn_dkv(const AttnArgs a, int splits, float* part) {
  constexpr int CH = DP / 8, NT = 256, NS = DP / 16, ND = DP / 32;
  constexpr int NL = kBN * CH / NT;
  __shared__ uint4 sq[kBN * CH], sg[kBN * CH];
  __shared__ floatx2 sst[kBN];

  const int tiles_k = (a.Sk + kKeys - 1) / kKeys;
  int id = xcd_order(blockIdx.x, gridDim.x);
  const int kt = id % tiles_k;
  id /= tiles_k;
  const int sp = id % splits;
  id /= splits;
  const int g = id % a.Hkv, b = id / a.Hkv;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r = lane & 31, h = lane >> 5;
  const int key = kt * kKeys + wave * 32 + r;
  const int nq = clamp_len(a.q_len, b, a.Sq), nk = clamp_len(a.kv_len, b, a.Sk);
  const bool ok = key < nk && (!a.mask || a.mask[b * a.mask_stride + key]);
  const int mrows = nq * a.G;
  int t1 = (mrows + kBN - 1) / kBN;
  const int per = (t1 + splits - 1) / splits, t0 = min(sp * per, t1);
  t1 = min(t0 + per, t1);
  if (kt * kKeys >= nk) t1 = t0;

  const uint16_t* kp = (const uint16_t*)a.k + b * a.ks[0] + (int64_t)key * a.ks[1] + g * a.ks[2];
  const uint16_t* vp = (const uint16_t*)a.v + b * a.vs[0] + (int64_t)key * a.vs[1] + g * a.vs[2];
  uint4 kf[NS], vf[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const int d = 16 * s + 8 * h, n = ok ? min(a.D - d, 8) : 0;
    kf[s] = load8<VEC>(kp + d, n);
    vf[s] = load8<VEC>(vp + d, n);
  }
  floatx16 dk[ND], dv[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i) dk[i] = dv[i] = floatx16{};

  const uint16_t* qp = (const uint16_t*)a.q + b * a.qs[0] + (int64_t)g * a.G * a.qs[2];
  const uint16_t* gp = (const uint16_t*)a.dout + b * a.dos[0] + (int64_t)g * a.G * a.dos[2];
  const floatx2* stat = reinterpret_cast<const floatx2*>(a.delta) + ((int64_t)b * a.Hkv + g) * a.M;

  uint4 rq[NL], rg[NL];
  floatx2 rs[NL];  // the row's (lse, delta), beside each of its chunks
  auto fetch = [&](int t) {
#pragma unroll
    for (int n = 0; n < NL; ++n) {
      const int e = tid + n * NT, row = t * kBN + e / CH, d = 8 * (e % CH);
      const int qi = row / a.G, hd = row % a.G;
      const int cnt = row < mrows ? min(a.D - d, 8) : 0;
      rs[n] = row < mrows ? stat[row] : floatx2{INFINITY, 0.0f};
      rq[n] = load8<VEC>(qp + (int64_t)qi * a.qs[1] + hd * a.qs[2] + d, cnt);
      rg[n] = load8<VEC>(gp + (int64_t)qi * a.dos[1] + hd * a.dos[2] + d, cnt);
    }
  };
  if (t0 < t1) fetch(t0);
  for (int t = t0; t < t1; ++t) {
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NL; ++n) {
      const int e = tid + n * NT, row = e / CH, p = swz<CH>(row, e % CH);
      const bool on = rs[n][0] != INFINITY;  // what a row without a key holds never enters a product
      sq[p] = on ? rq[n] : make_uint4(0, 0, 0, 0);
      sg[p] = on ? rg[n] : make_uint4(0, 0, 0, 0);
      if (e % CH == 0) sst[row] = rs[n];
    }
    __syncthreads();
    if (t + 1 < t1) fetch(t + 1);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      floatx16 s = {}, dp = {};
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        const int p = swz<CH>(32 * n + r, 2 * i + h);
        s = T::mma(sq[p], kf[i], s);
        dp = T::mma(sg[p], vf[i], dp);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const floatx2 st = sst[32 * n + 8 * (i / 4) + 4 * h + i % 4];
        s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], a.c, -st[0]));
        dp[i] = s[i] * (dp[i] - st[1]);
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
  if (splits > 1) {
    const int64_t keys = (int64_t)a.B * a.Hkv * a.Sk, at = ((int64_t)b * a.Hkv + g) * a.Sk + key;
    float* p = part + 2 * (sp * keys + at) * DP;
    store_part<DP>(dk, p, h);
    store_part<DP>(dv, p + DP, h);
  } else {
    const float back = ldexpf(1.0f, -a.shift);
    store_cols<T, DP, VEC>(dk, (uint16_t*)a.dk + b * a.dks[0] + (int64_t)key * a.dks[1] + g * a.dks[2],
                           a.scale * back, a.D, h);
    store_cols<T, DP, VEC>(dv, (uint16_t*)a.dv + b * a.dvs[0] + (int64_t)key * a.dvs[1] + g * a.dvs[2],
                           back, a.D, h);
  }
}

// Adds the parts up in order, one element a thread: dq (KV = false), dk and dv.
template <class T, int DP, bool KV>
__global__ __launch_bounds__(256) void k_attn_sum(const AttnArgs a, int splits, const float* part) {
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int len = KV ? a.Sk : a.M;
  const int64_t n = (int64_t)a.B * a.Hkv * len * (KV ? 2 : 1) * DP;
  const int d = (int)(e % DP);
  if (e >= n || d >= a.D) return;
  float x = 0.0f;
  for (int s = 0; s < splits; ++s) x += part[s * n + e];
  int64_t i = e / DP;
  const bool val = KV && (i & 1);
  if (KV) i >>= 1;
  const int at = (int)(i % len), bg = (int)(i / len), g = bg % a.Hkv, b = bg / a.Hkv;
  const float f = ldexpf(val ? 1.0f : a.scale, -a.shift);
  typename T::E* out;
  if (!KV)
    out = (typename T::E*)a.dq + b * a.dqs[0] + (int64_t)(at / a.G) * a.dqs[1] +
          (g * a.G + at % a.G) * a.dqs[2];
  else if (val)
    out = (typename T::E*)a.dv + b * a.dvs[0] + at * a.dvs[1] + g * a.dvs[2];
  else
    out = (typename T::E*)a.dk + b * a.dks[0] + at * a.dks[1] + g * a.dks[2];
  out[d] = (typename T::E)(x * f);
}

// Parts of the contracted axis, so that the chip is busy also where one axis is
// short: of at least 4 tiles each.
int dq_splits(const AttnArgs& a) {
  const int nw = a.M <= 32 ? 1 : 4;
  const int64_t wgs = (int64_t)((a.M + nw * 32 - 1) / (nw * 32)) * a.Hkv * a.B;
  const int64_t target = nw == 1 ? 4 * kCUs : 2 * kCUs, tiles = (a.Sk + kBN - 1) / kBN;
  return wgs ? (int)std::max<int64_t>(1, std::min(target / wgs, tiles / 4)) : 1;
}
int dkv_splits(const AttnArgs& a) {
  const int64_t wgs = (int64_t)((a.Sk + kKeys - 1) / kKeys) * a.Hkv * a.B;
  const int64_t tiles = ((int64_t)a.M + kBN - 1) / kBN;
  return wgs ? (int)std::max<int64_t>(1, std::min<int64_t>(kCUs / wgs, tiles / 4)) : 1;
}
int64_t stat_floats(const AttnArgs& a) { return ((int64_t)2 * a.B * a.Hkv * a.M + 3) / 4 * 4; }
int64_t dq_floats(const AttnArgs& a) {
  const int s = dq_splits(a);
  return s > 1 ? (int64_t)s * a.B * a.Hkv * a.M * padded(a.D) : 0;
}
int64_t dkv_floats(const AttnArgs& a) {
  const int s = dkv_splits(a);
  return s > 1 ? (int64_t)s * a.B * a.Hkv * a.Sk * 2 * padded(a.D) : 0;
}

template <class T, int DP, bool VEC>
void launch(const AttnArgs& a, float* part_q, float* part_kv, hipStream_t s) {
  const int64_t rows = (int64_t)a.B * a.Hkv * a.M, keys = (int64_t)a.B * a.Hkv * a.Sk;
  if (rows) {
    const int per = 256 / (DP / 8);
    k_attn_stat<T, DP, VEC><<<(unsigned)((rows + per - 1) / per), 256, 0, s>>>(a);
    const int ns = dq_splits(a), nw = a.M <= 32 ? 1 : 4;
    const int64_t n = (int64_t)((a.M + nw * 32 - 1) / (nw * 32)) * ns * a.Hkv * a.B;
    if (nw == 1)
      k_attn_dq<T, DP, 1, VEC><<<(unsigned)n, 64, 0, s>>>(a, ns, part_q);
    else
      k_attn_dq<T, DP, 4, VEC><<<(unsigned)n, 256, 0, s>>>(a, ns, part_q);
    if (ns > 1) k_attn_sum<T, DP, false><<<(unsigned)((rows * DP + 255) / 256), 256, 0, s>>>(a, ns, part_q);
  }
  if (keys) {
    const int ns = dkv_splits(a);
    const int64_t n = (int64_t)((a.Sk + kKeys - 1) / kKeys) * ns * a.Hkv * a.B;
    k_attn_dkv<T, DP, VEC><<<(unsigned)n, 256, 0, s>>>(a, ns, part_kv);
    if (ns > 1)
      k_attn_sum<T, DP, true><<<(unsigned)((keys * 2 * DP + 255) / 256), 256, 0, s>>>(a, ns, part_kv);
  }
}

template <class T>
void launch_t(const AttnArgs& a, float* pq, float* pk, hipStream_t s) {
  if (padded(a.D) == 128)
    a.vec ? launch<T, 128, true>(a, pq, pk, s) : launch<T, 128, false>(a, pq, pk, s);
  else
    a.vec ? launch<T, 64, true>(a, pq, pk, s) : launch<T, 64, false>(a, pq, pk, s);
}

}  // namespace

int64_t attn_bwd_bytes(const AttnArgs& a) {
  return 4 * (stat_floats(a) + dq_floats(a) + dkv_floats(a));
}

hipError_t launch_attn_bwd(const AttnArgs& a0, void* ws, hipStream_t s) {
  AttnArgs a = a0;
  a.delta = (float*)ws;
  float* pq = a.delta + stat_floats(a);
  float* pk = pq + dq_floats(a);
  if (a.B == 0) return hipSuccess;
  a.dtype == kF16 ? launch_t<F16>(a, pq, pk, s) : launch_t<BF16>(a, pq, pk, s);
  return hipGetLastError();
}

}  // namespace pnerf
