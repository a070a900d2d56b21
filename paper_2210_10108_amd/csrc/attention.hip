// Cross attention, forward: o_i = sum_j exp(a_ij - lse_i) v_j over the allowed
// keys j, a_ij = scale q_i . k_j, for queries and keys of different lengths.
//
// The query heads that share a kv head are rows of one product: row r of kv head
// g is query row r / G, head g G + r % G.  A wavefront owns 32 rows, a workgroup
// NW wavefronts' rows and one pass over tiles of 64 keys with the running
// maximum m and sum l of each row's softmax:
//   S^T = K Q^T     (A = keys from LDS, B = the rows' queries, in registers)
//   P = exp2(c S - m), l += sum P
//   O^T += V^T P^T  (A = values by transposed LDS reads, B = P)
// Both products have the row as their column, so that all of a row's scores are
// in two lanes (l and l + 32): the softmax needs one exchange a tile, and P is
// the second product's B operand as it stands -- lane half h holds keys
// 8 i + 4 h + 0..3, an order of the contraction that the value reads follow.
#define PNERF_LAYERS_DEVICE
#include <algorithm>

#include "layers_internal.h"

namespace pnerf {
namespace {

constexpr int kBN = 64;  // keys of a tile

// Position of 16-byte chunk c of row r in a tile row of CH chunks: a rotation
// of the row's low bits is xored in, so that 8 rows at one chunk (the 16-byte
// reads) and 4 rows at two adjacent chunks (the transposed reads) each cover
// all the banks.
template <int CH>
__device__ __forceinline__ int swz(int r, int c) {
  return r * CH + (c ^ (((r & 3) << 1) | ((r >> 2) & 1)));
}

template <class T, int DP, int NW, bool VEC, bool SPLIT>
__global__ __launch_bounds__(NW * 64) void k_attn_fwd(const AttnArgs a) {
  constexpr int CH = DP / 8, NT = NW * 64, NS = DP / 16, ND = DP / 32;
  constexpr int NL = kBN * CH / NT;  // 16-byte chunks per thread of a K or V tile
  __shared__ uint4 sk[kBN * CH], sv[kBN * CH];

  const int tiles_m = (a.M + NW * 32 - 1) / (NW * 32);
  int id = xcd_order(blockIdx.x, gridDim.x);
  const int mt = id % tiles_m;
  id /= tiles_m;
  const int sp = SPLIT ? id % a.splits : 0;
  if (SPLIT) id /= a.splits;
  const int g = id % a.Hkv, b = id / a.Hkv;

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int r = lane & 31, h = lane >> 5;
  const int row = mt * NW * 32 + wave * 32 + r;
  const int qi = row / a.G, head = g * a.G + row % a.G;
  const int nq = a.q_len ? min(max(a.q_len[b], 0), a.Sq) : a.Sq;
  const int nk = a.kv_len ? min(max(a.kv_len[b], 0), a.Sk) : a.Sk;
  const bool ok = row < a.M && qi < nq;

  // this part's tiles
  int t0 = 0, t1 = (nk + kBN - 1) / kBN;
  if (SPLIT) {
    const int per = (t1 + a.splits - 1) / a.splits;
    t0 = min(sp * per, t1);
    t1 = min(t0 + per, t1);
  }
  if ((mt * NW * 32) / a.G >= nq) t1 = t0;  // no row of this workgroup is valid

  const uint16_t* qp = (const uint16_t*)a.q + b * a.qs[0] + (int64_t)qi * a.qs[1] + head * a.qs[2];
  const uint16_t* kp = (const uint16_t*)a.k + b * a.ks[0] + g * a.ks[2];
  const uint16_t* vp = (const uint16_t*)a.v + b * a.vs[0] + g * a.vs[2];
  const uint8_t* mp = a.mask ? a.mask + b * a.mask_stride : nullptr;

  uint4 qf[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const int d = 16 * s + 8 * h;
    qf[s] = load8<VEC>(qp + d, ok ? min(a.D - d, 8) : 0);
  }

  floatx16 o[ND];
#pragma unroll
  for (int i = 0; i < ND; ++i) o[i] = floatx16{};
  float m = -INFINITY, l = 0.0f;

  uint4 rk[NL], rv[NL];
  bool allowed = false;  // key `lane` of the staged tile
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
      const int e = tid + n * NT, kr = e / CH, at = swz<CH>(kr, e % CH);
      const bool on = (vm >> kr) & 1;  // what a masked key or value holds never enters a product
      sk[at] = on ? rk[n] : make_uint4(0, 0, 0, 0);
      sv[at] = on ? rv[n] : make_uint4(0, 0, 0, 0);
    }
    __syncthreads();
    if (t + 1 < t1) fetch(t + 1);

    floatx16 s[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      s[n] = floatx16{};
#pragma unroll
      for (int i = 0; i < NS; ++i) s[n] = T::mma(sk[swz<CH>(32 * n + r, 2 * i + h)], qf[i], s[n]);
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
    const float mn = fmaxf(m, a.c * fmaxf(m0, m1));
    const float base = mn == -INFINITY ? 0.0f : mn;  // no allowed key yet
    const float alpha = __builtin_amdgcn_exp2f(m - base);
    m = mn;
    l *= alpha;
#pragma unroll
    for (int i = 0; i < ND; ++i) o[i] *= alpha;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[n][i] = __builtin_amdgcn_exp2f(fmaf(s[n][i], a.c, -base));
        l += s[n][i];
      }
#pragma unroll
    for (int n = 0; n < 4; ++n) {  // 16 keys each
      const floatx16& p = s[n / 2];
      const int i0 = 8 * (n % 2);
      const uint4 pf = make_uint4(T::pack(p[i0], p[i0 + 1]), T::pack(p[i0 + 2], p[i0 + 3]),
                                  T::pack(p[i0 + 4], p[i0 + 5]), T::pack(p[i0 + 6], p[i0 + 7]));
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        const int l16 = lane & 15, kr = 16 * n + 4 * h + l16 / 4;
        const int col = 32 * d + 16 * ((lane >> 4) & 1) + 4 * (l16 % 4);
        const char* lo = (const char*)(sv + swz<CH>(kr, col / 8)) + 2 * (col % 8);
        const char* hi = (const char*)(sv + swz<CH>(kr + 8, col / 8)) + 2 * (col % 8);
        const uint2 v0 = read_tr(lo), v1 = read_tr(hi);
        o[d] = T::mma(make_uint4(v0.x, v0.y, v1.x, v1.y), pf, o[d]);
      }
    }
  }

  float l0, l1;
  halves(l, l0, l1);
  l = l0 + l1;
  if (!ok) {  // past q_len, beside rows that are not
    m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int i = 0; i < ND; ++i) o[i] = floatx16{};
  }
  if (SPLIT) {
    if (row >= a.M) return;
    const int64_t rows = (int64_t)a.B * a.Hkv * a.M;
    const int64_t at = ((int64_t)b * a.Hkv + g) * a.M + row;
    if (h == 0) {
      floatx2* ml = reinterpret_cast<floatx2*>(a.part + (int64_t)a.splits * rows * DP);
      ml[sp * rows + at] = floatx2{m, l};
    }
    if (t0 == t1) return;  // the join does not read an empty part's sums
    float* po = a.part + (sp * rows + at) * DP;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<floatx4*>(po + 32 * d + 8 * i + 4 * h) =
            floatx4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
    return;
  }
  if (row >= a.M) return;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  uint16_t* op = (uint16_t*)a.o + b * a.os[0] + (int64_t)qi * a.os[1] + head * a.os[2];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int col = 32 * d + 8 * i + 4 * h;
      const floatx16& x = o[d];
      store4<VEC>(op + col, make_uint2(T::pack(x[4 * i] * inv, x[4 * i + 1] * inv),
                                       T::pack(x[4 * i + 2] * inv, x[4 * i + 3] * inv)),
                  min(a.D - col, 4));
    }
  if (a.lse && h == 0)
    a.lse[((int64_t)b * a.Hq + head) * a.Sq + qi] =
        l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

// Joins the parts of the key axis, a workgroup per row: the parts' sums meet at
// the largest of their maxima, in a fixed order.
template <class T, int DP>
__global__ __launch_bounds__(256) void k_attn_join(const AttnArgs a) {
  constexpr int NG = 256 / (DP / 4);  // groups of lanes, each with every NG-th part
  __shared__ float red[NG][DP];
  __shared__ float red_l[NG];
  const int row = blockIdx.x % a.M;
  const int bg = blockIdx.x / a.M, g = bg % a.Hkv, b = bg / a.Hkv;
  const int qi = row / a.G, head = g * a.G + row % a.G;
  const int64_t rows = (int64_t)a.B * a.Hkv * a.M, at = blockIdx.x;
  const floatx2* ml = reinterpret_cast<const floatx2*>(a.part + (int64_t)a.splits * rows * DP);
  float m = -INFINITY;
  for (int s = threadIdx.x & 63; s < a.splits; s += 64) m = fmaxf(m, ml[s * rows + at][0]);
  for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));

  const int grp = threadIdx.x / (DP / 4), d4 = 4 * (threadIdx.x % (DP / 4));
  floatx4 acc = {};
  float l = 0.0f;
  for (int s = grp; s < a.splits; s += NG) {
    const floatx2 v = ml[s * rows + at];
    // a part without an allowed key has no sums (NaN scores: the sum is NaN)
    if (v[0] == -INFINITY && v[1] == 0.0f) continue;
    const float w = __builtin_amdgcn_exp2f(v[0] - (m == -INFINITY ? 0.0f : m));
    l += w * v[1];
    acc += w * *reinterpret_cast<const floatx4*>(a.part + (s * rows + at) * DP + d4);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) red[grp][d4 + i] = acc[i];
  if (d4 == 0) red_l[grp] = l;
  __syncthreads();
  l = 0.0f;
  for (int i = 0; i < NG; ++i) l += red_l[i];
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  typename T::E* op = (typename T::E*)a.o + b * a.os[0] + (int64_t)qi * a.os[1] + head * a.os[2];
  for (int d = threadIdx.x; d < a.D; d += 256) {
    float x = 0.0f;
    for (int i = 0; i < NG; ++i) x += red[i][d];
    op[d] = (typename T::E)(x * inv);
  }
  if (a.lse && threadIdx.x == 0)
    a.lse[((int64_t)b * a.Hq + head) * a.Sq + qi] =
        l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

int padded(int D) { return D <= 64 ? 64 : 128; }
int waves(const AttnArgs& a) { return a.M <= 32 ? 1 : 4; }

template <class T, int DP, int NW, bool VEC>
void launch(const AttnArgs& a, hipStream_t s) {
  const int tiles = (a.M + NW * 32 - 1) / (NW * 32);
  const int64_t n = (int64_t)tiles * a.splits * a.Hkv * a.B;
  if (a.splits > 1)
    k_attn_fwd<T, DP, NW, VEC, true><<<(unsigned)n, NW * 64, 0, s>>>(a);
  else
    k_attn_fwd<T, DP, NW, VEC, false><<<(unsigned)n, NW * 64, 0, s>>>(a);
  if (a.splits > 1) k_attn_join<T, DP><<<(unsigned)(a.B * a.Hkv * a.M), 256, 0, s>>>(a);
}

template <class T>
void launch_t(const AttnArgs& a, hipStream_t s) {
  const bool wide = padded(a.D) == 128, many = waves(a) > 1;
  if (wide && many) a.vec ? launch<T, 128, 4, true>(a, s) : launch<T, 128, 4, false>(a, s);
  if (wide && !many) a.vec ? launch<T, 128, 1, true>(a, s) : launch<T, 128, 1, false>(a, s);
  if (!wide && many) a.vec ? launch<T, 64, 4, true>(a, s) : launch<T, 64, 4, false>(a, s);
  if (!wide && !many) a.vec ? launch<T, 64, 1, true>(a, s) : launch<T, 64, 1, false>(a, s);
}

}  // namespace

// Few rows leave compute units idle: the keys are then cut into parts, so that
// the chip's resident workgroups are all busy, of at least 4 tiles each.
int attn_fwd_splits(const AttnArgs& a) {
  const int nw = waves(a);
  const int64_t wgs = (int64_t)((a.M + nw * 32 - 1) / (nw * 32)) * a.Hkv * a.B;
  const int64_t target = nw == 1 ? 4 * kCUs : 2 * kCUs;
  const int64_t tiles = (a.Sk + kBN - 1) / kBN;
  if (wgs == 0) return 1;
  return (int)std::max<int64_t>(1, std::min(target / wgs, tiles / 4));
}

int64_t attn_fwd_bytes(const AttnArgs& a) {
  if (a.splits <= 1) return 0;
  return (int64_t)a.splits * a.B * a.Hkv * a.M * (padded(a.D) + 2) * 4;
}

hipError_t launch_attn_fwd(const AttnArgs& a0, void* ws, hipStream_t s) {
  AttnArgs a = a0;
  a.part = (float*)ws;
  if (a.B == 0 || a.M == 0) return hipSuccess;
  a.dtype == kF16 ? launch_t<F16>(a, s) : launch_t<BF16>(a, s);
  return hipGetLastError();
}

}  // namespace pnerf
