// Cross attention over states held in 8 bits, forward (what attention.hip does, its
// softmax and its products): over the allowed keys j
//   a_ij = scale ks[j / 64] q_i . k8_j,  o_i = sum_j exp(a_ij - lse_i) vs[j / 64] v8_j
// with k8, v8 of e4m3 and one scale for each block of 64 rows of a head, which is a
// tile here.  Every e4m3 number is a float16 and a bfloat16 number: tiles are widened
// on their way to LDS and the products are those of 16 bits, exact in what they
// multiply.  A tile's key scale is a factor of its scores.  Its value scale would be
// one of p, whose 16 bits might not hold it; instead the sums are kept in units of the
// current scale and rescaled, where the maximum's rescaling stands, when a tile has
// another one.
#define PNERF_LAYERS_DEVICE
#include <algorithm>

#include "attention_rows.h"

namespace pnerf {
namespace {

// 4 e4m3 numbers as two pairs of 16-bit ones.
template <class T>
__device__ __forceinline__ uint2 widen4(uint32_t w);
template <>
__device__ __forceinline__ uint2 widen4<F16>(uint32_t w) {
  return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true)));
}
template <>
__device__ __forceinline__ uint2 widen4<BF16>(uint32_t w) {
  return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true)));
}
template <class T>
__device__ __forceinline__ uint4 widen8(uint32_t lo, uint32_t hi) {
  const uint2 a = widen4<T>(lo), b = widen4<T>(hi);
  return make_uint4(a.x, a.y, b.x, b.y);
}

// Rows whose tiles have scales.  `factor` of the scores' unit, `unit` of the sums.
template <class T, int DP>
struct ScaledRows : Rows<T, DP> {
  float c, unit, unit_next;

  __device__ __forceinline__ void begin(const AttnArgs& a) { c = a.c, unit = unit_next = 1.0f; }
  // The scales of the next tile; one without an allowed key has none that count.
  __device__ __forceinline__ void scales(const AttnArgs& a, float ks, float vs, uint64_t vm) {
    if (vm) c = fmaxf(a.c * ks, 0x1p-126f), unit_next = vs;  // (0 times a masked key's -inf would be NaN)
  }
  template <class N, class V>
  __device__ __forceinline__ void run(int lane, N next, V values) {
    bool more = next();
    while (more) {
      this->rescale();
      if (unit_next != unit) {
        const float f = unit / unit_next;
        unit = unit_next;
#pragma unroll
        for (int i = 0; i < DP / 32; ++i) this->o[i] *= f;
      }
      do {
        this->add(values(), c, lane);
        more = next();
      } while (more && !this->grown() && unit_next == unit);
    }
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) this->o[i] *= unit;
  }
};

// A tile's scales (index of the tile below the number of blocks).
struct Scales {
  const float *k, *v;
  int64_t k_step, v_step;
  __device__ __forceinline__ Scales(const AttnArgs& a, int b, int g)
      : k(a.k_scale + b * a.kss[0] + g), v(a.v_scale + b * a.vss[0] + g), k_step(a.kss[1]), v_step(a.vss[1]) {}
};

// A tile by way of registers, element by element, 256 threads.
template <class T, int DP>
__device__ __forceinline__ void copy_tile8(uint4* lds, const void* p, const int64_t s[3], int b, int g, int D,
                                           int t, uint64_t vm) {
  constexpr int CH = DP / 8;
  const uint8_t* base = (const uint8_t*)p + b * s[0] + g * s[2];
  for (int e = threadIdx.x; e < kBN * CH; e += 256) {
    const int r = e / CH, d = 8 * (e % CH);
    uint32_t w[2] = {0, 0};
    if ((vm >> r) & 1) {
      const uint8_t* x = base + (int64_t)(t * kBN + r) * s[1] + d;
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (d + j < D) w[j / 4] |= (uint32_t)x[j] << (8 * (j & 3));
    }
    lds[swz<CH>(r, e % CH)] = widen8<T>(w[0], w[1]);
  }
}

// Any strides, alignment and head width.
template <class T, int DP>
__global__ __launch_bounds__(256) void k_attn_q8_any(const AttnArgs a, const Order order) {
  __shared__ uint4 sk[kBN * DP / 8], sv[kBN * DP / 8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
  const Place at(a, order, 128, wave * 32 + (lane & 31));
  const Scales sc(a, at.b, at.g);
  ScaledRows<T, DP> x;
  x.template init<false>(at.q, at.ok, a.D, h);
  x.begin(a);
  int t = at.t0;
  x.run(
      lane,
      [&] {
        if (t >= at.t1) return false;
        const uint64_t vm = __ballot(at.allowed(t * kBN + lane));
        __syncthreads();
        copy_tile8<T, DP>(sk, a.k, a.ks, at.b, at.g, a.D, t, vm);
        copy_tile8<T, DP>(sv, a.v, a.vs, at.b, at.g, a.D, t, vm);
        x.scales(a, sc.k[t * sc.k_step], sc.v[t * sc.v_step], vm);
        __syncthreads();
        x.scores(sk, vm, x.c, lane);
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

template <class T, int DP>
void launch(const AttnArgs& a, hipStream_t s) {
  const bool few = a.M <= 32;
  const int rows = few ? 32 : 128;
  const Order o = order_of(((int64_t)a.M + rows - 1) / rows, a.Hkv);
  const unsigned n = (unsigned)workgroups(o, a.splits, a);
  k_attn_q8_any<T, DP><<<n, 256, 0, s>>>(a, o);
  join<T, DP>(a, s);
}

}  // namespace

hipError_t launch_attn_q8(const AttnArgs& a0, void* ws, hipStream_t s) {
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
