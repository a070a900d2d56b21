// What the kernels that walk rows share: 8 elements at a time, sums over a row's lanes.
#pragma once
#include "layers_internal.h"

#if defined(__HIP_DEVICE_COMPILE__) || defined(PNERF_LAYERS_DEVICE)
namespace pnerf {

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

// (The instruction takes a subnormal number for zero.)
__device__ __forceinline__ float inv_rms(float mean, float eps) {
  const float x = mean + eps;
  const bool small = x < 0x1p-126f;
  return __builtin_amdgcn_rsqf(small ? x * 0x1p64f : x) * (small ? 0x1p32f : 1.0f);
}

}  // namespace pnerf
#endif
