// Keys and values in 8 bits: for each block of 64 rows of a head, scale = the least
// power of two, at least 2^-126, with which the block's largest value is at most 448,
// and x8 = x / scale to the nearest e4m3 number.  e4m3 is a floating type: a power of
// two costs none of its relative precision, makes the division exact, and leaves
// neighbouring blocks mostly with one scale, which the attention that reads them need
// not change then.
//
// A stream, bound by memory: a workgroup takes a block of a head, keeps it in registers
// while its largest value is found, and writes half of what it read.  Neighbouring
// workgroups, on different XCDs, take the keys and values of neighbouring heads, which
// lie side by side (64 x 2500 ragged rows, 8 heads of 128, f16: 166 us or 4.4 TB/s; 182 with
// neighbours on one XCD).
#define PNERF_LAYERS_DEVICE
#include "rows_common.h"

namespace pnerf {
namespace {

constexpr int kRows = 64;

// Two numbers of magnitude at most 448 to e4m3, to the nearest, in the low or high half of w.
template <bool HIGH>
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, uint32_t w) {
  return __builtin_amdgcn_cvt_pk_fp8_f32(a, b, w, HIGH);
}

// The largest finite magnitude; 0 for NaN and infinities, which become NaN.
__device__ __forceinline__ float finite_abs(float x) { return fabsf(x) < INFINITY ? fabsf(x) : 0.0f; }

// Exponent of the scale: 448 is 1.75 2^8, most = f 2^k.
__device__ __forceinline__ int scale_exponent(float most) {
  const uint32_t bits = __float_as_uint(most);
  if (bits == 0) return 0;
  const int k = (int)(bits >> 23) - 127;  // (a subnormal number's is below every bound)
  return max(k - 8 + ((bits & 0x7FFFFF) > 0x600000 ? 1 : 0), -126);
}

template <class E, bool VEC>
__global__ __launch_bounds__(256) void k_quantize(const QuantArgs a, int blocks) {
  __shared__ float red[4];
  int id = blockIdx.x;
  const QuantSide& x = a.side[id & 1];
  id >>= 1;
  const int h = id % a.H, t = id / a.H % blocks, b = id / a.H / blocks;
  const int len = a.len ? min(max(a.len[b], 0), a.S) : a.S;
  const E* in = (const E*)x.x + b * x.xs[0] + h * x.xs[2];
  uint8_t* out = x.y + b * x.ys[0] + h * x.ys[2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int chunks = (a.D + 7) / 8;  // of a row
  float v[4][8], most = 0.0f;
  int on[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {  // at most 16 chunks a row: 4 a thread
    const int e = threadIdx.x + 256 * i, r = e / chunks, d = 8 * (e % chunks), row = t * kRows + r;
    on[i] = r < kRows && row < len && (!a.mask || a.mask[b * a.mask_stride + row]);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
    if (on[i]) {
      const E* p = in + (int64_t)row * x.xs[1] + d;
      if (VEC) {
        load<E>(p, v[i]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (d + j < a.D) v[i][j] = (float)p[j];
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) most = fmaxf(most, finite_abs(v[i][j]));
  }
  for (int d = 32; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
  if (lane == 0) red[wave] = most;
  __syncthreads();
  most = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const int k = scale_exponent(most);
  if (threadIdx.x == 0) x.scale[b * x.ss[0] + t * x.ss[1] + h] = __uint_as_float((uint32_t)(k + 127) << 23);
  const float inv = __uint_as_float((uint32_t)(127 - k) << 23);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int e = threadIdx.x + 256 * i, r = e / chunks, d = 8 * (e % chunks), row = t * kRows + r;
    if (r >= kRows || row >= a.S) continue;
#pragma unroll
    for (int j = 0; j < 8; ++j) v[i][j] = fabsf(v[i][j]) < INFINITY ? v[i][j] * inv : __builtin_nanf("");
    uint2 w;
    w.x = to_e4m3<true>(v[i][2], v[i][3], to_e4m3<false>(v[i][0], v[i][1], 0));
    w.y = to_e4m3<true>(v[i][6], v[i][7], to_e4m3<false>(v[i][4], v[i][5], 0));
    uint8_t* p = out + (int64_t)row * x.ys[1] + d;
    if (VEC) {
      *reinterpret_cast<uint2*>(p) = w;
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (d + j < a.D) p[j] = (uint8_t)((j < 4 ? w.x : w.y) >> (8 * (j & 3)));
    }
  }
}

template <class E>
void launch(const QuantArgs& a, hipStream_t s) {
  const int blocks = (a.S + kRows - 1) / kRows;
  const unsigned n = 2u * a.B * blocks * a.H;
  if (a.vec)
    k_quantize<E, true><<<n, 256, 0, s>>>(a, blocks);
  else
    k_quantize<E, false><<<n, 256, 0, s>>>(a, blocks);
}

}  // namespace

hipError_t launch_quantize(const QuantArgs& a, hipStream_t s) {
  if (a.B == 0 || a.S == 0) return hipSuccess;
  if (a.dtype == kF16) launch<_Float16>(a, s);
  if (a.dtype == kBF16) launch<__bf16>(a, s);
  return hipGetLastError();
}

}  // namespace pnerf
