// Linear layer: y = act(x W + bias) + residual, and its gradient
//   dz = dy act'(z),  dx = dz W^T,  dW = x^T dz,  db = sum_m dz.
// Three matrix products of one kind, C[m][n] = sum_k A[m][k] B[k][n], which
// differ in which axis of each operand is contiguous in memory.
#define PNERF_LAYERS_DEVICE
#include <algorithm>

#include "layers_internal.h"

namespace pnerf {
namespace {

enum Act : int { kNone = 0, kRelu = 1, kGelu = 2, kSilu = 3 };

__device__ __forceinline__ float phi(float z) { return 0.5f * (1.0f + erff(z * 0.70710678118654752f)); }
__device__ __forceinline__ float gate(float z) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z));
}
__device__ __forceinline__ float act_value(int act, float z) {
  if (act == kRelu) return z < 0.0f ? 0.0f : z;
  if (act == kGelu) return z * phi(z);
  if (act == kSilu) return z * gate(z);
  return z;
}
__device__ __forceinline__ float act_slope(int act, float z) {
  if (act == kRelu) return z > 0.0f ? 1.0f : 0.0f;
  if (act == kGelu)
    return phi(z) + z * 0.3989422804014327f * __builtin_amdgcn_exp2f(-0.7213475204444817f * z * z);
  if (act == kSilu) {
    const float t = gate(z);
    return t * (1.0f + z * (1.0f - t));
  }
  return 1.0f;
}

// One operand of a product: element (i, k) at p + i * si + k * sk.  The kernels'
// AK, BK say which stride is 1: that of k, the contracted axis, or that of i.
struct Operand {
  const void* p;
  int64_t si, sk;
};
struct Product {
  int M, N, K;
  Operand a, b;  // rows of A (i = m), columns of B (i = n)
  void* c;
  int64_t cs;
  // epilogue of the forward product
  int act;
  const void *bias, *res;
  int64_t rs;
  void* z;
  int64_t zs;
};

// c[0..3] of row m, columns n..n+3: the epilogue.
template <class T, bool EPI, bool VEC>
__device__ __forceinline__ void finish4(const Product& p, int m, int n, float c[4]) {
  using E = typename T::E;
  const int cnt = min(p.N - n, 4);
  if (EPI) {
    if (p.bias)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < cnt) c[i] += (float)((const E*)p.bias)[n + i];
    if (p.z)
      store4<VEC>((uint16_t*)p.z + m * p.zs + n, make_uint2(T::pack(c[0], c[1]), T::pack(c[2], c[3])), cnt);
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = act_value(p.act, c[i]);
    if (p.res)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i < cnt) c[i] += (float)((const E*)p.res)[m * p.rs + n + i];
  }
  store4<VEC>((uint16_t*)p.c + m * p.cs + n, make_uint2(T::pack(c[0], c[1]), T::pack(c[2], c[3])), cnt);
}

// Any sizes, strides and alignment: 64 x 64 tiles, 32 deep, a 32 x 32 part a
// wavefront; both operands go through LDS with their contracted axis contiguous.
// The product is formed transposed (A operand: columns of B), so that a lane's
// result registers are neighbours in a row of C.
template <class T, bool EPI, bool AK, bool BK>
__global__ __launch_bounds__(256) void k_product_any(const Product p) {
  constexpr int kT = 64, kD = 32, kRow = kD + 8;  // padded rows: 16-byte reads spread over the banks
  __shared__ alignas(16) uint16_t sa[kT * kRow], sb[kT * kRow];
  const int tiles_n = (p.N + kT - 1) / kT;
  const int id = xcd_order(blockIdx.x, gridDim.x);
  const int n0 = id % tiles_n * kT, m0 = id / tiles_n * kT;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, r = lane & 31, h = lane >> 5;

  uint4 ra, rb;
  // 8 elements a thread, along whichever axis is contiguous
  auto fetch = [&](const Operand& o, bool along_k, int i0, int most, int k0) {
    const int i = i0 + (along_k ? tid / 4 : 8 * (tid % 8)), k = k0 + (along_k ? 8 * (tid % 4) : tid / 8);
    const uint16_t* q = (const uint16_t*)o.p + i * o.si + k * o.sk;
    const int n = along_k ? (i < most ? min(p.K - k, 8) : 0) : (k < p.K ? min(most - i, 8) : 0);
    return load8<false>(q, n);
  };
  auto put = [&](uint16_t* s, uint4 v, bool along_k) {
    if (along_k) {
      *reinterpret_cast<uint4*>(s + (tid / 4) * kRow + 8 * (tid % 4)) = v;
    } else {
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int j = 0; j < 8; ++j)
        s[(8 * (tid % 8) + j) * kRow + tid / 8] = (uint16_t)(w[j / 2] >> (16 * (j & 1)));
    }
  };
  floatx16 acc = {};
  ra = fetch(p.a, AK, m0, p.M, 0);
  rb = fetch(p.b, BK, n0, p.N, 0);
  for (int k0 = 0; k0 < p.K; k0 += kD) {
    __syncthreads();
    put(sa, ra, AK);
    put(sb, rb, BK);
    __syncthreads();
    if (k0 + kD < p.K) {
      ra = fetch(p.a, AK, m0, p.M, k0 + kD);
      rb = fetch(p.b, BK, n0, p.N, k0 + kD);
    }
#pragma unroll
    for (int s = 0; s < kD / 16; ++s) {
      const int at = 16 * s + 8 * h;
      const uint4 x = *reinterpret_cast<const uint4*>(sb + (32 * (wave & 1) + r) * kRow + at);
      const uint4 y = *reinterpret_cast<const uint4*>(sa + (32 * (wave >> 1) + r) * kRow + at);
      acc = T::mma(x, y, acc);
    }
  }
  const int m = m0 + 32 * (wave >> 1) + r;
  if (m >= p.M) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int n = n0 + 32 * (wave & 1) + 8 * i + 4 * h;
    float c[4] = {acc[4 * i], acc[4 * i + 1], acc[4 * i + 2], acc[4 * i + 3]};
    if (n < p.N) finish4<T, EPI, false>(p, m, n, c);
  }
}

// dz = dy act'(z) (left out where act is none: dz is dy) and the column sums of
// 64 rows each: 256 columns a workgroup, 8 a thread.
template <class T, bool VEC>
__global__ __launch_bounds__(256) void k_linear_dz(const LinearArgs a, uint16_t* dz, int64_t dz_stride,
                                                   float* part) {
  __shared__ float red[8][256];
  const int tiles_n = (a.N + 255) / 256;
  const int n = (blockIdx.x % tiles_n) * 256 + 8 * (threadIdx.x % 32);
  const int rb = blockIdx.x / tiles_n, grp = threadIdx.x / 32, cnt = min(a.N - n, 8);
  float sum[8] = {};
  for (int i = grp; i < 64; i += 8) {
    const int m = rb * 64 + i;
    if (m >= a.M || cnt <= 0) break;
    const uint4 w = load8<VEC>((const uint16_t*)a.dy + m * a.dys + n, cnt);
    float g[8] = {T::lo(w.x), T::hi(w.x), T::lo(w.y), T::hi(w.y), T::lo(w.z), T::hi(w.z), T::lo(w.w), T::hi(w.w)};
    if (a.act != kNone) {
      const uint4 u = load8<VEC>((const uint16_t*)a.z + m * a.zs + n, cnt);
      const float z[8] = {T::lo(u.x), T::hi(u.x), T::lo(u.y), T::hi(u.y), T::lo(u.z), T::hi(u.z), T::lo(u.w), T::hi(u.w)};
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] *= act_slope(a.act, z[j]);
      uint16_t* o = dz + m * dz_stride + n;
      store4<VEC>(o, make_uint2(T::pack(g[0], g[1]), T::pack(g[2], g[3])), cnt);
      store4<VEC>(o + 4, make_uint2(T::pack(g[4], g[5]), T::pack(g[6], g[7])), cnt - 4);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] += g[j];
  }
  if (!part) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) red[grp][8 * (threadIdx.x % 32) + j] = sum[j];
  __syncthreads();
  const int c = (blockIdx.x % tiles_n) * 256 + threadIdx.x;
  if (c < a.N) {
    float t = 0.0f;
    for (int i = 0; i < 8; ++i) t += red[i][threadIdx.x];
    part[(int64_t)rb * a.N + c] = t;
  }
}

// db: the row blocks' sums added up in order, 64 columns a workgroup, 4 rows at a time.
template <class T>
__global__ __launch_bounds__(256) void k_linear_db(const float* part, int blocks, int N, typename T::E* db) {
  __shared__ float red[4][64];
  const int c = blockIdx.x * 64 + threadIdx.x % 64, r = threadIdx.x / 64;
  float t = 0.0f;
  if (c < N)
    for (int i = r; i < blocks; i += 4) t += part[(int64_t)i * N + c];
  red[r][threadIdx.x % 64] = t;
  __syncthreads();
  if (r == 0 && c < N) db[c] = (typename T::E)(red[0][threadIdx.x] + red[1][threadIdx.x] +
                                               red[2][threadIdx.x] + red[3][threadIdx.x]);
}

template <class T, bool EPI, bool AK, bool BK>
void product(const Product& p, hipStream_t s) {
  if (p.M == 0) return;
  const int64_t n = (int64_t)((p.M + 63) / 64) * ((p.N + 63) / 64);
  k_product_any<T, EPI, AK, BK><<<(unsigned)n, 256, 0, s>>>(p);
}

template <class T>
void forward(const LinearArgs& a, void* ws, hipStream_t s) {
  Product p = {};
  p.M = a.M, p.N = a.N, p.K = a.K;
  p.a = {a.x, a.xs, 1};
  p.b = {a.w, 1, a.ws};
  p.c = a.y, p.cs = a.ys;
  p.act = a.act, p.bias = a.bias, p.res = a.res, p.rs = a.rs, p.z = a.z, p.zs = a.zs;
  product<T, true, true, false>(p, s);
}

int64_t dz_row(const LinearArgs& a) { return ((int64_t)a.N + 7) / 8 * 8; }
int64_t dz_bytes(const LinearArgs& a) {  // dz, where it is not dy itself
  return a.act == kNone ? 0 : ((int64_t)a.M * dz_row(a) * 2 + 15) / 16 * 16;
}

template <class T>
void backward(const LinearArgs& a, void* ws, hipStream_t s) {
  const int blocks = (a.M + 63) / 64;
  const void* dz = a.act == kNone ? a.dy : ws;
  const int64_t dzs = a.act == kNone ? a.dys : dz_row(a);
  float* part = a.db ? (float*)((char*)ws + dz_bytes(a)) : nullptr;
  if (blocks && (a.act != kNone || a.db)) {
    const int64_t n = (int64_t)blocks * ((a.N + 255) / 256);
    if (a.vec)
      k_linear_dz<T, true><<<(unsigned)n, 256, 0, s>>>(a, (uint16_t*)ws, dzs, part);
    else
      k_linear_dz<T, false><<<(unsigned)n, 256, 0, s>>>(a, (uint16_t*)ws, dzs, part);
  }
  if (a.db) k_linear_db<T><<<(a.N + 63) / 64, 256, 0, s>>>(part, blocks, a.N, (typename T::E*)a.db);
  if (a.dx) {  // [M][K], over N
    Product p = {};
    p.M = a.M, p.N = a.K, p.K = a.N;
    p.a = {dz, dzs, 1};
    p.b = {a.w, a.ws, 1};
    p.c = a.dx, p.cs = a.dxs;
    product<T, false, true, true>(p, s);
  }
  if (a.dw) {  // [K][N], over M
    Product p = {};
    p.M = a.K, p.N = a.N, p.K = a.M;
    p.a = {a.x, 1, a.xs};
    p.b = {dz, 1, dzs};
    p.c = a.dw, p.cs = a.dws;
    product<T, false, false, false>(p, s);
  }
}

}  // namespace

int64_t linear_fwd_bytes(const LinearArgs& a) { return 0; }

hipError_t launch_linear_fwd(const LinearArgs& a, void* ws, hipStream_t s) {
  a.dtype == kF16 ? forward<F16>(a, ws, s) : forward<BF16>(a, ws, s);
  return hipGetLastError();
}

int64_t linear_bwd_bytes(const LinearArgs& a) {
  return dz_bytes(a) + (int64_t)((a.M + 63) / 64) * a.N * 4;
}

hipError_t launch_linear_bwd(const LinearArgs& a, void* ws, hipStream_t s) {
  a.dtype == kF16 ? backward<F16>(a, ws, s) : backward<BF16>(a, ws, s);
  return hipGetLastError();
}

}  // namespace pnerf
