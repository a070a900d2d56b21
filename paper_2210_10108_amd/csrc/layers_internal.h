// Internal declarations of the layer operators (include/pnerf_layers.h): the
// kernels' arguments, the host launchers, and what the kernels share on the
// device (element types, matrix products, transposed LDS reads).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace pnerf {

constexpr int kCUs = 256;     // compute units of an MI355X
constexpr int kXCDs = 8;      // accelerator dies, each with its own L2

enum DType : int { kF32 = 0, kF16 = 1, kBF16 = 2 };

struct AttnArgs {
  int dtype;
  int B, Sq, Sk, Hq, Hkv, G, D;  // G = Hq / Hkv
  int M;                         // rows of one kv head: Sq * G, row r = query row r / G, head r % G
  int vec;                       // every row of every tensor starts on 16 bytes and D % 8 == 0
  float c;                       // scale * log2(e)
  float scale;
  const void *q, *k, *v;
  void* o;
  float* lse;
  int64_t qs[3], ks[3], vs[3], os[3];
  const int32_t *q_len, *kv_len;
  const uint8_t* mask;
  int64_t mask_stride;
  int splits;       // parts of the key axis (of the row axis in the dk, dv pass)
  float* part;      // partial results of the parts
  // backward
  const void* dout;
  void *dq, *dk, *dv;
  int64_t dos[3], dqs[3], dks[3], dvs[3];
  float* delta;     // (lse, delta) of every row [B][Hq][Sq]
  float *do_norm, *v_norm;  // float16: |do| of every row, |v| of every key [B][Hkv][Sk]
  // 8-bit states: k, v and their strides are of bytes; scales [B][blocks][Hkv], strides of batch and block
  const float *k_scale, *v_scale;
  int64_t kss[2], vss[2];
  int sorted;  // longest batch entries first
};

// Parts of the key axis and bytes of workspace of the forward pass.
int attn_fwd_splits(const AttnArgs& a);
int64_t attn_fwd_bytes(const AttnArgs& a);
hipError_t launch_attn_fwd(const AttnArgs& a, void* ws, hipStream_t s);
int64_t attn_bwd_bytes(const AttnArgs& a);
hipError_t launch_attn_bwd(const AttnArgs& a, void* ws, hipStream_t s);
hipError_t launch_attn_q8(const AttnArgs& a, void* ws, hipStream_t s);

struct QuantSide {
  const void* x;
  uint8_t* y;
  float* scale;
  int64_t xs[3], ys[3], ss[2];
};
struct QuantArgs {
  int dtype, B, S, H, D;
  int vec;  // every row of every tensor starts on 16 (outputs 8) bytes and D % 8 == 0
  QuantSide side[2];  // keys, values
  const int32_t* len;
  const uint8_t* mask;
  int64_t mask_stride;
};
hipError_t launch_quantize(const QuantArgs& a, hipStream_t s);

struct LayerNormArgs {
  int dtype, rows, W;
  int vec;  // every row of every tensor starts on 16 bytes and W % 8 == 0
  float eps;
  const void *x, *w, *b, *dy, *dres;
  void *y, *dx, *dw, *db;
  int64_t xs, ys, dys, drs, dxs;
};
hipError_t launch_layer_norm_fwd(const LayerNormArgs& a, hipStream_t s);
int64_t layer_norm_bwd_bytes(const LayerNormArgs& a);
hipError_t launch_layer_norm_bwd(const LayerNormArgs& a, void* ws, hipStream_t s);

// One gradient of a clipping call.
struct ClipEntry {
  const void* g;
  void* out;
  int64_t n;
  uint32_t first;  // its first chunk among all
  uint16_t dtype, out_dtype;
};
constexpr int kClipChunk = 8192;  // elements that a workgroup takes at a time
constexpr int kClipInline = 96;   // entries that a launch carries in its arguments
struct ClipArgs {
  double max_norm, eps;
  int count;        // entries; the first kClipInline of a group in e, or all in `table`
  uint32_t chunks;
  int parts;        // workgroups of the sum, each with its partial
  double* part;
  float* norm;
  ClipEntry* table;
  ClipEntry e[kClipInline];
};
int64_t clip_bytes(int64_t count);
hipError_t launch_clip(const ClipEntry* e, int count, double max_norm, double eps, float* norm, void* ws,
                       hipStream_t s);

struct NormSide {
  int rows, heads;
  const void *x, *w, *dy;
  void *y, *dx, *dw;
  const int32_t* pos;
  int64_t xs[2], ys[2], dys[2], dxs[2];
};
struct NormArgs {
  int dtype, D, R, interleaved, n_pos;
  int vec;  // 8 elements of every row load as one, and the rotation pairs whole such groups
  float eps;
  const float* table;
  NormSide side[2];  // queries, keys
  // rotation at positions of several axes (pos is then [rows][axes])
  int axes;
  int whole;         // the pairs of every 8 elements (of every 16 where they are interleaved) share an axis
  int norm;          // 0: the heads are turned as they are
  float sign;        // -1: turned back
  uint32_t pair_axis[8];  // 2 bits a pair
};
hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t s);
int64_t norm_bwd_bytes(const NormArgs& a);
hipError_t launch_norm_bwd(const NormArgs& a, void* ws, hipStream_t s);
hipError_t launch_axes_fwd(const NormArgs& a, hipStream_t s);
hipError_t launch_axes_bwd(const NormArgs& a, void* ws, hipStream_t s);  // workspace as for launch_norm_bwd

struct LinearArgs {
  int dtype, act;
  int M, N, K;
  const void *x, *w, *bias, *res, *dy;
  void *y, *z;            // forward: z is written; backward: z is read
  void *dx, *dw, *db;
  int64_t xs, ws, rs, ys, zs, dys, dxs, dws;
};
int64_t linear_fwd_bytes(const LinearArgs& a);
hipError_t launch_linear_fwd(const LinearArgs& a, void* ws, hipStream_t s);
int64_t linear_bwd_bytes(const LinearArgs& a);
hipError_t launch_linear_bwd(const LinearArgs& a, void* ws, hipStream_t s);

// ------------------------------------------------------------------ device
#if defined(__HIP_DEVICE_COMPILE__) || defined(PNERF_LAYERS_DEVICE)
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// The 16-bit element types: conversions, and the 32 x 32 x 16 product.  Operand
// layout of the product: lane l holds row (A) or column (B) l % 32 and the 8
// positions 8 (l / 32) .. + 7 of the 16-deep axis; result: column l % 32, and in
// register i row 8 (i / 4) + 4 (l / 32) + i % 4.
struct F16 {
  using E = _Float16;
  __device__ static __forceinline__ uint32_t pack(float a, float b) {
    const f16x2 h = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, h);
  }
  __device__ static __forceinline__ float lo(uint32_t w) { return (float)__builtin_bit_cast(f16x2, w)[0]; }
  __device__ static __forceinline__ float hi(uint32_t w) { return (float)__builtin_bit_cast(f16x2, w)[1]; }
  __device__ static __forceinline__ floatx16 mma(uint4 a, uint4 b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};
struct BF16 {
  using E = __bf16;
  __device__ static __forceinline__ uint32_t pack(float a, float b) {
    const bf16x2 h = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, h);
  }
  __device__ static __forceinline__ float lo(uint32_t w) { return __uint_as_float(w << 16); }
  __device__ static __forceinline__ float hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
  __device__ static __forceinline__ floatx16 mma(uint4 a, uint4 b, floatx16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};

// 8 consecutive 16-bit elements from p, n of them within bounds (the others 0):
// one 16-byte load where VEC (then n is 0 or 8), else element by element.
template <bool VEC>
__device__ __forceinline__ uint4 load8(const void* p, int n) {
  uint4 r = make_uint4(0, 0, 0, 0);
  if (VEC) {
    if (n > 0) r = *reinterpret_cast<const uint4*>(p);
  } else {
    const uint16_t* e = reinterpret_cast<const uint16_t*>(p);
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) w[j / 2] |= (uint32_t)e[j] << (16 * (j & 1));
    r = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return r;
}

// 4 consecutive elements to p, n of them within bounds.
template <bool VEC>
__device__ __forceinline__ void store4(void* p, uint2 v, int n) {
  if (VEC) {
    if (n > 0) *reinterpret_cast<uint2*>(p) = v;
  } else {
    uint16_t* e = reinterpret_cast<uint16_t*>(p);
    if (n > 0) e[0] = (uint16_t)v.x;
    if (n > 1) e[1] = (uint16_t)(v.x >> 16);
    if (n > 2) e[2] = (uint16_t)v.y;
    if (n > 3) e[3] = (uint16_t)(v.y >> 16);
  }
}

// Transposed LDS read: within each 16 lanes, lane 4 r + c gives the address of
// row r, elements 4c .. 4c + 3; lane i receives element i of rows 0 .. 3.
__device__ __forceinline__ uint2 read_tr(const void* lds) {
  const s16x4 t = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4*)lds);
  return __builtin_bit_cast(uint2, t);
}

// Values of both 32-lane halves: (lane % 32, lane % 32 + 32).
__device__ __forceinline__ void halves(float x, float& a, float& b) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  a = __uint_as_float(r[0]);
  b = __uint_as_float(r[1]);
}

// Loads that write LDS themselves: 16 bytes a lane, the lanes' 64 pieces one
// after the other from `lds` (a byte address, the same in all lanes).  `offset`
// is each lane's own, against a descriptor's base and bound: past the bound zeros
// are written, and kOutside is past every bound.  (m0, which holds the address, is
// no register that the compiler keeps anything in: nothing else here uses it.)
// The compiler does not see the loads: s_waitcnt is the kernel's own.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
constexpr uint32_t kOutside = 0x80000000u;
__device__ __forceinline__ void load_to_lds(uint32_t lds, uint32_t offset, u32x4 desc) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :: "s"(lds), "v"(offset), "s"(desc) : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p;
}
// Descriptor of `bytes` bytes from base (the same in all lanes), at most 2^31 - 1.
__device__ __forceinline__ u32x4 descriptor(const void* base, int64_t bytes) {
  u32x4 d;
  d[0] = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)base);
  d[1] = __builtin_amdgcn_readfirstlane((uint32_t)((uintptr_t)base >> 32) & 0xFFFFu);
  d[2] = __builtin_amdgcn_readfirstlane((uint32_t)min(bytes, (int64_t)0x7FFFFFFF));
  d[3] = 0x00027000u;
  return d;
}

// LDS written by lanes of this wavefront may be read by its others from here on
// (a wavefront's LDS accesses complete in order: this holds the compiler).
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Work item `id` of n such that consecutive items run on one XCD (workgroups
// go to the XCDs in turn): items that share operands share an L2.
__device__ __forceinline__ int xcd_order(int id, int n) {
  const int x = id % kXCDs, i = id / kXCDs, q = n / kXCDs, r = n % kXCDs;
  return x * q + min(x, r) + i;
}
#endif

}  // namespace pnerf
