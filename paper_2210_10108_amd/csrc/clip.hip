// The norm over all gradients and their scaling:
//   norm = sqrt(sum g^2),  c = min(1, max_norm / (norm + eps)),  out = c g
// Squares are taken and summed in float64: none of a float32 or bfloat16 gradient
// overflows or is lost, and the order of the sum, which is fixed, does not matter to
// the result's 32 bits.
//
// Bound by memory: every gradient is read twice and an output written (353 million
// bfloat16 elements in 150 tensors: 364 us for 2.1 GB, 706 MB at 5.9 TB/s and 1.4 GB at 5.8,
// what the last cache still holds of the first reading included).
//
// Two launches: the workgroups' partial sums, then every workgroup adds all of them
// up in the same order and scales its chunks.  The gradients of a call are one list
// of chunks, so that many small tensors cost no launches; up to kClipInline of them
// are described in the kernels' arguments, more in a table in the workspace that
// small launches fill.
#define PNERF_LAYERS_DEVICE
#include <algorithm>

#include "rows_common.h"

namespace pnerf {
namespace {

// Workgroups, with a partial sum each: 399 us at the size above with 4 a compute unit and
// chunks of 8192, 405 with 8; chunks of 16384: 409 and 425 (before the outputs went past the
// caches).
constexpr int kBlock = 256, kParts = 4 * kCUs;
constexpr uint32_t kPastChunks = (1u << 26) / kClipChunk;  // 128 MB of 16-bit gradients, and as much written

// Elements of a chunk before its first 16-byte boundary (n or less).
template <class E>
__device__ __forceinline__ int head_of(const E* p, int n) {
  return min((int)((16 - ((uintptr_t)p & 15)) & 15) / (int)sizeof(E), n);
}

// The sum of squares of a thread's share of a chunk.  A whole chunk on a 16-byte
// boundary (nearly all are): all its loads, then `meanwhile`, then their squares.
// Elsewhere 8 elements at a time from the first boundary on, the others one by one.
template <class E, class F>
__device__ __forceinline__ double squares(const void* p, int n, F meanwhile) {
  const E* g = (const E*)p;
  double t = 0.0;
  const int head = head_of(g, n);
  if (n == kClipChunk && head == 0) {
    constexpr int kLoads = kClipChunk / 8 / kBlock;
    typename Elem<E>::Raw raw[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k) raw[k] = Elem<E>::raw(g + 8 * (threadIdx.x + k * kBlock));
    meanwhile();
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      float v[8];
      Elem<E>::unpack(raw[k], v);
#pragma unroll
      for (int j = 0; j < 8; ++j) t = fma((double)v[j], (double)v[j], t);
    }
    return t;
  }
  const int groups = (n - head) / 8, tail = head + 8 * groups;
  for (int i = threadIdx.x; i < groups; i += kBlock) {
    float v[8];
    load<E>(g + head + 8 * i, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) t = fma((double)v[j], (double)v[j], t);
  }
  for (int i = threadIdx.x; i < head + n - tail; i += kBlock) {
    const double v = (double)(float)g[i < head ? i : tail + i - head];
    t = fma(v, v, t);
  }
  meanwhile();
  return t;
}

// 8 elements to memory; past: without a place in the caches.
template <class O>
__device__ __forceinline__ void store8(O* p, const float (&v)[8], bool past) {
  if (!past) return Elem<O>::store(p, v);
  if constexpr (sizeof(O) == 4) {
    __builtin_nontemporal_store(floatx4{v[0], v[1], v[2], v[3]}, (floatx4*)p);
    __builtin_nontemporal_store(floatx4{v[4], v[5], v[6], v[7]}, (floatx4*)p + 1);
  } else {
    alignas(16) O e[8];
    Elem<O>::store(e, v);
    __builtin_nontemporal_store(*reinterpret_cast<const u32x4*>(e), (u32x4*)p);
  }
}

// The same for scaling.  Where gradient and output do not reach a 16-byte boundary
// together, one by one.  (What a thread writes it has read before: they may be one.)
template <class E, class O, class F>
__device__ __forceinline__ void scaled(const void* p, void* q, int n, float c, bool past, F meanwhile) {
  const E* g = (const E*)p;
  O* out = (O*)q;
  const int first = head_of(g, n);
  const bool together = first == n || ((uintptr_t)(out + first) & 15) == 0;
  if (n == kClipChunk && first == 0 && together) {
    constexpr int kLoads = kClipChunk / 8 / kBlock;
    typename Elem<E>::Raw raw[kLoads];
#pragma unroll
    for (int k = 0; k < kLoads; ++k) raw[k] = Elem<E>::raw(g + 8 * (threadIdx.x + k * kBlock));
    meanwhile();
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
      float v[8];
      Elem<E>::unpack(raw[k], v);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= c;
      store8(out + 8 * (threadIdx.x + k * kBlock), v, past);
    }
    return;
  }
  const int head = together ? first : n, groups = (n - head) / 8, tail = head + 8 * groups;
  for (int i = threadIdx.x; i < groups; i += kBlock) {
    float v[8];
    load<E>(g + head + 8 * i, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] *= c;
    Elem<O>::store(out + head + 8 * i, v);
  }
  for (int i = threadIdx.x; i < head + n - tail; i += kBlock) {
    const int at = i < head ? i : tail + i - head;
    out[at] = (O)((float)g[at] * c);
  }
  meanwhile();
}

// Sum over the workgroup, in all threads, in an order that is always the same.
__device__ __forceinline__ double block_sum(double x) {
  __shared__ double red[kBlock];
  red[threadIdx.x] = x;
  __syncthreads();
#pragma unroll
  for (int d = kBlock / 2; d; d /= 2) {
    if ((int)threadIdx.x < d) red[threadIdx.x] += red[threadIdx.x + d];
    __syncthreads();
  }
  return red[0];
}

// A chunk and what it is part of: the last entry that starts at or before it.
struct Chunk {
  const char* g;
  char* out;
  int n;  // elements; 0: past the last chunk
  int dtype, out_dtype;
  __device__ __forceinline__ Chunk(const ClipEntry* table, int count, bool there, uint32_t chunk) : n(0) {
    if (!there) return;
    int lo = 0, hi = count;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (table[mid].first <= chunk) lo = mid; else hi = mid;
    }
    const ClipEntry& e = table[lo];
    const int64_t at = (int64_t)(chunk - e.first) * kClipChunk;
    dtype = e.dtype, out_dtype = e.out_dtype;
    n = (int)min(e.n - at, (int64_t)kClipChunk);
    g = (const char*)e.g + at * (dtype == kF32 ? 4 : 2);
    out = (char*)e.out + at * (out_dtype == kF32 ? 4 : 2);
  }
};

// (The search for a workgroup's next chunk, a chain of dependent loads, is made while
// the current chunk's elements are on their way.)
template <bool TABLE>
__global__ __launch_bounds__(kBlock) void k_clip_sum(const ClipArgs a) {
  const ClipEntry* table = TABLE ? a.table : a.e;
  double t = 0.0;
  uint32_t i = blockIdx.x;
  for (Chunk x(table, a.count, i < a.chunks, i); x.n;) {
    Chunk next = x;
    auto search = [&] { i += gridDim.x, next = Chunk(table, a.count, i < a.chunks, i); };
    if (x.dtype == kF32) t += squares<float>(x.g, x.n, search);
    else if (x.dtype == kF16) t += squares<_Float16>(x.g, x.n, search);
    else t += squares<__bf16>(x.g, x.n, search);
    x = next;
  }
  t = block_sum(t);
  if (threadIdx.x == 0) a.part[blockIdx.x] = t;
}

template <bool TABLE>
__global__ __launch_bounds__(kBlock) void k_clip_scale(const ClipArgs a) {
  const ClipEntry* table = TABLE ? a.table : a.e;
  double t = 0.0;
  for (int i = threadIdx.x; i < a.parts; i += kBlock) t += a.part[i];
  const double norm = sqrt(block_sum(t));
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.norm = (float)norm;
  const double ratio = a.max_norm / (norm + a.eps);
  // at most 1; a norm that is NaN makes all results NaN, and without a bound nothing is scaled
  const float c = a.max_norm == INFINITY || ratio >= 1.0 ? 1.0f : (float)ratio;
  // The chunks that were read last come first: they may still be in the last cache (256
  // MB), and where it does not hold the outputs as well these are kept out of it (353
  // million bfloat16 elements: 399 us, so 367).
  const bool past = a.chunks > kPastChunks;
  uint32_t i = blockIdx.x;
  for (Chunk x(table, a.count, i < a.chunks, a.chunks - 1 - i); x.n;) {
    Chunk next = x;
    auto search = [&] { i += gridDim.x, next = Chunk(table, a.count, i < a.chunks, a.chunks - 1 - i); };
    if (c == 1.0f && x.g == x.out) search();
    else if (x.dtype == kF32) scaled<float, float>(x.g, x.out, x.n, c, past, search);
    else if (x.dtype == kF16 && x.out_dtype == kF32) scaled<_Float16, float>(x.g, x.out, x.n, c, past, search);
    else if (x.dtype == kF16) scaled<_Float16, _Float16>(x.g, x.out, x.n, c, past, search);
    else if (x.out_dtype == kF32) scaled<__bf16, float>(x.g, x.out, x.n, c, past, search);
    else scaled<__bf16, __bf16>(x.g, x.out, x.n, c, past, search);
    x = next;
  }
}

// Entries of the arguments to their place in the table.
__global__ __launch_bounds__(128) void k_clip_table(const ClipArgs a, int first) {
  if ((int)threadIdx.x < a.count) a.table[first + threadIdx.x] = a.e[threadIdx.x];
}

}  // namespace

int64_t clip_bytes(int64_t count) {
  return kParts * 8 + (count > kClipInline ? count * (int64_t)sizeof(ClipEntry) : 0);
}

// e: the call's entries that have elements.
hipError_t launch_clip(const ClipEntry* e, int count, double max_norm, double eps, float* norm, void* ws,
                       hipStream_t s) {
  ClipArgs a = {};
  a.max_norm = max_norm, a.eps = eps, a.norm = norm;
  a.part = (double*)ws;
  a.table = (ClipEntry*)((char*)ws + kParts * 8);
  const bool table = count > kClipInline;
  for (int i = 0; i < count; i += kClipInline) {
    a.count = std::min(count - i, kClipInline);
    std::copy(e + i, e + i + a.count, a.e);
    if (table) k_clip_table<<<1, 128, 0, s>>>(a, i);
  }
  a.count = count;
  a.chunks = count ? e[count - 1].first + (uint32_t)((e[count - 1].n + kClipChunk - 1) / kClipChunk) : 0;
  a.parts = (int)std::min<uint32_t>(a.chunks, kParts);
  const unsigned n = (unsigned)std::max(a.parts, 1);
  if (table) {
    k_clip_sum<true><<<n, kBlock, 0, s>>>(a);
    k_clip_scale<true><<<n, kBlock, 0, s>>>(a);
  } else {
    if (a.parts) k_clip_sum<false><<<n, kBlock, 0, s>>>(a);
    k_clip_scale<false><<<n, kBlock, 0, s>>>(a);
  }
  return hipGetLastError();
}

}  // namespace pnerf
