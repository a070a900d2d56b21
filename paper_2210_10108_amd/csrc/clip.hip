// The norm over all gradients and their scaling:
//   norm = sqrt(sum g^2),  c = min(1, max_norm / (norm + eps)),  out = c g
// Squares are taken and summed in float64: none of a float32 or bfloat16 gradient
// overflows or is lost, and the order of the sum, which is fixed, does not matter to
// the result's 32 bits.
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

constexpr int kBlock = 256, kParts = 8 * kCUs;

// Elements of a chunk before its first 16-byte boundary (n or less).
template <class E>
__device__ __forceinline__ int head_of(const E* p, int n) {
  return min((int)((16 - ((uintptr_t)p & 15)) & 15) / (int)sizeof(E), n);
}

// The sum of squares of a thread's share of a chunk: 8 elements at a time from the
// first 16-byte boundary on, what is before and behind them one by one.
template <class E>
__device__ __forceinline__ double squares(const E* g, int n) {
  double t = 0.0;
  const int head = head_of(g, n), groups = (n - head) / 8, tail = head + 8 * groups;
#pragma unroll 4
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
  return t;
}

// Where gradient and output reach a 16-byte boundary together, 8 elements at a time,
// else one by one.  (The share of a thread is read before it is written: they may be one.)
template <class E, class O>
__device__ __forceinline__ void scaled(const E* g, O* out, int n, float c) {
  const int first = head_of(g, n);
  const bool together = first == n || ((uintptr_t)(out + first) & 15) == 0;
  const int head = together ? first : n, groups = (n - head) / 8, tail = head + 8 * groups;
#pragma unroll 4
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

// The entry that holds a chunk: the last one that starts at or before it.
__device__ __forceinline__ int entry_of(const ClipEntry* e, int count, uint32_t chunk) {
  int lo = 0, hi = count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (e[mid].first <= chunk) lo = mid; else hi = mid;
  }
  return lo;
}

template <bool TABLE>
__global__ __launch_bounds__(kBlock) void k_clip_sum(const ClipArgs a) {
  const ClipEntry* table = TABLE ? a.table : a.e;
  double t = 0.0;
  for (uint32_t chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
    const ClipEntry& e = table[entry_of(table, a.count, chunk)];
    const int64_t at = (int64_t)(chunk - e.first) * kClipChunk;
    const int n = (int)min(e.n - at, (int64_t)kClipChunk);
    if (e.dtype == kF32) t += squares((const float*)e.g + at, n);
    else if (e.dtype == kF16) t += squares((const _Float16*)e.g + at, n);
    else t += squares((const __bf16*)e.g + at, n);
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
  const double x = a.max_norm / (norm + a.eps);
  // at most 1; a norm that is NaN makes all results NaN, and without a bound nothing is scaled
  const float c = a.max_norm == INFINITY || x >= 1.0 ? 1.0f : (float)x;
  // the chunks that were read last come first: they may still be in a cache
  for (uint32_t i = blockIdx.x; i < a.chunks; i += gridDim.x) {
    const uint32_t chunk = a.chunks - 1 - i;
    const ClipEntry& e = table[entry_of(table, a.count, chunk)];
    if (c == 1.0f && e.g == e.out) continue;
    const int64_t at = (int64_t)(chunk - e.first) * kClipChunk;
    const int n = (int)min(e.n - at, (int64_t)kClipChunk);
    if (e.dtype == kF32) scaled((const float*)e.g + at, (float*)e.out + at, n, c);
    else if (e.dtype == kF16 && e.out_dtype == kF32) scaled((const _Float16*)e.g + at, (float*)e.out + at, n, c);
    else if (e.dtype == kF16) scaled((const _Float16*)e.g + at, (_Float16*)e.out + at, n, c);
    else if (e.out_dtype == kF32) scaled((const __bf16*)e.g + at, (float*)e.out + at, n, c);
    else scaled((const __bf16*)e.g + at, (__bf16*)e.out + at, n, c);
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
