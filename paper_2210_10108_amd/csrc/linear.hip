// Linear layer: y = act(x W + bias) + residual, and its gradient
//   dz = dy act'(z),  dx = dz W^T,  dW = x^T dz,  db = sum_m dz.
// Three matrix products of one kind, C[m][n] = sum_k A[m][k] B[k][n], which
// differ in which axis of each operand is contiguous in memory.
#define PNERF_LAYERS_DEVICE
#include <algorithm>
#include <type_traits>

#include "layers_internal.h"

namespace pnerf {
namespace {

enum Act : int { kNone = 0, kRelu = 1, kGelu = 2, kSilu = 3 };

// The normal distribution function and its density.  For z <= 0 it is the density's
// exponential times erfcx(-z / sqrt 2) / 2, a smooth function that t p(t) fits, t = 1 / (1 -
// 0.3625 z) and p of degree 6: by weighted least squares of the relative error
// over 0 >= z >= -14, at most 7.7e-7 of it there.  (GELU's tail is small but no less exact
// in 16 bits than other numbers, so an absolute bound will not do.)  In 32-bit steps the
// relative error is 2e-6 down to z = -6 and 8e-6 at -13, where the exponent's rounding
// weighs; above zero the error is 5e-7 at most.  One reciprocal and one exponential,
// which is the density's as well.
__device__ __forceinline__ float phi(float z, float& density) {
  const float e = __builtin_amdgcn_exp2f(-0.7213475204444817f * z * z);
  const float t = __builtin_amdgcn_rcpf(fmaf(0.3625f, fabsf(z), 1.0f));
  float q = fmaf(t, 0.048062854f, -0.17974228f);
  q = fmaf(t, q, 0.1751038f);
  q = fmaf(t, q, 0.029682558f);
  q = fmaf(t, q, 0.13925667f);
  q = fmaf(t, q, 0.1429364f);
  q = fmaf(t, q, 0.14470038f);
  q *= t * e;
  density = 0.3989422804014327f * e;
  return z < 0.0f ? q : 1.0f - q;
}
__device__ __forceinline__ float gate(float z) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z));
}
__device__ __forceinline__ float act_value(int act, float z) {
  if (act == kRelu) return z < 0.0f ? 0.0f : z;
  if (act == kGelu) {
    float d;
    return z * phi(z, d);
  }
  if (act == kSilu) return z * gate(z);
  return z;
}
__device__ __forceinline__ float act_slope(int act, float z) {
  if (act == kRelu) return z > 0.0f ? 1.0f : 0.0f;
  if (act == kGelu) {
    float d;
    const float f = phi(z, d);
    return fmaf(z, d, f);
  }
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
  int vec;       // rows of 8 elements of C and of the epilogue's tensors start on 16 bytes, N % 8 == 0
  int row;       // N rounded up to 8: a row of the parts' sums
  // epilogue of the forward product
  int act;
  const void *bias, *res;
  int64_t rs;
  void* z;
  int64_t zs;
};

// c[0..W-1] of row m, columns n0.. before N: the epilogue, element by element.
template <class T, bool EPI, int W>
__device__ __forceinline__ void finish_any(const Product& p, int m, int n0, float c[W]) {
  using E = typename T::E;
#pragma unroll
  for (int i = 0; i < W; ++i) {
    if (n0 + i >= p.N) break;
    float v = c[i];
    if (EPI) {
      if (p.bias) v += (float)((const E*)p.bias)[n0 + i];
      if (p.z) ((E*)p.z)[m * p.zs + n0 + i] = (E)v;
      v = act_value(p.act, v);
      if (p.res) v += (float)((const E*)p.res)[m * p.rs + n0 + i];
    }
    ((E*)p.c)[m * p.cs + n0 + i] = (E)v;
  }
}

// c[0..3] of row m, columns n..n+3: the epilogue.
template <class T, bool EPI>
__device__ __forceinline__ void finish4(const Product& p, int m, int n, float c[4]) {
  if (!p.vec) return finish_any<T, EPI, 4>(p, m, n, c);
  auto add = [&](const void* q) {
    const uint2 v = *reinterpret_cast<const uint2*>(q);
    c[0] += T::lo(v.x), c[1] += T::hi(v.x), c[2] += T::lo(v.y), c[3] += T::hi(v.y);
  };
  auto put = [&](void* q) { *reinterpret_cast<uint2*>(q) = make_uint2(T::pack(c[0], c[1]), T::pack(c[2], c[3])); };
  if (EPI) {
    if (p.bias) add((const uint16_t*)p.bias + n);
    if (p.z) put((uint16_t*)p.z + m * p.zs + n);
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = act_value(p.act, c[i]);
    if (p.res) add((const uint16_t*)p.res + m * p.rs + n);
  }
  put((uint16_t*)p.c + m * p.cs + n);
}

// c[0..7] of row m, columns n..n+7, where p.vec; bias and res: those 8 elements (zeros: none).
template <class T, bool EPI>
__device__ __forceinline__ void finish8(const Product& p, int m, int n, float c[8], uint4 bias, uint4 res) {
  auto add = [&](const uint4 v) {
    c[0] += T::lo(v.x), c[1] += T::hi(v.x), c[2] += T::lo(v.y), c[3] += T::hi(v.y);
    c[4] += T::lo(v.z), c[5] += T::hi(v.z), c[6] += T::lo(v.w), c[7] += T::hi(v.w);
  };
  auto packed = [&] { return make_uint4(T::pack(c[0], c[1]), T::pack(c[2], c[3]), T::pack(c[4], c[5]), T::pack(c[6], c[7])); };
  if (EPI) {
    add(bias);
    if (p.z) *reinterpret_cast<uint4*>((uint16_t*)p.z + m * p.zs + n) = packed();
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = act_value(p.act, c[i]);
    if (p.res) add(res);
  }
  *reinterpret_cast<uint4*>((uint16_t*)p.c + m * p.cs + n) = packed();
}

// Any sizes, strides and alignment: 64 x 64 tiles, 32 deep, a 32 x 32 part a
// wavefront; both operands go through LDS with their contracted axis contiguous.
// The product is formed transposed (A operand: columns of B), so that a lane's
// result registers are neighbours in a row of C.  A step waits for its element
// loads, about 2 us, so few tiles of a deep product are cut into parts of the
// depth (222 x 5690 x 101: 344 us in one part, 23 in 44 with their join).
template <class T, bool EPI, bool AK, bool BK>
__global__ __launch_bounds__(256) void k_product_any(const Product p, int splits, float* part) {
  constexpr int kT = 64, kD = 32, kRow = kD + 8;  // padded rows: 16-byte reads spread over the banks
  __shared__ alignas(16) uint16_t sa[kT * kRow], sb[kT * kRow];
  const int tiles_n = (p.N + kT - 1) / kT, tiles = (p.M + kT - 1) / kT * tiles_n;
  const int id = xcd_order(blockIdx.x, gridDim.x), sp = id / tiles;
  const int n0 = id % tiles % tiles_n * kT, m0 = id % tiles / tiles_n * kT;
  const int steps = (p.K + kD - 1) / kD, per = (steps + splits - 1) / splits;
  const int k_first = min(sp * per, steps) * kD, k_end = min((sp + 1) * per, steps) * kD;
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
  ra = fetch(p.a, AK, m0, p.M, k_first);
  rb = fetch(p.b, BK, n0, p.N, k_first);
  for (int k0 = k_first; k0 < k_end; k0 += kD) {
    __syncthreads();
    put(sa, ra, AK);
    put(sb, rb, BK);
    __syncthreads();
    if (k0 + kD < k_end) {
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
    if (n >= p.N) continue;
    if (splits > 1)
      *reinterpret_cast<floatx4*>(part + ((int64_t)sp * p.M + m) * p.row + n) = floatx4{c[0], c[1], c[2], c[3]};
    else
      finish_any<T, EPI, 4>(p, m, n, c);
  }
}

// ------------------------------------------------------------ aligned products
// Rows of 16-byte chunks go from memory to LDS by loads that write LDS
// themselves (load_to_lds); a chunk's place within its row is xored with bits of
// the row so that the fragment reads cover all banks, which the lanes' addresses
// in memory follow.  The buffer descriptor's bound gives zeros past the last row;
// lanes past the end of a row take an offset beyond any bound.
constexpr int kBK = 64;                      // depth of a tile in LDS
constexpr int64_t kMaxFastStride = 1 << 21;  // elements: a tile's offsets stay below 2^31 bytes

// One operand's tile of ROWS rows (of A, or columns of B) x 64: its loads and
// its fragments.  KC: the contracted axis is contiguous, an LDS row is a row of
// the operand, 8 chunks; else an LDS row is one k, ROWS / 8 chunks.
template <int ROWS, int NW, bool KC>
struct Tile {
  static constexpr int kChunks = KC ? kBK / 8 : ROWS / 8;        // of an LDS row
  static constexpr int kLoads = ROWS * kBK / 8 / 64 / NW;        // instructions a wavefront
  static constexpr int kStep = NW * 64 / kChunks;                // LDS rows between them
  static constexpr int kBytes = ROWS * kBK * 2;
  const char* base;   // of the current tile in memory
  int64_t row_bytes;  // between LDS rows
  int rows, inner;    // LDS rows left, and elements of one
  uint32_t off;       // this lane's first chunk
  int chunk;          // ... and which of its row it is
  uint32_t frag[KC ? 4 : 2];

  __device__ __forceinline__ void init(const Operand& o, int i0, int most, int k0, int K, int wave, int lane,
                                       int ifrag) {
    base = (const char*)o.p + 2 * (i0 * o.si + k0 * o.sk);
    row_bytes = 2 * (KC ? o.si : o.sk);
    rows = KC ? most - i0 : K - k0;
    inner = ((KC ? K - k0 : most - i0) + 7) & ~7;  // what a row holds past its end is zeros, to whole chunks
    const int p = wave * 64 + lane, r = p / kChunks;
    chunk = (p % kChunks) ^ (KC ? r & 7 : (r & 3) << 1);
    off = (uint32_t)(r * row_bytes + 16 * chunk);
    const int l32 = lane & 31, h = lane >> 5, l16 = lane & 15;
    if (KC) {
#pragma unroll
      for (int s = 0; s < 4; ++s) frag[s] = (ifrag + l32) * (2 * kBK) + 16 * ((2 * s + h) ^ (l32 & 7));
    } else {
      const int k = 8 * h + l16 / 4, col = ifrag + 16 * ((lane >> 4) & 1) + 4 * (l16 % 4);
#pragma unroll
      for (int s = 0; s < 2; ++s)
        frag[s] = k * (2 * ROWS) + 16 * (((col + 32 * s) / 8) ^ ((k & 3) << 1)) + 2 * (col % 8);
    }
  }
  // Loads n0 .. n1 - 1 of the tile, into LDS at lds.
  template <int N0, int N1>
  __device__ __forceinline__ void load(uint32_t lds, int wave) {
    const u32x4 desc = descriptor(base, (rows - 1) * row_bytes + 2 * inner);
    const uint32_t first = 8 * chunk < inner ? off : kOutside;
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds + wave * 1024);
#pragma unroll
    for (int n = N0; n < N1; ++n)
      load_to_lds(to + n * NW * 1024, first + (uint32_t)(n * kStep) * (uint32_t)row_bytes, desc);
  }
  __device__ __forceinline__ void next() {
    base += KC ? 2 * kBK : kBK * row_bytes;
    if (KC)
      inner -= kBK;
    else
      rows -= kBK;
  }
  // Fragment of 32 rows (number t of the wavefront's) at depth 16 s.
  __device__ __forceinline__ uint4 fragment(const char* lds, int t, int s) const {
    if (KC) return *reinterpret_cast<const uint4*>(lds + frag[s] + t * 32 * 2 * kBK);
    const char* p = lds + frag[t & 1] + (t / 2) * 128 + s * 16 * (2 * ROWS);
    const uint2 a = read_tr(p), b = read_tr(p + 4 * (2 * ROWS));
    return make_uint4(a.x, a.y, b.x, b.y);
  }
};

// Tells the scheduler to issue READS LDS reads evenly between MFMAS products.
template <int READS, int MFMAS, int I = 0>
__device__ __forceinline__ void spread_reads() {
  if constexpr (I < MFMAS) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a product
    constexpr int n = READS * (I + 1) / MFMAS - READS * I / MFMAS;
    if constexpr (n > 0) __builtin_amdgcn_sched_group_barrier(0x100, n, 0);  // LDS reads
    spread_reads<READS, MFMAS, I + 1>();
  }
}

// BM x BN tiles, 64 deep, two of them in LDS: while the products of one run, the
// loads of the one after the next fill the buffer just read.  2 x WN wavefronts;
// fragments are read one 16-deep step ahead, across the tiles' border, so that the
// one barrier a tile falls between the last reads of a tile and the last of its
// products.  LDS bounds the 256 x 256 tile: 192 KB read and 64 KB written for
// 2048 cycles of products a SIMD, all of the 128 bytes a cycle.  Eight wavefronts,
// two a SIMD, measured 1.05 to 1.12 PFLOP/s on 4096^3 where four, which read a third
// less, reached 0.88 to 0.97; with no branch in a tile and its LDS reads spread
// between its products 1.17 to 1.25 (8192^3: 1.19 to 1.26).
template <class T, bool EPI, bool AK, bool BK, int BM, int BN, int WN>
__global__ __launch_bounds__(128 * WN, BM == 256 ? 1 : 2) void k_product(const Product p, int splits, float* part) {
  constexpr int NW = 2 * WN, TM = BM / 64, TN = BN / WN / 32;  // wavefronts; 32 x 32 results of one
  using TA = Tile<BM, NW, AK>;
  using TB = Tile<BN, NW, BK>;
  constexpr int kBuf = TA::kBytes + TB::kBytes;
  constexpr int kLds = 2 * kBuf + (BN == 256 ? 8192 : 16384);  // the epilogue's need
  __shared__ alignas(128) char lds[kLds];

  // tiles in the order of the XCDs, and within one XCD's run 8 rows of tiles at a
  // time, so that the tiles in flight share operands in its L2
  const int tiles_m = (p.M + BM - 1) / BM, tiles_n = (p.N + BN - 1) / BN;
  int id = xcd_order(blockIdx.x, gridDim.x);
  const int sp = id / (tiles_m * tiles_n);
  id -= sp * tiles_m * tiles_n;
  const int band = id / (8 * tiles_n), in_band = id - band * 8 * tiles_n;
  const int height = min(8, tiles_m - band * 8);
  const int m0 = (band * 8 + in_band % height) * BM, n0 = in_band / height * BN;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / WN, wn = wave % WN;
  const int all = (p.K + kBK - 1) / kBK, per = (all + splits - 1) / splits;
  const int t0 = min(sp * per, all), nt = min(t0 + per, all) - t0;

  TA a;
  TB b;
  a.init(p.a, m0, p.M, t0 * kBK, p.K, wave, lane, wm * (BM / 2));
  b.init(p.b, n0, p.N, t0 * kBK, p.K, wave, lane, wn * (BN / WN));
  const uint32_t la = lds_address(lds), lb = la + TA::kBytes;

  floatx16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; ++i)
#pragma unroll
    for (int j = 0; j < TN; ++j) acc[i][j] = floatx16{};

  uint4 fa[2][TM], fb[2][TN];
  auto fragments = [&](int set, const char* buf, int s) {
#pragma unroll
    for (int i = 0; i < TM; ++i) fa[set][i] = a.fragment(buf, i, s);
#pragma unroll
    for (int j = 0; j < TN; ++j) fb[set][j] = b.fragment(buf + TA::kBytes, j, s);
  };
  constexpr int HA = TA::kLoads / 2, HB = TB::kLoads / 2;
  // One tile.  after: how many follow it (2: two or more).  No branches: the
  // fragment reads of the next step are spread between the products of this one.
  auto tile = [&](int cur, auto after) {
    const int oth = kBuf - cur;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if (s < 3) {
        fragments((s + 1) & 1, lds + cur, s + 1);
      } else if (after.value > 0) {
        // the next tile is in LDS, and every wavefront has read this one
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        fragments(0, lds + oth, 0);
      }
      // the tile after the next, into the buffer that the last barrier freed: its
      // first half now, its second during the next tile
      if (s == 3 && after.value > 1) {
        a.template load<0, HA>(la + cur, wave), b.template load<0, HB>(lb + cur, wave);
      }
      if (s == 0 && after.value > 0) {
        a.template load<HA, TA::kLoads>(la + oth, wave), b.template load<HB, TB::kLoads>(lb + oth, wave);
        a.next(), b.next();
      }
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = T::mma(fb[s & 1][j], fa[s & 1][i], acc[i][j]);
      if (s < 3 || after.value > 0) {
        constexpr int kReads = TM * (AK ? 1 : 2) + TN * (BK ? 1 : 2), kMfma = TM * TN;
        spread_reads<kReads, kMfma>();
      }
    }
  };
  if (nt > 0) {
    a.template load<0, TA::kLoads>(la, wave), b.template load<0, TB::kLoads>(lb, wave);
    a.next(), b.next();
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (nt > 1) a.template load<0, HA>(la + kBuf, wave), b.template load<0, HB>(lb + kBuf, wave);
    __builtin_amdgcn_s_barrier();
    fragments(0, lds, 0);
    int t = 0;
    for (; t + 2 < nt; ++t) tile((t & 1) * kBuf, std::integral_constant<int, 2>());
    if (t + 1 < nt) tile((t++ & 1) * kBuf, std::integral_constant<int, 1>());
    tile((t & 1) * kBuf, std::integral_constant<int, 0>());
  }

  // Results by way of LDS, 32 rows of the wavefront at a time, so that a lane
  // has 8 neighbours of a row and a row's lanes are neighbours.  The residual of
  // the next 32 rows is on its way into LDS (each lane's own pieces) meanwhile: a
  // wavefront is alone on its SIMD and nothing else would hide its latency.
  constexpr int kRow = BN / WN + 4, kLanes = BN / WN / 8, kStep = 64 / kLanes, kSteps = 32 / kStep;
  static_assert(BN / WN == 64, "a lane for every column");
  static_assert(NW * (32 * kRow * 4 + 2 * kSteps * 1024) <= kLds, "results and residual fit LDS");
  float* mine = reinterpret_cast<float*>(lds) + wave * 32 * kRow;
  const char* res = lds + NW * 32 * kRow * 4 + wave * 2 * kSteps * 1024;
  const int r = lane & 31, h = lane >> 5, n = n0 + wn * (BN / WN) + 8 * (lane % kLanes);
  const int first = m0 + wm * (BM / 2) + lane / kLanes;  // this lane's first row
  uint4 bias = make_uint4(0, 0, 0, 0);
  const bool with_res = EPI && p.res && p.vec && splits == 1, full = m0 + BM <= p.M && n0 + BN <= p.N;
  if (EPI && p.bias && p.vec && n < p.N) bias = *reinterpret_cast<const uint4*>((const uint16_t*)p.bias + n);
  auto load_res = [&](int i) {
    const char* base = (const char*)p.res + 2 * ((int64_t)(m0 + wm * (BM / 2) + 32 * i) * p.rs + n0 + wn * (BN / WN));
    const u32x4 desc = descriptor(base, 0x7FFFFFFF);
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds_address(res) + (i & 1) * kSteps * 1024);
    const uint32_t off = (uint32_t)(lane / kLanes) * (uint32_t)(2 * p.rs) + 16 * (lane % kLanes);
#pragma unroll
    for (int k = 0; k < kSteps; ++k)
      load_to_lds(to + 1024 * k, first + 32 * i + k * kStep < p.M && n < p.N ? off + k * kStep * (uint32_t)(2 * p.rs) : kOutside, desc);
  };
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __syncthreads();  // every wavefront has read its last fragments
  if (with_res) load_res(0);
#pragma unroll
  for (int i = 0; i < TM; ++i) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<floatx4*>(mine + r * kRow + 32 * j + 8 * q + 4 * h) =
            floatx4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    if (with_res) {
      // these 32 rows' residual is there; the stores of the 32 before, which were
      // issued after its loads, may still be on their way (their number is known
      // where no row or column of the tile is outside)
      if (i > 0 && full && p.z)
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * kSteps) : "memory");
      else if (i > 0 && full)
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kSteps) : "memory");
      else
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      if (i + 1 < TM) load_res(i + 1);
    }
    wave_fence();
    // An element a lane, 64 neighbours at a time (dx of 4001 x 4003 x 4005 134 us, 151 by
    // 8 elements a lane).
    if (!p.vec && splits == 1) {
      using E = typename T::E;
      const int col = n0 + wn * (BN / WN) + lane, row = m0 + wm * (BM / 2) + 32 * i;
      const int rows = col < p.N ? min(p.M - row, 32) : 0;
      const float add = EPI && p.bias && rows > 0 ? (float)((const E*)p.bias)[col] : 0.0f;
#pragma unroll 1
      for (int k = 0; k < rows; k += 8) {
        float v[8] = {}, u[8];
        if (EPI && p.res)  // all before the first store, which the compiler would not move them past
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (k + j < rows) v[j] = (float)((const E*)p.res)[(row + k + j) * p.rs + col];
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] = mine[(k + j) * kRow + lane] + add;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (k + j >= rows) break;
          if (EPI && p.z) ((E*)p.z)[(row + k + j) * p.zs + col] = (E)u[j];
          ((E*)p.c)[(row + k + j) * p.cs + col] = (E)(EPI ? act_value(p.act, u[j]) + v[j] : u[j]);
        }
      }
      wave_fence();
      continue;
    }
#pragma unroll 1
    for (int k = 0; k < kSteps; ++k) {
      const int m = first + 32 * i + k * kStep;
      if (m >= p.M || n >= p.N) continue;
      const floatx4* from = reinterpret_cast<const floatx4*>(mine + (lane / kLanes + k * kStep) * kRow + 8 * (lane % kLanes));
      const floatx4 x = from[0], y = from[1];
      if (splits > 1) {
        floatx4* to = reinterpret_cast<floatx4*>(part + ((int64_t)sp * p.M + m) * p.row + n);
        to[0] = x, to[1] = y;
      } else {
        float c[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
        const uint4 add = with_res ? *reinterpret_cast<const uint4*>(res + ((i & 1) * kSteps + k) * 1024 + 16 * lane)
                                   : make_uint4(0, 0, 0, 0);
        finish8<T, EPI>(p, m, n, c, bias, add);
      }
    }
    wave_fence();
  }
}

// The parts of the contracted axis added up in order, and the epilogue: 4
// elements of a row a thread.
template <class T, bool EPI>
__global__ __launch_bounds__(256) void k_product_join(const Product p, int splits, const float* part) {
  const int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, all = (int64_t)p.M * p.row;
  const int m = (int)(e / p.row), n = (int)(e - (int64_t)m * p.row);
  if (e >= all || n >= p.N) return;
  floatx4 x = *reinterpret_cast<const floatx4*>(part + e);
#pragma unroll 4
  for (int s = 1; s < splits; ++s) x += *reinterpret_cast<const floatx4*>(part + s * all + e);
  float c[4] = {x[0], x[1], x[2], x[3]};
  finish4<T, EPI>(p, m, n, c);
}

// Few rows (at most 32): the weights' bytes are the time.  They go from memory
// to registers, each once: lane l of a wavefront holds 4 neighbouring columns of
// W (4 (l % 16) ..) at depths 8 (l / 16) .. + 7, which two-register byte
// permutes turn into operands of the 16 x 16 x 32 product -- column j of every
// lane makes one.  A workgroup takes 64 columns, its 16 wavefronts the depths in
// turn; their sums meet in LDS.
template <class T>
struct Mma16;
template <>
struct Mma16<F16> {
  __device__ static __forceinline__ floatx4 mma(uint4 a, uint4 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};
template <>
struct Mma16<BF16> {
  __device__ static __forceinline__ floatx4 mma(uint4 a, uint4 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};

constexpr int kFewWaves = 16;
template <class T, int MT>
__global__ __launch_bounds__(kFewWaves * 64) void k_product_few(const Product p, int splits, float* part) {
  __shared__ float red[kFewWaves][16 * MT][64 + 4];
  const int tiles_n = (p.N + 63) / 64;
  const int n0 = blockIdx.x % tiles_n * 64, sp = blockIdx.x / tiles_n;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c16 = lane & 15, g = lane >> 4;
  const int steps = (p.K + 31) / 32, n = n0 + 4 * c16;
  const uint16_t* w = (const uint16_t*)p.b.p + n;
  const uint16_t* x = (const uint16_t*)p.a.p;
  floatx4 acc[MT][4];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = floatx4{};
  uint2 rw[2][8];
  uint4 rx[2][MT];
  auto fetch = [&](int set, int step) {
    const int k0 = 32 * step + 8 * g;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      rw[set][i] = n < p.N && k0 + i < p.K ? *reinterpret_cast<const uint2*>(w + (int64_t)(k0 + i) * p.b.sk)
                                           : make_uint2(0, 0);
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      const int m = 16 * i + c16;
      rx[set][i] = load8<true>(x + m * p.a.si + k0, m < p.M ? p.K - k0 : 0);
    }
  };
  auto multiply = [&](int set) {
    const uint2* v = rw[set];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;
      uint32_t f[4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
        f[i] = j < 2 ? __builtin_amdgcn_perm(v[2 * i + 1].x, v[2 * i].x, sel)
                     : __builtin_amdgcn_perm(v[2 * i + 1].y, v[2 * i].y, sel);
#pragma unroll
      for (int i = 0; i < MT; ++i)
        acc[i][j] = Mma16<T>::mma(make_uint4(f[0], f[1], f[2], f[3]), rx[set][i], acc[i][j]);
    }
  };
  const int stride = kFewWaves * splits, first = sp * kFewWaves + wave;
  if (first < steps) fetch(0, first);
  for (int s = first; s < steps; s += 2 * stride) {
    if (s + stride < steps) fetch(1, s + stride);
    multiply(0);
    if (s + stride < steps) {
      if (s + 2 * stride < steps) fetch(0, s + 2 * stride);
      multiply(1);
    }
  }
  // result: column m = lane % 16, row 4 g + i of product j is column 4 (4 g + i) + j of the tile
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<floatx4*>(&red[wave][16 * i + c16][4 * (4 * g + q)]) =
          floatx4{acc[i][0][q], acc[i][1][q], acc[i][2][q], acc[i][3][q]};
  __syncthreads();
  for (int e = threadIdx.x; e < 16 * MT * 16; e += kFewWaves * 64) {
    const int m = e / 16, c = 4 * (e % 16);
    if (m >= p.M || n0 + c >= p.N) continue;
    floatx4 t = {};
#pragma unroll
    for (int i = 0; i < kFewWaves; ++i) t += *reinterpret_cast<const floatx4*>(&red[i][m][c]);
    if (splits > 1) {
      *reinterpret_cast<floatx4*>(part + ((int64_t)sp * p.M + m) * p.row + n0 + c) = t;
    } else {
      float v[4] = {t[0], t[1], t[2], t[3]};
      finish4<T, true>(p, m, n0 + c, v);
    }
  }
}

// dz = dy act'(z) (left out where act is none: dz is dy) and the column sums of
// kDzRows rows each: 256 columns a workgroup, 8 a thread, all its rows' loads at
// once.  The bytes bound it (4095 x 4096, GELU, 101 MB: 23 us; with twice the rows a
// workgroup, half the wavefronts, 31).
constexpr int kDzRows = 32;
template <class T, bool VEC>
__global__ __launch_bounds__(256) void k_linear_dz(const LinearArgs a, uint16_t* dz, int64_t dz_stride,
                                                   float* part) {
  __shared__ float red[8][256];
  const int tiles_n = (a.N + 255) / 256;
  const int n = (blockIdx.x % tiles_n) * 256 + 8 * (threadIdx.x % 32);
  const int rb = blockIdx.x / tiles_n, grp = threadIdx.x / 32, cnt = min(a.N - n, 8);
  float sum[8] = {};
  uint4 w[4], u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = rb * kDzRows + 8 * i + grp, here = m < a.M ? cnt : 0;
    w[i] = load8<VEC>((const uint16_t*)a.dy + m * a.dys + n, here);
    if (a.act != kNone) u[i] = load8<VEC>((const uint16_t*)a.z + m * a.zs + n, here);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int m = rb * kDzRows + 8 * i + grp, here = m < a.M ? cnt : 0;
    float g[8] = {T::lo(w[i].x), T::hi(w[i].x), T::lo(w[i].y), T::hi(w[i].y),
                  T::lo(w[i].z), T::hi(w[i].z), T::lo(w[i].w), T::hi(w[i].w)};
    if (a.act != kNone) {
      const float z[8] = {T::lo(u[i].x), T::hi(u[i].x), T::lo(u[i].y), T::hi(u[i].y),
                          T::lo(u[i].z), T::hi(u[i].z), T::lo(u[i].w), T::hi(u[i].w)};
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] *= act_slope(a.act, z[j]);
      const uint4 o = make_uint4(T::pack(g[0], g[1]), T::pack(g[2], g[3]), T::pack(g[4], g[5]), T::pack(g[6], g[7]));
      // dz's own rows are of whole chunks; past N they are zeros, as g is
      if (here > 0) *reinterpret_cast<uint4*>(dz + m * dz_stride + n) = o;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) sum[j] += j < here ? g[j] : 0.0f;
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

// db: the row blocks' sums added up in order, 16 columns a workgroup, 16 rows at a time.
template <class T>
__global__ __launch_bounds__(256) void k_linear_db(const float* part, int blocks, int N, typename T::E* db) {
  __shared__ float red[16][17];
  const int c = blockIdx.x * 16 + threadIdx.x % 16, r = threadIdx.x / 16;
  float t = 0.0f;
  if (c < N)
#pragma unroll 4
    for (int i = r; i < blocks; i += 16) t += part[(int64_t)i * N + c];
  red[r][threadIdx.x % 16] = t;
  __syncthreads();
  if (r != 0 || c >= N) return;
  t = 0.0f;
  for (int i = 0; i < 16; ++i) t += red[i][threadIdx.x];
  db[c] = (typename T::E)t;
}

// Rows of a matrix copied to rows of whole 16-byte chunks, zeros past their end.
__global__ __launch_bounds__(256) void k_lay_out(const uint16_t* p, int64_t stride, int64_t rows, int inner, uint16_t* out) {
  const int chunks = (inner + 7) / 8;
  const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t r = e / chunks;
  const int d = 8 * (int)(e - r * chunks);
  if (r < rows) *reinterpret_cast<uint4*>(out + 8 * e) = load8<false>(p + r * stride + d, min(inner - d, 8));
}

// A matrix with contiguous rows, as the aligned products read it: rows of whole
// chunks on 16 bytes that do not overlap.
struct Mat {
  const void* p;
  int64_t rows, stride;
  int inner;
};
int64_t chunked(int64_t n) { return (n + 7) / 8 * 8; }
bool aligned16(const void* p) { return (uintptr_t)p % 16 == 0; }
bool laid_out(const Mat& m) {
  return m.inner % 8 == 0 &&
         (m.rows <= 1 || (m.stride % 8 == 0 && m.stride >= m.inner && m.stride <= kMaxFastStride));
}
bool ready(const Mat& m) { return laid_out(m) && aligned16(m.p); }
int64_t copy_bytes(const Mat& m) { return m.rows * chunked(m.inner) * 2; }
// The matrix itself where it is ready, else its copy at ws, which moves on in any case.
Mat lay_out(const Mat& m, char*& ws, hipStream_t s) {
  Mat r = m;
  if (!ready(m) && m.rows > 0) {
    r.p = ws, r.stride = chunked(m.inner);
    const int64_t n = m.rows * (r.stride / 8);
    k_lay_out<<<(unsigned)((n + 255) / 256), 256, 0, s>>>((const uint16_t*)m.p, m.stride, m.rows, m.inner, (uint16_t*)ws);
  }
  ws += copy_bytes(m);
  return r;
}
// Whether a product whose operands' sizes or strides are not those of whole chunks
// is worth their copies: two launches and the operands' bytes against a product
// element by element (55 TFLOP/s on 6355 x 3389 x 5488, where the copies and
// their products take a training step at 720 TFLOP/s; the weights of few rows at a
// fraction of the memory's rate).  Training steps with copies and without: 641 x 287
// x 317 78 and 65 us, 1933 x 2123 x 82 87 and 112.
bool worth_copies(int64_t M, int64_t N, int64_t K) {
  return std::max(N, K) <= kMaxFastStride && (M * N * K >= 1 << 27 || K * N >= 1 << 21);
}

// How a product is run: which kernel, and into how many parts its contracted
// axis is cut.
enum Kind { kAny, kFew, kTile128, kTile256 };
struct Plan {
  Kind kind;
  int splits;
};

// Tiles of 256 x 256 read the least from LDS and memory, but there must be
// enough of them to go round the compute units; smaller products take 128 x 128
// tiles, two workgroups a compute unit, and where those are still too few, parts
// of the depth of at least 4 tiles each.
Plan plan_of(int M, int N, int K, bool fast, bool few) {
  auto over = [](int a, int b) { return ((int64_t)a + b - 1) / b; };
  if (!fast) {
    const int64_t tiles = std::max<int64_t>(1, over(M, 64) * over(N, 64));
    return {kAny, (int)std::max<int64_t>(1, std::min<int64_t>(2 * kCUs / tiles, over(K, 32) / 4))};
  }
  if (few && M <= 32) {
    const int64_t wgs = over(N, 64), most = over(K, 32) / (2 * kFewWaves);
    return {kFew, (int)std::max<int64_t>(1, std::min<int64_t>(kCUs / wgs, most))};
  }
  const int64_t big = over(M, 256) * over(N, 256);
  if (big >= 3 * kCUs / 4) return {kTile256, 1};
  const int64_t small = std::max<int64_t>(1, over(M, 128) * over(N, 128));  // M may be 0
  return {kTile128, (int)std::max<int64_t>(1, std::min<int64_t>(2 * kCUs / small, over(K, kBK) / 4))};
}
// Its parts' sums, whether the operands turn out to be aligned or not.
int64_t plan_bytes(int M, int N, int K, bool few) {
  const int parts = std::max(plan_of(M, N, K, true, few).splits, plan_of(M, N, K, false, few).splits);
  return parts > 1 ? parts * (int64_t)M * chunked(N) * 4 : 0;
}

template <class T, bool EPI, bool AK, bool BK>
void product(Product p, bool fast, float* part, hipStream_t s) {
  if (p.M == 0) return;
  const Plan pl = plan_of(p.M, p.N, p.K, fast, EPI);
  auto whole = [&](const void* q, int64_t stride) { return !q || (aligned16(q) && (p.M == 1 || stride % 8 == 0)); };
  p.row = (int)chunked(p.N);
  p.vec = p.N % 8 == 0 && whole(p.c, p.cs) && whole(p.z, p.zs) && whole(p.res, p.rs) && p.rs <= kMaxFastStride && aligned16(p.bias);
  auto tiles = [&](int a, int b) { return (unsigned)(((int64_t)p.M + a - 1) / a * (((int64_t)p.N + b - 1) / b)); };
  switch (pl.kind) {
    case kAny:
      k_product_any<T, EPI, AK, BK><<<tiles(64, 64) * pl.splits, 256, 0, s>>>(p, pl.splits, part);
      break;
    case kFew:
      if constexpr (EPI) {
        const unsigned n = (p.N + 63) / 64 * pl.splits;
        if (p.M <= 16)
          k_product_few<T, 1><<<n, kFewWaves * 64, 0, s>>>(p, pl.splits, part);
        else
          k_product_few<T, 2><<<n, kFewWaves * 64, 0, s>>>(p, pl.splits, part);
      }
      break;
    case kTile128:
      k_product<T, EPI, AK, BK, 128, 128, 2><<<tiles(128, 128) * pl.splits, 256, 0, s>>>(p, pl.splits, part);
      break;
    case kTile256:
      k_product<T, EPI, AK, BK, 256, 256, 4><<<tiles(256, 256), 512, 0, s>>>(p, 1, part);
      break;
  }
  if (pl.splits > 1)
    k_product_join<T, EPI><<<(unsigned)(((int64_t)p.M * p.row / 4 + 255) / 256), 256, 0, s>>>(p, pl.splits, part);
}

// (The stride of a single row is not what the caller's may be.)
Mat mat(const void* p, int64_t rows, int64_t stride, int inner) { return {p, rows, rows <= 1 ? chunked(inner) : stride, inner}; }
Mat x_of(const LinearArgs& a) { return mat(a.x, a.M, a.xs, a.K); }
Mat w_of(const LinearArgs& a) { return mat(a.w, a.K, a.ws, a.N); }
Mat dy_of(const LinearArgs& a) { return mat(a.dy, a.M, a.dys, a.N); }

// dz, where it is not dy itself: rows of whole chunks in the workspace.
int64_t dz_bytes(const LinearArgs& a) { return a.act == kNone ? 0 : (int64_t)a.M * chunked(a.N) * 2; }
int64_t db_bytes(const LinearArgs& a) { return (int64_t)((a.M + kDzRows - 1) / kDzRows) * chunked(a.N) * 4; }
// Whether the operands are copied, by their sizes and strides alone.
bool copies(const LinearArgs& a, bool backward) {
  if (!worth_copies(a.M, a.N, a.K)) return false;
  return !laid_out(x_of(a)) || !laid_out(w_of(a)) || (backward && a.act == kNone && !laid_out(dy_of(a)));
}

template <class T>
void forward(const LinearArgs& a, void* ws, hipStream_t s) {
  Mat x = x_of(a), w = w_of(a);
  char* at = (char*)ws;
  const bool copy = a.M && copies(a, false);
  if (copy) x = lay_out(x, at, s), w = lay_out(w, at, s);
  Product p = {};
  p.M = a.M, p.N = a.N, p.K = a.K;
  p.a = {x.p, x.stride, 1};
  p.b = {w.p, 1, w.stride};
  p.c = a.y, p.cs = a.ys;
  p.act = a.act, p.bias = a.bias, p.res = a.res, p.rs = a.rs, p.z = a.z, p.zs = a.zs;
  product<T, true, true, false>(p, copy || (ready(x) && ready(w)), (float*)at, s);
}

template <class T>
void backward(const LinearArgs& a, void* ws, hipStream_t s) {
  const int blocks = (a.M + kDzRows - 1) / kDzRows;
  char* at = (char*)ws;
  Mat x = x_of(a), w = w_of(a), dz = dy_of(a);
  if (a.act != kNone) dz.p = at, dz.stride = chunked(a.N);
  at += dz_bytes(a);
  float* part = a.db ? (float*)at : nullptr;
  at += db_bytes(a);
  if (blocks && (a.act != kNone || a.db)) {
    const int64_t n = (int64_t)blocks * ((a.N + 255) / 256);
    auto whole = [&](const void* q, int64_t stride) { return aligned16(q) && (a.M == 1 || stride % 8 == 0); };
    if (a.N % 8 == 0 && whole(a.dy, a.dys) && (a.act == kNone || whole(a.z, a.zs)))
      k_linear_dz<T, true><<<(unsigned)n, 256, 0, s>>>(a, (uint16_t*)dz.p, dz.stride, part);
    else
      k_linear_dz<T, false><<<(unsigned)n, 256, 0, s>>>(a, (uint16_t*)dz.p, dz.stride, part);
  }
  if (a.db) k_linear_db<T><<<(a.N + 15) / 16, 256, 0, s>>>(part, blocks, a.N, (typename T::E*)a.db);
  // dz of the workspace is ready whatever N: past its end a row holds zeros
  const bool copy = a.M && copies(a, true);
  bool dz_ready = a.act != kNone ? dz.stride <= kMaxFastStride : ready(dz);
  if (copy) {
    if (a.dw)
      x = lay_out(x, at, s);
    else
      at += copy_bytes(x);
    if (a.dx)
      w = lay_out(w, at, s);
    else
      at += copy_bytes(w);
    if (a.act == kNone) dz = lay_out(dz, at, s), dz_ready = true;
  }
  if (a.dx) {  // [M][K], over N
    Product p = {};
    p.M = a.M, p.N = a.K, p.K = a.N;
    p.a = {dz.p, dz.stride, 1};
    p.b = {w.p, w.stride, 1};
    p.c = a.dx, p.cs = a.dxs;
    product<T, false, true, true>(p, dz_ready && (copy || ready(w)), (float*)at, s);
  }
  if (a.dw) {  // [K][N], over M
    Product p = {};
    p.M = a.K, p.N = a.N, p.K = a.M;
    p.a = {x.p, 1, x.stride};
    p.b = {dz.p, 1, dz.stride};
    p.c = a.dw, p.cs = a.dws;
    // the rows past a single one are beyond the descriptor's bound only while their
    // 32-bit offsets do not come round
    const bool near = std::max(x.stride, dz.stride) <= kMaxFastStride;
    product<T, false, false, false>(p, near && dz_ready && (copy || ready(x)), (float*)at, s);
  }
}

}  // namespace

// The workspace follows from sizes and strides alone, whatever the pointers' alignment.
int64_t linear_fwd_bytes(const LinearArgs& a) {
  return (copies(a, false) ? copy_bytes(x_of(a)) + copy_bytes(w_of(a)) : 0) +
         plan_bytes(a.M, a.N, a.K, true);
}

hipError_t launch_linear_fwd(const LinearArgs& a, void* ws, hipStream_t s) {
  a.dtype == kF16 ? forward<F16>(a, ws, s) : forward<BF16>(a, ws, s);
  return hipGetLastError();
}

int64_t linear_bwd_bytes(const LinearArgs& a) {
  const int64_t copied = copies(a, true) ? copy_bytes(x_of(a)) + copy_bytes(w_of(a)) + (a.act == kNone ? copy_bytes(dy_of(a)) : 0) : 0;
  return dz_bytes(a) + db_bytes(a) + copied + std::max(plan_bytes(a.M, a.K, a.N, false), plan_bytes(a.K, a.N, a.M, false));
}

hipError_t launch_linear_bwd(const LinearArgs& a, void* ws, hipStream_t s) {
  a.dtype == kF16 ? backward<F16>(a, ws, s) : backward<BF16>(a, ws, s);
  return hipGetLastError();
}

}  // namespace pnerf
