// What the attention kernels share: tiles of keys and values in LDS, fragments,
// results.
#pragma once
#include "layers_internal.h"

namespace pnerf {

constexpr int kBN = 64;                          // keys of a tile
constexpr int64_t kMaxTileStride = 1 << 22;      // elements: a tile's offsets stay below 2^31 bytes

inline int padded(int D) { return D <= 64 ? 64 : 128; }  // head width in the kernels
// Whether tiles can go to LDS by 16-byte loads with 32-bit offsets.
inline bool fast_loads(const AttnArgs& a) {
  return a.vec && a.ks[1] <= kMaxTileStride && a.vs[1] <= kMaxTileStride;
}
// Which workgroup takes which tile of rows (or keys), part, kv head and batch
// entry.  The tiles of one kv head read the same keys and values, so they go to
// one XCD; but batch entries may be of very different lengths, so every XCD takes
// its share of each: the order is kv head, chunk of its tiles, batch entry, part,
// tile, with as many chunks of tiles as make kv heads times chunks a multiple of
// the XCDs.  (With batch entries outermost, two of lengths 4 to 1 left half the
// XCDs idle most of the time.)  Single tiles share nothing and go round the XCDs.
struct Order {
  int tiles, chunks, per;  // per: tiles of a chunk
};
inline Order order_of(int64_t tiles, int Hkv) {
  int gcd = kXCDs;
  while (Hkv % gcd) gcd /= 2;
  const int chunks = (int)(tiles < kXCDs / gcd ? tiles : kXCDs / gcd);
  return {(int)tiles, chunks, (int)((tiles + chunks - 1) / chunks)};
}
inline int64_t workgroups(const Order& o, int splits, const AttnArgs& a) {
  return (int64_t)o.chunks * o.per * splits * a.Hkv * a.B;
}

// Whether two groups of wavefronts share a workgroup's rows (KS = 2): where the
// workgroups are fewer than the chip holds of that kind -- by registers two a
// compute unit at the narrow head, one at the wide one.  257 to 512 wide ones of
// equal length run better as single groups, two a compute unit (2048 rows and 4096
// keys, bf16, 17 / 24 / 32 heads: single 136 / 147 / 158 us and dq 182 / 197 / 212,
// two groups 147 / 153 / 164 and 203 / 213 / 226).  Where lengths are given they mostly
// differ, and a compute unit left with one long workgroup needs its second group
// (16 heads, rows and keys 2011 x 2500 and 502 x 625: 88 us against 95 and dq 108
// against 118; 2011 x 625 and 502 x 2500: 65 against 89 and 79 against 110).  The host
// does not see the lengths: given but equal ones pay the first line's difference.
inline bool two_groups(int64_t workgroups, const AttnArgs& a) {
  const bool two = padded(a.D) == 64 || a.q_len || a.kv_len;
  return workgroups <= (two ? 2 : 1) * kCUs && a.Sk > 2 * kBN;
}

#if defined(__HIP_DEVICE_COMPILE__) || defined(PNERF_LAYERS_DEVICE)
// The bits of row r that are xored into the position of its 16-byte chunks: 8
// rows at one chunk (the 16-byte reads) and 4 rows at two adjacent chunks (the
// transposed reads) each cover all the banks.
__device__ __forceinline__ int swz_bits(int r) { return ((r & 3) << 1) | ((r >> 2) & 1); }
// Position of chunk c of row r in a tile of CH chunks a row.
template <int CH>
__device__ __forceinline__ int swz(int r, int c) {
  return r * CH + (c ^ swz_bits(r));
}

struct Item {
  int tile, sp, g, b;  // tile may be past the last one: nothing to do
  __device__ __forceinline__ Item(const Order& o, int splits, int Hkv, int B) {
    if (o.tiles == 1) {
      int id = blockIdx.x;
      tile = 0, sp = id % splits;
      id /= splits;
      g = id % Hkv, b = id / Hkv;
      return;
    }
    int id = xcd_order(blockIdx.x, gridDim.x);
    const int t = id % o.per;
    id /= o.per;
    sp = id % splits;
    id /= splits;
    b = id % B;
    id /= B;
    tile = id % o.chunks * o.per + t;
    if (t >= o.per || tile >= o.tiles) tile = o.tiles;
    g = id / o.chunks;
  }
};

__device__ __forceinline__ int clamp_len(const int32_t* len, int b, int most) {
  return len ? min(max(len[b], 0), most) : most;
}
// Waits: for all loads (into LDS and registers) and LDS accesses; for LDS accesses.
// By the builtin, which the compiler takes into account: after a wait that it does
// not know it would wait again for its own earlier loads, at their first use, and
// with them for the loads into LDS that were issued since.
__device__ __forceinline__ void wait_loads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void wait_reads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
  asm volatile("" ::: "memory");
}

// The loads of tiles of N rows (keys, values, or the query rows of one head) into
// LDS, by NW wavefronts.
template <int DP, int NW, int N = kBN>
struct RowTile {
  static constexpr int kPieces = N * DP / 8;         // 16-byte chunks of a tile
  static constexpr int kLoads = kPieces / 64 / NW;   // of a wavefront
  static constexpr int kRows = 64 / (DP / 8);        // rows of one load
  static constexpr int kKinds = NW == 1 && kRows == 4 ? 2 : 1;  // see swz_bits: odd loads' rows differ in bit 2
  const char* base;
  int64_t row_bytes;
  int wave, D;
  uint32_t off[kKinds];  // this lane's chunk of the tile's first load (of each kind)
  __device__ __forceinline__ RowTile(const void* p, int64_t first, int64_t stride, int D_, int wave_, int lane)
      : base((const char*)p + 2 * first), row_bytes(2 * stride), wave(wave_), D(D_) {
#pragma unroll
    for (int i = 0; i < kKinds; ++i) {
      const int r = wave * kRows + lane / (DP / 8), c = (lane % (DP / 8)) ^ swz_bits(r + i * kRows);
      off[i] = 8 * c < D ? (uint32_t)r * (uint32_t)row_bytes + 16 * c : kOutside;
    }
  }
  // Tile t of n_rows rows to LDS at lds.  on: its rows that may be read; a row past
  // the last is beyond the descriptor's bound only where rows do not overlap.
  __device__ __forceinline__ void load(uint32_t lds, int t, int n_rows, uint64_t on, int lane) const {
    const u32x4 desc = descriptor(base + (int64_t)t * N * row_bytes,
                                  (int64_t)(n_rows - t * N - 1) * row_bytes + 2 * D);
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds + wave * 1024);
    const uint32_t step = NW * kRows * (uint32_t)row_bytes;
    if (on == ~0ull) {
#pragma unroll
      for (int n = 0; n < kLoads; ++n) load_to_lds(to + n * NW * 1024, off[n % kKinds] + n * step, desc);
    } else {
      uint64_t mine = on >> (wave * kRows + lane / (DP / 8));
#pragma unroll
      for (int n = 0; n < kLoads; ++n, mine >>= NW * kRows) {
        const uint32_t o = off[n % kKinds] + n * step;
        load_to_lds(to + n * NW * 1024, mine & 1 ? o : kOutside, desc);
      }
    }
  }
};

// A tile by way of registers, element by element, 256 threads.
template <int DP>
__device__ __forceinline__ void copy_tile(uint4* lds, const void* p, const int64_t s[3], int b, int g, int D,
                                          int t, uint64_t vm) {
  constexpr int CH = DP / 8;
  const uint16_t* base = (const uint16_t*)p + b * s[0] + g * s[2];
  for (int e = threadIdx.x; e < kBN * CH; e += 256) {
    const int r = e / CH, d = 8 * (e % CH);
    const bool on = (vm >> r) & 1;
    lds[swz<CH>(r, e % CH)] = load8<false>(base + (int64_t)(t * kBN + r) * s[1] + d, on ? min(D - d, 8) : 0);
  }
}

// A operand of 32 columns x 16 rows, transposed from a tile in LDS: rows row0 +
// 4 h + 0..3 and + 8, columns col0 + lane % 32 (the order of a result's registers).
template <int CH>
__device__ __forceinline__ uint4 tr_frag(const uint4* tile, int row0, int col0, int lane) {
  const int l16 = lane & 15, r = row0 + 4 * (lane >> 5) + l16 / 4;
  const int col = col0 + 16 * ((lane >> 4) & 1) + 4 * (l16 % 4);
  const uint2 a = read_tr((const char*)(tile + swz<CH>(r, col / 8)) + 2 * (col % 8));
  const uint2 b = read_tr((const char*)(tile + swz<CH>(r + 8, col / 8)) + 2 * (col % 8));
  return make_uint4(a.x, a.y, b.x, b.y);
}

// Registers i .. i + 7 of a result as the B operand of 16 of its rows.
template <class T>
__device__ __forceinline__ uint4 pack8(const floatx16& p, int i) {
  return make_uint4(T::pack(p[i], p[i + 1]), T::pack(p[i + 2], p[i + 3]),
                    T::pack(p[i + 4], p[i + 5]), T::pack(p[i + 6], p[i + 7]));
}

// A lane's column of a transposed result to memory: 16-bit elements times f, or
// 32-bit partial sums.
template <class T, int DP, bool VEC>
__device__ __forceinline__ void store_cols(const floatx16* acc, uint16_t* p, float f, int D, int h) {
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int col = 32 * d + 8 * i + 4 * h;
      const floatx16& x = acc[d];
      store4<VEC>(p + col, make_uint2(T::pack(x[4 * i] * f, x[4 * i + 1] * f),
                                      T::pack(x[4 * i + 2] * f, x[4 * i + 3] * f)),
                  min(D - col, 4));
    }
}
template <int DP>
__device__ __forceinline__ void store_part(const floatx16* acc, float* p, int h, float f = 1.0f) {
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      *reinterpret_cast<floatx4*>(p + 32 * d + 8 * i + 4 * h) =
          floatx4{acc[d][4 * i], acc[d][4 * i + 1], acc[d][4 * i + 2], acc[d][4 * i + 3]} * f;
}

__device__ __forceinline__ float log_sum(float m, float l) {  // m in units of ln 2
  return l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}
#endif

}  // namespace pnerf
