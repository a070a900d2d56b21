// Cross attention over states held in 8 bits, forward (what attention.hip does, its
// softmax and its products): over the allowed keys j
//   a_ij = scale ks[j / 64] q_i . k8_j,  o_i = sum_j exp(a_ij - lse_i) vs[j / 64] v8_j
// with k8, v8 of e4m3 and one scale for each block of 64 rows of a head, which is a
// tile here.  Every e4m3 number is a float16 and a bfloat16 number: tiles are widened on
// their way to LDS, or from it, and the products are those of 16 bits, exact in what they
// multiply.  A tile's key scale is a factor of its scores.  Its value scale is one of p, in
// the exponent that makes it, as far as the 16 bits of p hold it; for scales that lie
// further apart the sums change their unit, where the maximum's rescaling stands (see
// ScaledRows).
#define PNERF_LAYERS_DEVICE
#include <algorithm>
#include <type_traits>

#include "attention_rows.h"

namespace pnerf {
namespace {

// The batch entry whose length is the rank-th longest of its 64 (in every lane; equal
// ones in order).
__device__ __forceinline__ int by_length(const AttnArgs& a, int rank) {
  const int first = rank & ~63, n = min(a.B - first, 64), lane = threadIdx.x & 63;
  const int mine = lane < n ? clamp_len(a.kv_len, first + lane, a.Sk) : -1;
  int before = 0;
  for (int i = 0; i < n; ++i) {
    const int other = __builtin_amdgcn_readlane(mine, i);
    before += other > mine || (other == mine && i < lane);
  }
  return first + __builtin_ctzll(__ballot(lane < n && before == (rank & 63)));
}

// The workgroup's item.  Where batch entries differ in length and the chip does not hold
// all workgroups at once, the longest go first: one that starts late would leave the
// others waiting for it.  Each XCD then goes through the entries with all of its heads.
__device__ __forceinline__ Item item_of(const AttnArgs& a, const Order& o) {
  Item item(o, a.splits, a.Hkv, a.B);
  const int heads = a.Hkv * o.chunks / kXCDs;  // and chunks of an XCD
  if (!a.sorted) return item;
  if (o.tiles > 1 && a.Hkv * o.chunks % kXCDs == 0) {
    int id = blockIdx.x / kXCDs;
    const int t = id % o.per;
    id /= o.per;
    item.sp = id % a.splits;
    id /= a.splits;
    const int hc = blockIdx.x % kXCDs * heads + id % heads;
    item.b = id / heads;
    item.g = hc / o.chunks;
    item.tile = min(t * o.chunks + hc % o.chunks, o.tiles);  // in turn: short entries fill no chunk first
  }
  item.b = by_length(a, item.b);
  return item;
}

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

// Transposed read of bytes: within each 16 lanes, lane 2 r + c gives the address of row
// r, bytes 8c .. 8c + 7; lane i receives byte i of rows 0 .. 7.
__device__ __forceinline__ uint2 read_tr8(const char* lds) {
  typedef int i32x2 __attribute__((ext_vector_type(2)));
  const i32x2 t = __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2*)lds);
  return __builtin_bit_cast(uint2, t);
}

// Tiles of bytes in LDS: where 16-byte chunk c of row r is.  The chunks' positions are
// xored with bits of the row such that both reads cover all banks: 16 rows at one chunk
// (keys: a lane's 16 bytes are its share of two products), and 8 rows, 0..3 and 8..11,
// at two adjacent ones (values, transposed).
template <int DP>
__device__ __forceinline__ int bytes_bits(int r) {
  const int b1 = (r >> 1) & 1, b2 = (r >> 2) & 1, b3 = (r >> 3) & 1;
  return DP == 128 ? b2 | b1 << 1 | b3 << 2 : b2 | b3 << 1;
}
template <int DP>
__device__ __forceinline__ int bytes_swz(int r, int c) {
  return r * DP + 16 * (c ^ bytes_bits<DP>(r));
}

// The scales of 64 tiles at a time, a lane each: a load for each tile would have to be
// waited for, and with it the tiles that are on their way.
struct Scales {
  const float *k, *v;
  int64_t k_step, v_step;
  int last, first;  // the states' last tile; the first one held
  float ks, vs;
  __device__ __forceinline__ Scales(const AttnArgs& a, int b, int g)
      : k(a.k_scale + b * a.kss[0] + g), v(a.v_scale + b * a.vss[0] + g), k_step(a.kss[1]), v_step(a.vss[1]),
        last((a.Sk - 1) / kBN), first(-64), ks(1.0f), vs(1.0f) {}
  // Tiles are asked for in rising order, the same one in all lanes.
  __device__ __forceinline__ void of(int t, float& k_scale, float& v_scale) {
    if (t >= first + 64) {
      first = t;
      const int mine = min(t + (int)(threadIdx.x & 63), last);
      ks = k[mine * k_step], vs = v[mine * v_step];
    }
    k_scale = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(ks), t - first));
    v_scale = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(vs), t - first));
  }
};

// Rows whose tiles have scales: c of the scores, and the value scale, whose ratio to 2^e,
// the unit in which a row's sums are kept, is a factor of p, by way of its exponent.  p's
// data type has to hold that: in float16 ratios from 1 to 2^7 (p is at most 2^8, and what
// it loses below 2^-14 must not grow), in bfloat16, which has float32's range, from 2^-60
// to 2^60.  For a tile outside, the unit follows the scale and the sums are rescaled, as
// far as they stay numbers that count: scales may be any positive normal ones.
template <class T, int DP>
struct ScaledRows : Rows<T, DP> {
  static constexpr bool kNarrow = std::is_same<T, F16>::value;
  static constexpr float kLeast = kNarrow ? 0.0f : -60.0f, kMost = kNarrow ? 7.0f : 60.0f;
  static constexpr float kStart = kNarrow ? 3.0f : 0.0f;  // log2 of the ratio that a new unit begins with
  float c, e;
  float vk, vl;  // log2 of the tile's value scale: its whole part, the rest
  bool bad;      // the query holds an infinity or NaN

  __device__ __forceinline__ void begin(const AttnArgs& a) { c = a.c, e = 1e4f, vk = vl = 0.0f; }
  // A query with an infinity or NaN is taken as zeros: with it, the zeros that stand for
  // keys that may not be read would give NaN.  Its row's sum becomes NaN in the end if there
  // is an allowed key.  (To be called when other loads are on their way, too: it waits for
  // the queries.)
  __device__ __forceinline__ void clean() {
    // an exponent of ones carries into its number's sign bit
    constexpr uint32_t kExp = kNarrow ? 0x7C007C00u : 0x7F807F80u, kOne = kNarrow ? 0x04000400u : 0x00800080u;
    uint32_t carry = 0;
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) {
      const uint4 w = this->qf[i];
      carry |= ((w.x & kExp) + kOne) | ((w.y & kExp) + kOne) | ((w.z & kExp) + kOne) | ((w.w & kExp) + kOne);
    }
    const uint64_t here = __ballot((carry & 0x80008000u) != 0);  // a row is in lanes r and r + 32
    const uint32_t rows = (uint32_t)here | (uint32_t)(here >> 32);
    bad = rows >> (threadIdx.x & 31) & 1;
    if (rows)
#pragma unroll
      for (int i = 0; i < DP / 16; ++i) this->qf[i] = bad ? make_uint4(0, 0, 0, 0) : this->qf[i];
  }
  // The scales of the next tile; one without an allowed key has none that count.
  __device__ __forceinline__ void scales(const AttnArgs& a, Scales& sc, int t, uint64_t vm) {
    if (!vm) return;
    float ks, vs;
    sc.of(t, ks, vs);
    c = fmaxf(a.c * ks, 0x1p-126f);  // (0 times a masked key's -inf would be NaN)
    const uint32_t bits = __float_as_uint(vs);
    vk = (float)((int)(bits >> 23) - 127);
    vl = __builtin_amdgcn_logf(__uint_as_float((bits & 0x7FFFFFu) | 0x3F800000u));
  }
  __device__ __forceinline__ bool outside() const {
    const float r = vl + (vk - e);
    return r < kLeast || r > kMost;
  }
  // log2 of the ratio.  It is less than kLeast only where sums of 2^100 make what the tile
  // adds nothing (see unit); p itself, of which l is the sum, stays a number.
  __device__ __forceinline__ float shift() const { return fmaxf(vl + (vk - e), -60.0f); }
  // The largest of a lane's sums.
  __device__ __forceinline__ float largest() const {
    float x = 0.0f;
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) x = fmaxf(x, fabsf(this->o[i][j]));
    return x;
  }
  // The sums times 2^n.
  __device__ __forceinline__ void move(int n) {
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) this->o[i][j] = __builtin_amdgcn_ldexpf(this->o[i][j], n);
  }
  // The unit to use from here on, given that the new maximum leaves 2^d of the sums.
  __device__ __forceinline__ float unit(float d) const {
    float to = outside() ? vk - kStart : e;
    if (!__any(to != e)) return to;
    // Down, as far as the row's largest sum stays below 2^101: beside it the tile, of less
    // than 2^50 in that unit, is nothing.  Up, as far as that sum stays above 2^-91, where
    // nothing is lost, or is nothing beside the tile, whose largest weight keeps 2^8 then.
    float most = -INFINITY, x, y;
#pragma unroll
    for (int i = 0; i < 32; ++i) most = fmaxf(most, this->s[i / 16][i % 16]);
    halves(largest(), x, y);
    const float at = ceilf(e + d + __builtin_amdgcn_logf(fmaxf(x, y)));  // -inf: nothing yet
    halves(most, x, y);
    const float weight = ceilf(c * fmaxf(x, y) - this->top + vk + vl);
    if (to < e) to = fmaxf(to, at - 100.0f);
    if (to > e && at > -INFINITY) to = fminf(to, fmaxf(at + 90.0f, weight - 8.0f));
    return to;
  }
  // Queries in the order in which byte tiles hold the head's width (see bytes_swz).
  __device__ __forceinline__ void init_bytes(const uint16_t* q, bool ok, int D, int h) {
    this->template init<true>(q, false, D, h);
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) {
      const int d = 32 * (i / 2) + 16 * h + 8 * (i % 2);
      this->qf[i] = load8<true>(q + d, ok ? min(D - d, 8) : 0);
    }
  }
  // What the scores of 32 keys start from: 0, and -inf at those that may not be read,
  // whose rows in LDS are zeros.  (A register holds two keys, one a half wavefront.)
  __device__ __forceinline__ static floatx16 start(uint32_t keys) {
    floatx16 s = {};
    if (keys != ~0u)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int k = 8 * (i / 4) + i % 4;
        const uint32_t lo = (int32_t)(keys << (31 - k)) >> 31, hi = (int32_t)(keys << (27 - k)) >> 31;
        s[i] = __builtin_amdgcn_inverse_ballot_w64((uint64_t)hi << 32 | lo) ? 0.0f : -INFINITY;
      }
    return s;
  }
  __device__ __forceinline__ void scores(const uint4* sk, uint64_t vm, int lane) {
    constexpr int CH = DP / 8;
    const int r = lane & 31, h = lane >> 5;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      this->s[n] = start((uint32_t)(vm >> (32 * n)));
#pragma unroll
      for (int i = 0; i < DP / 16; ++i)
        this->s[n] = T::mma(sk[swz<CH>(32 * n + r, 2 * i + h)], this->qf[i], this->s[n]);
    }
    this->raise(c);
  }
  // The scores' exponentials times the ratio, and their sum.
  __device__ __forceinline__ void weights() {
    const float sh = shift(), base = (this->m == -INFINITY ? 0.0f : this->m) - sh;  // -inf: no allowed key yet
    float sum = 0.0f;
#pragma unroll
    for (int n = 0; n < 2; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        this->s[n][i] = __builtin_amdgcn_exp2f(fmaf(this->s[n][i], c, -base));
        sum += this->s[n][i];
      }
    this->l = fmaf(sum, __builtin_amdgcn_exp2f(-sh), this->l);
  }
  // (Rounding them to the data type, as the matrix instructions take them, leaves an error
  // against 64 bits of 1.8e-3 in bfloat16 and 2.1e-4 in float16, where the result's own
  // rounding makes 1.6e-3 and 2.1e-4.)
  __device__ __forceinline__ void add(const uint4* sv, int lane) {
    weights();
#pragma unroll
    for (int n = 0; n < 4; ++n) {  // 16 keys each
      const uint4 pf = pack8<T>(this->s[n / 2], 8 * (n % 2));
#pragma unroll
      for (int d = 0; d < DP / 32; ++d)
        this->o[d] = T::mma(tr_frag<DP / 8>(sv, 16 * n, 32 * d, lane), pf, this->o[d]);
    }
  }
  // The same as scores and add, of tiles of bytes.
  __device__ __forceinline__ void scores_bytes(const char* sk, uint64_t vm, int lane) {
    const int r = lane & 31, h = lane >> 5;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      this->s[n] = start((uint32_t)(vm >> (32 * n)));
#pragma unroll
      for (int i = 0; i < DP / 32; ++i) {
        const uint4 k = *reinterpret_cast<const uint4*>(sk + bytes_swz<DP>(32 * n + r, 2 * i + h));
        this->s[n] = T::mma(widen8<T>(k.x, k.y), this->qf[2 * i], this->s[n]);
        this->s[n] = T::mma(widen8<T>(k.z, k.w), this->qf[2 * i + 1], this->s[n]);
      }
    }
    this->raise(c);
  }
  __device__ __forceinline__ void add_bytes(const char* sv, int lane) {
    weights();
    const int l16 = lane & 15, r = 4 * (lane >> 5) + l16 / 2 + (l16 & 8 ? 4 : 0);  // keys 4 h + 0..3 and + 8
#pragma unroll
    for (int n = 0; n < 4; ++n) {  // 16 keys each
      const uint4 pf = pack8<T>(this->s[n / 2], 8 * (n % 2));
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) {
        const uint2 v = read_tr8(sv + bytes_swz<DP>(16 * n + r, 2 * d + ((lane >> 4) & 1)) + 8 * (l16 & 1));
        this->o[d] = T::mma(widen8<T>(v.x, v.y), pf, this->o[d]);
      }
    }
  }
  template <class N, class V>
  __device__ __forceinline__ void run(N next, V add_tile) {
    bool more = next();
    while (more) {
      // to the new maximum and unit: l by the first, the sums by both
      const float d = this->m - (this->top == -INFINITY ? 0.0f : this->top), to = unit(d);
      const float alpha = __builtin_amdgcn_exp2f(d);
      this->m = this->top;
      this->l *= alpha;
#pragma unroll
      for (int i = 0; i < DP / 32; ++i) this->o[i] *= alpha;
      if (__any(to != e)) move((int)(e - to));  // (2^(e - to) alone may be no number)
      e = to;
      do {
        add_tile();
        more = next();
      } while (more && !this->grown() && !__any(outside()));
    }
    // Sums in the unit 1.  Where those would pass float32's range (the results, which l
    // divides them by, need not) they and l are 2^-n of what they were, and m, of which
    // they are multiples by exp2, is n more.
    int n = 0;
    if (__any(e > 16.0f)) {
      float x, y;
      halves(largest(), x, y);
      const bool far = (int)e + __builtin_amdgcn_frexp_expf(fmaxf(x, y)) > 100;
      halves(this->l, x, y);
      if (far) n = 16 + __builtin_amdgcn_frexp_expf(x + y);
      this->m += (float)n;
      this->l = __builtin_amdgcn_ldexpf(this->l, -n);
    }
    move((int)e - n);
    if (bad && this->l != 0.0f) this->l = __builtin_nanf("");
  }
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

// The loads of tiles of 64 rows of bytes into registers by NW wavefronts, and their way
// to LDS as 16-bit elements.  A lane takes 8 bytes, 16 when they are widened: 8
// neighbouring lanes then write 8 neighbouring chunks, which cover all banks.  (Of 16
// bytes a lane they would write every other chunk: half of all LDS cycles were conflicts.)
template <class T, int DP, int NW>
struct ByteTile {
  static constexpr int kChunks = DP / 8;                 // of a row
  static constexpr int kRows = 64 / kChunks * NW;        // of one load of all wavefronts
  static constexpr int kLoads = kBN / kRows;             // of a wavefront
  const char* base;
  int64_t row_bytes;
  int D, row, chunk;  // this lane's row of the first load, its chunk
  uint2 raw[kLoads];
  __device__ __forceinline__ ByteTile(const void* p, int64_t first, int64_t stride, int D_, int wave, int lane)
      : base((const char*)p + first), row_bytes(stride), D(D_), row(wave * (64 / kChunks) + lane / kChunks),
        chunk(lane % kChunks) {}
  // Tile t of n_rows rows.  on: its rows that may be read; the others, and what lies
  // past the head's width, are zeros (a row past the last is beyond the bound only
  // where rows do not overlap).
  __device__ __forceinline__ void load(int t, int n_rows, uint64_t on) {
    const u32x4 d = descriptor(base + (int64_t)t * kBN * row_bytes, (int64_t)(n_rows - t * kBN - 1) * row_bytes + D);
    const __amdgpu_buffer_rsrc_t desc = __builtin_amdgcn_make_buffer_rsrc(
        reinterpret_cast<void*>((uint64_t)d[1] << 32 | d[0]), 0, d[2], d[3]);
    const uint32_t off = 8 * chunk < D ? (uint32_t)row * (uint32_t)row_bytes + 8 * chunk : kOutside;
    const uint32_t step = kRows * (uint32_t)row_bytes;
    const uint64_t mine = on >> row;
#pragma unroll
    for (int n = 0; n < kLoads; ++n) {
      const uint32_t o = on == ~0ull || (mine >> (n * kRows) & 1) ? off + n * step : kOutside;
      raw[n] = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(desc, o, 0, 0));
    }
  }
  __device__ __forceinline__ void widen(uint4* lds) const {
#pragma unroll
    for (int n = 0; n < kLoads; ++n) lds[swz<DP / 8>(row + n * kRows, chunk)] = widen8<T>(raw[n].x, raw[n].y);
  }
};

// Many rows: four wavefronts of 32 rows share the tiles, two of them in LDS and the
// next in registers on its way there.  One barrier a tile.  KS = 2: as in k_attn_fwd.
// Matrix products, exponentials and LDS reads bound it, as with 16-bit states, and the
// widening on top: 13 vector instructions for each product of 32 cycles (2 x 4096 rows, 8192
// keys, 32 heads of 128 over 8, bf16: 1202 us or 0.91 PFLOP/s where 16-bit states take 1112; 5%
// of the keys masked: 1245 and 1240).  Tried and slower: the next tile widened beside the
// scores' products (spills), or by one group after them, and sums of unmasked tiles that
// start from the instruction's own zero.
template <class T, int DP, int KS>
__global__ __launch_bounds__(256 * KS, 3 - KS) void k_attn_q8_fwd(const AttnArgs a, const Order order) {
  using Tile = ByteTile<T, DP, 4>;
  constexpr int kPieces = kBN * DP / 8;
  __shared__ uint4 lds[KS][2][2 * kPieces];  // keys, then values
  const int lane = threadIdx.x & 63, all_waves = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int wave = all_waves & 3, grp = all_waves >> 2;
  const Place at(a, item_of(a, order), 128, wave * 32 + (lane & 31));
  Scales sc(a, at.b, at.g);
  Tile kt(a.k, at.b * a.ks[0] + at.g * a.ks[2], a.ks[1], a.D, wave, lane);
  Tile vt(a.v, at.b * a.vs[0] + at.g * a.vs[2], a.vs[1], a.D, wave, lane);
  ScaledRows<T, DP> x;
  x.template init<true>(at.q, at.ok, a.D, h);
  x.begin(a);
  uint64_t vm = 0, vm_next = 0;
  int t = at.t0 + grp;
  uint32_t mask = at.mask_at(t * kBN + lane);  // of key `lane` of the tile to be fetched next
  auto fetch = [&](int tile) {  // the tile after the one in LDS, if there is one
    if (tile >= at.t1) return;
    vm_next = at.allowed_of(mask, tile * kBN + lane);
    mask = at.mask_at((tile + KS) * kBN + lane);
    kt.load(tile, at.nk, vm_next);
    vt.load(tile, at.nk, vm_next);
  };
  auto put = [&](int buf) {
    kt.widen(lds[grp][buf]);
    vt.widen(lds[grp][buf] + kPieces);
    vm = vm_next;
  };
  fetch(t);
  if (t < at.t1) put(0);
  fetch(t + KS);
  x.clean();
  const int rounds = (at.t1 - at.t0 + KS - 1) / KS;  // the same for both groups: they share the barrier
  int round = 0;
  x.run(
      [&] {
        if (round == rounds) return false;
        const int buf = round & 1;
        wait_reads();
        __builtin_amdgcn_s_barrier();  // this tile is there, and the one before has been read
        const bool here = t < at.t1;  // the last round may have no tile for the second group
        const uint64_t on = vm;
        if (here) x.scales(a, sc, t, on);
        t += KS;
        if (t < at.t1) {
          put(buf ^ 1);
          fetch(t + KS);
        }
        if (!here) return false;
        x.scores(lds[grp][buf], on, lane);
        ++round;
        return true;
      },
      [&] { x.add(lds[grp][(round - 1) & 1] + kPieces, lane); });
  if constexpr (KS == 2) {
    static_assert(kGroupsLds<DP> <= sizeof(lds), "a group's sums fit LDS");
    if (!join_groups<T, DP>(x, lds, wave, grp, lane)) return;
  }
  x.close(at.ok);
  if (at.row >= a.M) return;
  if (a.splits > 1)
    x.store_partial(a, at.sp, ((int64_t)at.b * a.Hkv + at.g) * a.M + at.row, h, at.t0 < at.t1);
  else
    x.template store<true>(a, at.b, at.qi, at.head, h);
}

// The loads of tiles of 64 rows of bytes straight into LDS, by one wavefront.
template <int DP>
struct ByteRows {
  static constexpr int kChunks = DP / 16, kRows = 64 / kChunks, kLoads = kBN / kRows;
  static_assert(kRows % 8 == 0 && (DP == 64 ? kRows == 16 : true), "see off: rows of the other loads");
  const char* base;
  int64_t row_bytes;
  int D;
  uint32_t off[DP == 128 ? 2 : 1];  // this lane's chunk of the first load (of even and odd ones: bytes_bits)
  __device__ __forceinline__ ByteRows(const void* p, int64_t first, int64_t stride, int D_, int lane)
      : base((const char*)p + first), row_bytes(stride), D(D_) {
#pragma unroll
    for (int i = 0; i < (DP == 128 ? 2 : 1); ++i) {
      const int r = lane / kChunks, c = (lane % kChunks) ^ bytes_bits<DP>(r + i * kRows);
      off[i] = 16 * c < D ? (uint32_t)r * (uint32_t)row_bytes + 16 * c : kOutside;
    }
  }
  __device__ __forceinline__ void load(uint32_t lds, int t, int n_rows, uint64_t on, int lane) const {
    const u32x4 desc = descriptor(base + (int64_t)t * kBN * row_bytes, (int64_t)(n_rows - t * kBN - 1) * row_bytes + D);
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds), step = kRows * (uint32_t)row_bytes;
    const uint64_t mine = on >> (lane / kChunks);
#pragma unroll
    for (int n = 0; n < kLoads; ++n) {
      const uint32_t o = off[DP == 128 ? n % 2 : 0] + n * step;
      load_to_lds(to + n * 1024, on == ~0ull || (mine >> (n * kRows) & 1) ? o : kOutside, desc);
    }
  }
};

// At most 32 rows of a kv head (single tokens): the bytes of the states are the time.
// Eight wavefronts with the same rows take the tiles in turn, each with its own keys
// and values in LDS, as bytes, and no barrier; keys are loaded again as soon as the
// scores are there, values as soon as they have been used.  The bytes are widened on
// the way from LDS to the products: each is read once.  (One token over 131109 rows, 32
// heads of 128 over 8: 59 us or 4.6 TB/s and the join's 5; 64 ragged entries of up to 2500
// rows, 16 heads over 4: 26.7 us, 42 with four wavefronts and tiles widened through registers.)
template <class T, int DP>
__global__ __launch_bounds__(512) void k_attn_q8_few(const AttnArgs a, const Order order) {
  constexpr int kWaves = 8, kTile = kBN * DP;
  __shared__ uint4 lds[(kWaves * 2 * kTile > kFewLds<DP, kWaves> ? kWaves * 2 * kTile : kFewLds<DP, kWaves>) / 16];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const Place at(a, item_of(a, order), 32, lane & 31);
  Scales sc(a, at.b, at.g);
  const ByteRows<DP> kt(a.k, at.b * a.ks[0] + at.g * a.ks[2], a.ks[1], a.D, lane);
  const ByteRows<DP> vt(a.v, at.b * a.vs[0] + at.g * a.vs[2], a.vs[1], a.D, lane);
  ScaledRows<T, DP> x;
  x.init_bytes(at.q, at.ok, a.D, h);
  x.begin(a);
  const char *sk = (const char*)lds + wave * 2 * kTile, *sv = sk + kTile;
  const uint32_t to_k = lds_address(sk), to_v = lds_address(sv);
  int t = at.t0 + wave;    // of the next scores
  uint64_t vm_next = 0;    // its keys that may be read
  uint32_t mask = 1;
  bool first = true;
  if (t < at.t1) {
    vm_next = __ballot(at.allowed(t * kBN + lane));
    mask = at.mask_at((t + kWaves) * kBN + lane);
    kt.load(to_k, t, at.nk, vm_next, lane);
    vt.load(to_v, t, at.nk, vm_next, lane);
  }
  x.clean();
  x.run(
      [&] {
        if (!first) {
          wait_reads();  // the values before have been used
          if (t < at.t1) vt.load(to_v, t, at.nk, vm_next, lane);
        }
        if (t >= at.t1) return false;
        first = false;
        wait_loads();
        const uint64_t vm = vm_next;
        vm_next = at.allowed_of(mask, (t + kWaves) * kBN + lane);
        x.scales(a, sc, t, vm);
        x.scores_bytes(sk, vm, lane);
        wait_reads();
        t += kWaves;
        if (t < at.t1) {
          mask = at.mask_at((t + kWaves) * kBN + lane);
          kt.load(to_k, t, at.nk, vm_next, lane);
        }
        return true;
      },
      [&] { x.add_bytes(sv, lane); });
  finish_few<T, DP, kWaves>(a, at, x, lds, wave, lane, h);
}

// Any strides, alignment and head width.
template <class T, int DP>
__global__ __launch_bounds__(256, 2) void k_attn_q8_any(const AttnArgs a, const Order order) {
  __shared__ uint4 sk[kBN * DP / 8], sv[kBN * DP / 8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
  const Place at(a, item_of(a, order), 128, wave * 32 + (lane & 31));
  Scales sc(a, at.b, at.g);
  ScaledRows<T, DP> x;
  x.template init<false>(at.q, at.ok, a.D, h);
  x.begin(a);
  x.clean();
  int t = at.t0;
  x.run(
      [&] {
        if (t >= at.t1) return false;
        const uint64_t vm = __ballot(at.allowed(t * kBN + lane));
        __syncthreads();
        copy_tile8<T, DP>(sk, a.k, a.ks, at.b, at.g, a.D, t, vm);
        copy_tile8<T, DP>(sv, a.v, a.vs, at.b, at.g, a.D, t, vm);
        x.scales(a, sc, t, vm);
        __syncthreads();
        x.scores(sk, vm, lane);
        ++t;
        return true;
      },
      [&] { x.add(sv, lane); });
  x.close(at.ok);
  if (at.row >= a.M) return;
  if (a.splits > 1)
    x.store_partial(a, at.sp, ((int64_t)at.b * a.Hkv + at.g) * a.M + at.row, h, at.t0 < at.t1);
  else
    x.template store<false>(a, at.b, at.qi, at.head, h);
}

template <class T, int DP>
void launch(AttnArgs a, hipStream_t s) {
  const bool few = a.M <= 32;
  const int rows = few ? 32 : 128;
  const Order o = order_of(((int64_t)a.M + rows - 1) / rows, a.Hkv);
  const unsigned n = (unsigned)workgroups(o, a.splits, a);
  a.sorted = a.kv_len && a.B > 1 && n > kCUs;
  if (!fast_loads(a))
    k_attn_q8_any<T, DP><<<n, 256, 0, s>>>(a, o);
  else if (few)
    k_attn_q8_few<T, DP><<<n, 512, 0, s>>>(a, o);
  else if (two_groups(n, a))
    k_attn_q8_fwd<T, DP, 2><<<n, 512, 0, s>>>(a, o);
  else
    k_attn_q8_fwd<T, DP, 1><<<n, 256, 0, s>>>(a, o);
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
