// Cross attention, forward: o_i = sum_j exp(a_ij - lse_i) v_j over the allowed
// keys j, a_ij = scale q_i . k_j, for queries and keys of different lengths.
//
// The query heads that share a kv head are rows of one product: row r of kv head
// g is query row r / G, head g G + r % G.  A wavefront holds 32 rows and passes
// over tiles of 64 keys with the running maximum m and sum l of each row's
// softmax:
//   S^T = K Q^T     (A = keys from LDS, B = the rows' queries, in registers)
//   P = exp2(c S - m), l += sum P
//   O^T += V^T P^T  (A = values by transposed LDS reads, B = P)
// Both products have the row as their column, so that all of a row's scores are
// in two lanes (l and l + 32): the softmax needs one exchange a tile, and P is
// the second product's B operand as it stands -- lane half h holds keys
// 8 i + 4 h + 0..3, an order of the contraction that the value reads follow.
//
// Keys and values go from memory to LDS by loads that write LDS themselves.  A
// key that may not be read (past its length, masked) and the elements past the
// head's width are zeros there: its lanes take an offset beyond the descriptor's
// bound, so that what such a place holds never enters a product.
#define PNERF_LAYERS_DEVICE
#include <algorithm>

#include "attention_rows.h"

namespace pnerf {
namespace {

// Many rows: four wavefronts of 32 rows share the tiles, two of them in LDS: the
// loads of the next run while the products of one do.  One barrier a tile.
// KS = 2: two such groups with the same rows take the tiles in turn, each with its
// own LDS, and join at the end: where workgroups are few (two_groups) that puts a
// second wavefront on every SIMD (1024 rows, 1200 keys, 2 x 16 heads of 64, one
// workgroup a CU: 33 us with one group, 22 with two; 2048 rows, 4096 keys, 16 heads
// of 128: 0.84 PFLOP/s with two, 0.54 with one on 17 heads).
template <class T, int DP, int KS>
__global__ __launch_bounds__(256 * KS, 3 - KS) void k_attn_fwd(const AttnArgs a, const Order order) {
  using Tile = RowTile<DP, 4>;
  __shared__ uint4 lds[KS][2][2 * Tile::kPieces];  // keys, then values
  const int lane = threadIdx.x & 63, all_waves = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int wave = all_waves & 3, grp = all_waves >> 2;
  const Place at(a, order, 128, wave * 32 + (lane & 31));
  const Tile kt(a.k, at.b * a.ks[0] + at.g * a.ks[2], a.ks[1], a.D, wave, lane);
  const Tile vt(a.v, at.b * a.vs[0] + at.g * a.vs[2], a.vs[1], a.D, wave, lane);
  Rows<T, DP> x;
  x.template init<true>(at.q, at.ok, a.D, h);
  const uint32_t to[2] = {lds_address(lds[grp][0]), lds_address(lds[grp][1])};
  auto load = [&](int buf, int t, uint64_t vm) {
    kt.load(to[buf], t, at.nk, vm, lane);
    vt.load(to[buf] + 16 * Tile::kPieces, t, at.nk, vm, lane);
  };
  uint64_t vm = 0, vm_next = 0;
  bool allowed = false;  // key `lane` of the tile after the next
  int t = at.t0 + grp;
  if (t < at.t1) {
    vm_next = __ballot(at.allowed(t * kBN + lane));
    load(0, t, vm_next);
    allowed = at.allowed((t + KS) * kBN + lane);
  }
  const int rounds = (at.t1 - at.t0 + KS - 1) / KS;  // the same for both groups: they share the barrier
  int round = 0;
  x.run(
      a.c, lane,
      [&] {
        if (round == rounds) return false;
        const int buf = round & 1;
        wait_loads();
        __builtin_amdgcn_s_barrier();  // this tile is there, and the one before has been read
        vm = vm_next;
        vm_next = __ballot(allowed);
        const bool here = t < at.t1;  // the last round may have no tile for the second group
        t += KS;
        if (t < at.t1) {
          load(buf ^ 1, t, vm_next);
          allowed = at.allowed((t + KS) * kBN + lane);
        }
        if (!here) return false;
        x.scores(lds[grp][buf], vm, a.c, lane);
        ++round;
        return true;
      },
      [&] { return lds[grp][(round - 1) & 1] + Tile::kPieces; });
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

// At most 32 rows of a kv head (single tokens): the bytes of the states are the
// time.  Four wavefronts with the same rows take the tiles in turn, each with its
// own keys and values in LDS and no barrier; keys are loaded again as soon as the
// scores are there, values as soon as they have been used.  At the end the
// wavefronts' sums meet in LDS.
template <class T, int DP>
__global__ __launch_bounds__(256) void k_attn_few(const AttnArgs a, const Order order) {
  using Tile = RowTile<DP, 1>;
  __shared__ uint4 lds[4][2 * Tile::kPieces];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const Place at(a, order, 32, lane & 31);
  const Tile kt(a.k, at.b * a.ks[0] + at.g * a.ks[2], a.ks[1], a.D, 0, lane);
  const Tile vt(a.v, at.b * a.vs[0] + at.g * a.vs[2], a.vs[1], a.D, 0, lane);
  Rows<T, DP> x;
  x.template init<true>(at.q, at.ok, a.D, h);
  uint4 *sk = lds[wave], *sv = sk + Tile::kPieces;
  const uint32_t to_k = lds_address(sk), to_v = lds_address(sv);
  int t = at.t0 + wave;    // of the next scores
  uint64_t vm_next = 0;    // its keys that may be read
  bool allowed = false, first = true;
  if (t < at.t1) {
    vm_next = __ballot(at.allowed(t * kBN + lane));
    kt.load(to_k, t, at.nk, vm_next, lane);
    vt.load(to_v, t, at.nk, vm_next, lane);
    allowed = at.allowed((t + 4) * kBN + lane);
  }
  x.run(
      a.c, lane,
      [&] {
        if (!first) {
          wait_reads();  // the values before have been used
          if (t < at.t1) vt.load(to_v, t, at.nk, vm_next, lane);
        }
        if (t >= at.t1) return false;
        first = false;
        wait_loads();
        const uint64_t vm = vm_next;
        vm_next = __ballot(allowed);
        x.scores(sk, vm, a.c, lane);
        wait_reads();
        t += 4;
        if (t < at.t1) {
          kt.load(to_k, t, at.nk, vm_next, lane);
          allowed = at.allowed((t + 4) * kBN + lane);
        }
        return true;
      },
      [&] { return sv; });

  static_assert(kFewLds<DP> <= sizeof(lds), "the sums fit the tiles' LDS");
  finish_few<T, DP>(a, at, x, lds, wave, lane, h);
}

// Any strides, alignment and head width: as k_attn_fwd, the tiles by way of
// registers, element by element.
template <class T, int DP>
__global__ __launch_bounds__(256) void k_attn_any(const AttnArgs a, const Order order) {
  __shared__ uint4 sk[kBN * DP / 8], sv[kBN * DP / 8];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
  const Place at(a, order, 128, wave * 32 + (lane & 31));
  Rows<T, DP> x;
  x.template init<false>(at.q, at.ok, a.D, h);
  int t = at.t0;
  x.run(
      a.c, lane,
      [&] {
        if (t >= at.t1) return false;
        const uint64_t vm = __ballot(at.allowed(t * kBN + lane));
        __syncthreads();
        copy_tile<DP>(sk, a.k, a.ks, at.b, at.g, a.D, t, vm);
        copy_tile<DP>(sv, a.v, a.vs, at.b, at.g, a.D, t, vm);
        __syncthreads();
        x.scores(sk, vm, a.c, lane);
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
  if (!fast_loads(a))
    k_attn_any<T, DP><<<n, 256, 0, s>>>(a, o);
  else if (few)
    k_attn_few<T, DP><<<n, 256, 0, s>>>(a, o);
  else if (two_groups(n, a))
    k_attn_fwd<T, DP, 2><<<n, 512, 0, s>>>(a, o);
  else
    k_attn_fwd<T, DP, 1><<<n, 256, 0, s>>>(a, o);
  join<T, DP>(a, s);
}

}  // namespace

// Few workgroups leave compute units idle: where there are not enough for half of
// them, the keys are cut into parts, of at least 4 tiles (16 for few rows, where
// 4 wavefronts share a part) each.
int attn_fwd_splits(const AttnArgs& a) {
  const bool few = a.M <= 32;
  const int rows = few ? 32 : 128;
  const int64_t wgs = (int64_t)((a.M + rows - 1) / rows) * a.Hkv * a.B;
  const int64_t tiles = (a.Sk + kBN - 1) / kBN;
  if (wgs == 0) return 1;
  return (int)std::max<int64_t>(1, std::min(kCUs / wgs, tiles / (few ? 16 : 4)));
}

int64_t attn_fwd_bytes(const AttnArgs& a) {
  if (a.splits <= 1) return 0;
  return (int64_t)a.splits * a.B * a.Hkv * a.M * (padded(a.D) + 2) * 4;
}

hipError_t launch_attn_fwd(const AttnArgs& a0, void* ws, hipStream_t s) {
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
