// Attention of several new tokens per request over the cache and themselves
// (dsa_tree_attention), as templates over the cache's element type.
#pragma once

#include <type_traits>

#include "device.h"
#include "tree.h"

namespace dsa {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr float kTreeMin = -3.0e38f;  // "no score yet": finite, below every finite score in use
constexpr float kTreeSlack = 8.f;

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {  // nearest even
  const f32x2 x = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}

// High halves of two fp32 values as a bf16 pair (truncation).
__device__ __forceinline__ uint32_t high_halves(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}

// Bit 15 of the result: any of eight bf16 values is infinite or NaN (an exponent
// of ones carries into the bit above it).
__device__ __forceinline__ uint32_t nonfinite_bit(const uint4& x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t carry = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    carry |= ((w[i] & 0x7f80u) + 0x80u) | (((w[i] >> 16) & 0x7f80u) + 0x80u);
  return carry;
}

// K/V rows that other workgroups read too: without the hint of load_stream16.
__device__ __forceinline__ uint4 load16(const uint8_t* p) {
  return *reinterpret_cast<const uint4*>(p);
}

// Sixteen E4M3 values as bf16 (exact: 4 significant bits, exponents -9 .. 8).
__device__ __forceinline__ void widen_fp8(const uint4& r, uint4& lo, uint4& hi) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
  uint32_t o[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[i]), false);
    const auto b = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[i]), true);
    o[2 * i] = high_halves(a[0], a[1]);
    o[2 * i + 1] = high_halves(b[0], b[1]);
  }
  lo = make_uint4(o[0], o[1], o[2], o[3]);
  hi = make_uint4(o[4], o[5], o[6], o[7]);
}

// The sign bit of every byte of x that is an E4M3 NaN (seven ones).
__device__ __forceinline__ uint32_t nan_bytes(uint32_t x) {
  return ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
}

// x with every infinity and NaN replaced by 0.
__device__ __forceinline__ uint32_t finite_pair(uint32_t w) {
  const uint32_t lo = (w & 0x7f80u) == 0x7f80u ? 0u : w & 0xffffu;
  const uint32_t hi = (w & 0x7f800000u) == 0x7f800000u ? 0u : w & 0xffff0000u;
  return lo | hi;
}

// The lowest x of 32 bits (none for x <= 0, all for x >= 32).
__device__ __forceinline__ uint32_t low_bits(int x) {
  return x <= 0 ? 0u : x >= 32 ? ~0u : (1u << x) - 1u;
}

// The (request, KV head) pair of a workgroup and its place among the pair's
// per_pair workgroups, which share K and V.  Workgroup ids go round the eight XCDs,
// each with an L2 of its own, so a pair stays on one XCD, and neighbouring pairs (a
// request's heads, with its length) go to different ones.  Where the pairs do not
// go evenly round, the workgroups are cut into eight equal runs instead.  (Equal
// runs for all, a request's heads on one XCD: 49.5 us where this takes 43.4 for 16
// ragged prompts, 68.2 and 61.8 for 24 trees of 61 nodes, 76.3 and 73.5 for 32 ragged
// fp8 requests; 60.0 both for 32 ragged requests of one row tile.)
struct TreeItem {
  int pair, sub;  // pair < 0: nothing to do
};
__device__ __forceinline__ TreeItem tree_item(int pairs, int per_pair) {
  const int xcd = blockIdx.x & 7, at = blockIdx.x >> 3;
  if (pairs % 8 == 0 || pairs >= 64) {
    const int pair = at / per_pair * 8 + xcd;
    return {pair < pairs ? pair : -1, at % per_pair};
  }
  const int items = pairs * per_pair, per = (items + 7) / 8, item = xcd * per + at;
  if (at >= per || item >= items) return {-1, 0};
  return {item / per_pair, item % per_pair};
}
// Workgroups to launch for it.
inline uint32_t tree_grid(int64_t pairs, int64_t per_pair) {
  return static_cast<uint32_t>(pairs % 8 == 0 || pairs >= 64
                                   ? (pairs + 7) / 8 * 8 * per_pair
                                   : (pairs * per_pair + 7) / 8 * 8);
}

// The request at place r of the batch.  RANKED: of up to 64 requests those with the
// most work (row tiles times keys) first, so that long ones neither share a CU nor
// come last; every wave ranks them for itself, a request per lane.  Where
// arithmetic and not bytes bound the kernel: 32 ragged requests of 8 KV heads, 13
// nodes, fp8: 73.5 us a layer instead of 75.7; 24 of 61 nodes over a ring: 61.8 and
// 67.1; 16 ragged prompts: 43.4 and 47.1.
struct TreePlace {
  int b;
  TreeReq rq;
};
template <bool RANKED>
__device__ __forceinline__ TreePlace tree_place(const TreeArgs& a, int r, int tile_rows) {
  if (!RANKED || a.B == 1 || a.B > 64)
    return {r, tree_request(a.base, a.count, r, a.N, a.Lp, a.Ldec)};
  const int lane = threadIdx.x & 63;
  const TreeReq rq = tree_request(a.base, a.count, min(lane, a.B - 1), a.N, a.Lp, a.Ldec);
  const float tiles = static_cast<float>((rq.n * a.G + tile_rows - 1) / tile_rows);
  const float work = rq.n ? tiles * (a.Lp + min(rq.base, a.W) + rq.n) : 0.f;
  // positive floats compare as their bits; the lowest six tell requests apart
  const int mine = (__float_as_int(work) & ~63) | (63 - lane);
  int before = 0;
#pragma unroll 4
  for (int j = 0; j < a.B; ++j) before += __builtin_amdgcn_readlane(mine, j) > mine;
  const int b = __builtin_ctzll(__ballot(lane < a.B && before == r));
  return {b, {__builtin_amdgcn_readlane(rq.n, b), __builtin_amdgcn_readlane(rq.base, b)}};
}

template <int D>
constexpr int kPartRow = D + 4;  // fp32 of a partial row: values, maximum, sum, padding

// Output element pairs: four consecutive values of a row.
template <bool F32>
__device__ __forceinline__ void store4(void* out, int64_t at, float a, float b, float c, float d) {
  if constexpr (F32)
    *reinterpret_cast<float4*>(static_cast<float*>(out) + at) = make_float4(a, b, c, d);
  else
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + at) =
        make_uint2(pack_bf16(a, b), pack_bf16(c, d));
}

// What a lane needs of its query row (node, query head).
struct TreeRow {
  int node, dep;  // the node and its depth (a chain: the same)
  int thr;        // cached entries past the prefix are seen above this one
};

__device__ __forceinline__ TreeRow tree_row(const TreeArgs& a, const TreeReq& rq,
                                            const TreeKeys& ks, int b, int row) {
  TreeRow r;
  r.node = row / a.G;
  r.dep = a.depth ? a.depth[static_cast<int64_t>(b) * a.N + r.node] : r.node;
  r.thr = ks.cached.pre + rq.base + r.dep - a.W - ks.j0;
  return r;
}

// What is the same for all rows of a row tile.
struct TreeTile {
  int n0, n1, deepest, sink;  // nodes, largest depth; smaller depths stand at sink positions
};

// Which of 32 cached entries from e on the row sees.
__device__ __forceinline__ uint32_t see_cached(const TreeKeys& ks, const TreeRow& r, int e) {
  return low_bits(ks.cached.n - e) & (low_bits(ks.cached.pre - e) | ~low_bits(r.thr + 1 - e));
}

// Which of 32 new entries from e on the row sees.
__device__ __forceinline__ uint32_t see_fresh(const TreeArgs& a, const TreeKeys& ks,
                                              const TreeTile& tt, const TreeRow& r, int b, int e) {
  const KeyList& k = ks.fresh;
  uint32_t see = low_bits(k.n - e);
  if (!a.depth) {  // entries from k.pre on are nodes in order; every node sees those before
    const int f = -k.shift - e;
    return see & low_bits(r.node + 1 + f) &
           (low_bits(k.pre - e) | low_bits(tt.sink + f) | ~low_bits(r.node - a.W + 1 + f));
  }
  const int64_t at = static_cast<int64_t>(b) * a.N;
  see &= e / 32 < a.words ? a.anc[(at + r.node) * a.words + e / 32] : 0u;
  if (tt.deepest >= a.W)  // some node has ancestors out of its window
    for (uint32_t m = see; m; m &= m - 1) {
      const int i = __builtin_ctz(m), de = a.depth[at + e + i];
      if (de >= tt.sink && r.dep - de >= a.W) see &= ~(1u << i);
    }
  return see;
}

// Whether some row of the tile must not see some of the `keys` entries from e on.
__device__ __forceinline__ bool hides_cached(const TreeArgs& a, const TreeReq& rq,
                                             const TreeKeys& ks, const TreeTile& tt, int e,
                                             int keys) {
  const KeyList& k = ks.cached;
  const int thr = k.pre + rq.base + tt.deepest - a.W - ks.j0;
  return e + keys > k.n || (e + keys > k.pre && max(e, k.pre) <= thr);
}
__device__ __forceinline__ bool hides_fresh(const TreeArgs& a, const TreeKeys& ks,
                                            const TreeTile& tt, int e, int keys) {
  const KeyList& k = ks.fresh;
  return a.depth || !(e + keys <= k.pre || (e >= k.pre && e + keys <= k.n &&
                                            k.row(e + keys - 1) <= tt.n0 && k.row(e) > tt.n1 - a.W));
}

// Elements of a K or V row in LDS.  Padded so that neither the K operand's
// reads (16 rows, 16 bytes each, side by side) nor the transposed V reads
// (8 rows, 32 bytes each) meet in a bank; addresses are then a lane's base and
// constants (swizzled rows without padding cost a register per address).
template <int D>
constexpr int kKRow = D + 8;
template <int D>
constexpr int kVRow = D + 16;

// Order of a row's 16-byte chunks (8 elements) in LDS.  A lane widens 16 fp8
// elements to two chunks; stored side by side, the first chunks of all lanes
// would take every second place and meet in the banks, so fp8 builds put the even
// chunks ahead of the odd ones: chunk at place j.
template <int D, bool EVEN>
__host__ __device__ constexpr int chunk_at(int j) {
  return !EVEN ? j : j < D / 16 ? 2 * j : 2 * (j - D / 16) + 1;
}
template <int D, bool EVEN>
__host__ __device__ constexpr int place_of(int c) {
  return !EVEN ? c : c / 2 + D / 16 * (c % 2);
}

// A wave's 32 query rows against tiles of keys in LDS.
//
// Both products run on the matrix cores with the keys as rows, S^T = K Q^T and
// O^T = V^T P^T (v_mfma_f32_32x32x16_bf16).  A lane then holds scores, weights
// and outputs of one query row (lane % 32) only: the running maximum and the
// rescale need one exchange, with the lane's other half, and the weights are the
// second product's operand where they are.  V comes back from LDS transposed
// (ds_read_b64_tr_b16) in the order of keys the weights have.
template <int D, bool F32, bool FP8>
struct TreeWave {
  bf16x8 qf[D / 16];
  f32x16 o[D / 32];
  float m, l;

  // Queries: the second operand of S^T, in the order of K's elements in LDS.
  __device__ __forceinline__ void start(const TreeArgs& a, int lane, const uint16_t* q) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      uint4 x = *reinterpret_cast<const uint4*>(q + (lane >> 5 ? 8 * chunk_at<D, FP8>(2 * s + 1)
                                                              : 8 * chunk_at<D, FP8>(2 * s)));
      x.x ^= a.q_sign;
      x.y ^= a.q_sign;
      x.z ^= a.q_sign;
      x.w ^= a.q_sign;
      qf[s] = __builtin_bit_cast(bf16x8, x);
    }
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[c][i] = 0.f;
    m = kTreeMin;
    l = 0.f;
  }

  // Four keys from `key` on of a lane's column of block c: of sixteen lanes that name
  // four rows of 16 columns, each gets a column (ds_read_b64_tr_b16).
  static __device__ __forceinline__ uint2 vread(const uint16_t* lv, int lane, int key, int c) {
    const int s16 = lane & 15, r = key + (s16 >> 2);
    return __builtin_bit_cast(
        uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                   (__attribute__((address_space(3))) s16x4*)(
                       lv + r * kVRow<D> + 32 * c + 16 * ((lane >> 4) & 1) + 4 * (s16 & 3))));
  }

  // S^T of 32 keys: lane (lq, hh) gets row lq's scores of keys 8 (i / 4) + 4 hh +
  // i % 4, times `turn`, -inf where `hides` and the row does not see them.
  __device__ __forceinline__ void scores(int lane, const uint16_t* lk, float turn, bool hides,
                                         uint32_t see, f32x16& sc) {
    const int hh = lane >> 5;
#pragma unroll
    for (int i = 0; i < 16; ++i) sc[i] = 0.f;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      const bf16x8 kf = *reinterpret_cast<const bf16x8*>(lk + (lane & 31) * kKRow<D> + 16 * s + 8 * hh);
      sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[s], sc, 0, 0, 0);
    }
    if (turn != 1.f) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] *= turn;
    }
    if (hides) {
      const uint32_t w = see >> (4 * hh);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        sc[i] = w & (1u << (8 * (i / 4) + i % 4)) ? sc[i] : -__builtin_inff();
    }
  }

  // The running maximum takes the scores in.  Weights stay relative to the maximum
  // of an earlier tile as long as none passes 2^kTreeSlack: every sum keeps its
  // relative precision, and the rescale (a multiply per output, and per
  // weight in `held`, not yet in the outputs) leaves most tiles.
  template <bool HELD>
  __device__ __forceinline__ void raise(float sl, const f32x16& sc, f32x16& held) {
    float mx = sc[0];
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sc[i]);
    float x1, x2;
    xor_pair<32>(mx, x1, x2);
    const float mnew = fmaxf(m, fmaxf(x1, x2) * sl);
    if (__ballot(mnew > m + kTreeSlack)) {
      const float alpha = fast_exp2(m - mnew);
      l *= alpha;
#pragma unroll
      for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[c][i] *= alpha;
      if constexpr (HELD) {
#pragma unroll
        for (int i = 0; i < 16; ++i) held[i] *= alpha;
      }
      m = mnew;
    }
  }

  // Scores to weights, in place, times V's scale.  A hidden key's weight of 0 stays one
  // where that is infinite or NaN.
  __device__ __forceinline__ void weights(float sl, float vs, f32x16& sc) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      sc[i] = fast_exp2(fmaf(sc[i], sl, -m));
      l += sc[i];
    }
    if (vs == 1.f) return;
    if (__builtin_expect(vs - vs == 0.f, 1)) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] *= vs;
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[i] = sc[i] == 0.f ? 0.f : sc[i] * vs;
    }
  }

  // O += P V of 32 keys, 16 a step.  Half hh's eight operand slots are the keys
  // 4 hh .. + 3 and 8 + 4 hh .. + 3 of the step, and V is read in that order.
  // For fp32 outputs the weights go in as three bf16 terms, which hold all their
  // 24 bits; for bf16 outputs as two, each nearest, so that what is left out of a
  // weight, 2^-16 of it, is a 256th of the output's own half step (with one term an
  // element was off by up to 7 of those).
  __device__ __forceinline__ void values(int lane, const uint16_t* lv, const f32x16& p) {
    constexpr int NE = F32 ? 3 : 2;
    const int hh = lane >> 5;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      bf16x8 pf[NE];
      uint32_t w[NE][4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float u = p[8 * s + 2 * j], v = p[8 * s + 2 * j + 1];
        if constexpr (F32) {
#pragma unroll
          for (int e = 0; e < NE; ++e) {
            w[e][j] = high_halves(u, v);
            u -= __uint_as_float(__float_as_uint(u) & 0xffff0000u);
            v -= __uint_as_float(__float_as_uint(v) & 0xffff0000u);
          }
        } else {
          w[0][j] = pack_bf16(u, v);
          w[1][j] = pack_bf16(u - __uint_as_float(w[0][j] << 16),
                              v - __uint_as_float(w[0][j] & 0xffff0000u));
        }
      }
#pragma unroll
      for (int e = 0; e < NE; ++e)
        pf[e] = __builtin_bit_cast(bf16x8, make_uint4(w[e][0], w[e][1], w[e][2], w[e][3]));
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        const uint2 va = vread(lv, lane, 16 * s + 4 * hh, c);
        const uint2 vb = vread(lv, lane, 16 * s + 8 + 4 * hh, c);
        const bf16x8 vf = __builtin_bit_cast(bf16x8, make_uint4(va.x, va.y, vb.x, vb.y));
#pragma unroll
        for (int e = 0; e < NE; ++e)
          o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[e], o[c], 0, 0, 0);
      }
    }
  }

  // A tile of 32 keys.  sl: score scale (positive), turn: what it lacks, -1 or NaN
  // (else 1); vs: scale of V; see: the keys each row sees, used where `hides`.
  __device__ __forceinline__ void tile(int lane, const uint16_t* lk, const uint16_t* lv, float sl,
                                       float turn, float vs, bool hides, uint32_t see) {
    f32x16 sc;
    scores(lane, lk, turn, hides, see, sc);
    raise<false>(sl, sc, sc);
    weights(sl, vs, sc);
    values(lane, lv, sc);
  }

  // 64 keys: the second half's scores are under way while the first's
  // weights are computed, and the first half's values while the second's are.
  __device__ __forceinline__ void tile2(int lane, const uint16_t* lk, const uint16_t* lv, float sl,
                                        float turn, float vs, bool hides,
                                        const uint32_t (&see)[2]) {
    f32x16 s0, s1;
    scores(lane, lk, turn, hides, see[0], s0);
    raise<false>(sl, s0, s0);
    scores(lane, lk + 32 * kKRow<D>, turn, hides, see[1], s1);
    weights(sl, vs, s0);
    raise<true>(sl, s1, s0);
    values(lane, lv, s0);
    weights(sl, vs, s1);
    values(lane, lv + 32 * kVRow<D>, s1);
  }

  // Whether the lane's outputs are finite, and its n-th four of them.
  __device__ __forceinline__ bool all_finite() const {
    float s[4] = {};
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i & 3] = fmaf(o[c][i], 0.f, s[i & 3]);
    return s[0] + s[1] + s[2] + s[3] == 0.f;
  }
  __device__ __forceinline__ void four(int n, float (&x)[4]) const {
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i & 3] = n == 4 * c + i / 4 ? o[c][i] : x[i & 3];
  }
  __device__ __forceinline__ void set_four(int n, const float (&x)[4]) {
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[c][i] = n == 4 * c + i / 4 ? x[i & 3] : o[c][i];
  }

  // Adds the infinities and NaN of V row v (fp8 where CODES) to the rows that see
  // its key: as products of 1 and the largest bf16 values, whose sum overflows, and of
  // 0 where the key is hidden.  A NaN is both infinities, one after the other.  (Summed
  // up by themselves: an infinity stays one where the matrix core adds these to it.)
  template <bool CODES>
  __device__ __forceinline__ void add_nonfinite(int lane, const uint8_t* v, bool mine) {
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      const int place = 4 * c + ((lane & 31) >> 3);  // (chunk_at of a lane's place)
      const int at = FP8 ? (place < D / 16 ? 2 * place : 2 * (place - D / 16) + 1) : place;
      const int col = 8 * at + (lane & 7);
      const uint32_t x = CODES ? ((v[col] & 0x7fu) == 0x7fu ? 0x7fc0u : 0u)
                               : reinterpret_cast<const uint16_t*>(v)[col];
      const uint32_t size = x & 0x7fffu;
      const uint32_t up = x == 0x7f80u || size > 0x7f80u ? 0x7f7f7f7fu : 0u;
      const uint32_t down = x == 0xff80u || size > 0x7f80u ? 0xff7fff7fu : 0u;
      const uint32_t one = mine ? 0x3f803f80u : 0u;
      const bf16x8 p = __builtin_bit_cast(bf16x8, make_uint4(one, one, one, one));
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t big = e ? down : up;
        f32x16 t;
#pragma unroll
        for (int i = 0; i < 16; ++i) t[i] = 0.f;
        t = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            __builtin_bit_cast(bf16x8, make_uint4(big, big, big, big)), p, t, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 16; ++i) o[c][i] += t[i];
        __builtin_amdgcn_sched_barrier(0);  // one t at a time
      }
    }
  }
};

// Scales of the scores and of V over the cache.  Scores are compared before they
// are scaled, so the scale is positive: a negative one turns the scores, a
// zero one is as good as the smallest, and a NaN makes the scores NaN before the
// hidden ones are left out.
struct CacheScale {
  float sl, vs, turn;
};
template <bool FP8>
__device__ __forceinline__ CacheScale cache_scale(const TreeArgs& a, int pair) {
  CacheScale c{a.scale_log2, 1.f, 1.f};
  if constexpr (FP8) {
    if (a.ks) c.sl *= a.ks[pair];
    if (a.vs) c.vs = a.vs[pair];
    c.turn = c.sl != c.sl ? c.sl : c.sl < 0.f ? -1.f : 1.f;
    c.sl = fmaxf(fabsf(c.sl), kTreeMinScale);  // (the smallest for a NaN)
  }
  return c;
}

// In a tile with hidden keys a V row's infinity or NaN would reach queries that
// must not see it, as 0 times it.  Such elements become 0 in LDS, and
// add_nonfinite adds them where they are seen.  x: the N chunks of 16 bytes that
// each lane has just stored, chunk i at `v` + i * step, D / 8 lanes to a row;
// returns the rows that had any: bit i * (512 / D) + g for row g of pass i.  (The
// rare second pass goes over LDS: on the registers it cost 20 of them.)
template <int D, int N>
__device__ __forceinline__ uint32_t clean_rows(const uint4* x, uint16_t* v, int step) {
  constexpr int CPR = D / 8, RPW = 64 / CPR;
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) any |= nonfinite_bit(x[i]);
  if (!__ballot((any & 0x8000u) != 0)) return 0;
  uint32_t rows = 0;
#pragma unroll 1
  for (int i = 0; i < N; ++i, v += step) {
    const uint4 y = *reinterpret_cast<const uint4*>(v);
    const bool mine = (nonfinite_bit(y) & 0x8000u) != 0;
    const uint64_t who = __ballot(mine);
    if (mine)
      *reinterpret_cast<uint4*>(v) =
          make_uint4(finite_pair(y.x), finite_pair(y.y), finite_pair(y.z), finite_pair(y.w));
#pragma unroll
    for (int g = 0; g < RPW; ++g)
      rows |= (who >> (g * CPR) & ((1ull << CPR) - 1)) ? 1u << (i * RPW + g) : 0u;
  }
  return rows;
}

// The same of fp8 rows, in registers: x: N chunks of 16 elements, D / 16 lanes to a
// row; bit i * (1024 / D) + g of the result for row g of pass i.
template <int D, int N>
__device__ __forceinline__ uint32_t clean_codes(uint4* x) {
  constexpr int CPR = D / 16, RPW = 64 / CPR;
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < N; ++i)
    any |= nan_bytes(x[i].x) | nan_bytes(x[i].y) | nan_bytes(x[i].z) | nan_bytes(x[i].w);
  if (!__ballot(any != 0)) return 0;
  uint32_t rows = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w}, bad = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t b = nan_bytes(w[e]);
      bad |= b;
      w[e] &= ~((b >> 7) * 0xffu);
    }
    x[i] = make_uint4(w[0], w[1], w[2], w[3]);
    const uint64_t who = __ballot(bad != 0);
#pragma unroll
    for (int g = 0; g < RPW; ++g)
      rows |= (who >> (g * CPR)) & ((1ull << CPR) - 1) ? 1u << (i * RPW + g) : 0u;
  }
  return rows;
}

// A weight's terms, or a weight that underflows, make NaN of an infinity in V
// where one of them is 0.  So four elements of a row that are not all finite are
// settled once more: what each sees of infinities and NaN, over the tiles of 32 keys
// t0 .. t1 - 1 or until all of them are NaN, takes its place.  v_old, v_new: the
// elements' columns of V.
template <bool FP8>
__device__ __forceinline__ void settle_nonfinite(const TreeArgs& a, const TreeKeys& ks,
                                                 const TreeTile& tt, const TreeRow& my, int b,
                                                 const uint8_t* v_old, const uint8_t* v_new, int t0,
                                                 int t1, float (&x)[4]) {
  const int t_old = (ks.cached.n + 31) / 32;
  uint32_t up = 0, down = 0;  // bit per element: an infinity, or both for a NaN
  uint32_t open = 0;          // those to settle
#pragma unroll
  for (int k = 0; k < 4; ++k) open |= x[k] - x[k] == 0.f ? 0u : 1u << k;
#pragma unroll 1
  for (int t = t0; t < t1 && (open & ~(up & down)); ++t) {
    const bool old = t < t_old;
    const int e0 = (t - (old ? 0 : t_old)) * 32;
    const KeyList list = pick_list(old, ks.cached, ks.fresh);
    const uint8_t* v = old ? v_old : v_new;
    const int64_t step = old ? a.sr : a.nsn * 2;
    const uint32_t see = old ? see_cached(ks, my, e0) : see_fresh(a, ks, tt, my, b, e0);
#pragma unroll 1
    for (int i = 0; i < 32; i += 8) {
      uint32_t h[8][2];  // bf16 bits; of fp8 codes the NaN ones alone
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint8_t* at = v + list.near(e0 + i + e) * step;
        if (FP8 && old) {
          const uint32_t n = nan_bytes(*reinterpret_cast<const uint32_t*>(at)) >> 7;
          h[e][0] = ((n & 1u) | (n & 0x100u) << 8) * 0x7fc0u;
          h[e][1] = ((n >> 16 & 1u) | (n >> 8 & 0x10000u)) * 0x7fc0u;
        } else {
          const uint2 y = *reinterpret_cast<const uint2*>(at);
          h[e][0] = y.x;
          h[e][1] = y.y;
        }
      }
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t y = h[e][k / 2] >> (16 * (k & 1)), size = y & 0x7fffu;
          if (size < 0x7f80u || !(see >> (i + e) & 1u)) continue;
          if (size > 0x7f80u || !(y & 0x8000u)) up |= 1u << k;
          if (size > 0x7f80u || (y & 0x8000u)) down |= 1u << k;
        }
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const bool u = up & open & 1u << k, d = down & open & 1u << k;
    if (u || d) x[k] = u && d ? __builtin_nanf("") : u ? __builtin_inff() : -__builtin_inff();
  }
}

// Whether four values are finite numbers.
__device__ __forceinline__ bool all_finite(float a, float b, float c, float d) {
  return fmaf(a, 0.f, fmaf(b, 0.f, fmaf(c, 0.f, d * 0.f))) == 0.f;
}

// Columns of output registers 4 k .. of block c (k = 0 .. 3), half hh's four.
template <int D, bool FP8>
__device__ __forceinline__ int out_col(int c, int k, int hh) {
  return 8 * chunk_at<D, FP8>(4 * c + k) + 4 * hh;
}

// Splits of a row tile that have keys, and the tiles of 'part' of 'parts'.
__device__ __forceinline__ int tree_splits(const TreeArgs& a, int tiles) {
  return min(a.splits, (tiles + a.split_tiles - 1) / a.split_tiles);
}
__device__ __forceinline__ int tree_cut(int tiles, int part, int parts) {
  return static_cast<int>(static_cast<int64_t>(tiles) * part / parts);
}

// ---- many query rows -----------------------------------------------------------

constexpr int kTileKeys = 64;   // keys of a tile
constexpr int kTileRows = 128;  // query rows of a workgroup

// A workgroup of four waves takes 128 query rows (node, query head of the KV
// head's group) of one request and KV head.  Tiles of 64 keys go through LDS for all
// four waves, two buffers in turn.
//
// Bound by the waves' own instructions: two images of 4096 tokens at once (32 heads
// over 8, d = 128, bf16 outputs) take 465 to 478 us, 0.66 PFLOP/s, where a library
// product of 8192^3 reaches 1.19; the matrix cores are busy for 43 % of the time, the
// softmax's exponentials, maxima and packing beside them.  With the weights in one
// bf16 term they took 375: 286 for the arithmetic without loads and stores to LDS, 51
// for the loads, 32 for the LDS stores.  The second term adds half as many products
// and 49 instructions per 32 keys.  Measured with one term and left: 64 rows per wave
// (490 us: one wave per SIMD), 32-key tiles with three waves per SIMD (376), 256 rows
// per workgroup (377, and 52 us where 16 ragged prompts take 38).
template <bool FP8, int D, bool F32>
__global__ __launch_bounds__(256, 2) void tree_tile_kernel(TreeArgs a) {
  constexpr int CPR = D / 8;           // 16-byte chunks of a bf16 row
  constexpr int NP = CPR * kTileKeys / 256;
  constexpr int RPP = 256 / CPR;       // rows per pass of the workgroup
  constexpr int CP8 = D / 16, NP8 = CP8 * kTileKeys / 256, RP8 = 256 / CP8;
  __shared__ __align__(16) uint16_t lk[2][kTileKeys * kKRow<D>];
  __shared__ __align__(16) uint16_t lv[2][kTileKeys * kVRow<D>];
  __shared__ uint32_t lbad[2][4];  // V rows of a tile that are not finite, by wave (clean_rows)

  const TreeItem item = tree_item(a.B * a.Hkv, a.row_tiles);
  if (item.pair < 0) return;
  const TreePlace place = tree_place<true>(a, item.pair / a.Hkv, kTileRows);
  const TreeReq rq = place.rq;
  const int b = place.b;
  const int h = item.pair % a.Hkv, pair = b * a.Hkv + h;
  const int qt = a.row_tiles - 1 - item.sub;  // longest first
  const int rows = rq.n * a.G, r0 = qt * kTileRows;
  if (r0 >= rows) return;
  TreeTile tt{r0 / a.G, (min(r0 + kTileRows, rows) - 1) / a.G, 0, a.S - rq.base};
  tt.deepest = a.depth ? a.max_depth[b] : tt.n1;
  const TreeKeys ks = tree_keys(a, rq, tt.n0, tt.n1);
  const int t_old = (ks.cached.n + kTileKeys - 1) / kTileKeys;
  const int tiles = t_old + (ks.fresh.n + kTileKeys - 1) / kTileKeys;

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = r0 + 32 * wave + (lane & 31);
  const bool wave_on = r0 + 32 * wave < rows;
  const CacheScale cs = cache_scale<FP8>(a, pair);
  const TreeRow my = tree_row(a, rq, ks, b, min(row, rows - 1));
  TreeWave<D, F32, FP8> w;
  w.start(a, lane,
          a.q + b * a.qsb + my.node * a.qsn + (h * a.G + min(row, rows - 1) % a.G) * a.qsh);

  const uint8_t* kc = a.k + tree_cache_base(a, b, h, FP8 ? 1 : 2);
  const uint8_t* vc = a.v + tree_cache_base(a, b, h, FP8 ? 1 : 2);
  const uint8_t* kn = reinterpret_cast<const uint8_t*>(a.kn + b * a.nsb + h * a.nsh);
  const uint8_t* vn = reinterpret_cast<const uint8_t*>(a.vn + b * a.nsb + h * a.nsh);
  uint4 rk[NP], rv[NP];

  // Tile t, of bf16 rows: of the new tokens, or of a bf16 cache.
  auto load = [&](int t) {
    const bool old = !FP8 && t < t_old;
    const KeyList list = pick_list(old, ks.cached, ks.fresh);
    const uint8_t* k = old ? kc : kn;
    const uint8_t* v = old ? vc : vn;
    const int64_t step = old ? a.sr : a.nsn * 2;
    const int e0 = (t - (t < t_old ? 0 : t_old)) * kTileKeys + tid / CPR;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int64_t at = list.near(e0 + i * RPP) * step + (tid % CPR) * 16;
      rk[i] = load16(k + at);
      rv[i] = load16(v + at);
    }
  };
  auto hides = [&](int t) {
    return t < t_old ? hides_cached(a, rq, ks, tt, t * kTileKeys, kTileKeys)
                     : hides_fresh(a, ks, tt, (t - t_old) * kTileKeys, kTileKeys);
  };
  auto put = [&](int t, int buf) {
    const int c = place_of<D, FP8>(tid % CPR);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int r = i * RPP + tid / CPR;
      *reinterpret_cast<uint4*>(lk[buf] + r * kKRow<D> + c * 8) = rk[i];
      *reinterpret_cast<uint4*>(lv[buf] + r * kVRow<D> + c * 8) = rv[i];
    }
    uint32_t bad = 0;
    if (hides(t))
      bad = clean_rows<D, NP>(rv, lv[buf] + (tid / CPR) * kVRow<D> + c * 8, RPP * kVRow<D>);
    if (lane == 0) lbad[buf][wave] = bad;
  };
  // The same of an fp8 cache: sixteen elements a load.
  auto load8 = [&](int t) {
#pragma unroll
    for (int i = 0; i < NP8; ++i) {
      const int64_t at = ks.cached.near(t * kTileKeys + i * RP8 + tid / CP8) * a.sr + (tid % CP8) * 16;
      rk[i] = load16(kc + at);
      rv[i] = load16(vc + at);
    }
  };
  auto put8 = [&](int t, int buf) {
    uint32_t bad = 0;
    if (hides(t)) bad = clean_codes<D, NP8>(rv);
    if (lane == 0) lbad[buf][wave] = bad;
#pragma unroll
    for (int i = 0; i < NP8; ++i) {
      const int r = i * RP8 + tid / CP8, c = tid % CP8;
      uint4 lo, hi;
      widen_fp8(rk[i], lo, hi);
      *reinterpret_cast<uint4*>(lk[buf] + r * kKRow<D> + c * 8) = lo;
      *reinterpret_cast<uint4*>(lk[buf] + r * kKRow<D> + c * 8 + D / 2) = hi;
      widen_fp8(rv[i], lo, hi);
      *reinterpret_cast<uint4*>(lv[buf] + r * kVRow<D> + c * 8) = lo;
      *reinterpret_cast<uint4*>(lv[buf] + r * kVRow<D> + c * 8 + D / 2) = hi;
    }
  };
  auto see_of = [&](int t, uint32_t (&see)[2]) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      see[i] = t < t_old ? see_cached(ks, my, t * kTileKeys + 32 * i)
                         : see_fresh(a, ks, tt, my, b, (t - t_old) * kTileKeys + 32 * i);
  };
  auto add_hidden = [&](int t, int buf, const uint32_t (&see)[2], auto codes) {
    constexpr int per = codes.value ? RP8 : RPP;  // rows of a pass of all waves, of one wave
    constexpr int own = per / 4;
    const bool old = t < t_old;
#pragma unroll 1
    for (int i = 0; i < 4; ++i)
#pragma unroll 1
      for (uint32_t bad = lbad[buf][i]; bad; bad &= bad - 1) {
        const int at = __builtin_ctz(bad), e = at / own * per + i * own + at % own;
        const bool mine = (see[e >> 5] >> (e & 31)) & 1u;
        const uint8_t* v = old ? vc + ks.cached.near(t * kTileKeys + e) * a.sr
                               : vn + ks.fresh.near((t - t_old) * kTileKeys + e) * a.nsn * 2;
        w.template add_nonfinite<codes.value>(lane, v, mine);
      }
  };

  // A tile's rows go into LDS at the start of the tile before, when they have had a
  // whole tile's time to arrive, and the tile after them is asked for.
  int t = 0, buf = 0;
  if constexpr (FP8) {
    const int end = t_old;
    if (t < end) {
      load8(t);
      put8(t, 0);
      if (t + 1 < end) load8(t + 1);
      __syncthreads();
    }
    for (; t < end; ++t, buf ^= 1) {
      if (t + 1 < end) put8(t + 1, buf ^ 1);
      if (t + 2 < end) load8(t + 2);
      asm volatile("" ::: "memory");
      if (wave_on) {
        uint32_t see[2] = {};
        const bool hide = hides(t);
        if (hide) see_of(t, see);
        w.tile2(lane, lk[buf], lv[buf], cs.sl, cs.turn, cs.vs, hide, see);
        if (hide) add_hidden(t, buf, see, std::true_type());
      }
      __syncthreads();
    }
  }
  if (t < tiles) {
    load(t);
    put(t, buf);
    if (t + 1 < tiles) load(t + 1);
    __syncthreads();
  }
  for (; t < tiles; ++t, buf ^= 1) {
    if (t + 1 < tiles) put(t + 1, buf ^ 1);
    if (t + 2 < tiles) load(t + 2);
    asm volatile("" ::: "memory");  // the loads stay ahead of the tile
    if (wave_on) {
      uint32_t see[2] = {};
      const bool hide = hides(t);
      if (hide) see_of(t, see);
      w.tile2(lane, lk[buf], lv[buf], a.scale_log2, 1.f, 1.f, hide, see);
      if (hide) add_hidden(t, buf, see, std::false_type());
    }
    __syncthreads();
  }

  float l1, l2;
  xor_pair<32>(w.l, l1, l2);
  const float l = l1 + l2;
  if (row >= rows) return;
  const int hh = lane >> 5;
  const float inv = 1.f / l;
  if (__builtin_expect(!w.all_finite(), 0) && l - l == 0.f && cs.vs - cs.vs == 0.f) {
#pragma unroll 1
    for (int n = 0; n < D / 8; ++n) {
      const int col = out_col<D, FP8>(n / 4, n % 4, hh);
      float x[4] = {};
      w.four(n, x);
      if (all_finite(x[0], x[1], x[2], x[3])) continue;
      settle_nonfinite<FP8>(a, ks, tt, my, b, vc + col * (FP8 ? 1 : 2), vn + col * 2, 0,
                            (ks.cached.n + 31) / 32 + (ks.fresh.n + 31) / 32, x);
      w.set_four(n, x);
    }
  }
  const int64_t out =
      ((static_cast<int64_t>(b) * a.N + my.node) * a.Hq + h * a.G + row % a.G) * D;
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int i = 0; i < 16; i += 4)
      store4<F32>(a.out, out + out_col<D, FP8>(c, i / 4, hh), w.o[c][i] * inv, w.o[c][i + 1] * inv,
                  w.o[c][i + 2] * inv, w.o[c][i + 3] * inv);
}

// ---- few query rows --------------------------------------------------------------

constexpr int kStreamKeys = 32;  // keys of a wave's tile
constexpr int kStreamRows = 32;  // query rows of a workgroup

template <int D>
constexpr uint32_t kStreamLds = kStreamKeys * (kKRow<D> + kVRow<D>) * 2;  // a wave's K and V tile

// At most 32 query rows per workgroup.  Every wave streams tiles of 32 keys of
// its own for all rows, through registers (the next tiles are on their way while
// one is computed) and an LDS region of its own, so the waves of a workgroup wait
// for each other only to join their results at the end.
//
// Bound by the cache's bytes with one row tile and a full chip: 32 requests of 32
// heads, 265 to 807 keys, d = 128, bf16, fp32 outputs, take 57 us (5.1 TB/s; a large
// copy reaches 4.8, a stream that only reads 6.6).  K straight into the matrix
// operand, a row per lane, halves the LDS traffic but reads 32 bytes of a row at a time
// (67 us); loads without the streaming hint take 66 where these take 60, replayed.
// With few workgroups bound by what a CU reads (32 workgroups of 552 keys, unsplit: 14.6
// us), with two row tiles over fp8 by widening and arithmetic, done for both (32
// requests of 8 KV heads, 256 to 4339 keys: 67 us for 13 nodes of four heads, 48 for 7).
template <bool FP8, int D, bool F32, int NW>
__global__ __launch_bounds__(64 * NW, 2) void tree_stream_kernel(TreeArgs a) {
  constexpr int CPR = D / 8, RPP = 64 / CPR, NP = kStreamKeys / RPP;  // bf16 rows of V
  constexpr int C = FP8 ? D / 16 : CPR, R = 64 / C, N = kStreamKeys / R;  // the cache's
  constexpr int PF = N > 4 ? 1 : 2;  // tiles in flight ahead of the one at hand
  __shared__ __align__(16) uint16_t lds[NW * (kStreamLds<D> / 2)];
  __shared__ float lm[NW][32], ll[NW][32];

  const TreeItem item = tree_item(a.B * a.Hkv, a.row_tiles * a.splits);
  if (item.pair < 0) return;
  const int r = item.pair / a.Hkv;
  const TreePlace place =
      a.row_tiles == 1 ? tree_place<false>(a, r, 32) : tree_place<true>(a, r, 32);
  const TreeReq rq = place.rq;
  const int b = place.b;
  const int h = item.pair % a.Hkv, pair = b * a.Hkv + h;
  const int sp = item.sub / a.row_tiles, qt = item.sub % a.row_tiles;
  const int rows = rq.n * a.G, r0 = qt * 32;
  if (r0 >= rows) return;
  TreeTile tt{r0 / a.G, (min(r0 + 32, rows) - 1) / a.G, 0, a.S - rq.base};
  tt.deepest = a.depth ? a.max_depth[b] : tt.n1;
  const TreeKeys ks = tree_keys(a, rq, tt.n0, tt.n1);
  const int t_old = (ks.cached.n + kStreamKeys - 1) / kStreamKeys;
  const int tiles = t_old + (ks.fresh.n + kStreamKeys - 1) / kStreamKeys;
  const int nsp = tree_splits(a, tiles);
  if (sp >= nsp) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t0 = tree_cut(tiles, sp * NW + wave, nsp * NW);
  const int t1 = tree_cut(tiles, sp * NW + wave + 1, nsp * NW);

  uint16_t* lk = lds + wave * (kStreamLds<D> / 2);
  uint16_t* lv = lk + kStreamKeys * kKRow<D>;
  const uint8_t* kc = a.k + tree_cache_base(a, b, h, FP8 ? 1 : 2);
  const uint8_t* vc = a.v + tree_cache_base(a, b, h, FP8 ? 1 : 2);
  const uint8_t* kn = reinterpret_cast<const uint8_t*>(a.kn + b * a.nsb + h * a.nsh);
  const uint8_t* vn = reinterpret_cast<const uint8_t*>(a.vn + b * a.nsb + h * a.nsh);
  uint4 rk[PF * N], rv[PF * N];
  static_assert(PF * N >= NP, "the registers of the cache's tiles hold a tile of new rows");

  // Tile t, of bf16 rows: of the new tokens, or of a bf16 cache.
  auto load = [&](int t, int set) {
    const bool old = !FP8 && t < t_old;
    const KeyList list = pick_list(old, ks.cached, ks.fresh);
    const int64_t step = old ? a.sr : a.nsn * 2;
    const int e0 = (t - (t < t_old ? 0 : t_old)) * kStreamKeys;
    const uint8_t* k = old ? kc : kn;
    const uint8_t* v = old ? vc : vn;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int64_t at = list.near(e0 + i * RPP + lane / CPR) * step + (lane % CPR) * 16;
      rk[set + i] = load_stream16(k + at);
      rv[set + i] = load_stream16(v + at);
    }
  };
  // The same of an fp8 cache: sixteen elements a load.
  auto load8 = [&](int t, int set) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t at = ks.cached.near(t * kStreamKeys + i * R + lane / C) * a.sr + (lane % C) * 16;
      rk[set + i] = load_stream16(kc + at);
      rv[set + i] = load_stream16(vc + at);
    }
  };
  const int end8 = FP8 ? min(t1, t_old) : t0;  // tiles before it are of an fp8 cache
#pragma unroll
  for (int j = 0; j < PF; ++j) {
    if constexpr (FP8) {
      if (t0 + j < end8) load8(t0 + j, j * N);
    } else {
      if (t0 + j < t1) load(t0 + j, j * NP);
    }
  }

  const int lane_row = min(r0 + (lane & 31), rows - 1);
  const TreeRow my = tree_row(a, rq, ks, b, lane_row);
  TreeWave<D, F32, FP8> w;
  w.start(a, lane, a.q + b * a.qsb + my.node * a.qsn + (h * a.G + lane_row % a.G) * a.qsh);
  const CacheScale cs = cache_scale<FP8>(a, pair);

  // V rows of `bad`, from their place in memory, to the rows that see them.
  auto add_hidden = [&](uint32_t bad, uint32_t see, auto codes, auto&& row_at) {
#pragma unroll 1
    for (; bad; bad &= bad - 1) {
      const int e = __builtin_ctz(bad);
      w.template add_nonfinite<codes.value>(lane, row_at(e), (see >> e) & 1u);
    }
  };

  // A tile of bf16 rows in registers [set, set + NP); `next` fills them again.
  auto tile = [&](int t, int set, auto&& next) {
    const bool old = !FP8 && t < t_old;
    const int e0 = (t - (t < t_old ? 0 : t_old)) * kStreamKeys;
    const bool hide = old ? hides_cached(a, rq, ks, tt, e0, kStreamKeys)
                          : hides_fresh(a, ks, tt, e0, kStreamKeys);
    uint32_t see = 0;
    if (hide) see = old ? see_cached(ks, my, e0) : see_fresh(a, ks, tt, my, b, e0);
    const int c = place_of<D, FP8>(lane % CPR);
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int r = i * RPP + lane / CPR;
      *reinterpret_cast<uint4*>(lk + r * kKRow<D> + c * 8) = rk[set + i];
      *reinterpret_cast<uint4*>(lv + r * kVRow<D> + c * 8) = rv[set + i];
    }
    uint32_t bad = 0;
    if (hide)
      bad = clean_rows<D, NP>(rv + set, lv + (lane / CPR) * kVRow<D> + c * 8, RPP * kVRow<D>);
    next();
    fence_wave();
    w.tile(lane, lk, lv, a.scale_log2, 1.f, 1.f, hide, see);
    add_hidden(bad, see, std::false_type(), [&](int e) {
      return old ? vc + ks.cached.near(e0 + e) * a.sr : vn + ks.fresh.near(e0 + e) * a.nsn * 2;
    });
    fence_wave();
  };

  if constexpr (FP8) {
    for (int t = t0; t < end8; t += PF) {
#pragma unroll
      for (int j = 0; j < PF; ++j) {
        if (t + j >= end8) break;
        const int e0 = (t + j) * kStreamKeys;
        const bool hide = hides_cached(a, rq, ks, tt, e0, kStreamKeys);
        const uint32_t see = hide ? see_cached(ks, my, e0) : 0u;
        const uint32_t bad = hide ? clean_codes<D, N>(rv + j * N) : 0u;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int r = i * R + lane / C, c = lane % C;
          uint4 lo, hi;
          widen_fp8(rk[j * N + i], lo, hi);
          *reinterpret_cast<uint4*>(lk + r * kKRow<D> + c * 8) = lo;
          *reinterpret_cast<uint4*>(lk + r * kKRow<D> + c * 8 + D / 2) = hi;
          widen_fp8(rv[j * N + i], lo, hi);
          *reinterpret_cast<uint4*>(lv + r * kVRow<D> + c * 8) = lo;
          *reinterpret_cast<uint4*>(lv + r * kVRow<D> + c * 8 + D / 2) = hi;
        }
        if (t + j + PF < end8) load8(t + j + PF, j * N);
        fence_wave();
        w.tile(lane, lk, lv, cs.sl, cs.turn, cs.vs, hide, see);
        add_hidden(bad, see, std::true_type(),
                   [&](int e) { return vc + ks.cached.near(e0 + e) * a.sr; });
        fence_wave();
      }
    }
    for (int t = max(t0, t_old); t < t1; ++t) {
      load(t, 0);
      tile(t, 0, [] {});
    }
  } else {
    for (int t = t0; t < t1; t += PF) {
#pragma unroll
      for (int j = 0; j < PF; ++j) {
        if (t + j >= t1) break;
        tile(t + j, j * NP, [&] {
          if (t + j + PF < t1) load(t + j + PF, j * NP);
        });
      }
    }
  }

  // Join the waves' results: every wave scales its own to the common maximum and
  // leaves them in its LDS region, then the workgroup's threads add them up.
  const bool split = nsp > 1;
  float* part = a.part + ((static_cast<int64_t>(pair) * a.row_tiles + qt) * a.splits + sp) *
                             32 * kPartRow<D>;
  float l1, l2;
  xor_pair<32>(w.l, l1, l2);
  if (lane < 32) {
    lm[wave][lane] = w.m;
    ll[wave][lane] = l1 + l2;
  }
  __syncthreads();
  float M = kTreeMin;
#pragma unroll
  for (int i = 0; i < NW; ++i) M = fmaxf(M, lm[i][lane & 31]);
  const float mine = fast_exp2(w.m - M);
  float* red = reinterpret_cast<float*>(lk);  // [32 rows][D], groups of 4 columns swizzled
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const int g = out_col<D, FP8>(c, i / 4, lane >> 5) / 4, r = lane & 31;
      *reinterpret_cast<float4*>(red + r * D + ((g ^ (r & 15)) * 4)) =
          make_float4(w.o[c][i] * mine, w.o[c][i + 1] * mine, w.o[c][i + 2] * mine,
                      w.o[c][i + 3] * mine);
    }
  __syncthreads();
  for (int at = threadIdx.x; at < 32 * (D / 4); at += 64 * NW) {
    const int r = at / (D / 4), g = at % (D / 4), row = r0 + r;
    if (row >= rows) break;
    float mr = kTreeMin, lr = 0.f;
#pragma unroll
    for (int i = 0; i < NW; ++i) mr = fmaxf(mr, lm[i][r]);
#pragma unroll
    for (int i = 0; i < NW; ++i) lr = fmaf(ll[i][r], fast_exp2(lm[i][r] - mr), lr);
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      const float4 x = *reinterpret_cast<const float4*>(
          reinterpret_cast<const float*>(lds + i * (kStreamLds<D> / 2)) + r * D +
          ((g ^ (r & 15)) * 4));
      s.x += x.x;
      s.y += x.y;
      s.z += x.z;
      s.w += x.w;
    }
    if (__builtin_expect(!all_finite(s.x, s.y, s.z, s.w), 0) && lr - lr == 0.f && cs.vs - cs.vs == 0.f) {
      float x[4] = {s.x, s.y, s.z, s.w};
      settle_nonfinite<FP8>(a, ks, tt, tree_row(a, rq, ks, b, row), b, vc + 4 * g * (FP8 ? 1 : 2),
                            vn + 8 * g, tree_cut(tiles, sp * NW, nsp * NW),
                            tree_cut(tiles, sp * NW + NW, nsp * NW), x);
      s = make_float4(x[0], x[1], x[2], x[3]);
    }
    if (split) {
      float* p = part + (row - r0) * kPartRow<D>;
      *reinterpret_cast<float4*>(p + 4 * g) = s;
      if (g == 0) *reinterpret_cast<float2*>(p + D) = make_float2(mr, lr);
    } else {
      const float inv = 1.f / lr;
      const int64_t out = (static_cast<int64_t>(b) * a.N + row / a.G) * a.Hq + h * a.G + row % a.G;
      store4<F32>(a.out, out * D + 4 * g, s.x * inv, s.y * inv, s.z * inv, s.w * inv);
    }
  }
}

// acc plus a split's value x of weight w; an infinity or NaN counts whole, also
// where w has underflowed.
__device__ __forceinline__ float add_split(float x, float w, float acc) {
  return x - x == 0.f ? fmaf(x, w, acc) : acc + x;
}

// Joins a row's splits: out = sum_s 2^(m_s - M) acc_s / sum_s 2^(m_s - M) l_s.
// One wave per query row.  Bound by its chain of memory latencies, so the first
// kAhead splits are read before it is known how many there are.
template <int D, bool F32>
__global__ __launch_bounds__(256) void tree_combine_kernel(TreeArgs a) {
  constexpr int E = D / 64, kAhead = 8;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t at = static_cast<int64_t>(blockIdx.x) * 4 + wave;
  const int per_pair = a.row_tiles * kStreamRows;
  const int pair = static_cast<int>(at / per_pair), row = static_cast<int>(at % per_pair);
  if (pair >= a.B * a.Hkv) return;
  const int b = pair / a.Hkv, h = pair % a.Hkv, qt = row / kStreamRows, r0 = qt * kStreamRows;
  constexpr int64_t step = kStreamRows * kPartRow<D>;
  const float* part = a.part + (static_cast<int64_t>(pair) * a.row_tiles + qt) * a.splits * step +
                      (row - r0) * kPartRow<D>;
  float pm[kAhead], pl[kAhead], px[kAhead][E];
#pragma unroll
  for (int s = 0; s < kAhead; ++s) {
    if (s >= a.splits) break;
    const float* x = part + s * step;
    pm[s] = x[D];
    pl[s] = x[D + 1];
#pragma unroll
    for (int e = 0; e < E; ++e) px[s][e] = x[lane * E + e];
  }
  const TreeReq rq = tree_request(a.base, a.count, b, a.N, a.Lp, a.Ldec);
  const int rows = rq.n * a.G;
  if (row >= rows) return;
  const TreeKeys ks = tree_keys(a, rq, r0 / a.G, (min(r0 + kStreamRows, rows) - 1) / a.G);
  const int tiles = (ks.cached.n + kStreamKeys - 1) / kStreamKeys +
                    (ks.fresh.n + kStreamKeys - 1) / kStreamKeys;
  const int nsp = tree_splits(a, tiles);
  if (nsp <= 1) return;
  float M = kTreeMin, L = 0.f, acc[E] = {};
#pragma unroll
  for (int s = 0; s < kAhead; ++s)
    if (s < nsp) M = fmaxf(M, pm[s]);
  for (int s = kAhead; s < nsp; ++s) M = fmaxf(M, part[s * step + D]);
#pragma unroll
  for (int s = 0; s < kAhead; ++s)
    if (s < nsp) {
      const float w = fast_exp2(pm[s] - M);
      L = fmaf(pl[s], w, L);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] = add_split(px[s][e], w, acc[e]);
    }
#pragma unroll 4
  for (int s = kAhead; s < nsp; ++s) {
    const float* x = part + s * step;
    const float w = fast_exp2(x[D] - M);
    L = fmaf(x[D + 1], w, L);
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = add_split(x[lane * E + e], w, acc[e]);
  }
  const float inv = 1.f / L;
  const int64_t to =
      ((static_cast<int64_t>(b) * a.N + row / a.G) * a.Hq + h * a.G + row % a.G) * D + lane * E;
  if constexpr (F32) {
#pragma unroll
    for (int e = 0; e < E; ++e) static_cast<float*>(a.out)[to + e] = acc[e] * inv;
  } else if constexpr (E == 2) {
    *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + to) =
        pack_bf16(acc[0] * inv, acc[1] * inv);
  } else {
    static_cast<uint16_t*>(a.out)[to] = static_cast<uint16_t>(pack_bf16(acc[0] * inv, 0.f));
  }
}

template <bool FP8, int D, bool F32>
hipError_t launch_one(const TreeLaunch& l, const TreeArgs& a, hipStream_t st) {
  const int64_t pairs = static_cast<int64_t>(a.B) * a.Hkv;
  const dim3 grid(tree_grid(pairs, a.row_tiles * a.splits));
  if (l.rows == kTileRows)
    tree_tile_kernel<FP8, D, F32><<<grid, dim3(256), 0, st>>>(a);
  else if (l.waves == 8)
    tree_stream_kernel<FP8, D, F32, 8><<<grid, dim3(512), 0, st>>>(a);
  else
    tree_stream_kernel<FP8, D, F32, 4><<<grid, dim3(256), 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || l.splits == 1) return e;
  const int64_t waves = pairs * a.row_tiles * kStreamRows;
  tree_combine_kernel<D, F32><<<dim3(static_cast<uint32_t>((waves + 3) / 4)), dim3(256), 0, st>>>(a);
  return hipGetLastError();
}

template <bool FP8>
hipError_t launch_tree(const Derived& d, const TreeLaunch& l, const TreeArgs& a, bool f32,
                       hipStream_t st) {
  if (d.D == 64)
    return f32 ? launch_one<FP8, 64, true>(l, a, st) : launch_one<FP8, 64, false>(l, a, st);
  return f32 ? launch_one<FP8, 128, true>(l, a, st) : launch_one<FP8, 128, false>(l, a, st);
}

}  // namespace
}  // namespace dsa
