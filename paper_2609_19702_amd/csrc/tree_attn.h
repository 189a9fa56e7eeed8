// Attention of several new tokens per request over the cache and themselves
// (dsa_tree_attention), as templates over the cache's element type.
#pragma once

#include "device.h"
#include "tree.h"

namespace dsa {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr float kTreeMin = -3.0e38f;  // "no score yet": finite, below every finite score in use

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

// Work item of a workgroup: consecutive items share K and V, and the eight
// XCDs (workgroup id mod 8) take an eighth of the items each, in order, so what
// one workgroup brings into an XCD's L2 the next finds there.
__device__ __forceinline__ int xcd_item(int items) {
  const int per = (items + 7) / 8, at = blockIdx.x >> 3;
  const int item = (blockIdx.x & 7) * per + at;
  return at < per && item < items ? item : -1;
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

// What a wave needs of one query row (node, query head): its lane's row.
struct TreeRow {
  int node, dep;  // the node and its depth (a chain: the same)
  int thr;        // cached entries past the prefix are seen above this one
  int64_t out;    // element offset of the output row
};

__device__ __forceinline__ TreeRow tree_row(const TreeArgs& a, const TreeReq& rq,
                                            const TreeKeys& ks, int b, int h, int row) {
  TreeRow r;
  r.node = row / a.G;
  const int head = h * a.G + row % a.G;
  r.dep = a.depth ? a.depth[static_cast<int64_t>(b) * a.N + r.node] : r.node;
  r.thr = ks.pre + rq.base + r.dep - a.W - ks.j0;
  r.out = (static_cast<int64_t>(b) * a.N + r.node) * a.Hq + head;
  return r;
}

// Which of 32 cached entries from e on the row sees.
__device__ __forceinline__ uint32_t see_cached(const TreeKeys& ks, const TreeRow& r, int e) {
  return low_bits(ks.nold - e) & (low_bits(ks.pre - e) | ~low_bits(r.thr + 1 - e));
}

// Which of 32 new entries from e on the row sees.  sink: nodes of smaller depth
// stand at sink positions; deep: some node is a window or more deep.
__device__ __forceinline__ uint32_t see_new(const TreeArgs& a, const TreeKeys& ks, const TreeRow& r,
                                            int b, int e, int sink, bool deep) {
  uint32_t see = low_bits(ks.nnew - e);
  if (!a.depth) {  // nodes from a1 on follow the first a0, which every node sees
    const int f = ks.a0 - ks.a1 - e;
    return see & low_bits(r.node + 1 + f) &
           (low_bits(ks.a0 - e) | low_bits(sink + f) | ~low_bits(r.node - a.W + 1 + f));
  }
  const int64_t at = static_cast<int64_t>(b) * a.N;
  see &= e / 32 < a.words ? a.anc[(at + r.node) * a.words + e / 32] : 0u;
  if (deep)
    for (uint32_t m = see; m; m &= m - 1) {
      const int i = __builtin_ctz(m), de = a.depth[at + e + i];
      if (de >= sink && r.dep - de >= a.W) see &= ~(1u << i);
    }
  return see;
}

// Whether some row of nodes n0 .. n1 (the deepest at depth `deepest`) must not
// see some of the `keys` cached (new) entries from e on.
__device__ __forceinline__ bool hides_cached(const TreeArgs& a, const TreeReq& rq,
                                             const TreeKeys& ks, int e, int keys, int deepest) {
  const int thr = ks.pre + rq.base + deepest - a.W - ks.j0;
  return e + keys > ks.nold || (e + keys > ks.pre && max(e, ks.pre) <= thr);
}
__device__ __forceinline__ bool hides_new(const TreeArgs& a, const TreeKeys& ks, int e, int keys,
                                          int n0, int n1) {
  return a.depth || !(e + keys <= ks.a0 ||
                      (e >= ks.a0 && e + keys <= ks.nnew && ks.node(e + keys - 1) <= n0 &&
                       ks.node(e) > n1 - a.W));
}

// Elements of a K or V row in LDS.  Padded so that neither the K operand's
// reads (16 rows, 16 bytes each, side by side) nor the transposed V reads
// (8 rows, 32 bytes each) meet in a bank; addresses are then a lane's base and
// constants (swizzled rows without padding cost a register per address).
template <int D>
constexpr int kKRow = D + 8;
template <int D>
constexpr int kVRow = D + 16;

// A wave's NB blocks of 32 query rows against tiles of keys in LDS.
//
// Both products run on the matrix cores with the keys as rows, S^T = K Q^T and
// O^T = V^T P^T (v_mfma_f32_32x32x16_bf16).  A lane then holds scores, weights
// and outputs of one query row of each block (lane % 32) only: the running
// maximum and the rescale need one exchange, with the lane's other half, and the
// weights are the second product's operand where they are.  V comes back from
// LDS transposed (ds_read_b64_tr_b16) in the order of keys the weights have.
template <int D, bool F32, int NB>
struct TreeWave {
  bf16x8 qf[NB][D / 16];
  f32x16 o[NB][D / 32];
  float m[NB], l[NB];

  // Queries: the second operand of S^T, elements 16 s + 8 hh .. of the row.
  __device__ __forceinline__ void start(const TreeArgs& a, int lane, int nb, const uint16_t* q) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      uint4 x = *reinterpret_cast<const uint4*>(q + 16 * s + 8 * (lane >> 5));
      x.x ^= a.q_sign;
      x.y ^= a.q_sign;
      x.z ^= a.q_sign;
      x.w ^= a.q_sign;
      qf[nb][s] = __builtin_bit_cast(bf16x8, x);
    }
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[nb][c][i] = 0.f;
    m[nb] = kTreeMin;
    l[nb] = 0.f;
  }

  // Four keys from `key` on, 16 columns of block c: see kernels above.
  static __device__ __forceinline__ uint2 vread(const uint16_t* lv, int lane, int key, int c) {
    const int s16 = lane & 15, r = key + (s16 >> 2);
    return __builtin_bit_cast(
        uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                   (__attribute__((address_space(3))) s16x4*)(
                       lv + r * kVRow<D> + 32 * c + 16 * ((lane >> 4) & 1) + 4 * (s16 & 3))));
  }

  // A tile of 32 KB keys.  sl: score scale (positive), flip: of negated scores;
  // vs: scale of V; see: the keys each row sees, used where `hides`.
  template <int KB>
  __device__ __forceinline__ void tile(int lane, const uint16_t* lk, const uint16_t* lv, float sl,
                                       bool flip, float vs, bool hides,
                                       const uint32_t (&see)[NB][KB]) {
    const int lq = lane & 31, hh = lane >> 5;
    f32x16 sc[NB][KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[nb][kb][i] = 0.f;
#pragma unroll
      for (int s = 0; s < D / 16; ++s) {
        const bf16x8 kf =
            *reinterpret_cast<const bf16x8*>(lk + (32 * kb + lq) * kKRow<D> + 16 * s + 8 * hh);
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
          sc[nb][kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[nb][s], sc[nb][kb], 0, 0, 0);
      }
    }
    // Lane (lq, hh) holds row lq's scores of keys 32 kb + 8 (i / 4) + 4 hh + i % 4.
    if (flip) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 16; ++i) sc[nb][kb][i] = -sc[nb][kb][i];
    }
    if (hides) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          const uint32_t w = see[nb][kb] >> (4 * hh);
#pragma unroll
          for (int i = 0; i < 16; ++i)
            sc[nb][kb][i] =
                w & (1u << (8 * (i / 4) + i % 4)) ? sc[nb][kb][i] : -__builtin_inff();
        }
    }
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float mx = sc[nb][0][0];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sc[nb][kb][i]);
      float x1, x2;
      xor_pair<32>(mx, x1, x2);
      const float mnew = fmaxf(m[nb], fmaxf(x1, x2) * sl);
      if (__ballot(mnew > m[nb])) {
        const float alpha = fast_exp2(m[nb] - mnew);
        l[nb] *= alpha;
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[nb][c][i] *= alpha;
        m[nb] = mnew;
      }
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          sc[nb][kb][i] = fast_exp2(fmaf(sc[nb][kb][i], sl, -m[nb]));
          l[nb] += sc[nb][kb][i];
          if (vs != 1.f) sc[nb][kb][i] *= vs;
        }
    }
    // P.V, 16 keys a step.  Half hh's eight operand slots are the keys 4 hh ..
    // + 3 and 8 + 4 hh .. + 3 of the step, and V is read in that order.  For
    // fp32 outputs the weights go in as three bf16 terms, which hold all their
    // 24 bits; for bf16 outputs rounded to one, off by half a step as the
    // outputs are.
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        constexpr int NE = F32 ? 3 : 1;
        bf16x8 pf[NB][NE];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          uint32_t w[NE][4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float u = sc[nb][kb][8 * s + 2 * j], v = sc[nb][kb][8 * s + 2 * j + 1];
            if constexpr (F32) {
#pragma unroll
              for (int e = 0; e < NE; ++e) {
                w[e][j] = high_halves(u, v);
                u -= __uint_as_float(__float_as_uint(u) & 0xffff0000u);
                v -= __uint_as_float(__float_as_uint(v) & 0xffff0000u);
              }
            } else {
              w[0][j] = pack_bf16(u, v);
            }
          }
#pragma unroll
          for (int e = 0; e < NE; ++e)
            pf[nb][e] = __builtin_bit_cast(bf16x8, make_uint4(w[e][0], w[e][1], w[e][2], w[e][3]));
        }
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          const uint2 va = vread(lv, lane, 32 * kb + 16 * s + 4 * hh, c);
          const uint2 vb = vread(lv, lane, 32 * kb + 16 * s + 8 + 4 * hh, c);
          const bf16x8 vf = __builtin_bit_cast(bf16x8, make_uint4(va.x, va.y, vb.x, vb.y));
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < NE; ++e)
              o[nb][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[nb][e], o[nb][c], 0, 0, 0);
        }
      }
  }

  // Adds the infinities and NaN of V row v to the rows that see its key: as
  // products of 1 and the largest bf16 values, whose sum overflows where it is
  // added, and of 0 where the key is hidden.  A NaN is both infinities.
  __device__ __forceinline__ void add_nonfinite(int lane, const uint16_t* v,
                                                const bool (&mine)[NB]) {
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      const uint32_t x = v[32 * c + (lane & 31)], size = x & 0x7fffu;
      const uint32_t up = x == 0x7f80u || size > 0x7f80u ? 0x7f7f7f7fu : 0u;
      const uint32_t down = x == 0xff80u || size > 0x7f80u ? 0xff7fff7fu : 0u;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const uint32_t one = mine[nb] ? 0x3f803f80u : 0u;
        const bf16x8 p = __builtin_bit_cast(bf16x8, make_uint4(one, one, one, one));
        o[nb][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            __builtin_bit_cast(bf16x8, make_uint4(up, up, up, up)), p, o[nb][c], 0, 0, 0);
        o[nb][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            __builtin_bit_cast(bf16x8, make_uint4(down, down, down, down)), p, o[nb][c], 0, 0, 0);
      }
    }
  }
};

// Scales of the scores and of V over the cache.  Scores are compared before they
// are scaled, so the scale is positive: a negative one flips the scores, a
// zero one is as good as the smallest.
struct CacheScale {
  float sl, vs;
  bool flip;
};
template <bool FP8>
__device__ __forceinline__ CacheScale cache_scale(const TreeArgs& a, int pair) {
  CacheScale c{a.scale_log2, 1.f, false};
  if constexpr (FP8) {
    if (a.ks) c.sl *= a.ks[pair];
    if (a.vs) c.vs = a.vs[pair];
    c.flip = c.sl < 0.f;
    c.sl = fmaxf(fabsf(c.sl), kTreeMinScale);
  }
  return c;
}

// In a tile with hidden keys a V row's infinity or NaN would reach queries that
// must not see it, as 0 times it.  Such elements become 0 in LDS, and
// add_nonfinite adds them where they are seen.  Each lane takes the N chunks of 16
// bytes it has just stored, chunk i at `v` + i * step, D / 8 lanes to a row;
// returns the rows that had any: bit i * (512 / D) + g for row g of pass i.  (A
// loop over LDS: the same on the registers before they are stored costs 20 more.)
template <int D>
__device__ __forceinline__ uint32_t clean_rows(uint16_t* v, int n, int step) {
  constexpr int CPR = D / 8, RPW = 64 / CPR;
  uint32_t rows = 0;
#pragma unroll 1
  for (int i = 0; i < n; ++i, v += step) {
    const uint4 x = *reinterpret_cast<const uint4*>(v);
    const bool mine = (nonfinite_bit(x) & 0x8000u) != 0;
    const uint64_t who = __ballot(mine);
    if (!who) continue;
    if (mine)
      *reinterpret_cast<uint4*>(v) =
          make_uint4(finite_pair(x.x), finite_pair(x.y), finite_pair(x.z), finite_pair(x.w));
#pragma unroll
    for (int g = 0; g < RPW; ++g)
      rows |= (who >> (g * CPR) & ((1ull << CPR) - 1)) ? 1u << (i * RPW + g) : 0u;
  }
  return rows;
}

// Outputs of a finished block of 32 rows, or its partial result.
template <int D, bool F32>
__device__ __forceinline__ void tree_write(const TreeArgs& a, int lane, const f32x16 (&o)[D / 32],
                                           float inv, int64_t out) {
  const int64_t at = out * D + 4 * (lane >> 5);
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int i = 0; i < 16; i += 4)
      store4<F32>(a.out, at + 32 * c + 2 * i, o[c][i] * inv, o[c][i + 1] * inv, o[c][i + 2] * inv,
                  o[c][i + 3] * inv);
}

// Splits of a row tile that have keys, and the tiles of 'part' of 'parts'.
__device__ __forceinline__ int tree_splits(const TreeArgs& a, int tiles) {
  return min(a.splits, (tiles + a.split_tiles - 1) / a.split_tiles);
}
__device__ __forceinline__ int tree_cut(int tiles, int part, int parts) {
  return static_cast<int>(static_cast<int64_t>(tiles) * part / parts);
}

// ---- many query rows -----------------------------------------------------------

constexpr int kTileRows = 128;  // query rows of a workgroup: four waves of 32
constexpr int kTileKeys = 64;   // keys of a tile

// A workgroup of four waves takes 128 query rows (node, query head of the KV
// head's group) of one request and KV head, and a share of the keys.  Tiles of
// 64 keys go through LDS for all four waves, two buffers in turn.
template <bool FP8, int D, bool F32>
__global__ __launch_bounds__(256, 2) void tree_tile_kernel(TreeArgs a) {
  constexpr int CPR = D / 8;           // 16-byte chunks of a bf16 row
  constexpr int NP = CPR * kTileKeys / 256;
  constexpr int RPP = 256 / CPR;       // rows per pass of the workgroup
  constexpr int CP8 = D / 16, NP8 = CP8 * kTileKeys / 256, RP8 = 256 / CP8;
  __shared__ __align__(16) uint16_t lk[2][kTileKeys * kKRow<D>];
  __shared__ __align__(16) uint16_t lv[2][kTileKeys * kVRow<D>];
  __shared__ uint32_t lbad[2][4];  // V rows of a tile that are not finite, by wave (clean_rows)

  const int per_pair = a.row_tiles * a.splits;
  const int item = xcd_item(a.B * a.Hkv * per_pair);
  if (item < 0) return;
  const int pair = item / per_pair, sub = item % per_pair;
  const int b = pair / a.Hkv, h = pair % a.Hkv;
  const int qt = sub / a.splits, sp = sub % a.splits;
  const TreeReq rq = tree_request(a.base, a.count, b, a.N, a.Lp, a.Ldec);
  const int rows = rq.n * a.G, r0 = qt * kTileRows;
  if (r0 >= rows) return;
  const int n0 = r0 / a.G, n1 = (min(r0 + kTileRows, rows) - 1) / a.G;
  const TreeKeys ks = tree_keys(a, rq, n0, n1);
  const int t_old = (ks.nold + kTileKeys - 1) / kTileKeys;
  const int tiles = t_old + (ks.nnew + kTileKeys - 1) / kTileKeys;
  const int nsp = tree_splits(a, tiles);
  if (sp >= nsp) return;
  const int t0 = tree_cut(tiles, sp, nsp), t1 = tree_cut(tiles, sp + 1, nsp);

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = r0 + 32 * wave + (lane & 31);
  const bool wave_on = r0 + 32 * wave < rows;
  const TreeRow my = tree_row(a, rq, ks, b, h, min(row, rows - 1));
  const int deepest = a.depth ? a.max_depth[b] : n1;
  const int sink = a.S - rq.base;
  const CacheScale cs = cache_scale<FP8>(a, pair);
  TreeWave<D, F32, 1> w;
  w.start(a, lane, 0,
          a.q + b * a.qsb + my.node * a.qsn + (h * a.G + min(row, rows - 1) % a.G) * a.qsh);

  const int64_t cbase = tree_cache_base(a, b, h, FP8 ? 1 : 2);
  const uint16_t* kn = a.kn + b * a.nsb + h * a.nsh;
  const uint16_t* vn = a.vn + b * a.nsb + h * a.nsh;
  uint4 rk[NP], rv[NP];

  // A tile of bf16 rows (new ones, or the cache's) into LDS.
  auto put = [&](int buf, bool hides) {
    const int c = tid % CPR;
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int r = i * RPP + tid / CPR;
      *reinterpret_cast<uint4*>(lk[buf] + r * kKRow<D> + (c) * 8) = rk[i];
      *reinterpret_cast<uint4*>(lv[buf] + r * kVRow<D> + (c) * 8) = rv[i];
    }
    uint32_t bad = 0;
    if (hides) bad = clean_rows<D>(lv[buf] + (tid / CPR) * kVRow<D> + c * 8, NP, RPP * kVRow<D>);
    if (lane == 0) lbad[buf][wave] = bad;
  };
  auto add_hidden = [&](int buf, const uint32_t (&see)[1][2], auto&& row_of) {
    constexpr int RPW = 64 / CPR;  // rows of a wave's pass
#pragma unroll 1
    for (int i = 0; i < 4; ++i)
#pragma unroll 1
      for (uint32_t bad = lbad[buf][i]; bad; bad &= bad - 1) {
        const int at = __builtin_ctz(bad), e = at / RPW * RPP + i * RPW + at % RPW;
        const bool mine[1] = {static_cast<bool>((see[0][e >> 5] >> (e & 31)) & 1u)};
        w.add_nonfinite(lane, row_of(e), mine);
      }
  };

  // The cache's tiles.
  auto load_old = [&](int t) {
    constexpr int N = FP8 ? NP8 : NP, R = FP8 ? RP8 : RPP, C = FP8 ? CP8 : CPR;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = min(t * kTileKeys + i * R + tid / C, ks.nold - 1);
      const int64_t at = cbase + ks.row(r) * a.sr + (tid % C) * 16;
      rk[i] = load_stream16(a.k + at);
      rv[i] = load_stream16(a.v + at);
    }
  };
  auto hides_old = [&](int t) {
    return hides_cached(a, rq, ks, t * kTileKeys, kTileKeys, deepest);
  };
  auto put_old = [&](int t, int buf) {
    if constexpr (FP8) {
#pragma unroll
      for (int i = 0; i < NP8; ++i) {
        const int r = i * RP8 + tid / CP8, c = 2 * (tid % CP8);
        uint4 lo, hi;
        widen_fp8(rk[i], lo, hi);
        *reinterpret_cast<uint4*>(lk[buf] + r * kKRow<D> + (c) * 8) = lo;
        *reinterpret_cast<uint4*>(lk[buf] + r * kKRow<D> + (c + 1) * 8) = hi;
        widen_fp8(rv[i], lo, hi);
        *reinterpret_cast<uint4*>(lv[buf] + r * kVRow<D> + (c) * 8) = lo;
        *reinterpret_cast<uint4*>(lv[buf] + r * kVRow<D> + (c + 1) * 8) = hi;
      }
    } else {
      put(buf, hides_old(t));
    }
  };
  int t = t0, buf = 0;
  const int e_old = min(t1, t_old);
  if (t < e_old) {
    load_old(t);
    put_old(t, 0);
    __syncthreads();
    for (; t < e_old; ++t, buf ^= 1) {
      if (t + 1 < e_old) load_old(t + 1);
      if (wave_on) {
        const bool hides = hides_old(t);
        uint32_t see[1][2] = {};
        if (hides) {
          see[0][0] = see_cached(ks, my, t * kTileKeys);
          see[0][1] = see_cached(ks, my, t * kTileKeys + 32);
        }
        w.template tile<2>(lane, lk[buf], lv[buf], cs.sl, FP8 && cs.flip, FP8 ? cs.vs : 1.f, hides,
                           see);
        if (!FP8 && hides)
          add_hidden(buf, see, [&](int e) {
            return reinterpret_cast<const uint16_t*>(a.v + cbase + ks.row(t * kTileKeys + e) * a.sr);
          });
      }
      if (t + 1 < e_old) put_old(t + 1, buf ^ 1);
      __syncthreads();
    }
  }

  // The new tokens' tiles.
  auto load_new = [&](int x0) {
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int x = min(x0 + i * RPP + tid / CPR, ks.nnew - 1);
      const int64_t at = ks.node(x) * a.nsn + (tid % CPR) * 8;
      rk[i] = *reinterpret_cast<const uint4*>(kn + at);
      rv[i] = *reinterpret_cast<const uint4*>(vn + at);
    }
  };
  auto hides_at = [&](int x) { return hides_new(a, ks, x, kTileKeys, n0, n1); };
  if (t < t1) {
    const int end = (t1 - t_old) * kTileKeys;
    int x = (t - t_old) * kTileKeys;
    load_new(x);
    put(buf, hides_at(x));
    __syncthreads();
    for (; x < end; x += kTileKeys, buf ^= 1) {
      if (x + kTileKeys < end) load_new(x + kTileKeys);
      if (wave_on) {
        const bool hides = hides_at(x);
        uint32_t see[1][2] = {};
        if (hides) {
          see[0][0] = see_new(a, ks, my, b, x, sink, deepest >= a.W);
          see[0][1] = see_new(a, ks, my, b, x + 32, sink, deepest >= a.W);
        }
        w.template tile<2>(lane, lk[buf], lv[buf], a.scale_log2, false, 1.f, hides, see);
        if (hides)
          add_hidden(buf, see, [&](int e) { return vn + ks.node(x + e) * a.nsn; });
      }
      if (x + kTileKeys < end) put(buf ^ 1, hides_at(x + kTileKeys));
      __syncthreads();
    }
  }

  float l1, l2;
  xor_pair<32>(w.l[0], l1, l2);
  const float l = l1 + l2;
  if (row >= rows) return;
  if (nsp == 1) {
    tree_write<D, F32>(a, lane, w.o[0], 1.f / l, my.out);
    return;
  }
  float* part = a.part + ((static_cast<int64_t>(pair) * a.row_tiles + qt) * a.splits + sp) *
                             kTileRows * kPartRow<D> +
                (row - r0) * kPartRow<D>;
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int i = 0; i < 16; i += 4)
      *reinterpret_cast<float4*>(part + 32 * c + 2 * i + 4 * (lane >> 5)) =
          make_float4(w.o[0][c][i], w.o[0][c][i + 1], w.o[0][c][i + 2], w.o[0][c][i + 3]);
  if (lane < 32) *reinterpret_cast<float2*>(part + D) = make_float2(w.m[0], l);
}

// ---- few query rows --------------------------------------------------------------

constexpr int kStreamKeys = 32;  // keys of a wave's tile

template <int D>
constexpr uint32_t kStreamLds = kStreamKeys * (kKRow<D> + kVRow<D>) * 2;  // a wave's K and V tile, bytes

// At most 32 NB query rows per (request, KV head): bound by the cache's bytes.
// Every wave streams tiles of 32 keys of its own for all rows, through registers
// (the next tiles are on their way while one is computed) and an LDS region of
// its own, so the waves of a workgroup wait for each other only to join
// their results at the end.
template <bool FP8, int D, bool F32, int NB, int NW>
__global__ __launch_bounds__(64 * NW, NB == 1 ? 2 : 1) void tree_stream_kernel(TreeArgs a) {
  constexpr int CPR = D / 8, RPP = 64 / CPR, NP = kStreamKeys / RPP;  // bf16 rows
  constexpr int C = FP8 ? D / 16 : CPR, R = 64 / C, N = kStreamKeys / R;  // the cache's
  constexpr int PF = N > 4 ? 1 : 2;  // tiles in flight ahead of the one at hand
  __shared__ __align__(16) uint16_t lds[NW * (kStreamLds<D> / 2)];
  __shared__ float lm[NW][32], ll[NW][32];

  const int item = xcd_item(a.B * a.Hkv * a.splits);
  if (item < 0) return;
  const int pair = item / a.splits, sp = item % a.splits;
  const int b = pair / a.Hkv, h = pair % a.Hkv;
  const TreeReq rq = tree_request(a.base, a.count, b, a.N, a.Lp, a.Ldec);
  const int rows = rq.n * a.G;
  if (rows == 0) return;
  const int n1 = rq.n - 1;
  const TreeKeys ks = tree_keys(a, rq, 0, n1);
  const int t_old = (ks.nold + kStreamKeys - 1) / kStreamKeys;
  const int tiles = t_old + (ks.nnew + kStreamKeys - 1) / kStreamKeys;
  const int nsp = tree_splits(a, tiles);
  if (sp >= nsp) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t0 = tree_cut(tiles, sp * NW + wave, nsp * NW);
  const int t1 = tree_cut(tiles, sp * NW + wave + 1, nsp * NW);

  uint16_t* lk = lds + wave * (kStreamLds<D> / 2);
  uint16_t* lv = lk + kStreamKeys * kKRow<D>;
  const int64_t cbase = tree_cache_base(a, b, h, FP8 ? 1 : 2);
  uint4 rk[PF][N], rv[PF][N];
  auto load_old = [&](int t, uint4 (&k)[N], uint4 (&v)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int r = min(t * kStreamKeys + i * R + lane / C, ks.nold - 1);
      const int64_t at = cbase + ks.row(r) * a.sr + (lane % C) * 16;
      k[i] = load_stream16(a.k + at);
      v[i] = load_stream16(a.v + at);
    }
  };
  const int e_old = min(t1, t_old);
#pragma unroll
  for (int j = 0; j < PF; ++j)
    if (t0 + j < e_old) load_old(t0 + j, rk[j], rv[j]);

  TreeRow my[NB];
  TreeWave<D, F32, NB> w;
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int row = min(32 * nb + (lane & 31), rows - 1);
    my[nb] = tree_row(a, rq, ks, b, h, row);
    w.start(a, lane, nb,
            a.q + b * a.qsb + my[nb].node * a.qsn + (h * a.G + row % a.G) * a.qsh);
  }
  const int deepest = a.depth ? a.max_depth[b] : n1;
  const CacheScale cs = cache_scale<FP8>(a, pair);

  auto add_hidden = [&](uint32_t bad, const uint32_t (&see)[NB][1], auto&& row_of) {
#pragma unroll 1
    for (; bad; bad &= bad - 1) {
      const int e = __builtin_ctz(bad);
      bool mine[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) mine[nb] = (see[nb][0] >> e) & 1u;
      w.add_nonfinite(lane, row_of(e), mine);
    }
  };

  for (int t = t0; t < e_old; t += PF) {
#pragma unroll
    for (int j = 0; j < PF; ++j) {
      if (t + j >= e_old) break;
      const int e0 = (t + j) * kStreamKeys;
      const bool hides = hides_cached(a, rq, ks, e0, kStreamKeys, deepest);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int r = i * R + lane / C;
        if constexpr (FP8) {
          const int c = 2 * (lane % C);
          uint4 lo, hi;
          widen_fp8(rk[j][i], lo, hi);
          *reinterpret_cast<uint4*>(lk + r * kKRow<D> + (c) * 8) = lo;
          *reinterpret_cast<uint4*>(lk + r * kKRow<D> + (c + 1) * 8) = hi;
          widen_fp8(rv[j][i], lo, hi);
          *reinterpret_cast<uint4*>(lv + r * kVRow<D> + (c) * 8) = lo;
          *reinterpret_cast<uint4*>(lv + r * kVRow<D> + (c + 1) * 8) = hi;
        } else {
          *reinterpret_cast<uint4*>(lk + r * kKRow<D> + (lane % C) * 8) = rk[j][i];
          *reinterpret_cast<uint4*>(lv + r * kVRow<D> + (lane % C) * 8) = rv[j][i];
        }
      }
      if (t + j + PF < e_old) load_old(t + j + PF, rk[j], rv[j]);
      uint32_t bad = 0;
      if (!FP8 && hides) bad = clean_rows<D>(lv + (lane / C) * kVRow<D> + (lane % C) * 8, N, R * kVRow<D>);
      fence_wave();
      uint32_t see[NB][1] = {};
      if (hides)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) see[nb][0] = see_cached(ks, my[nb], e0);
      w.template tile<1>(lane, lk, lv, cs.sl, FP8 && cs.flip, FP8 ? cs.vs : 1.f, hides, see);
      if (!FP8 && bad)
        add_hidden(bad, see, [&](int e) {
          return reinterpret_cast<const uint16_t*>(a.v + cbase + ks.row(e0 + e) * a.sr);
        });
      fence_wave();
    }
  }

  const uint16_t* kn = a.kn + b * a.nsb + h * a.nsh;
  const uint16_t* vn = a.vn + b * a.nsb + h * a.nsh;
  for (int t = max(t0, t_old); t < t1; ++t) {
    const int x0 = (t - t_old) * kStreamKeys;
    uint4 k[NP], v[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int x = min(x0 + i * RPP + lane / CPR, ks.nnew - 1);
      const int64_t at = ks.node(x) * a.nsn + (lane % CPR) * 8;
      k[i] = *reinterpret_cast<const uint4*>(kn + at);
      v[i] = *reinterpret_cast<const uint4*>(vn + at);
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int r = i * RPP + lane / CPR;
      *reinterpret_cast<uint4*>(lk + r * kKRow<D> + (lane % CPR) * 8) = k[i];
      *reinterpret_cast<uint4*>(lv + r * kVRow<D> + (lane % CPR) * 8) = v[i];
    }
    const uint32_t bad =
        clean_rows<D>(lv + (lane / CPR) * kVRow<D> + (lane % CPR) * 8, NP, RPP * kVRow<D>);
    fence_wave();
    uint32_t see[NB][1];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
      see[nb][0] = see_new(a, ks, my[nb], b, x0, a.S - rq.base, deepest >= a.W);
    w.template tile<1>(lane, lk, lv, a.scale_log2, false, 1.f, true, see);
    add_hidden(bad, see, [&](int e) { return vn + ks.node(x0 + e) * a.nsn; });
    fence_wave();
  }

  // Join the waves' results, a block of rows at a time: every wave scales its own
  // to the common maximum and leaves them in its LDS region, 32 columns of a row
  // per step, then the workgroup's threads add them up.
  const bool split = nsp > 1;
  float* part = a.part + (static_cast<int64_t>(pair) * a.splits + sp) * (32 * NB) * kPartRow<D>;
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    float l1, l2;
    xor_pair<32>(w.l[nb], l1, l2);
    if (lane < 32) {
      lm[wave][lane] = w.m[nb];
      ll[wave][lane] = l1 + l2;
    }
    __syncthreads();
    float M = kTreeMin;
#pragma unroll
    for (int i = 0; i < NW; ++i) M = fmaxf(M, lm[i][lane & 31]);
    const float mine = fast_exp2(w.m[nb] - M);
    float* red = reinterpret_cast<float*>(lk);  // [32 rows][D], groups of 4 columns swizzled
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int g = 8 * c + i / 2 + (lane >> 5), r = lane & 31;
        *reinterpret_cast<float4*>(red + r * D + ((g ^ (r & 15)) * 4)) =
            make_float4(w.o[nb][c][i] * mine, w.o[nb][c][i + 1] * mine, w.o[nb][c][i + 2] * mine,
                        w.o[nb][c][i + 3] * mine);
      }
    __syncthreads();
    for (int at = threadIdx.x; at < 32 * (D / 4); at += 64 * NW) {
      const int r = at / (D / 4), g = at % (D / 4), row = 32 * nb + r;
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
      if (split) {
        float* p = part + row * kPartRow<D>;
        *reinterpret_cast<float4*>(p + 4 * g) = s;
        if (g == 0) *reinterpret_cast<float2*>(p + D) = make_float2(mr, lr);
      } else {
        const float inv = 1.f / lr;
        const int64_t out = (static_cast<int64_t>(b) * a.N + row / a.G) * a.Hq + h * a.G + row % a.G;
        store4<F32>(a.out, out * D + 4 * g, s.x * inv, s.y * inv, s.z * inv, s.w * inv);
      }
    }
    if (nb + 1 < NB) __syncthreads();
  }
}

// Joins a row's splits: out = sum_s 2^(m_s - M) acc_s / sum_s 2^(m_s - M) l_s.
// One wave per query row.
template <int D, bool F32>
__global__ __launch_bounds__(256) void tree_combine_kernel(TreeArgs a, int tile_rows,
                                                           int tile_keys) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x & 63;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int per_pair = a.row_tiles * tile_rows;
  const int pair = static_cast<int>(at / per_pair), row = static_cast<int>(at % per_pair);
  if (pair >= a.B * a.Hkv) return;
  const int b = pair / a.Hkv, h = pair % a.Hkv, qt = row / tile_rows;
  const TreeReq rq = tree_request(a.base, a.count, b, a.N, a.Lp, a.Ldec);
  const int rows = rq.n * a.G, r0 = qt * tile_rows;
  if (row >= rows) return;
  const TreeKeys ks = tree_keys(a, rq, r0 / a.G, (min(r0 + tile_rows, rows) - 1) / a.G);
  const int tiles = (ks.nold + tile_keys - 1) / tile_keys + (ks.nnew + tile_keys - 1) / tile_keys;
  const int nsp = tree_splits(a, tiles);
  if (nsp <= 1) return;
  const int64_t step = static_cast<int64_t>(tile_rows) * kPartRow<D>;
  const float* part = a.part + (static_cast<int64_t>(pair) * a.row_tiles + qt) * a.splits * step +
                      (row - r0) * kPartRow<D>;
  float M = kTreeMin;
  for (int s = 0; s < nsp; ++s) M = fmaxf(M, part[s * step + D]);
  float L = 0.f, acc[E] = {};
  for (int s = 0; s < nsp; ++s) {
    const float* x = part + s * step;
    const float w = fast_exp2(x[D] - M);
    L = fmaf(x[D + 1], w, L);
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = fmaf(x[lane * E + e], w, acc[e]);
  }
  const float inv = 1.f / L;
  const int64_t to = ((static_cast<int64_t>(b) * a.N + row / a.G) * a.Hq + h * a.G + row % a.G) * D +
                     lane * E;
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

template <bool FP8, int D, bool F32, int NB, int NW>
hipError_t launch_stream(const TreeLaunch& l, const TreeArgs& a, hipStream_t st) {
  tree_stream_kernel<FP8, D, F32, NB, NW><<<dim3(static_cast<uint32_t>((l.workgroups + 7) / 8 * 8)),
                                            dim3(64 * NW), 0, st>>>(a);
  return hipGetLastError();
}

template <bool FP8, int D, bool F32>
hipError_t launch_one(const TreeLaunch& l, const TreeArgs& a, hipStream_t st) {
  hipError_t e;
  if (l.rows > 64) {
    tree_tile_kernel<FP8, D, F32><<<dim3(static_cast<uint32_t>((l.workgroups + 7) / 8 * 8)),
                                    dim3(256), 0, st>>>(a);
    e = hipGetLastError();
  } else if (l.rows > 32) {
    e = launch_stream<FP8, D, F32, 2, 4>(l, a, st);
  } else {
    e = l.waves == 8 ? launch_stream<FP8, D, F32, 1, 8>(l, a, st)
                     : launch_stream<FP8, D, F32, 1, 4>(l, a, st);
  }
  if (e != hipSuccess || l.splits == 1) return e;
  const int64_t waves = static_cast<int64_t>(a.B) * a.Hkv * a.row_tiles * l.rows;
  tree_combine_kernel<D, F32><<<dim3(static_cast<uint32_t>((waves + 3) / 4)), dim3(256), 0, st>>>(
      a, l.rows, l.keys);
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
