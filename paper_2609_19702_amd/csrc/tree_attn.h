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


constexpr int kTileRows = 128;  // query rows of a workgroup: four waves of 32
constexpr int kTileKeys = 64;   // keys of a tile

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {  // nearest even
  const f32x2 x = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}

// High halves of two fp32 values as a bf16 pair (truncation).
__device__ __forceinline__ uint32_t high_halves(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}

__device__ __forceinline__ bool has_nonfinite(const uint4& x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    bad |= (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
  return bad;
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

// A workgroup of four waves takes 128 query rows (node, query head of the KV
// head's group) of one request and KV head, and a share of the keys.  Tiles of
// 64 keys go through LDS, two buffers in turn.  Both products run on the matrix
// cores with the keys as rows, S^T = K Q^T and O^T = V^T P^T
// (v_mfma_f32_32x32x16_bf16): a lane then holds scores, weights and outputs of
// one query row (lane % 32) only, so the running maximum and the rescale need
// no exchange but one with the lane's other half, and the weights are the second
// product's operand where they are.  V comes back from LDS transposed
// (ds_read_b64_tr_b16) in the key order the weights have.
template <bool FP8, int D, bool F32>
__global__ __launch_bounds__(256, FP8 && D == 128 ? 1 : 2) void tree_tile_kernel(TreeArgs a) {
  constexpr int CPR = D / 8;           // 16-byte chunks of a bf16 row
  constexpr int NP = CPR * kTileKeys / 256;
  constexpr int RPP = 256 / CPR;       // rows per pass of the workgroup
  constexpr int CP8 = D / 16, NP8 = CP8 * kTileKeys / 256, RP8 = 256 / CP8;
  __shared__ __align__(16) uint16_t lk[2][kTileKeys * D];
  __shared__ __align__(16) uint16_t lv[2][kTileKeys * D];
  __shared__ uint64_t lbad[2][4];  // keys of a tile whose V row is not finite, by wave

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
  const int nsp = min(a.splits, tiles);
  if (sp >= nsp) return;
  const int t0 = static_cast<int>(static_cast<int64_t>(tiles) * sp / nsp);
  const int t1 = static_cast<int>(static_cast<int64_t>(tiles) * (sp + 1) / nsp);

  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int lq = lane & 31, hh = lane >> 5;
  const int row = r0 + 32 * wave + lq;
  const bool wave_on = r0 + 32 * wave < rows;
  const int node = min(row, rows - 1) / a.G, head = h * a.G + min(row, rows - 1) % a.G;
  const bool chain = a.depth == nullptr;
  const int dep = chain ? node : a.depth[b * a.N + node];
  const int deepest = chain ? n1 : a.max_depth[b];
  const int p = rq.base + dep;
  const int thr = ks.pre + p - a.W - ks.j0;                       // cached entries past pre: visible above
  const int thr_max = ks.pre + rq.base + deepest - a.W - ks.j0;
  const int sink_node = a.S - rq.base;                            // depths below stand at sink positions
  const uint32_t* anc = chain ? nullptr : a.anc + (static_cast<int64_t>(b) * a.N + node) * a.words;
  const int32_t* depths = chain ? nullptr : a.depth + static_cast<int64_t>(b) * a.N;

  // Scores are compared before they are scaled, so scales are positive here: a
  // negative one flips the scores, a zero one is as good as the smallest.
  float kscale = a.scale_log2, vscale = 1.f;
  bool flip = false;
  if constexpr (FP8) {
    if (a.ks) kscale *= a.ks[pair];
    if (a.vs) vscale = a.vs[pair];
    flip = kscale < 0.f;
    kscale = fmaxf(fabsf(kscale), kTreeMinScale);
  }

  // Queries: the second operand of S^T, lane (row lq, elements 16 s + 8 hh ..).
  bf16x8 qf[D / 16];
  {
    const uint16_t* q = a.q + b * a.qsb + node * a.qsn + head * a.qsh;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      uint4 x = *reinterpret_cast<const uint4*>(q + 16 * s + 8 * hh);
      x.x ^= a.q_sign;
      x.y ^= a.q_sign;
      x.z ^= a.q_sign;
      x.w ^= a.q_sign;
      qf[s] = __builtin_bit_cast(bf16x8, x);
    }
  }

  const int64_t cbase = tree_cache_base(a, b, h, FP8 ? 1 : 2);
  const uint16_t* kn = a.kn + b * a.nsb + h * a.nsh;
  const uint16_t* vn = a.vn + b * a.nsb + h * a.nsh;
  uint4 rk[NP], rv[NP];
  const uint4 zero = make_uint4(0, 0, 0, 0);
  auto load = [&](int t) {
    if (t < t_old) {
      if constexpr (FP8) {
#pragma unroll
        for (int i = 0; i < NP8; ++i) {
          const int r = t * kTileKeys + i * RP8 + tid / CP8;
          rk[i] = rv[i] = zero;
          if (r < ks.nold) {
            const int64_t at = cbase + ks.row(r) * a.sr + (tid % CP8) * 16;
            rk[i] = load_stream16(a.k + at);
            rv[i] = load_stream16(a.v + at);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < NP; ++i) {
          const int r = t * kTileKeys + i * RPP + tid / CPR;
          rk[i] = rv[i] = zero;
          if (r < ks.nold) {
            const int64_t at = cbase + ks.row(r) * a.sr + (tid % CPR) * 16;
            rk[i] = load_stream16(a.k + at);
            rv[i] = load_stream16(a.v + at);
          }
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const int x = (t - t_old) * kTileKeys + i * RPP + tid / CPR;
        rk[i] = rv[i] = zero;
        if (x < ks.nnew) {
          const int64_t at = ks.node(x) * a.nsn + (tid % CPR) * 8;
          rk[i] = *reinterpret_cast<const uint4*>(kn + at);
          rv[i] = *reinterpret_cast<const uint4*>(vn + at);
        }
      }
    }
  };
  // Chunk c of row r lies at chunk c ^ (r mod CPR) of its row: rows start at
  // the same banks, and the lanes of a read go down the rows.
  auto put = [&](uint16_t* buf, int r, int c, const uint4& x) {
    *reinterpret_cast<uint4*>(buf + r * D + ((c ^ (r & (CPR - 1))) * 8)) = x;
  };
  // Whether some query of the workgroup must not see some key of tile t.
  auto masked = [&](int t) {
    if (t < t_old) {
      const int r = t * kTileKeys;
      return r + kTileKeys > ks.nold || (r + kTileKeys > ks.pre && max(r, ks.pre) <= thr_max);
    }
    const int x = (t - t_old) * kTileKeys;
    return !chain || !(x + kTileKeys <= ks.a0 ||
                       (x >= ks.a0 && x + kTileKeys <= ks.nnew &&
                        ks.node(x + kTileKeys - 1) <= n0 && ks.node(x) > n1 - a.W));
  };
  auto store = [&](int t, int buf) {
    if (FP8 && t < t_old) {
#pragma unroll
      for (int i = 0; i < NP8; ++i) {
        const int r = i * RP8 + tid / CP8, c = 2 * (tid % CP8);
        uint4 lo, hi;
        widen_fp8(rk[i], lo, hi);
        put(lk[buf], r, c, lo);
        put(lk[buf], r, c + 1, hi);
        widen_fp8(rv[i], lo, hi);
        put(lv[buf], r, c, lo);
        put(lv[buf], r, c + 1, hi);
      }
      if (lane == 0) lbad[buf][wave] = 0;
      return;
    }
    // In a tile with hidden keys a V row's infinity or NaN would reach queries
    // that must not see it, as 0 times it.  Such elements go in as 0, and
    // compute() adds them where they are seen.
    uint64_t bad = 0;
    if (masked(t)) {
#pragma unroll
      for (int i = 0; i < NP; ++i) {
        const bool mine = has_nonfinite(rv[i]);
        const uint64_t who = __ballot(mine);
        if (who) {
          if (mine)
            rv[i] = make_uint4(finite_pair(rv[i].x), finite_pair(rv[i].y), finite_pair(rv[i].z),
                               finite_pair(rv[i].w));
#pragma unroll 1
          for (int g = 0; g < 64 / CPR; ++g)
            if (who >> (g * CPR) & ((1ull << CPR) - 1))
              bad |= 1ull << (i * RPP + wave * (64 / CPR) + g);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int r = i * RPP + tid / CPR, c = tid % CPR;
      put(lk[buf], r, c, rk[i]);
      put(lv[buf], r, c, rv[i]);
    }
    if (lane == 0) lbad[buf][wave] = bad;
  };

  f32x16 o[D / 32];
#pragma unroll
  for (int c = 0; c < D / 32; ++c)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[c][i] = 0.f;
  float m = kTreeMin, l = 0.f;

  // Transposed V reads: see the two row orders in the comment above pv.
  const int s16 = lane & 15;
  auto vread = [&](const uint16_t* buf, int key, int c) {  // 4 keys from `key`, 16 columns
    const int r = key + (s16 >> 2);
    const int ch = 4 * c + 2 * ((lane >> 4) & 1) + ((s16 & 3) >> 1);
    return __builtin_bit_cast(
        uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                   (__attribute__((address_space(3))) s16x4*)(
                       buf + r * D + ((ch ^ (r & (CPR - 1))) * 8) + 4 * (s16 & 1))));
  };

  auto compute = [&](int t, int buf) {
    f32x16 sc[2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[kb][i] = 0.f;
      const int r = 32 * kb + lq;
#pragma unroll
      for (int s = 0; s < D / 16; ++s) {
        const bf16x8 kf = *reinterpret_cast<const bf16x8*>(
            lk[buf] + r * D + (((2 * s + hh) ^ (r & (CPR - 1))) * 8));
        sc[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[s], sc[kb], 0, 0, 0);
      }
    }
    // Lane (lq, hh) holds row lq's scores of keys 32 kb + 8 (i / 4) + 4 hh + i % 4.
    const bool old = t < t_old;
    const float sl = FP8 && old ? kscale : a.scale_log2;
    const bool hides = masked(t);
    if (FP8 && old && flip) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[kb][i] = -sc[kb][i];
    }
    uint32_t see[2] = {~0u, ~0u};
    if (hides) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) {
        if (old) {
          const int e = t * kTileKeys + 32 * kb;
          see[kb] = low_bits(ks.nold - e) & (low_bits(ks.pre - e) | ~low_bits(thr + 1 - e));
        } else {
          const int e = (t - t_old) * kTileKeys + 32 * kb;
          see[kb] = low_bits(ks.nnew - e);
          if (chain) {  // nodes from a1 on follow the first a0, which every node sees
            const int f = ks.a0 - ks.a1 - e;
            see[kb] &= low_bits(node + 1 + f) & (low_bits(ks.a0 - e) | low_bits(sink_node + f) |
                                                 ~low_bits(node - a.W + 1 + f));
          } else {
            uint32_t m = e / 32 < a.words ? anc[e / 32] : 0u;
            see[kb] &= m;
            if (deepest >= a.W) {
              m = see[kb];
              while (m) {
                const int i = __builtin_ctz(m), de = depths[e + i];
                m &= m - 1;
                if (de >= sink_node && dep - de >= a.W) see[kb] &= ~(1u << i);
              }
            }
          }
        }
        const uint32_t w = see[kb] >> (4 * hh);
#pragma unroll
        for (int i = 0; i < 16; ++i)
          sc[kb][i] = w & (1u << (8 * (i / 4) + i % 4)) ? sc[kb][i] : -__builtin_inff();
      }
    }
    float mx = sc[0][0];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sc[kb][i]);
    float x1, x2;
    xor_pair<32>(mx, x1, x2);
    const float mnew = fmaxf(m, fmaxf(x1, x2) * sl);
    if (__ballot(mnew > m)) {
      const float alpha = fast_exp2(m - mnew);
      l *= alpha;
#pragma unroll
      for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[c][i] *= alpha;
      m = mnew;
    }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        sc[kb][i] = fast_exp2(fmaf(sc[kb][i], sl, -m));
        l += sc[kb][i];
        if (FP8) sc[kb][i] *= old ? vscale : 1.f;
      }
    // P.V.  A step takes 16 keys; the weights' order gives half hh's eight
    // operand slots the keys 4 hh .. + 3 and 8 + 4 hh .. + 3 of the step, and V
    // is read in the same order.
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        bf16x8 pf[F32 ? 3 : 1];
        if constexpr (F32) {
          uint32_t w[3][4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float u = sc[kb][8 * s + 2 * j], v = sc[kb][8 * s + 2 * j + 1];
#pragma unroll
            for (int e = 0; e < 3; ++e) {
              w[e][j] = high_halves(u, v);
              u -= __uint_as_float(__float_as_uint(u) & 0xffff0000u);
              v -= __uint_as_float(__float_as_uint(v) & 0xffff0000u);
            }
          }
#pragma unroll
          for (int e = 0; e < 3; ++e)
            pf[e] = __builtin_bit_cast(bf16x8, make_uint4(w[e][0], w[e][1], w[e][2], w[e][3]));
        } else {
          uint32_t w[4];
#pragma unroll
          for (int j = 0; j < 4; ++j)
            w[j] = pack_bf16(sc[kb][8 * s + 2 * j], sc[kb][8 * s + 2 * j + 1]);
          pf[0] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
        }
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          const uint2 va = vread(lv[buf], 32 * kb + 16 * s + 4 * hh, c);
          const uint2 vb = vread(lv[buf], 32 * kb + 16 * s + 8 + 4 * hh, c);
          const bf16x8 vf = __builtin_bit_cast(bf16x8, make_uint4(va.x, va.y, vb.x, vb.y));
#pragma unroll
          for (int e = 0; e < (F32 ? 3 : 1); ++e)
            o[c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf[e], o[c], 0, 0, 0);
        }
      }
    if (!hides) return;
    uint64_t bad = lbad[buf][0] | lbad[buf][1] | lbad[buf][2] | lbad[buf][3];
#pragma unroll 1
    for (; bad; bad &= bad - 1) {
      const int e = __builtin_ctzll(bad), at = (old ? t : t - t_old) * kTileKeys + e;
      const bool mine = (see[e >> 5] >> (e & 31)) & 1u;
      const uint16_t* vr = old ? reinterpret_cast<const uint16_t*>(a.v + cbase + ks.row(at) * a.sr)
                               : vn + ks.node(at) * a.nsn;
#pragma unroll
      for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const uint2 x = *reinterpret_cast<const uint2*>(vr + 32 * c + 2 * i + 4 * hh);
          const float f[4] = {bf16_lo(x.x), bf16_hi(x.x), bf16_lo(x.y), bf16_hi(x.y)};
#pragma unroll
          for (int j = 0; j < 4; ++j)
            o[c][i + j] += mine && !__builtin_isfinite(f[j]) ? f[j] : 0.f;
        }
    }
  };

  load(t0);
  store(t0, 0);
  __syncthreads();
  for (int t = t0; t < t1; ++t) {
    const int buf = (t - t0) & 1;
    if (t + 1 < t1) load(t + 1);
    if (wave_on) compute(t, buf);
    if (t + 1 < t1) store(t + 1, buf ^ 1);
    __syncthreads();
  }

  float l1, l2;
  xor_pair<32>(l, l1, l2);
  l = l1 + l2;
  if (row >= rows) return;
  if (nsp == 1) {
    const float inv = 1.f / l;
    const int64_t at = ((static_cast<int64_t>(b) * a.N + node) * a.Hq + head) * D + 4 * hh;
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        store4<F32>(a.out, at + 32 * c + 2 * i, o[c][i] * inv, o[c][i + 1] * inv,
                    o[c][i + 2] * inv, o[c][i + 3] * inv);
  } else {
    float* part = a.part + ((static_cast<int64_t>(pair) * a.row_tiles + qt) * a.splits + sp) *
                               kTileRows * kPartRow<D> +
                  (row - r0) * kPartRow<D>;
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<float4*>(part + 32 * c + 2 * i + 4 * hh) =
            make_float4(o[c][i], o[c][i + 1], o[c][i + 2], o[c][i + 3]);
    if (hh == 0) *reinterpret_cast<float2*>(part + D) = make_float2(m, l);
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
  const int nsp = min(a.splits, tiles);
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

template <bool FP8, int D, bool F32>
hipError_t launch_one(const TreeLaunch& l, const TreeArgs& a, hipStream_t st) {
  tree_tile_kernel<FP8, D, F32><<<dim3(static_cast<uint32_t>((l.workgroups + 7) / 8 * 8)),
                                  dim3(256), 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || l.splits == 1) return e;
  const int64_t waves = static_cast<int64_t>(a.B) * a.Hkv * a.row_tiles * l.rows;
  tree_combine_kernel<D, F32><<<dim3(static_cast<uint32_t>((waves + 3) / 4)), dim3(256), 0, st>>>(
      a, l.rows, kTileKeys);
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
