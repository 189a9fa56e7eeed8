// Attention of one token per request over a cache in pages
// (dsa_paged_attention), as templates over the cache's element type.
#pragma once

#include "device.h"
#include "paged.h"

namespace dsa {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

constexpr float kLowest = -3.402823466e38f;  // "no score yet": no finite score is below
constexpr int kTile = 32;                    // rows of a wave's tile
constexpr int kPad = 16;  // V rows in LDS are D + kPad bf16 apart: four of them in distinct banks

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {  // nearest even
  const f32x2 x = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}

// Eight elements of a row as bf16, from 16 (bf16) or 8 (fp8) of its bytes.  Every
// E4M3 value is a bf16 value.
__device__ __forceinline__ bf16x8 widen_e4m3(uint32_t a, uint32_t b) {
  const auto x0 = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(a), false);
  const auto x1 = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(a), true);
  const auto x2 = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(b), false);
  const auto x3 = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(b), true);
  auto high = [](float lo, float hi) {
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
  };
  return __builtin_bit_cast(bf16x8, make_uint4(high(x0[0], x0[1]), high(x1[0], x1[1]),
                                               high(x2[0], x2[1]), high(x3[0], x3[1])));
}
template <bool FP8>
__device__ __forceinline__ bf16x8 to_bf16(const uint4& r, int half) {
  if constexpr (FP8)
    return half ? widen_e4m3(r.z, r.w) : widen_e4m3(r.x, r.y);
  else
    return __builtin_bit_cast(bf16x8, r);
}

// Rows of a request that its step attends: its prompt, then decode rows.
struct PagedRows {
  int n, t, front;  // rows, decode position, prompt rows
};

__device__ __forceinline__ PagedRows paged_rows(const PagedArgs& a, int b, int pair) {
  PagedRows r{0, -1, 0};
  const int pos = a.pos[b];
  if (pos < 0) return r;
  r.t = min(pos, a.Ldec - 1);
  r.front = a.prompt ? min(max(a.prompt[b], 0), a.Lp) : a.Lp;
  const int kept = a.mode == DSA_MODE_DENSE    ? r.t + 1
                   : a.mode == DSA_MODE_WINDOW ? min(r.t + 1, a.cap)
                                               : min(max(a.count[pair], 0), a.cap);
  r.n = r.front + kept;
  return r;
}

// The cache row of attended row i.
__device__ __forceinline__ int paged_row(const PagedArgs& a, const PagedRows& r, const int32_t* idx,
                                         int i) {
  const int j = i - r.front;
  if (j < 0 || a.mode == DSA_MODE_DENSE) return i;
  if (a.mode == DSA_MODE_WINDOW)
    return r.front + (j < a.Ns ? j : max(r.t - a.W + 1, a.Ns) + j - a.Ns);
  return r.front + min(max(idx[j], 0), r.t);
}

// Dynamic LDS: places of the split's rows, a V tile per wave, the waves' results.
template <int D>
__host__ __device__ constexpr uint32_t paged_lds(int C, int waves, int G) {
  return C * 8u + waves * kTile * (D + kPad) * 2u + waves * G * (D + 2) * 4u;
}

// A workgroup takes C rows of a (request, KV head), its waves tiles of 32 of them by
// turns.  Scores on the matrix cores with K as the A operand straight from memory
// (lane l: row l % 16, eight elements) and the group's queries as B; they arrive
// with head l % 16 in lane l, for rows 4 * (l / 16) + j of each half of the tile, and
// so do the softmax weights, which are then the A operand of the product with V for
// these rows in order; V goes through LDS and comes back transposed as B.  A
// weight is taken apart into TERMS bf16 ones: three hold all of its 24 bits, for
// fp32 outputs; two are off by 2^-18 at most, a thousandth of a bf16 output's step.
template <bool FP8, int D, int TERMS>
__global__ __launch_bounds__(512) void paged_kernel(PagedArgs a) {
  constexpr int E = FP8 ? 1 : 2;    // bytes per element
  constexpr int EPL = 16 / E;       // elements per load
  constexpr int KPL = EPL / 8;      // k-steps per load
  constexpr int LPR = D / EPL;      // lanes per V row
  constexpr int RPI = 64 / LPR;     // V rows per load instruction
  constexpr int NV = kTile / RPI;
  constexpr int NK = D / 32;        // k-steps
  constexpr int VROW = D + kPad;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int lr = lane & 15, lq = lane >> 4, rg = lane / LPR, col = lane % LPR;
  const int s = blockIdx.x % a.S, pair = blockIdx.x / a.S;
  const int h = pair % a.Hkv, b = pair / a.Hkv, G = a.G;
  int64_t* place = reinterpret_cast<int64_t*>(lds);
  uint16_t* vt = reinterpret_cast<uint16_t*>(lds + a.C * 8) + wave * kTile * VROW;
  float* red = reinterpret_cast<float*>(lds + a.C * 8 + waves * kTile * VROW * 2);

  bf16x8 q[NK];
#pragma unroll
  for (int i = 0; i < NK; ++i) {
    uint4 x = make_uint4(0, 0, 0, 0);
    if (lr < G)
      x = *reinterpret_cast<const uint4*>(a.q + (static_cast<size_t>(b) * a.Hq + h * G + lr) * D +
                                          32 * KPL * (i / KPL) + EPL * lq + 8 * (i % KPL));
    q[i] = __builtin_bit_cast(bf16x8, x);
  }
  const PagedRows r = paged_rows(a, b, pair);
  const int r0 = s * a.C, r1 = min(r.n, r0 + a.C);
  if (s > 0 && r0 >= r.n) return;
  const int32_t* idx = a.mode == DSA_MODE_DIAGONAL ? a.idx + static_cast<size_t>(pair) * a.cap
                                                   : nullptr;
  const int32_t* table = a.table + static_cast<int64_t>(b) * a.M;
  for (int i = threadIdx.x; i < a.C; i += blockDim.x) {
    int64_t at = -1;
    if (r0 + i < r1) {
      const int row = paged_row(a, r, idx, r0 + i), entry = row >> a.lg;
      const int page = entry < a.M ? table[entry] : -1;
      if (static_cast<unsigned>(page) < static_cast<unsigned>(a.pool))
        at = page * a.sp + (row & ((1 << a.lg) - 1)) * a.sr;
    }
    place[i] = at;
  }
  const float ks = FP8 && a.ks ? a.ks[h] : 1.f, vs = FP8 && a.vs ? a.vs[h] : 1.f;
  const float sl = a.scale * ks, sl2 = a.scale_log2 * ks;
  __syncthreads();

  const uint8_t* kb = a.k + h * a.sh + 16 * lq;
  const uint8_t* vb = a.v + h * a.sh + 16 * col;
  float m = kLowest, l = 0.f;  // of head lr, over the rows that this lane holds
  f32x4 o[D / 16];             // lane l: heads 4 * (l / 16) + r, column l % 16 of each block
#pragma unroll
  for (int c = 0; c < D / 16; ++c) o[c] = f32x4{0.f, 0.f, 0.f, 0.f};

  for (int t0 = wave * kTile; r0 + t0 < r1; t0 += waves * kTile) {
    const int64_t* tp = place + t0;
    const uint32_t there = static_cast<uint32_t>(__ballot(tp[lane & 31] >= 0));
    if (!there && !a.wlog) continue;
    uint4 kr[2][NK / KPL], vr[NV];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const uint8_t* at = kb + max(tp[16 * hf + lr], int64_t{0});  // a row left out: the first
#pragma unroll
      for (int i = 0; i < NK / KPL; ++i) kr[hf][i] = load_stream16(at + 64 * i);
    }
#pragma unroll
    for (int u = 0; u < NV; ++u)
      vr[u] = load_stream16(vb + max(tp[u * RPI + rg], int64_t{0}));
    __builtin_amdgcn_sched_barrier(0);  // every load before any arithmetic

    f32x4 sc[2];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      sc[hf] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NK; ++i)
        sc[hf] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(to_bf16<FP8>(kr[hf][i / KPL], i % KPL),
                                                         q[i], sc[hf], 0, 0, 0);
    }
    if (a.wlog && lr < G) {
      float* to = a.wlog + (static_cast<size_t>(b) * a.Hq + h * G + lr) * a.cap;
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int e = 16 * hf + 4 * lq + j, i = r0 + t0 + e;
          if (i >= r.front && i < r1)
            to[i - r.front] = (there >> e) & 1 ? sc[hf][j] * sl : -__builtin_inff();
        }
    }
    // What is left out is 0 in the product with V, whatever the memory holds.
    if (there != 0xffffffffu) {
#pragma unroll
      for (int u = 0; u < NV; ++u)
        if (!((there >> (u * RPI + rg)) & 1)) vr[u] = make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < NV; ++u)
#pragma unroll
      for (int x = 0; x < KPL; ++x)
        *reinterpret_cast<bf16x8*>(vt + (u * RPI + rg) * VROW + col * EPL + 8 * x) =
            to_bf16<FP8>(vr[u], x);

    float z[2][4], mx = kLowest;
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool ok = (there >> (16 * hf + 4 * lq + j)) & 1;
        z[hf][j] = ok ? sc[hf][j] * sl2 : -__builtin_inff();
        mx = fmaxf(mx, z[hf][j]);
      }
    {
      float x1, x2;
      xor_pair<16>(mx, x1, x2);
      mx = fmaxf(x1, x2);
      xor_pair<32>(mx, x1, x2);
      mx = fmaxf(x1, x2);
    }
    const float mnew = fmaxf(m, mx), alpha = fast_exp2(m - mnew);
    m = mnew;
    l *= alpha;
    uint32_t w[TERMS][4];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int j = 0; j < 4; j += 2) {
        float p0 = fast_exp2(z[hf][j] - mnew), p1 = fast_exp2(z[hf][j + 1] - mnew);
        l += p0;
        l += p1;
#pragma unroll
        for (int x = 0; x < TERMS; ++x) {
          const uint32_t u = pack_bf16(p0, p1);
          w[x][2 * hf + j / 2] = u;
          p0 -= bf16_lo(u);
          p1 -= bf16_hi(u);
        }
      }
    float al[4];  // of the heads whose outputs this lane holds
#pragma unroll
    for (int i = 0; i < 4; ++i) al[i] = __shfl(alpha, 4 * lq + i, 64);
#pragma unroll
    for (int c = 0; c < D / 16; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[c][i] *= al[i];
    fence_wave();  // the V tile is written
    const uint16_t* vsrc = vt + (4 * lq + (lr >> 2)) * VROW + 4 * (lr & 3);
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
      const s16x4 b0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) s16x4*)(vsrc + 16 * c));
      const s16x4 b1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) s16x4*)(vsrc + 16 * VROW + 16 * c));
      const bf16x8 v = __builtin_bit_cast(
          bf16x8, __builtin_shufflevector(b0, b1, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int x = 0; x < TERMS; ++x)
        o[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            __builtin_bit_cast(bf16x8, make_uint4(w[x][0], w[x][1], w[x][2], w[x][3])), v, o[c], 0,
            0, 0);
    }
    fence_wave();  // and read
  }

  {
    float x1, x2;
    xor_pair<16>(l, x1, x2);
    l = x1 + x2;
    xor_pair<32>(l, x1, x2);
    l = x1 + x2;
  }
  float* mine = red + wave * G * (D + 2);
#pragma unroll
  for (int c = 0; c < D / 16; ++c)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (4 * lq + i < G) mine[(4 * lq + i) * (D + 2) + 16 * c + lr] = o[c][i];
  if (lane < G) {
    mine[lane * (D + 2) + D] = m;
    mine[lane * (D + 2) + D + 1] = l;
  }
  __syncthreads();

  const int splits = (r.n + a.C - 1) / a.C;
  for (int e = threadIdx.x; e < G * D; e += blockDim.x) {
    const int g = e / D, d = e % D;
    float M = kLowest;
    for (int x = 0; x < waves; ++x) M = fmaxf(M, red[(x * G + g) * (D + 2) + D]);
    float L = 0.f, O = 0.f;
    for (int x = 0; x < waves; ++x) {
      const float* p = red + (x * G + g) * (D + 2);
      const float f = fast_exp2(p[D] - M);
      L = fmaf(p[D + 1], f, L);
      O = fmaf(p[d], f, O);
    }
    if (splits > 1) {
      float* to = a.part + ((static_cast<size_t>(pair) * a.S + s) * G + g) * (D + 2);
      to[d] = O;
      if (d == 0) {
        to[D] = M;
        to[D + 1] = L;
      }
    } else {
      const float y = L == 0.f ? 0.f : O * vs / L;
      const size_t to = (static_cast<size_t>(b) * a.Hq + h * G + g) * D + d;
      if (a.f32)
        static_cast<float*>(a.out)[to] = y;
      else
        static_cast<uint16_t*>(a.out)[to] = static_cast<uint16_t>(pack_bf16(y, y));
    }
  }
}

// Joins the splits of a (request, query head): a wave each.
template <int D>
__global__ __launch_bounds__(256) void paged_combine_kernel(PagedArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t at = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (at >= static_cast<int64_t>(a.B) * a.Hq) return;
  const int b = static_cast<int>(at / a.Hq), hq = static_cast<int>(at % a.Hq);
  const int h = hq / a.G, g = hq % a.G, pair = b * a.Hkv + h;
  const PagedRows r = paged_rows(a, b, pair);
  const int splits = (r.n + a.C - 1) / a.C;
  if (splits < 2) return;
  const int64_t step = static_cast<int64_t>(a.G) * (D + 2);
  const float* p = a.part + (static_cast<size_t>(pair) * a.S * a.G + g) * (D + 2);
  float M = kLowest;
  for (int x = lane; x < splits; x += 64) M = fmaxf(M, p[x * step + D]);
  M = wave_max(M);
  float L = 0.f, O[D / 64] = {};
  for (int x = 0; x < splits; ++x) {
    const float f = fast_exp2(p[x * step + D] - M);
    L = fmaf(p[x * step + D + 1], f, L);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) O[i] = fmaf(p[x * step + lane + 64 * i], f, O[i]);
  }
  const float vs = a.vs ? a.vs[h] : 1.f;
#pragma unroll
  for (int i = 0; i < D / 64; ++i) {
    const float y = L == 0.f ? 0.f : O[i] * vs / L;
    const size_t to = at * D + lane + 64 * i;
    if (a.f32)
      static_cast<float*>(a.out)[to] = y;
    else
      static_cast<uint16_t*>(a.out)[to] = static_cast<uint16_t>(pack_bf16(y, y));
  }
}

template <bool FP8, int D>
hipError_t launch_paged(const PagedLaunch& l, const PagedArgs& a, hipStream_t st) {
  const dim3 grid(static_cast<uint32_t>(l.workgroups)), block(64 * l.waves);
  const uint32_t lds = paged_lds<D>(l.C, l.waves, a.G);
  if (a.f32)
    paged_kernel<FP8, D, 3><<<grid, block, lds, st>>>(a);
  else
    paged_kernel<FP8, D, 2><<<grid, block, lds, st>>>(a);
  if (l.S > 1) {
    const int64_t rows = static_cast<int64_t>(a.B) * a.Hq;
    paged_combine_kernel<D><<<dim3(static_cast<uint32_t>((rows + 3) / 4)), dim3(256), 0, st>>>(a);
  }
  return hipGetLastError();
}

}  // namespace
}  // namespace dsa
