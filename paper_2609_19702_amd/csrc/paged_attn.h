// Attention of one token per request over a cache in pages
// (dsa_paged_attention), as templates over the cache's element type.
#pragma once

#include <type_traits>

#include "device.h"
#include "paged.h"

namespace dsa {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

constexpr float kLowest = -3.402823466e38f;  // "no score yet": no finite score is below
constexpr int kTile = 32;                    // rows of a wave's tile
constexpr float kSlack = 8.f;
constexpr int kPad = 16;  // V rows in LDS are D + kPad bf16 apart: four of them in distinct banks

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {  // nearest even
  const f32x2 x = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}

// Eight E4M3 values as bf16, which every one of them is.
__device__ __forceinline__ bf16x8 widen_e4m3(uint32_t a, uint32_t b) {
  auto two = [](uint32_t w, auto high) {
    return __builtin_bit_cast(
        uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(w), 1.f, high.value));
  };
  return __builtin_bit_cast(
      bf16x8, make_uint4(two(a, std::false_type{}), two(a, std::true_type{}),
                         two(b, std::false_type{}), two(b, std::true_type{})));
}

// Elements 8 * half .. 8 * half + 7 of a load.
template <bool FP8>
__device__ __forceinline__ bf16x8 to_bf16(const uint4& r, int half) {
  if constexpr (FP8)
    return half ? widen_e4m3(r.z, r.w) : widen_e4m3(r.x, r.y);
  else
    return __builtin_bit_cast(bf16x8, r);
}

// A quotient of uniform values is one too, which the compiler does not see: its vector
// registers are then kept for all that follows from it.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Rows of a request that its step attends: its prompt, then decode rows.
struct PagedRows {
  int n, t, front;  // rows, decode position, prompt rows
};

__device__ __forceinline__ PagedRows paged_rows(const PagedArgs& a, int b, int pair) {
  PagedRows r{0, -1, 0};
  const int pos = a.pos[b], prompt = a.prompt ? a.prompt[b] : a.Lp;
  const int kept = a.mode == DSA_MODE_DIAGONAL ? a.count[pair] : a.cap;
  if (pos < 0) return r;
  r.t = min(pos, a.Ldec - 1);
  r.front = min(max(prompt, 0), a.Lp);
  r.n = r.front + min(r.t + 1, min(max(kept, 0), a.cap));
  return r;
}

// What a workgroup does: rows first .. first + rows - 1 of a (request, KV head), split s of
// those that it is cut into.
struct PagedWork {
  PagedRows r;
  int b, h, s, first, rows, splits;
};

// The workgroup's rows, their places in memory (a row left out reads the first one)
// and which of them there are, 32 to a word; false for a split behind the last row.
__device__ __forceinline__ bool paged_work(const PagedArgs& a, int lane, int wave, int waves,
                                           int64_t* place, uint32_t* mask, PagedWork& w) {
  const int pairs = a.B * a.Hkv;
  const uint32_t group = a.first + blockIdx.x;
  w.s = uniform(group / pairs);
  const int pair = group - w.s * pairs;
  w.b = uniform(pair / a.Hkv);
  w.h = pair - w.b * a.Hkv;
  w.first = w.s * a.C;
  w.r = paged_rows(a, w.b, pair);
  w.splits = (w.r.n + a.C - 1) / a.C;
  w.rows = min(w.r.n - w.first, a.C);
  if (w.s > 0 && w.rows <= 0) return false;
  const bool planned = a.mode == DSA_MODE_DIAGONAL;
  const int32_t* idx = planned ? a.idx + static_cast<size_t>(pair) * a.cap : nullptr;
  const int32_t* table = a.table + static_cast<int64_t>(w.b) * a.M;
  for (int i0 = wave * 64; i0 < w.rows; i0 += waves * 64) {
    const int i = i0 + lane;
    int64_t at = 0;
    bool ok = false;
    if (i < w.rows) {
      const int e = w.first + i, j = e - w.r.front;
      int row = e;
      if (j >= 0 && planned)
        row = w.r.front + min(max(idx[j], 0), w.r.t);
      else if (j >= 0 && a.mode == DSA_MODE_WINDOW)
        row = w.r.front + (j < a.Ns ? j : max(w.r.t - a.W + 1, a.Ns) + j - a.Ns);
      const int entry = row >> a.lg, page = entry < a.M ? table[entry] : -1;
      ok = static_cast<unsigned>(page) < static_cast<unsigned>(a.pool);
      if (ok) at = page * a.sp + (row & ((1 << a.lg) - 1)) * a.sr;
    }
    const uint64_t there = __ballot(ok);
    place[i] = at;
    if (lane < 2) mask[i0 / 32 + lane] = static_cast<uint32_t>(there >> (32 * lane));
  }
  return true;
}

// Joins the waves' sums of G heads, for the combine or into the output.
template <int D>
__device__ __forceinline__ void paged_finish(const PagedArgs& a, const PagedWork& w, int G, int waves,
                                             const float* red, float vs) {
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
    if (w.splits > 1) {
      float* to = a.part + ((static_cast<size_t>(w.s) * a.B * a.Hkv + w.b * a.Hkv + w.h) * G + g) *
                             (D + 2);
      to[d] = O;
      if (d == 0) {
        to[D] = M;
        to[D + 1] = L;
      }
    } else {
      const float y = L == 0.f ? 0.f : O / L * vs;  // O * vs can pass fp32 where y does not
      const size_t to = (static_cast<size_t>(w.b) * a.Hq + w.h * G + g) * D + d;
      if (a.f32)
        static_cast<float*>(a.out)[to] = y;
      else
        static_cast<uint16_t*>(a.out)[to] = static_cast<uint16_t>(pack_bf16(y, y));
    }
  }
}

// A lane's sums with those of lane ^ OFF.
template <int OFF, int N>
__device__ __forceinline__ void join_lanes(float& m, float& l, float (&o)[N]) {
  float m1, m2, l1, l2;
  xor_pair<OFF>(m, m1, m2);
  xor_pair<OFF>(l, l1, l2);
  m = fmaxf(m1, m2);
  const float f1 = fast_exp2(m1 - m), f2 = fast_exp2(m2 - m);
  l = fmaf(l1, f1, l2 * f2);
#pragma unroll
  for (int e = 0; e < N; ++e) {
    float x1, x2;
    xor_pair<OFF>(o[e], x1, x2);
    o[e] = fmaf(x1, f1, x2 * f2);
  }
}

// The elements of a load in fp32.
template <bool FP8>
__device__ __forceinline__ void widen(const uint4& r, float (&f)[FP8 ? 16 : 8]) {
  if constexpr (FP8) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[i]), false);
      const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(w[i]), true);
      f[4 * i] = lo[0];
      f[4 * i + 1] = lo[1];
      f[4 * i + 2] = hi[0];
      f[4 * i + 3] = hi[1];
    }
  } else {
    unpack8(r, f);
  }
}

// Dynamic LDS: places of the split's rows, which of them there are, the queries, a V tile
// per wave (its last row without the pad: that leaves room for two workgroups of 768 rows
// and eight heads on a CU) and over the tiles the waves' results.
template <bool FP8, int D>
__host__ __device__ constexpr uint32_t paged_vt_bytes() {
  return (kTile - 1) * (FP8 ? D + 16 : 2 * (D + kPad)) + (FP8 ? D : 2 * D);
}
template <bool FP8, int D>
__host__ __device__ constexpr uint32_t paged_lds(int C, int waves, int G) {
  const uint32_t vt = paged_vt_bytes<FP8, D>(), red = G * (D + 2) * 4;
  return C * 8u + ((C / 8 + 15) & ~15) + G * D * 2 + waves * (vt > red ? vt : red);
}

// A tile of a wave as loaded.
template <bool FP8, int D>
struct PagedTile {
  static constexpr int E = FP8 ? 1 : 2;   // bytes per element
  static constexpr int EPL = 16 / E;      // elements per load
  static constexpr int KPL = EPL / 8;     // k-steps per load
  static constexpr int LPR = D / EPL;     // lanes per V row
  static constexpr int RPI = 64 / LPR;    // V rows per load instruction
  static constexpr int NV = kTile / RPI;
  static constexpr int NK = D / 32;       // k-steps
  uint4 k[2][NK / KPL], v[NV];
  uint32_t there;
};

// A workgroup takes C rows of a (request, KV head), its waves tiles of 32 of them by
// turns.  Scores on the matrix cores with K as the A operand straight from memory
// (lane l: row l % 16, eight elements) and the group's queries as B; they arrive
// with head l % 16 in lane l, for rows 4 * (l / 16) + j of each half of the tile, and
// so do the softmax weights, which are then the A operand of the product with V for
// these rows in order; V goes through LDS and comes back transposed as B.  A
// weight is taken apart into TERMS bf16 ones: three hold all of its 24 bits, for
// fp32 outputs; two are off by 2^-18 at most, a thousandth of a bf16 output's step.
// The queries are read from LDS each time and the waves' sums lie over their V tiles: with
// 128 registers and 768 rows, two workgroups share a CU.  Bound by memory and by how evenly
// the CUs end: 32 requests of 8 heads, 2304 rows each, d = 128, four queries a head, 56 us
// or 5.4 TB/s of reads (bf16); of 200 to 4300 rows, 69 us and 4.4, fp8 42 and 3.6, where waves
// wait for their one tile at a time: the vector units are busy for 35% of the kernel, the
// matrix cores for 12%.
template <bool FP8, int D, int TERMS>
__global__ __launch_bounds__(512, 4) void paged_kernel(PagedArgs a) {
  using T = PagedTile<FP8, D>;
  constexpr int EPL = T::EPL, KPL = T::KPL, LPR = T::LPR, RPI = T::RPI, NV = T::NV, NK = T::NK;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int lr = lane & 15, lq = lane >> 4, rg = lane / LPR, col = lane % LPR;
  const int pair = uniform((a.first + blockIdx.x) % (a.B * a.Hkv)), b = uniform(pair / a.Hkv);
  const int h = pair - b * a.Hkv, G = a.G;
  int64_t* place = reinterpret_cast<int64_t*>(lds);
  uint32_t* mask = reinterpret_cast<uint32_t*>(lds + a.C * 8);
  unsigned char* qs = lds + a.C * 8 + ((a.C / 8 + 15) & ~15);
  unsigned char* vts = qs + G * D * 2;
  unsigned char* vt = vts + wave * paged_vt_bytes<FP8, D>();
  float* red = reinterpret_cast<float*>(vts);  // the waves' sums, after their last tiles

  // Queries of heads past the group are any; nothing of theirs comes out.
  const uint16_t* qg = a.q + (static_cast<size_t>(b) * a.Hq + h * G) * D;
  if (threadIdx.x < G * D / 8)
    reinterpret_cast<uint4*>(qs)[threadIdx.x] = reinterpret_cast<const uint4*>(qg)[threadIdx.x];
  PagedWork work;
  if (!paged_work(a, lane, wave, waves, place, mask, work)) return;
  const float ks = FP8 && a.ks ? a.ks[h] : 1.f, vs = FP8 && a.vs ? a.vs[h] : 1.f;
  const float sl = a.scale * ks, sl2 = a.scale_log2 * ks;
  __syncthreads();

  const unsigned char* qat = qs + ((lr & (G - 1)) * D + EPL * lq) * 2;
  const uint8_t* kb = a.k + h * a.sh + 16 * lq;
  const uint8_t* vb = a.v + h * a.sh + 16 * col;
  float m = kLowest, l = 0.f;  // of head lr, over the rows that this lane holds
  f32x4 o[D / 16];             // lane l: heads 4 * (l / 16) + r, column l % 16 of each block
#pragma unroll
  for (int c = 0; c < D / 16; ++c) o[c] = f32x4{0.f, 0.f, 0.f, 0.f};

  auto load = [&](int t0, T& t) {
    const int64_t* tp = place + t0;
    t.there = mask[t0 / 32];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const uint8_t* at = kb + tp[16 * hf + lr];
#pragma unroll
      for (int i = 0; i < NK / KPL; ++i) t.k[hf][i] = load_stream16(at + 64 * i);
    }
#pragma unroll
    for (int u = 0; u < NV; ++u) t.v[u] = load_stream16(vb + tp[u * RPI + rg]);
  };

  auto compute = [&](int t0, T& t) {
    f32x4 sc[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      const bf16x8 q = *reinterpret_cast<const bf16x8*>(qat + 64 * KPL * (i / KPL) + 16 * (i % KPL));
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
        sc[hf] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(to_bf16<FP8>(t.k[hf][i / KPL], i % KPL), q,
                                                         sc[hf], 0, 0, 0);
    }
    const uint32_t there = __builtin_amdgcn_readfirstlane(t.there), mine = there >> (4 * lq);
    if (a.wlog && lr < G) {
      float* to = a.wlog + (static_cast<size_t>(b) * a.Hq + h * G + lr) * a.cap;
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int e = 16 * hf + 4 * lq + j, i = work.first + t0 + e;
          if (i >= work.r.front && i < work.first + work.rows)
            to[i - work.r.front] = (mine >> (16 * hf + j)) & 1 ? sc[hf][j] * sl : -__builtin_inff();
        }
    }
    float z[2][4], mx = kLowest;
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int j = 0; j < 4; ++j) z[hf][j] = sc[hf][j] * sl2;
    if (there != 0xffffffffu) {
      // What is left out is 0 in the product with V, whatever the memory holds.
      const uint32_t rows = there >> rg;
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const uint32_t keep = 0u - ((rows >> (u * RPI)) & 1);
        t.v[u].x &= keep;
        t.v[u].y &= keep;
        t.v[u].z &= keep;
        t.v[u].w &= keep;
      }
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (!((mine >> (16 * hf + j)) & 1)) z[hf][j] = -__builtin_inff();
    }
    // V rows in the order of the weights: those of lanes 16 * g .. are eight in turn.
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int row = u * RPI + rg;
      const int at = FP8 ? (row & 12) * 2 + (row >> 4) * 4 + (row & 3) : row;
      if constexpr (FP8)
        *reinterpret_cast<uint4*>(vt + at * (D + 16) + 16 * col) = t.v[u];
      else
        *reinterpret_cast<uint4*>(vt + at * 2 * (D + kPad) + 16 * col) = t.v[u];
    }
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int j = 0; j < 4; ++j) mx = fmaxf(mx, z[hf][j]);
    {
      float x1, x2;
      xor_pair<16>(mx, x1, x2);
      mx = fmaxf(x1, x2);
      xor_pair<32>(mx, x1, x2);
      mx = fmaxf(x1, x2);
    }
    // The sums are scaled by a maximum that lags behind by kSlack at most.
    const bool grow = mx > m + kSlack;
    if (__any(grow)) {
      const float mnew = grow ? mx : m, alpha = fast_exp2(m - mnew);
      m = mnew;
      l *= alpha;
      float al[4];  // of the heads whose outputs this lane holds
#pragma unroll
      for (int i = 0; i < 4; ++i) al[i] = __shfl(alpha, 4 * lq + i, 64);
#pragma unroll
      for (int c = 0; c < D / 16; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[c][i] *= al[i];
    }
    uint32_t w[TERMS][4];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int j = 0; j < 4; j += 2) {
        float p0 = fast_exp2(z[hf][j] - m), p1 = fast_exp2(z[hf][j + 1] - m);
        l += p0;
        l += p1;
#pragma unroll
        for (int x = 0; x < TERMS; ++x) {
          const uint32_t u = pack_bf16(p0, p1);
          w[x][2 * hf + j / 2] = u;
          if (x + 1 < TERMS) {
            p0 -= bf16_lo(u);
            p1 -= bf16_hi(u);
          }
        }
      }
    fence_wave();  // the V tile is written
#pragma unroll
    for (int c = 0; c < D / 16; ++c) {
      bf16x8 v;
      if constexpr (FP8) {
        const auto x = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
            (__attribute__((address_space(3))) i32x2*)(vt + (8 * lq + (lr >> 1)) * (D + 16) +
                                                       16 * c + 8 * (lr & 1)));
        v = widen_e4m3(static_cast<uint32_t>(x[0]), static_cast<uint32_t>(x[1]));
      } else {
        const unsigned char* at = vt + (4 * lq + (lr >> 2)) * 2 * (D + kPad) + 8 * (lr & 3) + 32 * c;
        const s16x4 b0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)(at));
        const s16x4 b1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)(at + 32 * (D + kPad)));
        v = __builtin_bit_cast(bf16x8, __builtin_shufflevector(b0, b1, 0, 1, 2, 3, 4, 5, 6, 7));
      }
#pragma unroll
      for (int x = 0; x < TERMS; ++x)
        o[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            __builtin_bit_cast(bf16x8, make_uint4(w[x][0], w[x][1], w[x][2], w[x][3])), v, o[c], 0,
            0, 0);
    }
    fence_wave();  // and read
  };

  for (int t0 = wave * kTile; t0 < work.rows; t0 += waves * kTile) {
    T x;
    load(t0, x);
    __builtin_amdgcn_sched_barrier(0);
    compute(t0, x);
  }

  {
    float x1, x2;
    xor_pair<16>(l, x1, x2);
    l = x1 + x2;
    xor_pair<32>(l, x1, x2);
    l = x1 + x2;
  }
  __syncthreads();  // the tiles are done with
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

  paged_finish<D>(a, work, G, waves, red, vs);
}

// One query head per KV head: the vector units.  A lane holds 16 bytes of a row, LPR
// lanes a row, U loads of each operand a tile of a wave; a row's score is summed over
// its lanes by DPP and all of them then hold it, so its weight needs no way to the
// row's V.  Every group of LPR lanes keeps a maximum and sums of its own up to the end.
// U is as many loads as 128 registers hold.  Bound by memory: 128 requests of 32 heads,
// 280 to 832 rows, d = 128, bf16, 154 us or 6.5 TB/s, what a stream that only reads reaches.
template <bool FP8, int D, int U>
__global__ __launch_bounds__(512, 4) void paged_row_kernel(PagedArgs a) {
  constexpr int E = FP8 ? 1 : 2, EPL = 16 / E, LPR = D / EPL, RPI = 64 / LPR, T = RPI * U;
  static_assert(T == 32 || T == 64, "a split is a multiple of 64 rows");
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int rg = lane / LPR, col = lane % LPR;
  int64_t* place = reinterpret_cast<int64_t*>(lds);
  uint32_t* mask = reinterpret_cast<uint32_t*>(lds + a.C * 8);
  float* red = reinterpret_cast<float*>(lds + a.C * 8 + ((a.C / 8 + 15) & ~15));

  const int pair = uniform((a.first + blockIdx.x) % (a.B * a.Hkv)), h = uniform(pair % a.Hkv);
  uint4 qr[EPL / 8];
#pragma unroll
  for (int i = 0; i < EPL / 8; ++i)
    qr[i] = *reinterpret_cast<const uint4*>(a.q + static_cast<size_t>(pair) * D + col * EPL + 8 * i);
  PagedWork work;
  if (!paged_work(a, lane, wave, waves, place, mask, work)) return;
  const int rows = work.rows;
  const float ks = FP8 && a.ks ? a.ks[h] : 1.f, vs = FP8 && a.vs ? a.vs[h] : 1.f;
  const float sl = a.scale * ks, sl2 = a.scale_log2 * ks;
  __syncthreads();

  float q[EPL], o[EPL];
#pragma unroll
  for (int i = 0; i < EPL / 8; ++i) {
    float f[8];
    unpack8(qr[i], f);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      q[8 * i + e] = f[e];
      o[8 * i + e] = 0.f;
    }
  }
  float m = kLowest, l = 0.f;
  const uint8_t* kb = a.k + h * a.sh + 16 * col;
  const uint8_t* vb = a.v + h * a.sh + 16 * col;
  for (int t0 = wave * T; t0 < rows; t0 += waves * T) {
    uint4 kr[U], vr[U];
    int64_t at[U];
#pragma unroll
    for (int u = 0; u < U; ++u) at[u] = place[t0 + u * RPI + rg];
#pragma unroll
    for (int u = 0; u < U; ++u) kr[u] = load_stream16(kb + at[u]);
#pragma unroll
    for (int u = 0; u < U; ++u) vr[u] = load_stream16(vb + at[u]);
    // bit u * RPI + rg of the tile's words: whether the lane's row u is there
    uint64_t there = mask[t0 / 32];
    if constexpr (T == 64) there |= static_cast<uint64_t>(mask[t0 / 32 + 1]) << 32;
    __builtin_amdgcn_sched_barrier(0);  // every load before any arithmetic
    float z[U], mx = kLowest;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float f[EPL], x = 0.f;
      widen<FP8>(kr[u], f);
#pragma unroll
      for (int e = 0; e < EPL; ++e) x = fmaf(q[e], f[e], x);
      z[u] = group_sum<LPR>(x);
    }
    const bool full = there == ~uint64_t{0} >> (64 - T);
    if (a.wlog && col == 0) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int e = u * RPI + rg, i = work.first + t0 + e;
        if (i >= work.r.front && i < work.first + rows)
          a.wlog[static_cast<size_t>(pair) * a.cap + i - work.r.front] =
              (there >> e) & 1 ? z[u] * sl : -__builtin_inff();
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) z[u] *= sl2;
    if (!full) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (!((there >> (u * RPI + rg)) & 1)) {
          z[u] = -__builtin_inff();
          vr[u] = make_uint4(0, 0, 0, 0);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) mx = fmaxf(mx, z[u]);
    const float mnew = fmaxf(m, mx), alpha = fast_exp2(m - mnew);
    m = mnew;
    l *= alpha;
#pragma unroll
    for (int e = 0; e < EPL; ++e) o[e] *= alpha;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float f[EPL];
      widen<FP8>(vr[u], f);
      const float p = fast_exp2(z[u] - m);
      l += p;
#pragma unroll
      for (int e = 0; e < EPL; ++e) o[e] = fmaf(p, f[e], o[e]);
    }
  }
  if constexpr (LPR <= 4) join_lanes<4, EPL>(m, l, o);
  if constexpr (LPR <= 8) join_lanes<8, EPL>(m, l, o);
  join_lanes<16, EPL>(m, l, o);
  join_lanes<32, EPL>(m, l, o);
  if (lane < LPR) {
    float* mine = red + wave * (D + 2);
#pragma unroll
    for (int e = 0; e < EPL; ++e) mine[col * EPL + e] = o[e];
    if (lane == 0) {
      mine[D] = m;
      mine[D + 1] = l;
    }
  }
  __syncthreads();
  paged_finish<D>(a, work, 1, waves, red, vs);
}

// Joins the splits of a (request, query head): `each` waves of a workgroup for one, by
// turns, four splits at a time.  3.9 us for two splits of 768 heads, 4.5 for six of 1024.
template <int D>
__global__ __launch_bounds__(256) void paged_combine_kernel(PagedArgs a, int each, int most) {
  constexpr int N = D / 64;
  __shared__ float red[4][D + 2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t group = a.first + blockIdx.x;
  const int at = uniform(each > 1 ? group : group * 4 + wave);
  if (at >= a.B * a.Hq) return;
  const int b = uniform(at / a.Hq), hq = at - b * a.Hq, h = uniform(hq / a.G), g = hq - h * a.G;
  const int pair = b * a.Hkv + h;
  const int64_t step = static_cast<int64_t>(a.B) * a.Hkv * a.G * (D + 2);
  const float* p = a.part + (static_cast<size_t>(pair) * a.G + g) * (D + 2);
  float mx[4], lx[4], ox[4][N];
  auto load = [&](int x0) {
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float* px = p + min(x0 + x, most - 1) * step;
      mx[x] = px[D];
      lx[x] = px[D + 1];
#pragma unroll
      for (int i = 0; i < N; ++i) ox[x][i] = px[lane + 64 * i];
    }
  };
  int x0 = each > 1 ? 4 * wave : 0;
  load(x0);  // on their way before it is known how many there are
  const int splits = (paged_rows(a, b, pair).n + a.C - 1) / a.C;
  if (splits < 2) return;
  float M = kLowest, L = 0.f, O[N] = {};
  while (x0 < splits) {
    float top = M;
#pragma unroll
    for (int x = 0; x < 4; ++x) top = x0 + x < splits ? fmaxf(top, mx[x]) : top;
    const float f = fast_exp2(M - top);
    M = top;
    L *= f;
#pragma unroll
    for (int i = 0; i < N; ++i) O[i] *= f;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      if (x0 + x >= splits) break;
      const float fx = fast_exp2(mx[x] - M);
      L = fmaf(lx[x], fx, L);
#pragma unroll
      for (int i = 0; i < N; ++i) O[i] = fmaf(ox[x][i], fx, O[i]);
    }
    x0 += 4 * each;
    if (x0 < splits) load(x0);
  }
  if (each > 1) {
    red[wave][D] = M;
    red[wave][D + 1] = L;
#pragma unroll
    for (int i = 0; i < N; ++i) red[wave][lane + 64 * i] = O[i];
    __syncthreads();
    if (wave) return;
    for (int w = 1; w < 4; ++w) M = fmaxf(M, red[w][D]);
    L = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) O[i] = 0.f;
    for (int w = 0; w < 4; ++w) {
      const float f = fast_exp2(red[w][D] - M);
      L = fmaf(red[w][D + 1], f, L);
#pragma unroll
      for (int i = 0; i < N; ++i) O[i] = fmaf(red[w][lane + 64 * i], f, O[i]);
    }
  }
  const float vs = a.vs ? a.vs[h] : 1.f;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float y = L == 0.f ? 0.f : O[i] / L * vs;
    const size_t to = static_cast<size_t>(at) * D + lane + 64 * i;
    if (a.f32)
      static_cast<float*>(a.out)[to] = y;
    else
      static_cast<uint16_t*>(a.out)[to] = static_cast<uint16_t>(pack_bf16(y, y));
  }
}

template <bool FP8, int D>
hipError_t launch_paged(const PagedLaunch& l, PagedArgs a, hipStream_t st) {
  const dim3 block(64 * l.waves);
  const hipError_t e = launch_parts(l.workgroups, 64 * l.waves, [&](uint32_t first, dim3 grid) {
    const uint32_t lds = paged_lds<FP8, D>(l.C, l.waves, a.G);
    a.first = first;
    if (a.G == 1) {
      const uint32_t row_lds = l.C * 8u + ((l.C / 8 + 15) & ~15) + l.waves * (D + 2) * 4u;
      paged_row_kernel<FP8, D, FP8 ? 4 : 8><<<grid, block, row_lds, st>>>(a);
    } else if (a.f32) {
      paged_kernel<FP8, D, 3><<<grid, block, lds, st>>>(a);
    } else {
      paged_kernel<FP8, D, 2><<<grid, block, lds, st>>>(a);
    }
  });
  if (e != hipSuccess || l.S == 1) return e;
  const int64_t rows = static_cast<int64_t>(a.B) * a.Hq;
  const int each = l.S > 4 ? 4 : 1;
  return launch_parts(each > 1 ? rows : (rows + 3) / 4, 256, [&](uint32_t first, dim3 grid) {
    a.first = first;
    paged_combine_kernel<D><<<grid, dim3(256), 0, st>>>(a, each, l.S);
  });
}

}  // namespace
}  // namespace dsa
