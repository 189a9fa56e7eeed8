// One step of a beam search: the best candidates over beams and vocabulary.
#include "device.h"
#include "paged.h"

namespace dsa {
namespace {

constexpr int kBeamThreads = 256;
constexpr int kBeamWaves = kBeamThreads / 64;
constexpr int kFew = 8, kMany = 32;  // values per thread

// Sixteen bytes anywhere.
typedef unsigned int Piece __attribute__((ext_vector_type(4), aligned(2)));

// A value of the logits and its place as one number, larger ones first, equal
// ones by the lower place; 0 for what is no candidate (NaN, -infinity).
__device__ __forceinline__ uint64_t beam_key(float x, int place) {
  return x > -__builtin_inff()
             ? (static_cast<uint64_t>(ordered_bits(x)) << 32) | static_cast<uint32_t>(~place)
             : 0;
}
__device__ __forceinline__ float from_ordered(uint32_t u) {
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ float key_value(uint64_t k) {
  return from_ordered(static_cast<uint32_t>(k >> 32));
}

__device__ __forceinline__ uint64_t wave_max_u64(uint64_t x) { return ~wave_min_u64(~x); }

// Sum over the wave by DPP and lane swaps, as wave_allreduce.
template <typename Get>
__device__ __forceinline__ double add_f64(double x, Get get) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = get(static_cast<uint32_t>(u)), hi = get(static_cast<uint32_t>(u >> 32));
  return x + __builtin_bit_cast(double, (static_cast<uint64_t>(hi) << 32) | lo);
}
template <int OFF>
__device__ __forceinline__ double add_swapped(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  float lo0, lo1, hi0, hi1;
  xor_pair<OFF>(__uint_as_float(static_cast<uint32_t>(u)), lo0, lo1);
  xor_pair<OFF>(__uint_as_float(static_cast<uint32_t>(u >> 32)), hi0, hi1);
  auto join = [](float hi, float lo) {
    return __builtin_bit_cast(double, (static_cast<uint64_t>(__float_as_uint(hi)) << 32) |
                                          __float_as_uint(lo));
  };
  return join(hi0, lo0) + join(hi1, lo1);
}
__device__ __forceinline__ double wave_sum_f64(double x) {
  x = add_f64(x, [](uint32_t y) { return dpp_i<kDppQuadSwap1>(y); });
  x = add_f64(x, [](uint32_t y) { return dpp_i<kDppQuadSwap2>(y); });
  x = add_f64(x, [](uint32_t y) { return dpp_i<kDppHalfMirror>(y); });
  x = add_f64(x, [](uint32_t y) { return dpp_i<kDppRowMirror>(y); });
  return add_swapped<32>(add_swapped<16>(x));
}

// How many of the n keys of a list in LDS are larger than `key`; n a multiple of 4.
__device__ __forceinline__ int key_rank(uint64_t key, const uint64_t* list, int n) {
  int rank = 0;
  for (int j = 0; j < n; j += 4) {
    uint64_t k[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) k[i] = list[j + i];
#pragma unroll
    for (int i = 0; i < 4; ++i) rank += k[i] > key;
  }
  return rank;
}

// A workgroup takes R values per thread of a row: their maximum, the sum of their
// exponentials (fours in fp32, the rest in fp64), and their W largest in order.
//
// The W largest are not below the W-th largest of the maxima of the workgroup's 32
// groups of eight lanes (here cut to 27 bits, with the group's number below), and few
// values are (about 10 of 8192 for eight beams, 22 for sixteen): those go into a list,
// where each is placed by the larger ones' number.  With more than 64 of them (equal
// values) every wave takes its largest out one at a time, from memory once more.
//
// Bound by the arithmetic between two barriers, and by whole rounds of workgroups: 256 rows of
// 65539 bf16 values take 12 us, 2.8 TB/s, with the vector units busy for 72% of them (16
// instructions a value), in 2304 workgroups where 2048 are resident; widened once and kept, in
// twice the registers, 16; 64 values a thread 14.
template <bool BF16, int R>
__global__ __launch_bounds__(kBeamThreads) void beam_row_kernel(BeamArgs a) {
  constexpr int VL = BF16 ? 8 : 4, NV = R / VL;  // values of a load, loads
  constexpr int kGroups = kBeamThreads / 8;
  static_assert(kGroups >= DSA_MAX_BEAMS && kGroups == 32 && kBeamWaves * DSA_MAX_BEAMS <= 64,
                "a lane each");
  __shared__ float top_s[kGroups];
  __shared__ __attribute__((aligned(16))) uint32_t order_s[kGroups];
  __shared__ double sum_s[kBeamWaves];
  __shared__ __attribute__((aligned(16))) uint64_t list_s[64];
  __shared__ int n_s;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t part = a.first + blockIdx.x;
  const int chunk = part % a.chunks, row = part / a.chunks;
  // Pieces of VL values, which begin at any value: a row's sums do not depend on where it
  // lies, so equal rows tie.
  const uint8_t* start = static_cast<const uint8_t*>(a.x) + row * a.stride * (16 / VL);
  const int first = chunk * a.per, end = min(first + a.per, (a.V + VL - 1) / VL);
  auto load = [&](int k) {
    const int piece = first + k * kBeamThreads + threadIdx.x, v = piece * VL;
    if (piece < end && v + VL <= a.V)
      return static_cast<u32x4>(__builtin_nontemporal_load(
          reinterpret_cast<const Piece*>(start + static_cast<int64_t>(v) * (16 / VL))));
    u32x4 w;  // the row's end, value by value, and what lies behind
#pragma unroll
    for (int i = 0; i < VL; ++i) {
      const bool there = piece < end && v + i < a.V;
      if constexpr (BF16) {
        const uint32_t u = there ? reinterpret_cast<const uint16_t*>(start)[v + i] : 0xff80u;
        w[i / 2] = i & 1 ? w[i / 2] | u << 16 : u;
      } else {
        w[i] = there ? reinterpret_cast<const uint32_t*>(start)[v + i] : 0xff800000u;
      }
    }
    return w;
  };
  auto value = [&](const u32x4& w, int i) {
    if constexpr (BF16)
      return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    else
      return __uint_as_float(w[i]);
  };
  u32x4 w[NV];  // as they lie: half the registers for bf16, so more waves
#pragma unroll
  for (int k = 0; k < NV; ++k) w[k] = load(k);
  auto place = [&](int k, int i) {
    return (first + k * kBeamThreads + static_cast<int>(threadIdx.x)) * VL + i;
  };

  float most[NV], mine = -__builtin_inff();
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    most[k] = value(w[k], 0);
#pragma unroll
    for (int i = 1; i < VL; ++i) most[k] = fmaxf(most[k], value(w[k], i));
    mine = fmaxf(mine, most[k]);
  }
  mine = fmaxf(mine, dpp<kDppQuadSwap1>(mine));
  mine = fmaxf(mine, dpp<kDppQuadSwap2>(mine));
  mine = fmaxf(mine, dpp<kDppHalfMirror>(mine));
  if ((lane & 7) == 0) {
    const int group = threadIdx.x >> 3;
    top_s[group] = mine;
    order_s[group] = (ordered_bits(mine) & ~(kGroups - 1u)) | group;
  }
  if (threadIdx.x < 64) list_s[threadIdx.x] = 0;
  if (threadIdx.x == 0) n_s = 0;
  __syncthreads();
  const float top = wave_max(top_s[lane % kGroups]);
  const uint32_t group = order_s[lane % kGroups];
  int larger = 0;  // of the groups of half the lanes
  const uint32_t* others = order_s + lane / kGroups * (kGroups / 2);
#pragma unroll
  for (int j = 0; j < kGroups / 2; ++j) larger += others[j] > group;
  larger += __shfl_xor(larger, kGroups, 64);
  const int at_w = __builtin_ctzll(__ballot(larger == a.W - 1));
  const float least = fmaxf(from_ordered(__shfl(group, at_w, 64) & ~(kGroups - 1u)), -3.402823466e38f);

  // A chunk of -infinities adds nothing; a NaN or +infinity makes the sum a NaN.
  double sum = 0.;
  const float base = top > -__builtin_inff() ? top : 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    asm volatile("" : "+v"(w[k]));  // the values are widened once more, not kept
#pragma unroll
    for (int i = 0; i < VL; i += 4) {
      float e[4];
#pragma unroll
      for (int j = 0; j < 4; ++j)
        e[j] = fast_exp2((value(w[k], i + j) - base) * 1.4426950408889634f);
      sum += static_cast<double>((e[0] + e[1]) + (e[2] + e[3]));
    }
  }
  sum = wave_sum_f64(sum);
  if (lane == 0) sum_s[wave] = sum;

#pragma unroll
  for (int k = 0; k < NV; ++k)
    if (most[k] >= least) {
#pragma unroll
      for (int i = 0; i < VL; ++i)
        if (value(w[k], i) >= least) {
          const int at = atomicAdd(&n_s, 1);
          if (at < 64) list_s[at] = beam_key(value(w[k], i), place(k, i));
        }
    }
  __syncthreads();
  int n = n_s;
  if (n > 64) {
    uint64_t best = 0, under = ~uint64_t{0};  // lane i: the wave's i-th
    for (int k = 0; k < a.W; ++k) {
      uint64_t next = 0;
#pragma unroll 1
      for (int q = 0; q < NV; ++q) {  // read again: rare, and no registers held for it
        const u32x4 x = load(q);
#pragma unroll
        for (int i = 0; i < VL; ++i) {
          const uint64_t key = beam_key(value(x, i), place(q, i));
          next = key < under && key > next ? key : next;
        }
      }
      under = wave_max_u64(next);
      if (lane == k) best = under;
    }
    __syncthreads();  // all have read n_s, and the list ends
    if (lane < a.W) list_s[wave * a.W + lane] = best;
    __syncthreads();
    n = kBeamWaves * a.W;
  }
  if (wave) return;
  const uint64_t key = lane < n ? list_s[lane] : 0;
  const int rank = key_rank(key, list_s, (n + 3) & ~3);
  uint64_t* to = a.cands + static_cast<int64_t>(part) * a.W;
  const int some = __popcll(__ballot(key != 0));
  if (key && rank < a.W) to[rank] = key;
  if (lane >= some && lane < a.W) to[lane] = 0;
  if (lane == 0) {
    double s = 0.;
    for (int w = 0; w < kBeamWaves; ++w) s += sum_s[w];
    a.sums[part] = s;
    a.tops[part] = top;
  }
}

// A candidate of the last steps: its score, and what decides between equal ones, larger ones
// first: beam, logit and token (4, 32 and 24 bits, beam and token counted from above).  A
// beam's scores grow with its logits but for their rounding, so its candidates come as its
// keys do.
struct BeamCand {
  double z;
  uint64_t tie;
};
// A value's distance to its row's maximum comes first: large logits (`off` is the beam's score less
// the log of its sum) would round the rest away.
__device__ __forceinline__ BeamCand beam_cand(float top, double off, int w, uint64_t key) {
  const double z = (static_cast<double>(key_value(key)) - static_cast<double>(top)) + off;
  const bool ok = key && z > -__builtin_inf();  // not so for a NaN
  const uint64_t tie = (static_cast<uint64_t>(DSA_MAX_BEAMS - 1 - w) << 56) | ((key >> 32) << 24) |
                       (key & 0xffffff);
  return {ok ? z : -__builtin_inf(), ok ? tie : 0};
}
__device__ __forceinline__ int cand_beam(uint64_t tie) {
  return DSA_MAX_BEAMS - 1 - static_cast<int>(tie >> 56);
}
__device__ __forceinline__ int cand_token(uint64_t tie) { return ~static_cast<int>(tie) & 0xffffff; }

// How many of n candidates come before each of them, into rank[n] (zeros): the workgroup's
// threads share the comparisons.
__device__ __forceinline__ void cand_ranks(const double* z, const uint64_t* tie, int n, int* rank) {
  const int tid = threadIdx.x, i = tid % n, parts = blockDim.x / n;
  const double zi = z[i];
  const uint64_t at = tie[i];
  int before = 0;
  if (tid < parts * n)
    for (int j = tid / n; j < n; j += parts) before += z[j] > zi || (z[j] == zi && tie[j] > at);
  if (before) atomicAdd(rank + i, before);
}

// A workgroup per request, a wave per beam.  The wave joins its chunks' sums and finds
// its W best chunks, by the first of their sorted keys; of all beams' the W best
// chunks hold the W best candidates.  A thread each, ranked by how many come before.
// Bound by the way through fp64 exponentials and three barriers: 3.6 us for four beams, 5.9
// for 32 requests of eight.
__global__ __launch_bounds__(64 * DSA_MAX_BEAMS) void beam_pick_kernel(BeamArgs a) {
  constexpr int kAll = DSA_MAX_BEAMS * DSA_MAX_BEAMS;
  __shared__ double z_s[kAll];
  __shared__ uint64_t tie_s[kAll];
  __shared__ int chunk_s[kAll], best_s[DSA_MAX_BEAMS];
  __shared__ double off_s[DSA_MAX_BEAMS];
  __shared__ float top_s[DSA_MAX_BEAMS];
  __shared__ int rank_s[2][kAll], some_s;
  __shared__ __attribute__((aligned(16))) uint64_t head_s[DSA_MAX_BEAMS][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b = blockIdx.x, n = a.W * a.W;
  const int64_t beam = static_cast<int64_t>(b) * a.W + wave, part = beam * a.chunks;
  const uint64_t* keys = a.cands + part * a.W;
  const float old = a.score[beam];
  const bool one = lane < a.chunks;
  const float t0 = one ? a.tops[part + lane] : -__builtin_inff();
  const double s0 = one ? a.sums[part + lane] : 0.;
  const uint64_t k0 = one ? keys[static_cast<int64_t>(lane) * a.W] : 0;
  if (tid < DSA_MAX_BEAMS) best_s[tid] = -1;
  if (tid < n) rank_s[0][tid] = rank_s[1][tid] = 0;
  if (tid == 0) some_s = 0;

  float top = t0;
  for (int c = lane + 64; c < a.chunks; c += 64) top = fmaxf(top, a.tops[part + c]);
  top = wave_max(top);
  auto scaled = [&](float t, double s) {
    return t > -__builtin_inff() ? s * exp(static_cast<double>(t) - static_cast<double>(top)) : s;
  };
  double sum = scaled(t0, s0);
  for (int c = lane + 64; c < a.chunks; c += 64) sum += scaled(a.tops[part + c], a.sums[part + c]);
  sum = wave_sum_f64(sum);
  const double off = static_cast<double>(old) - log(sum);
  if (lane == 0) {
    off_s[wave] = off;
    top_s[wave] = top;
  }

  // The beam's best chunks (keys are all different but for 0, which is none).
  const int mine = wave * a.W;
  if (lane < a.W) {
    z_s[mine + lane] = -__builtin_inf();
    tie_s[mine + lane] = 0;
    chunk_s[mine + lane] = -1;
  }
  fence_wave();
  if (a.chunks <= 64) {
    head_s[wave][lane] = k0;
    fence_wave();
    const int rank = key_rank(k0, head_s[wave], (a.chunks + 3) & ~3);
    if (k0 && rank < a.W) {
      const BeamCand c = beam_cand(top, off, wave, k0);
      z_s[mine + rank] = c.z;
      tie_s[mine + rank] = c.tie;
      chunk_s[mine + rank] = mine / a.W * a.chunks + lane;
    }
  } else {
    uint64_t under = ~uint64_t{0};
    for (int k = 0; k < a.W; ++k) {
      uint64_t most = 0;
      int at = -1;
      for (int c = lane; c < a.chunks; c += 64) {
        const uint64_t key = keys[static_cast<int64_t>(c) * a.W];
        if (key < under && key > most) {
          most = key;
          at = c;
        }
      }
      under = wave_max_u64(most);
      if (under && most == under) {
        const BeamCand c = beam_cand(top, off, wave, most);
        z_s[mine + k] = c.z;
        tie_s[mine + k] = c.tie;
        chunk_s[mine + k] = mine / a.W * a.chunks + at;
      }
    }
  }
  __syncthreads();
  cand_ranks(z_s, tie_s, n, rank_s[0]);
  __syncthreads();
  if (tid < n && z_s[tid] > -__builtin_inf() && rank_s[0][tid] < a.W)
    best_s[rank_s[0][tid]] = chunk_s[tid];
  __syncthreads();
  if (tid < n) {  // the best chunks' keys
    const int chunk = best_s[tid / a.W], w = chunk < 0 ? 0 : chunk / a.chunks;
    const uint64_t key = chunk < 0 ? 0
                                   : a.cands[(static_cast<int64_t>(b) * a.W * a.chunks + chunk) * a.W +
                                             tid % a.W];
    const BeamCand c = beam_cand(top_s[w], off_s[w], w, key);
    z_s[tid] = c.z;
    tie_s[tid] = c.tie;
    if (c.z > -__builtin_inf()) atomicAdd(&some_s, 1);
  }
  __syncthreads();
  cand_ranks(z_s, tie_s, n, rank_s[1]);
  __syncthreads();
  if (tid >= n) return;
  const int rank = rank_s[1][tid];
  const int64_t to = static_cast<int64_t>(b) * a.W;
  if (z_s[tid] > -__builtin_inf() && rank < a.W) {
    a.next[to + rank] = static_cast<float>(z_s[tid]);
    a.parent[to + rank] = b * a.W + cand_beam(tie_s[tid]);
    a.token[to + rank] = cand_token(tie_s[tid]);
  }
  if (tid >= some_s && tid < a.W) {  // where there are fewer
    a.next[to + tid] = -__builtin_inff();
    a.parent[to + tid] = -1;
    a.token[to + tid] = -1;
  }
}

}  // namespace

// About two workgroups per CU or more, a row in equal chunks of 16-byte pieces.
BeamLaunch beam_launch(int B, int W, int V, bool bf16) {
  BeamLaunch l{};
  const int vl = bf16 ? 8 : 4;
  l.many = static_cast<int64_t>(B) * W * V > int64_t{512} * kBeamThreads * kFew;
  const int64_t pieces = (V + vl - 1) / vl;
  const int64_t most = kBeamThreads * (l.many ? kMany : kFew) / vl;
  l.chunks = static_cast<int>((pieces + most - 1) / most);
  l.per = static_cast<int>((pieces + l.chunks - 1) / l.chunks);
  const size_t n = static_cast<size_t>(B) * W * l.chunks;
  l.cands = 0;
  l.sums = l.cands + n * W * 8;
  l.tops = l.sums + n * 8;
  l.bytes = (l.tops + n * 4 + 255) / 256 * 256;
  return l;
}

hipError_t launch_beam(BeamArgs a, hipStream_t st) {
  const int64_t parts = static_cast<int64_t>(a.B) * a.W * a.chunks;
  const hipError_t e = launch_parts(parts, kBeamThreads, [&](uint32_t first, dim3 grid) {
    const dim3 block(kBeamThreads);
    a.first = first;
    if (a.bf16)
      a.many ? beam_row_kernel<true, kMany><<<grid, block, 0, st>>>(a)
             : beam_row_kernel<true, kFew><<<grid, block, 0, st>>>(a);
    else
      a.many ? beam_row_kernel<false, kMany><<<grid, block, 0, st>>>(a)
             : beam_row_kernel<false, kFew><<<grid, block, 0, st>>>(a);
  });
  if (e != hipSuccess) return e;
  beam_pick_kernel<<<dim3(a.B), dim3(64 * a.W), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace dsa
