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
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t u = static_cast<uint32_t>(k >> 32);
  return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
__device__ __forceinline__ int key_place(uint64_t k) { return ~static_cast<int>(k); }

__device__ __forceinline__ uint64_t wave_max_u64(uint64_t x) { return ~wave_min_u64(~x); }

__device__ __forceinline__ double wave_sum_f64(double x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}

// Lane's key among the first n lanes' (all different but for 0): how many are larger.
__device__ __forceinline__ int key_rank(uint64_t key, int n) {
  int rank = 0;
  for (int j = 0; j < n; ++j) {
    const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(key >> 32), j);
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(key), j);
    rank += ((static_cast<uint64_t>(hi) << 32) | lo) > key;
  }
  return rank;
}

// A workgroup takes R values per thread of a row: their maximum, the sum of their
// exponentials (fours in fp32, the rest in fp64), and their W largest in order.
//
// A wave's W largest are at least its W-th largest of the lanes' own maxima, and
// few values are: those go into a list, where each is placed by the larger ones' number.
// With more than 64 of them (equal values) the largest are taken out one at a time.
template <bool BF16, int R>
__global__ __launch_bounds__(kBeamThreads) void beam_row_kernel(BeamArgs a) {
  constexpr int VL = BF16 ? 8 : 4, NV = R / VL;  // values of a load, loads
  __shared__ float top_s[kBeamWaves];
  __shared__ double sum_s[kBeamWaves];
  __shared__ uint64_t list_s[kBeamWaves][64];
  __shared__ uint64_t best_s[64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int chunk = blockIdx.x % a.chunks, row = blockIdx.x / a.chunks;
  // Pieces of VL values, which begin at any value: a row's sums do not depend on where it
  // lies, so equal rows tie.
  const uint8_t* start = static_cast<const uint8_t*>(a.x) + row * a.stride * (16 / VL);
  const int first = chunk * a.per, end = min(first + a.per, (a.V + VL - 1) / VL);
  float x[R];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int piece = first + k * kBeamThreads + threadIdx.x, v = piece * VL;
    const bool whole = piece < end && v + VL <= a.V;
    u32x4 w = {0, 0, 0, 0};
    if (whole)
      w = __builtin_nontemporal_load(
          reinterpret_cast<const Piece*>(start + static_cast<int64_t>(v) * (16 / VL)));
    if constexpr (BF16) {
      float f[8];
      unpack8(make_uint4(w.x, w.y, w.z, w.w), f);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[8 * k + i] = f[i];
    } else {
      x[4 * k] = __uint_as_float(w.x);
      x[4 * k + 1] = __uint_as_float(w.y);
      x[4 * k + 2] = __uint_as_float(w.z);
      x[4 * k + 3] = __uint_as_float(w.w);
    }
    if (!whole) {  // the row's end, value by value, and what lies behind
#pragma unroll
      for (int i = 0; i < VL; ++i) {
        x[VL * k + i] = -__builtin_inff();
        if (piece < end && v + i < a.V) {
          if constexpr (BF16)
            x[VL * k + i] = bf16_lo(reinterpret_cast<const uint16_t*>(start)[v + i]);
          else
            x[VL * k + i] = reinterpret_cast<const float*>(start)[v + i];
        }
      }
    }
  }
  auto place = [&](int i) {
    return (first + i / VL * kBeamThreads + static_cast<int>(threadIdx.x)) * VL + i % VL;
  };

  float mine = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < R; ++i) mine = fmaxf(mine, x[i]);
  float top = wave_max(mine);
  if (lane == 0) top_s[wave] = top;
  __syncthreads();
  for (int w = 0; w < kBeamWaves; ++w) top = fmaxf(top, top_s[w]);
  // A chunk of -infinities adds nothing; a NaN or +infinity makes the sum a NaN.
  double sum = 0.;
  const float base = top > -__builtin_inff() ? top : 0.f;
#pragma unroll
  for (int i = 0; i < R; i += 4) {
    float e[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) e[k] = fast_exp2((x[i + k] - base) * 1.4426950408889634f);
    sum += static_cast<double>((e[0] + e[1]) + (e[2] + e[3]));
  }
  sum = wave_sum_f64(sum);
  if (lane == 0) sum_s[wave] = sum;

  // The W-th largest of the lanes' maxima.
  float least = -__builtin_inff(), left = mine;
  for (int k = 0; k < a.W; ++k) {
    least = wave_max(left);
    if (lane == __builtin_ctzll(__ballot(left == least))) left = -__builtin_inff();
  }
  int n = 0;
  uint64_t* list = list_s[wave];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const bool in = x[i] >= least && x[i] > -__builtin_inff();
    const uint64_t some = __ballot(in);
    if (some) {
      const int at = n + __popcll(some & ((uint64_t(1) << lane) - 1));
      if (in && at < 64) list[at] = beam_key(x[i], place(i));
      n += __popcll(some);
    }
  }
  fence_wave();
  uint64_t best = 0;  // lane i: the i-th
  if (n <= 64) {
    const uint64_t key = lane < n ? list[lane] : 0;
    const int rank = key_rank(key, n);
    fence_wave();
    if (lane < n && rank < a.W) list[rank] = key;
    fence_wave();
    best = lane < min(n, a.W) ? list[lane] : 0;
  } else {
    uint64_t under = ~uint64_t{0};
    for (int k = 0; k < a.W; ++k) {
      uint64_t most = 0;
#pragma unroll
      for (int i = 0; i < R; ++i) {
        const uint64_t key = beam_key(x[i], place(i));
        most = key < under && key > most ? key : most;
      }
      under = wave_max_u64(most);
      if (lane == k) best = under;
    }
  }
  if (lane < a.W) best_s[wave * a.W + lane] = best;
  __syncthreads();
  if (wave) return;
  const int all = kBeamWaves * a.W;  // at most 64
  const uint64_t key = lane < all ? best_s[lane] : 0;
  const int rank = key_rank(key, all);
  uint64_t* to = a.cands + static_cast<int64_t>(blockIdx.x) * a.W;
  const int some = __popcll(__ballot(key != 0));
  if (key && rank < a.W) to[rank] = key;
  if (lane >= some && lane < a.W) to[lane] = 0;
  if (lane == 0) {
    double s = 0.;
    for (int w = 0; w < kBeamWaves; ++w) s += sum_s[w];
    a.sums[blockIdx.x] = s;
    a.tops[blockIdx.x] = top;
  }
}

// A workgroup per request, a wave per beam: the wave joins its chunks, all take the
// best of the beams' W * W candidates, a thread each.
__global__ __launch_bounds__(64 * DSA_MAX_BEAMS) void beam_pick_kernel(BeamArgs a) {
  __shared__ double score_s[DSA_MAX_BEAMS * DSA_MAX_BEAMS];
  __shared__ int64_t place_s[DSA_MAX_BEAMS * DSA_MAX_BEAMS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b = blockIdx.x, n = a.W * a.W;
  const int64_t beam = static_cast<int64_t>(b) * a.W + wave, part = beam * a.chunks;
  const double none = -__builtin_inf();
  const float old = a.score[beam];

  // The first chunks, and the first keys, a lane each.
  const uint64_t* keys = a.cands + part * a.W;
  const int held = a.chunks * a.W;
  uint64_t k0 = lane < held ? keys[lane] : 0, k1 = lane + 64 < held ? keys[lane + 64] : 0;
  float t0 = lane < a.chunks ? a.tops[part + lane] : -__builtin_inff();
  const double s0 = lane < a.chunks ? a.sums[part + lane] : 0.;
  float top = t0;
  for (int c = lane + 64; c < a.chunks; c += 64) top = fmaxf(top, a.tops[part + c]);
  top = wave_max(top);
  auto scaled = [&](float t, double s) {
    return t > -__builtin_inff() ? s * exp(static_cast<double>(t) - static_cast<double>(top)) : s;
  };
  double sum = scaled(t0, s0);
  for (int c = lane + 64; c < a.chunks; c += 64) sum += scaled(a.tops[part + c], a.sums[part + c]);
  sum = wave_sum_f64(sum);
  const double off = static_cast<double>(old) - (static_cast<double>(top) + log(sum));

  // The beam's W largest logits, one at a time.
  uint64_t under = ~uint64_t{0}, best = 0;
  for (int k = 0; k < a.W; ++k) {
    uint64_t most = k0 < under ? k0 : 0;
    most = k1 < under && k1 > most ? k1 : most;
    for (int e = lane + 128; e < held; e += 64) {
      const uint64_t key = keys[e];
      most = key < under && key > most ? key : most;
    }
    under = wave_max_u64(most);
    if (lane == k) best = under;
  }
  if (lane < a.W) {
    const double z = off + static_cast<double>(key_value(best));
    score_s[wave * a.W + lane] = best && z > none ? z : none;
    place_s[wave * a.W + lane] = static_cast<int64_t>(wave) * a.V + key_place(best);
  }
  __syncthreads();
  if (tid >= n) return;
  const double z = score_s[tid];
  const int64_t at = place_s[tid];
  int rank = 0, some = 0;
  for (int j = 0; j < n; ++j) {
    const double y = score_s[j];
    rank += y > z || (y == z && place_s[j] < at);
    some += y > none;
  }
  const int64_t to = static_cast<int64_t>(b) * a.W;
  if (z > none && rank < a.W) {
    a.next[to + rank] = static_cast<float>(z);
    a.parent[to + rank] = b * a.W + static_cast<int>(at / a.V);
    a.token[to + rank] = static_cast<int>(at % a.V);
  }
  if (tid >= some && tid < a.W) {
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

hipError_t launch_beam(const BeamArgs& a, hipStream_t st) {
  const dim3 grid(static_cast<uint32_t>(static_cast<int64_t>(a.B) * a.W * a.chunks));
  const dim3 block(kBeamThreads);
  if (a.bf16)
    a.many ? beam_row_kernel<true, kMany><<<grid, block, 0, st>>>(a)
           : beam_row_kernel<true, kFew><<<grid, block, 0, st>>>(a);
  else
    a.many ? beam_row_kernel<false, kMany><<<grid, block, 0, st>>>(a)
           : beam_row_kernel<false, kFew><<<grid, block, 0, st>>>(a);
  beam_pick_kernel<<<dim3(a.B), dim3(64 * a.W), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace dsa
