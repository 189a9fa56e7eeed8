// One step of a beam search: the best candidates over beams and vocabulary.
#include "device.h"
#include "paged.h"

namespace dsa {
namespace {

constexpr int kBeamThreads = 256;
constexpr int kBeamWaves = kBeamThreads / 64;

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

// A workgroup takes R values per thread of a row: their maximum, the sum of their
// exponentials in fp64, and their W largest in order.
template <bool BF16, int R>
__global__ __launch_bounds__(kBeamThreads) void beam_row_kernel(BeamArgs a) {
  __shared__ float top_s[kBeamWaves];
  __shared__ double sum_s[kBeamWaves];
  __shared__ uint64_t best_s[64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int chunk = blockIdx.x % a.chunks, row = blockIdx.x / a.chunks;
  const int first = chunk * a.per;
  float x[R];
#pragma unroll
  for (int i = 0; i < R; ++i) {
    const int v = first + i * kBeamThreads + threadIdx.x;
    const int64_t at = row * a.stride + min(v, a.V - 1);
    float y;
    if constexpr (BF16)
      y = bf16_lo(static_cast<const uint16_t*>(a.x)[at]);
    else
      y = static_cast<const float*>(a.x)[at];
    x[i] = v < a.V ? y : -__builtin_inff();
  }
  float top = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < R; ++i) top = fmaxf(top, x[i]);
  top = wave_max(top);
  if (lane == 0) top_s[wave] = top;
  __syncthreads();
  for (int w = 0; w < kBeamWaves; ++w) top = fmaxf(top, top_s[w]);
  // A chunk of -infinities adds nothing; a NaN or +infinity makes the sum a NaN.
  double sum = 0.;
  const float base = top > -__builtin_inff() ? top : 0.f;
#pragma unroll
  for (int i = 0; i < R; ++i) sum += static_cast<double>(fast_exp2((x[i] - base) * 1.4426950408889634f));
  sum = wave_sum_f64(sum);
  if (lane == 0) sum_s[wave] = sum;

  // The wave's W largest, one at a time.
  uint64_t best = 0;  // lane i: the i-th
  uint64_t under = ~uint64_t{0};
  for (int k = 0; k < a.W; ++k) {
    uint64_t mine = 0;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const uint64_t key = beam_key(x[i], first + i * kBeamThreads + static_cast<int>(threadIdx.x));
      mine = key < under && key > mine ? key : mine;
    }
    under = wave_max_u64(mine);
    if (lane == k) best = under;
  }
  if (lane < a.W) best_s[wave * a.W + lane] = best;
  __syncthreads();
  if (wave) return;
  uint64_t mine = lane < kBeamWaves * a.W ? best_s[lane] : 0;
  uint64_t* to = a.cands + static_cast<int64_t>(blockIdx.x) * a.W;
  for (int k = 0; k < a.W; ++k) {
    const uint64_t y = wave_max_u64(mine);
    if (mine == y) mine = 0;
    if (lane == 0) to[k] = y;
  }
  if (lane == 0) {
    double s = 0.;
    for (int w = 0; w < kBeamWaves; ++w) s += sum_s[w];
    a.sums[blockIdx.x] = s;
    a.tops[blockIdx.x] = top;
  }
}

// A workgroup per request joins its beams' parts and takes the best.
__global__ __launch_bounds__(kBeamThreads) void beam_pick_kernel(BeamArgs a) {
  __shared__ double off_s[DSA_MAX_BEAMS];  // score - log of the sum of exponentials
  __shared__ double best_s[kBeamWaves];
  __shared__ int64_t place_s[kBeamWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b = blockIdx.x;
  const int64_t part = static_cast<int64_t>(b) * a.W * a.chunks;
  for (int w = wave; w < a.W; w += kBeamWaves) {
    float top = -__builtin_inff();
    for (int c = lane; c < a.chunks; c += 64) top = fmaxf(top, a.tops[part + w * a.chunks + c]);
    top = wave_max(top);
    double sum = 0.;
    for (int c = lane; c < a.chunks; c += 64) {
      const float t = a.tops[part + w * a.chunks + c];
      const double s = a.sums[part + w * a.chunks + c];
      sum += t > -__builtin_inff() ? s * exp(static_cast<double>(t) - static_cast<double>(top)) : s;
    }
    sum = wave_sum_f64(sum);
    if (lane == 0)
      off_s[w] = static_cast<double>(a.score[static_cast<int64_t>(b) * a.W + w]) -
                 (static_cast<double>(top) + log(sum));
  }
  __syncthreads();
  const int per = a.chunks * a.W, n = a.W * per;
  const double none = -__builtin_inf();
  double under = __builtin_inf();
  int64_t under_place = -1;
  for (int k = 0; k < a.W; ++k) {
    double best = none;
    int64_t place = (int64_t{1} << 62);
    for (int e = tid; e < n; e += kBeamThreads) {
      const uint64_t key = a.cands[part * a.W + e];
      const int w = e / per;
      if (!key) continue;
      const double z = off_s[w] + static_cast<double>(key_value(key));
      const int64_t at = static_cast<int64_t>(w) * a.V + key_place(key);
      if (!(z > none)) continue;
      if (!(z < under || (z == under && at > under_place))) continue;  // taken already
      if (z > best || (z == best && at < place)) {
        best = z;
        place = at;
      }
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) {
      const double z = __shfl_xor(best, o, 64);
      const int64_t at = __shfl_xor(static_cast<long long>(place), o, 64);
      if (z > best || (z == best && at < place)) {
        best = z;
        place = at;
      }
    }
    if (lane == 0) {
      best_s[wave] = best;
      place_s[wave] = place;
    }
    __syncthreads();
    for (int w = 0; w < kBeamWaves; ++w)
      if (best_s[w] > best || (best_s[w] == best && place_s[w] < place)) {
        best = best_s[w];
        place = place_s[w];
      }
    __syncthreads();
    const bool some = best > none;
    under = some ? best : none;
    under_place = some ? place : (int64_t{1} << 62);
    if (tid == 0) {
      const int64_t to = static_cast<int64_t>(b) * a.W + k;
      a.next[to] = some ? static_cast<float>(best) : -__builtin_inff();
      a.parent[to] = some ? b * a.W + static_cast<int>(place / a.V) : -1;
      a.token[to] = some ? static_cast<int>(place % a.V) : -1;
    }
  }
}

}  // namespace

BeamLaunch beam_launch(int B, int W, int V) {
  BeamLaunch l{};
  l.per = kBeamThreads * (static_cast<int64_t>(B) * W * V <= (1 << 20) ? 8 : 32);
  l.chunks = (V + l.per - 1) / l.per;
  const size_t n = static_cast<size_t>(B) * W * l.chunks;
  l.cands = 0;
  l.sums = l.cands + n * W * 8;
  l.tops = l.sums + n * 8;
  l.bytes = (l.tops + n * 4 + 255) / 256 * 256;
  return l;
}

hipError_t launch_beam(const BeamArgs& a, hipStream_t st) {
  const dim3 grid(static_cast<uint32_t>(static_cast<int64_t>(a.B) * a.W * a.chunks));
  const bool many = a.per > 8 * kBeamThreads;
  if (a.bf16)
    many ? beam_row_kernel<true, 32><<<grid, dim3(kBeamThreads), 0, st>>>(a)
         : beam_row_kernel<true, 8><<<grid, dim3(kBeamThreads), 0, st>>>(a);
  else
    many ? beam_row_kernel<false, 32><<<grid, dim3(kBeamThreads), 0, st>>>(a)
         : beam_row_kernel<false, 8><<<grid, dim3(kBeamThreads), 0, st>>>(a);
  beam_pick_kernel<<<dim3(a.B), dim3(kBeamThreads), 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace dsa
