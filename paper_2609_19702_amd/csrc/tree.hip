// Trees of drafted tokens: their plan, their verification, and the accepted
// rows' way into the caches.
#include "device.h"
#include "tree.h"

namespace dsa {
namespace {

constexpr int kMaxNodes = DSA_MAX_TREE_NODES;
constexpr int kMaxWords = kMaxNodes / 32;

// Depth and ancestors by pointer doubling: after round k a node knows its 2^k
// nearest ancestors (itself among them) and how far it looked, so eight rounds
// reach the root of any tree, where a walk would take a step per level.  One
// workgroup per request, one thread per node.  Bound by its launch and the rounds'
// latency: 3.6 us for one tree of 7 nodes, 6.4 for 24 of 61.
__global__ __launch_bounds__(kMaxNodes) void tree_plan_kernel(TreePlanArgs a) {
  __shared__ uint32_t anc[kMaxNodes][kMaxWords + 1];
  __shared__ int up[kMaxNodes], dep[kMaxNodes];
  __shared__ int flag, deepest;
  const int b = blockIdx.x, i = threadIdx.x;
  const int n = a.count ? min(max(a.count[b], 0), a.N) : a.N;
  if (i == 0) flag = deepest = 0;
  __syncthreads();
  int p = -1;
  if (i < n) {
    p = a.parent[b * a.N + i];
    if (p < -1 || p >= i) {
      p = -1;
      flag = DSA_TREE_FLAG_BAD_PARENT;
    }
  }
  const int parent = p;
  uint32_t m[kMaxWords];
#pragma unroll
  for (int w = 0; w < kMaxWords; ++w) m[w] = w == i / 32 ? 1u << (i & 31) : 0u;
  int d = p >= 0;
  while (__syncthreads_or(p >= 0)) {
#pragma unroll
    for (int w = 0; w < kMaxWords; ++w) anc[i][w] = m[w];
    up[i] = p;
    dep[i] = d;
    __syncthreads();
    if (p >= 0) {
#pragma unroll
      for (int w = 0; w < kMaxWords; ++w) m[w] |= anc[p][w];
      d += dep[p];
      p = up[p];
    }
  }
  if (i < n) atomicMax(&deepest, d);
  __syncthreads();
  if (i < a.N) {
    a.depth[b * a.N + i] = d;
    a.out_parent[b * a.N + i] = parent;
#pragma unroll
    for (int w = 0; w < kMaxWords; ++w)
      if (w < a.words) a.anc[(static_cast<int64_t>(b) * a.N + i) * a.words + w] = m[w];
  }
  if (i == 0) {
    a.flags[b] = flag;
    a.max_depth[b] = deepest;
  }
}

constexpr int kVerifyWaves = 16;
constexpr int kVerifyBlock = 64 * kVerifyWaves;
constexpr int kScan = 1024;  // tokens a wave takes at a time, 16 to a lane

__device__ __forceinline__ double wave_add(double x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o, 64);
  return x;
}

// Sum over lanes 0 .. l of a wave.
__device__ __forceinline__ double wave_upto(double x, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double y = __shfl_up(x, o, 64);
    if (lane >= o) x += y;
  }
  return x;
}

// What the rejected children of a node leave of its distribution, up to a
// factor.  With draft rows, P_0 = p and P_k+1 = max(P_k - q, 0) / its sum is
// max(p - a_k q, 0) / s_k with a_0 = 0, s_0 = 1, a_k+1 = a_k + s_k and s_k the sum
// of max(p - a_k q, 0): one multiply-add per token, however many were rejected.
// Without, the tokens taken out are gone.
struct Rest {
  const float* p;  // target row
  const float* q;  // draft row, or nullptr
  double a;
  const int* taken;
  int ntaken;

  // fmax gives 0 for NaN.
  __device__ __forceinline__ static double of(float p, float q, double a) {
    return fmax(fma(-a, static_cast<double>(fmaxf(q, 0.f)), static_cast<double>(p)), 0.);
  }
  // Some taken token in [lo, hi): then every value there is checked.
  __device__ __forceinline__ bool any(int lo, int hi) const {
    bool yes = false;
    for (int i = 0; i < ntaken; ++i) yes |= taken[i] >= lo && taken[i] < hi;
    return yes;
  }
  __device__ __forceinline__ bool gone(int v) const {
    bool yes = false;
    for (int i = 0; i < ntaken; ++i) yes |= taken[i] == v;
    return yes;
  }
  __device__ __forceinline__ double at(int v) const {
    return gone(v) ? 0. : of(p[v], q ? q[v] : 0.f, a);
  }
  // A lane's sum over the tokens [lo, hi) that it takes.  1024 at a time with 8
  // loads of 16 bytes on their way (4 where nothing was rejected yet, a = 0): one CU
  // reads a row, and only bytes in flight make it fast.  Rows need not be
  // 16-byte aligned.
  __device__ __forceinline__ double sum(int lane, int lo, int hi) const {
    struct __attribute__((packed, aligned(4))) Four {
      float f[4];
    };
    constexpr int kWide = 4;
    double s = 0.;
    if (any(lo, hi)) {
      for (int v = lo + lane; v < hi; v += 64) s += at(v);
      return s;
    }
    for (; hi - lo >= 256 * kWide; lo += 256 * kWide) {
      Four x[kWide], y[kWide];
      const Four* px = reinterpret_cast<const Four*>(p + lo) + lane;
      const Four* qx = reinterpret_cast<const Four*>(q + lo) + lane;
#pragma unroll
      for (int e = 0; e < kWide; ++e) x[e] = px[64 * e];
      if (a != 0.) {
#pragma unroll
        for (int e = 0; e < kWide; ++e) y[e] = qx[64 * e];
#pragma unroll
        for (int e = 0; e < kWide; ++e)
#pragma unroll
          for (int k = 0; k < 4; ++k) s += of(x[e].f[k], y[e].f[k], a);
      } else {
#pragma unroll
        for (int e = 0; e < kWide; ++e)
#pragma unroll
          for (int k = 0; k < 4; ++k) s += fmax(static_cast<double>(x[e].f[k]), 0.);
      }
    }
    for (; lo < hi; lo += kScan) {
      float x[16], y[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int v = min(lo + 64 * e + lane, hi - 1);
        x[e] = p[v];
        y[e] = a != 0. ? q[v] : 0.f;
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) s += of(lo + 64 * e + lane < hi ? x[e] : 0.f, y[e], a);
    }
    return s;
  }
};

// One workgroup per request.  What the decisions read of the distributions, two
// numbers per drafted token, is gathered for all nodes at once; the walk down
// the tree then runs on LDS.  The vocabulary is only streamed where a child was
// rejected and the residual's sum is needed (draft rows), and for the next
// token, where the sums of that last pass, a sixteenth of the vocabulary per
// wave, lead to the sixteenth it lies in, and so on down.  Sums and comparisons
// are in fp64: every difference of two fp32 values that is compared with a
// random number is then exact or nearly so.  Bound by latency and by what one CU
// reads of a row from memory (about 40 GB/s, 6.5 us for 65536 fp32 numbers): 8 us for a
// chain of 6 over 16384 tokens, 37 to 50 for 64 trees of 24 nodes over 65539, both with
// draft rows.  A request spread over workgroups would need a workspace
// and a launch per rejection.
__global__ __launch_bounds__(kVerifyBlock) void tree_verify_kernel(VerifyArgs a) {
  __shared__ int parent[kMaxNodes], token[kMaxNodes], path[kMaxNodes], taken[kMaxNodes];
  __shared__ float uni[kMaxNodes], px[kMaxNodes], qx[kMaxNodes];
  __shared__ double part[2][kVerifyWaves];  // sums of the waves' shares, two passes in turn
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = a.count ? min(max(a.count[b], 0), a.N) : a.N;
  const int V = a.V;
  const bool draft = a.draft != nullptr;
  const float last = a.uniform[static_cast<int64_t>(b) * (a.N + 1) + a.N];
  if (tid < kMaxNodes) {
    int par = -1, tok = -1;
    float u = 1.f, p = 0.f, q = 0.f;
    if (tid < n) {
      par = a.parent ? a.parent[b * a.N + tid] : tid - 1;
      tok = a.tokens[b * a.N + tid];
      u = a.uniform[static_cast<int64_t>(b) * (a.N + 1) + tid];
      if (par < 0 || par >= tid) par = -1;
      if (par >= 0 && tok >= 0 && tok < V) {
        const int64_t at = (static_cast<int64_t>(b) * a.N + par) * V + tok;
        p = a.target[at];
        if (draft) q = a.draft[at];
      }
    }
    parent[tid] = par;
    token[tid] = tok;
    uni[tid] = u;
    px[tid] = p > 0.f ? p : 0.f;
    qx[tid] = q > 0.f ? q : 0.f;
    path[tid] = -1;
  }
  __syncthreads();

  Rest rest{nullptr, nullptr, 0., taken, 0};
  const int share = V / kVerifyWaves;  // tokens per wave; the last one takes the rest, too
  int turn = 0;
  // The residual's sum; the waves' shares of it stay in part[turn].
  auto pass = [&]() {
    turn ^= 1;
    const double s = wave_add(rest.sum(lane, wave * share, wave == kVerifyWaves - 1 ? V : (wave + 1) * share));
    if (lane == 0) part[turn][wave] = s;
    __syncthreads();
    double all = 0.;
#pragma unroll
    for (int i = 0; i < kVerifyWaves; ++i) all += part[turn][i];
    return all;
  };

  int cur = 0, len = 0;
  double sum = 0.;
  if (n > 0) {
    bool summed = false;  // part[turn] belongs to `rest`
    for (;;) {
      if (tid == 0) path[len] = cur;
      ++len;
      const int64_t row = (static_cast<int64_t>(b) * a.N + cur) * V;
      rest.p = a.target + row;
      rest.q = draft ? a.draft + row : nullptr;
      rest.a = 0.;
      rest.ntaken = 0;
      double s = 1.;       // the residual's sum (draft rows), or what is not taken out
      bool spent = false;  // nothing is left of the residual
      summed = false;
      int next = -1;
      for (int w = 0; w < a.N && next < 0; w += 64) {
        uint64_t kids = __ballot(w + lane > cur && parent[w + lane] == cur);
        while (kids && next < 0) {
          const int i = w + __builtin_ctzll(kids);
          kids &= kids - 1;
          const double u = uni[i], p = px[i];
          if (draft) {
            if (spent) continue;
            if (u * static_cast<double>(qx[i]) * s < Rest::of(px[i], qx[i], rest.a)) {
              next = i;
              break;
            }
            const double before = rest.a;
            rest.a += s;
            const double left = pass();
            summed = spent = left <= 0.;
            if (spent) {
              rest.a = before;
              summed = false;
            } else {
              s = sum = left;
              summed = true;
            }
          } else {
            bool again = false;
            for (int e = 0; e < rest.ntaken; ++e) again |= taken[e] == token[i];
            if (again) continue;
            if (p > 0. && u * s < p) {
              next = i;
              break;
            }
            s -= p;
            if (tid == 0) taken[rest.ntaken] = token[i];
            ++rest.ntaken;
            __syncthreads();
          }
        }
      }
      if (next < 0) break;
      cur = next;
      __syncthreads();  // `taken` starts anew
    }
    if (!summed) sum = pass();
  }
  if (tid < a.N) a.path[static_cast<int64_t>(b) * a.N + tid] = path[tid];
  if (tid == 0) a.accepted[b] = len;

  // The next token: the first share whose running sum passes the target, then the
  // first of its sixteenths, down to what one wave holds.  Rounding can leave the
  // target unpassed at the very end: then the last share with any mass, and the
  // last token of it.
  if (!(n > 0 && sum > 0.)) {
    if (tid == 0) a.next[b] = -1;
    return;
  }
  const double aim = static_cast<double>(last) * sum;
  double before = 0.;  // sum ahead of `lo`
  bool past = false;   // the target was not passed
  int lo = 0, hi = V;
  // The share that the target lies in, of those in part[turn].
  auto pick = [&]() {
    int at = -1, some = 0;
    for (int i = 0; i < kVerifyWaves && at < 0; ++i) {
      const double x = part[turn][i];
      if (x > 0.) some = i;
      if (x > 0. && !past && before + x > aim)
        at = i;
      else
        before += x;
    }
    past |= at < 0;
    return at < 0 ? some : at;
  };
  int size = share, at = pick();
  for (;;) {
    lo += at * size;
    hi = at == kVerifyWaves - 1 ? hi : lo + size;
    turn ^= 1;
    if (hi - lo <= 64 * kVerifyWaves) break;
    size = (hi - lo) / kVerifyWaves;
    const int from = lo + wave * size;
    const double s =
        wave_add(rest.sum(lane, from, wave == kVerifyWaves - 1 ? hi : from + size));
    if (lane == 0) part[turn][wave] = s;
    __syncthreads();
    at = pick();
  }
  // A token per thread.
  const int v = lo + tid;
  const double r = v < hi ? rest.at(v) : 0.;
  const double s = wave_add(r);
  if (lane == 0) part[turn][wave] = s;
  __syncthreads();
  at = pick();
  if (wave != at) return;
  const double upto = before + wave_upto(r, lane);
  const uint64_t hit = __ballot(!past && r > 0. && upto > aim), mass = __ballot(r > 0.);
  const int found = hit ? __builtin_ctzll(hit) : 63 - __builtin_clzll(mass | 1);
  if (lane == 0) a.next[b] = lo + 64 * wave + found;
}

// Eight elements of a row and of its V row per thread: 16 bytes in, 16 (bf16)
// or 8 (fp8) out.  Bound by the bytes it moves: 43 us for 201 MB, 4.7 TB/s (4
// layers of 32 prompts of 256 tokens, 8 heads of 128, into fp8).
template <bool FP8>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a, int chunks, int blocks) {
  const int64_t lb = blockIdx.x / blocks;  // layer and request
  const int b = static_cast<int>(lb % a.B), layer = static_cast<int>(lb / a.B);
  const int at = (blockIdx.x % blocks) * 256 + threadIdx.x;
  const int c = at % chunks, h = at / chunks % a.Hkv, e = at / chunks / a.Hkv;
  const TreeReq rq = tree_request(a.base, a.count, b, a.N, a.Lp, a.Ldec);
  const int n = a.accepted ? min(max(a.accepted[b], 0), rq.n) : rq.n;
  if (e >= n) return;
  const int pos = rq.base + e, last = min(rq.base + n, a.Ldec) - 1;
  if (pos >= a.Ldec) return;
  const int32_t* path = a.path ? a.path + b * static_cast<int64_t>(a.N) : nullptr;
  const int node = path ? path[e] : e;
  if (node < 0 || node >= rq.n) return;
  int row = a.Lp + pos;
  if (a.ring && pos >= a.S) {
    // a later row of this call takes the slot, but for one that is skipped
    for (int f = e + a.ring; rq.base + f <= last; f += a.ring)
      if (!path || (path[f] >= 0 && path[f] < rq.n)) return;
    row = a.Lp + a.S + (pos - a.S) % a.ring;
  }
  const int64_t from = layer * a.nsl + b * a.nsb + node * a.nsn + h * a.nsh + c * 8;
  const int64_t base = layer * a.sl + (a.row_base ? a.row_base[b] * (FP8 ? 1 : 2) : b * a.sb) +
                       h * a.sh + row * a.sr + c * (FP8 ? 8 : 16);
  const uint4 xk = *reinterpret_cast<const uint4*>(a.kn + from);
  const uint4 xv = *reinterpret_cast<const uint4*>(a.vn + from);
  if constexpr (FP8) {
    const int64_t s = (static_cast<int64_t>(layer) * a.B + b) * a.Hkv + h;
    auto code = [](const uint4& x, float scale) {
      float f[8];
      unpack8(x, f);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float y = f[i] / scale;
        f[i] = y != y ? y : fminf(fmaxf(y, -448.f), 448.f);
      }
      uint2 w;
      w.x = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
      w.x = __builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], w.x, true);
      w.y = __builtin_amdgcn_cvt_pk_fp8_f32(f[4], f[5], 0, false);
      w.y = __builtin_amdgcn_cvt_pk_fp8_f32(f[6], f[7], w.y, true);
      return w;
    };
    *reinterpret_cast<uint2*>(a.k + base) = code(xk, a.ks ? a.ks[s] : 1.f);
    *reinterpret_cast<uint2*>(a.v + base) = code(xv, a.vs ? a.vs[s] : 1.f);
  } else {
    *reinterpret_cast<uint4*>(a.k + base) = xk;
    *reinterpret_cast<uint4*>(a.v + base) = xv;
  }
}

}  // namespace

hipError_t launch_tree_plan(const TreePlanArgs& a, hipStream_t st) {
  tree_plan_kernel<<<dim3(a.B), dim3(kMaxNodes), 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_verify(const VerifyArgs& a, int B, hipStream_t st) {
  tree_verify_kernel<<<dim3(B), dim3(kVerifyBlock), 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_append(const AppendArgs& a, int D, int dtype, hipStream_t st) {
  const int chunks = D / 8;
  const int blocks = static_cast<int>((static_cast<int64_t>(a.N) * a.Hkv * chunks + 255) / 256);
  const dim3 grid(static_cast<uint32_t>(static_cast<int64_t>(blocks) * a.layers * a.B));
  if (dtype == DSA_KV_FP8_E4M3)
    append_kernel<true><<<grid, dim3(256), 0, st>>>(a, chunks, blocks);
  else
    append_kernel<false><<<grid, dim3(256), 0, st>>>(a, chunks, blocks);
  return hipGetLastError();
}

}  // namespace dsa
