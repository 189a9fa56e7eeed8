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
// workgroup per request, one thread per node.
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
constexpr int kMaxBlocks = 1024;  // of a vocabulary, each a multiple of kScan tokens
constexpr int kScan = 1024;       // tokens a wave takes at a time

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

// One workgroup per request.  What the decisions read of the distributions, two
// numbers per drafted token, is gathered for all nodes at once; the walk down
// the tree then runs on LDS.  The vocabulary is only streamed where a child was
// rejected and the residual's sum is needed (draft rows), and for the next
// token; the blocks' sums of that last pass lead to the block it lies in.
// Sums and comparisons are in fp64: every difference of two fp32 values that
// is compared with a random number is then exact or nearly so.
__global__ __launch_bounds__(kVerifyBlock) void tree_verify_kernel(VerifyArgs a) {
  __shared__ int parent[kMaxNodes], token[kMaxNodes], path[kMaxNodes], taken[kMaxNodes];
  __shared__ float uni[kMaxNodes], px[kMaxNodes], qx[kMaxNodes];
  __shared__ double z[kMaxNodes + 1], zinv[kMaxNodes + 1];  // residual sums of the node at hand
  __shared__ double block_sum[kMaxBlocks];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = a.count ? min(max(a.count[b], 0), a.N) : a.N;
  const int V = a.V;
  const bool draft = a.draft != nullptr;
  if (tid < kMaxNodes) {
    int par = -1, tok = -1;
    float u = 1.f, p = 0.f, q = 0.f;
    if (tid < n) {
      par = a.parent ? a.parent[b * a.N + tid] : tid - 1;
      if (par < 0 || par >= tid) par = -1;
      tok = a.tokens[b * a.N + tid];
      u = a.uniform[static_cast<int64_t>(b) * (a.N + 1) + tid];
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

  const int span = kScan * ((V + kScan * kMaxBlocks - 1) / (kScan * kMaxBlocks));  // tokens per block
  const int blocks = (V + span - 1) / span;
  const float* tr = nullptr;
  const float* dr = nullptr;
  int ntaken = 0;
  // What is left of token v's probability after k rejected children.
  auto residual = [&](float pf, float qf, int k) {
    double r = pf > 0.f ? pf : 0.f;
    const double q = qf > 0.f ? qf : 0.f;
    for (int i = 0; i < k; ++i) {
      r = r * zinv[i] - q;
      r = r > 0. ? r : 0.;
    }
    return r;
  };
  auto left = [&](int v, float pf, float qf, int k) {
    if (draft) return residual(pf, qf, k);
    double r = pf > 0.f ? pf : 0.f;
    for (int i = 0; i < ntaken; ++i)
      if (taken[i] == v) r = 0.;
    return r;
  };
  // Block sums of the residual after k rejected children of the node at hand.
  auto pass = [&](int k) {
    for (int j = wave; j < blocks; j += kVerifyWaves) {
      double s = 0.;
      for (int v0 = j * span; v0 < min((j + 1) * span, V); v0 += kScan) {
        float p[16], q[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int v = v0 + 64 * e + lane;
          p[e] = v < V ? tr[v] : 0.f;
          q[e] = draft && v < V ? dr[v] : 0.f;
        }
#pragma unroll
        for (int e = 0; e < 16; ++e) s += left(v0 + 64 * e + lane, p[e], q[e], k);
      }
      s = wave_add(s);
      if (lane == 0) block_sum[j] = s;
    }
    __syncthreads();
  };
  // Their total: every wave computes it alike.
  auto total = [&]() {
    double s = 0.;
    for (int j = lane; j < blocks; j += 64) s += block_sum[j];
    return wave_add(s);
  };

  int cur = 0, len = 0, k = 0;
  bool summed = false;  // block_sum holds the sums for (cur, k)
  double sum = 0.;
  if (n > 0) {
    for (;;) {
      if (tid == 0) {
        path[len] = cur;
        z[0] = zinv[0] = 1.;
      }
      ++len;
      tr = a.target + (static_cast<int64_t>(b) * a.N + cur) * V;
      dr = draft ? a.draft + (static_cast<int64_t>(b) * a.N + cur) * V : nullptr;
      k = ntaken = 0;
      summed = false;
      double rest = 1.;
      bool spent = false;
      int next = -1;
      __syncthreads();
      for (int w = 0; w < kMaxNodes && next < 0; w += 64) {
        uint64_t kids = __ballot(w + lane > cur && parent[w + lane] == cur);
        while (kids && next < 0) {
          const int i = w + __builtin_ctzll(kids);
          kids &= kids - 1;
          const double u = uni[i];
          if (draft) {
            if (spent) continue;
            const double r = residual(px[i], qx[i], k);
            if (u * static_cast<double>(qx[i]) * z[k] < r) {
              next = i;
              break;
            }
            pass(k + 1);
            const double s = total();
            __syncthreads();
            if (s > 0.) {
              ++k;
              if (tid == 0) {
                z[k] = s;
                zinv[k] = 1. / s;
              }
              sum = s;
              summed = true;
              __syncthreads();
            } else {
              spent = true;
              summed = false;
            }
          } else {
            const double p = px[i];
            bool again = false;
            for (int e = 0; e < ntaken; ++e) again |= taken[e] == token[i];
            if (!again && p > 0. && u * rest < p) {
              next = i;
              break;
            }
            if (!again) {
              rest -= p;
              __syncthreads();
              if (tid == 0) taken[ntaken] = token[i];
              ++ntaken;
              __syncthreads();
            }
          }
        }
      }
      if (next < 0) break;
      cur = next;
      __syncthreads();
    }
    if (!summed) {
      pass(k);
      sum = total();
    }
  }
  if (tid < a.N) a.path[b * a.N + tid] = path[tid];
  if (tid == 0) a.accepted[b] = len;
  if (wave) return;

  // The next token, by the first wave: the first block whose running sum passes
  // the target, then the first token in it.
  int found = -1;
  if (n > 0 && sum > 0.) {
    const double aim = static_cast<double>(a.uniform[static_cast<int64_t>(b) * (a.N + 1) + a.N]) * sum;
    double before = 0.;
    int at = -1, some = -1;  // the block, and the last one with any mass
    for (int j0 = 0; j0 < blocks && at < 0; j0 += 64) {
      const double x = j0 + lane < blocks ? block_sum[j0 + lane] : 0.;
      const double upto = before + wave_upto(x, lane);
      const uint64_t over = __ballot(upto > aim && x > 0.);
      const uint64_t mass = __ballot(x > 0.);
      if (mass) some = j0 + 63 - __builtin_clzll(mass);
      if (over) {
        const int w = __builtin_ctzll(over);
        at = j0 + w;
        before = __shfl(upto - x, w, 64);
      } else {
        before = __shfl(upto, 63, 64);
      }
    }
    const bool past = at < 0;  // rounding only: take the last token with mass
    if (past) at = some;
    int last = -1;
    for (int v0 = at * span; v0 < min((at + 1) * span, V) && found < 0; v0 += kScan) {
      double r[16], s = 0.;
      const int v1 = v0 + lane * 16;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const bool in = v1 + e < V;
        r[e] = left(v1 + e, in ? tr[v1 + e] : 0.f, in && draft ? dr[v1 + e] : 0.f, k);
        s += r[e];
      }
      double upto = before + wave_upto(s, lane) - s;
      int mine = -1, tail = -1;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        upto += r[e];
        if (r[e] > 0.) {
          tail = v1 + e;
          if (mine < 0 && !past && upto > aim) mine = v1 + e;
        }
      }
      const uint64_t hit = __ballot(mine >= 0), any = __ballot(tail >= 0);
      if (any) last = __shfl(tail, 63 - __builtin_clzll(any), 64);
      if (hit) found = __shfl(mine, __builtin_ctzll(hit), 64);
      before = __shfl(upto, 63, 64);
    }
    if (found < 0) found = last;
  }
  if (lane == 0) a.next[b] = found;
}

// Eight elements of a row and of its V row per thread: 16 bytes in, 16 (bf16)
// or 8 (fp8) out.  Bound by the bytes it moves.
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
  int row = a.Lp + pos;
  if (a.ring && pos >= a.S) {
    if (pos + a.ring <= last) return;  // a later row of this call takes the slot
    row = a.Lp + a.S + (pos - a.S) % a.ring;
  }
  const int node = a.path ? a.path[b * static_cast<int64_t>(a.N) + e] : e;
  if (node < 0 || node >= rq.n) return;
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
