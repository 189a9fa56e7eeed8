// Several tokens of a request at once (dsa_tree_*, dsa_kv_append): kernel
// argument blocks, launchers, and the key lists both attention kernels walk.
#pragma once

#include "internal.h"

namespace dsa {

// Checks a K/V cache layout against a call's parameters (as every call that takes one).
dsa_status check_kv(const dsa_kv_layout* kv, const Derived& d);
// Ring slots after the sinks, or 0 where every position maps to itself.
int ring_slots(const dsa_kv_layout* kv, const Derived& d);

constexpr int kTreeNone = 1 << 30;  // "no window": further back than any position
constexpr float kTreeMinScale = 1.1754944e-38f;  // smallest scale of scores: -inf keeps its sign

struct TreePlanArgs {
  const int32_t* parent;
  const int32_t* count;
  int32_t* flags;
  int32_t* max_depth;
  int32_t* depth;
  int32_t* out_parent;
  uint32_t* anc;
  int B, N, words;
};

struct TreeArgs {
  const uint16_t* q;
  const uint16_t* kn;  // new K / V rows, bf16
  const uint16_t* vn;
  const uint8_t* k;    // caches, addressed in bytes
  const uint8_t* v;
  int64_t qsb, qsn, qsh;    // strides in elements
  int64_t nsb, nsn, nsh;
  const int64_t* row_base;  // per-request cache offsets in elements, or nullptr
  int64_t sb, sh, sr;       // cache strides in bytes
  const float* ks;          // fp8: per-(request, KV head) K / V scales, or nullptr
  const float* vs;
  const int32_t* base;
  const int32_t* count;
  const int32_t* max_depth;  // tree plan (nullptr: a chain)
  const int32_t* depth;
  const uint32_t* anc;
  int words;
  float scale_log2;  // |sm_scale| * log2(e), at least kTreeMinScale
  uint32_t q_sign;   // 0x80008000 where sm_scale < 0: the queries' sign flips instead
  void* out;
  float* part;       // split partials (splits > 1)
  int B, Hq, Hkv, G, N, Lp, Ldec;
  int S, W;          // sinks, recent window (kTreeNone: none)
  int ring;          // positions >= S rotate through this many slots (0: linear)
  int row_tiles, splits;
  int split_tiles;   // key tiles of a split, at least (but the last)
};

// Launch of dsa_tree_attention.
struct TreeLaunch {
  int rows;       // query rows per workgroup
  int waves;      // waves per workgroup (streaming)
  int split_tiles;  // tiles of 32 keys per split, at least
  int row_tiles;  // per (request, KV head)
  int splits;
  int64_t workgroups;
  size_t ws_bytes;
};
TreeLaunch tree_launch(const Derived& d, int nodes);

struct VerifyArgs {
  const int32_t* count;
  const int32_t* parent;  // tree plan (nullptr: a chain)
  const int32_t* tokens;
  const float* target;
  const float* draft;
  const float* uniform;
  int32_t* path;
  int32_t* accepted;
  int32_t* next;
  int N, V;
};

struct AppendArgs {
  const uint16_t* kn;
  const uint16_t* vn;
  int64_t nsl, nsb, nsn, nsh;  // strides in elements
  const int32_t* base;
  const int32_t* count;
  const int32_t* path;
  const int32_t* accepted;
  uint8_t* k;
  uint8_t* v;
  const int64_t* row_base;
  int64_t sl, sb, sh, sr;  // cache strides in bytes
  const float* ks;
  const float* vs;
  int layers, B, Hkv, N, Lp, Ldec, S, ring;
};

hipError_t launch_tree_plan(const TreePlanArgs& a, hipStream_t st);
hipError_t launch_tree_bf16(const Derived& d, const TreeLaunch& l, const TreeArgs& a, bool f32,
                            hipStream_t st);
hipError_t launch_tree_fp8(const Derived& d, const TreeLaunch& l, const TreeArgs& a, bool f32,
                           hipStream_t st);
hipError_t launch_verify(const VerifyArgs& a, int B, hipStream_t st);
hipError_t launch_append(const AppendArgs& a, int D, int dtype, hipStream_t st);

// ---- device side ------------------------------------------------------------

// Nodes of request b and its first position; n = 0 for an unused slot.
struct TreeReq {
  int n, base;
};

__device__ __forceinline__ TreeReq tree_request(const int32_t* base, const int32_t* count, int b,
                                                int N, int Lp, int Ldec) {
  TreeReq r;
  r.base = min(base[b], Ldec);
  r.n = count ? min(max(count[b], 0), N) : N;
  if (r.base < -Lp) r.n = 0;
  return r;
}

// A list of keys: entries 0 .. pre - 1 are rows 0 .. pre - 1 of an array, the ones
// after them consecutive rows from pre + shift on, which pass the end of a ring
// of rows (`wrap`: the row after its last) once at most.
struct KeyList {
  int n, pre, shift, wrap, ring;
  __device__ __forceinline__ int row(int e) const {
    const int x = e + shift;
    return e < pre ? e : x >= wrap ? x - ring : x;
  }
  // Row of entry e, of the last one for those after it: a tile's end.
  __device__ __forceinline__ int64_t near(int e) const { return row(min(e, n - 1)); }
};

// One of two lists, field by field (a reference to either would put both into memory).
__device__ __forceinline__ KeyList pick_list(bool first, const KeyList& a, const KeyList& b) {
  return {first ? a.n : b.n, first ? a.pre : b.pre, first ? a.shift : b.shift,
          first ? a.wrap : b.wrap, first ? a.ring : b.ring};
}

// The keys that nodes n0 .. n1 of a request can attend.
//   cached: rows 0 .. pre - 1 of the cache (prompt and sinks), which every node
//           attends, then the positions from j0 on
//   fresh:  nodes 0 .. pre - 1 (at prompt or sink positions), then the last
//           fresh.n - fresh.pre up to n1
// Positions that the window of the lowest node hides from all are left out.
struct TreeKeys {
  KeyList cached, fresh;
  int j0;
};

__device__ __forceinline__ TreeKeys tree_keys(const TreeArgs& a, const TreeReq& r, int n0, int n1) {
  TreeKeys k;
  const bool chain = a.depth == nullptr;
  const int low = r.base + (chain ? n0 : 0);  // lowest position of the nodes
  const int first = low - a.W + 1;            // lowest position of their windows
  const int s = r.base < 0 ? r.base : min(a.S, r.base);
  k.j0 = r.base < 0 ? 0 : min(max(s, first), r.base);
  k.cached.pre = a.Lp + s;
  k.cached.n = k.cached.pre + (r.base < 0 ? 0 : r.base - k.j0);
  // The window fits in the ring (check_kv).
  k.cached.ring = a.ring;
  k.cached.wrap = a.ring ? a.Lp + a.S + a.ring : 0x7fffffff;
  k.cached.shift =
      a.Lp - k.cached.pre + (a.ring && k.j0 >= a.S ? a.S + (k.j0 - a.S) % a.ring : k.j0);
  const int a1 = chain ? min(max(first - r.base, 0), n0) : 0;
  k.fresh.pre = min(max(a.S - r.base, 0), a1);
  k.fresh.n = k.fresh.pre + n1 + 1 - a1;
  k.fresh.shift = a1 - k.fresh.pre;
  k.fresh.wrap = 0x7fffffff;
  k.fresh.ring = 0;
  return k;
}

__device__ __forceinline__ int64_t tree_cache_base(const TreeArgs& a, int b, int h,
                                                   int elem_bytes) {
  return (a.row_base ? a.row_base[b] * elem_bytes : b * a.sb) + h * a.sh;
}

}  // namespace dsa
