// A KV cache in pages (dsa_page_*, dsa_paged_*) and the beam selection: kernel
// argument blocks and launchers.
#pragma once

#include <algorithm>

#include "internal.h"

namespace dsa {

// A launch holds fewer than 2^32 threads: `launch(first, grid)` for every part of `groups`
// workgroups, the first of which is workgroup `first` of them all.
template <typename Launch>
hipError_t launch_parts(int64_t groups, int threads, Launch launch) {
  const int64_t most = ((int64_t{1} << 32) - 1) / threads;
  for (int64_t first = 0; first < groups; first += most) {
    launch(static_cast<uint32_t>(first), dim3(static_cast<uint32_t>(std::min(most, groups - first))));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

struct PageUpdateArgs {
  const int32_t* length;
  const int32_t* fresh;  // new rows per request, or nullptr: 1 each
  const int32_t* prompt;
  int32_t* table;
  int32_t* refs;
  int32_t* cursor;
  int32_t* slots;
  int32_t* pos;
  int32_t* copies;
  int32_t* flags;
  int B, M, N, pool, lg;  // lg: log2 of the rows of a page
  int Lp, S, W;           // W: window of the rows kept after the sinks (0: all)
};

struct PageReorderArgs {
  const int32_t* parent;
  int32_t* table;
  int32_t* refs;
  int B, M, pool;
};

struct PagedAppendArgs {
  const int32_t* slots;
  const int32_t* copies;  // or nullptr
  const uint16_t* kn;
  const uint16_t* vn;
  int64_t nsl, nsb, nsn, nsh;  // strides in elements
  uint8_t* k;
  uint8_t* v;
  int64_t sl, sp, sh, sr;  // cache strides in bytes
  const float* ks;
  const float* vs;
  int layers, B, N, Hkv, D, pool, lg;
  uint32_t first;  // workgroup of the launch's first
};

struct PagedArgs {
  const uint16_t* q;
  const uint8_t* k;  // caches, addressed in bytes
  const uint8_t* v;
  int64_t sp, sh, sr;  // strides in bytes
  const float* ks;     // fp8: scales of the KV heads, or nullptr
  const float* vs;
  const int32_t* table;
  const int32_t* prompt;
  const int32_t* pos;
  const int32_t* count;  // plan (diagonal mode)
  const int32_t* idx;
  float scale;
  float scale_log2;  // sm_scale * log2(e)
  void* out;
  float* wlog;
  float* part;  // split partials (splits > 1)
  int B, Hq, Hkv, G, Lp, Ldec, mode, Ns, W, cap;
  int M, pool, lg;
  int C;    // rows of a split
  int f32;  // output in fp32
  uint32_t first;  // workgroup of the launch's first
};

// Launch of dsa_paged_attention.
struct PagedLaunch {
  int C, S, waves;  // rows of a split, splits at most
  int64_t workgroups;
  size_t ws_bytes;
};
PagedLaunch paged_launch(const Derived& d);

struct BeamArgs {
  const void* x;
  int64_t stride;
  const float* score;
  float* next;
  int32_t* parent;
  int32_t* token;
  double* sums;     // [B * W][chunks] sums of exp(x - max)
  float* tops;      // [B * W][chunks] maxima
  uint64_t* cands;  // [B * W][chunks][W] the largest values and their places
  int B, W, V, chunks, per;  // per: 16-byte pieces of a row that a workgroup takes
  bool bf16, many;
  uint32_t first;  // workgroup of the launch's first
};
struct BeamLaunch {
  int per, chunks;
  bool many;  // values per thread
  size_t sums, tops, cands, bytes;  // offsets in the workspace
};
BeamLaunch beam_launch(int B, int W, int V, bool bf16);

hipError_t launch_page_update(const PageUpdateArgs& a, hipStream_t st);
hipError_t launch_page_reorder(const PageReorderArgs& a, hipStream_t st);
hipError_t launch_paged_append(const PagedAppendArgs& a, int dtype, hipStream_t st);
hipError_t launch_paged_bf16(const Derived& d, const PagedLaunch& l, const PagedArgs& a,
                             hipStream_t st);
hipError_t launch_paged_fp8(const Derived& d, const PagedLaunch& l, const PagedArgs& a,
                            hipStream_t st);
hipError_t launch_beam(BeamArgs a, hipStream_t st);

}  // namespace dsa
