// Page tables: pages for new rows and back, requests that go on from others'
// pages, and the new K/V rows' way into their slots.
#include <algorithm>

#include "device.h"
#include "paged.h"

namespace dsa {
namespace {

constexpr int kUpdateThreads = 1024;
constexpr int kUpdateWaves = kUpdateThreads / 64;
constexpr int kLook = 4;  // pages that a thread looks at together

// Counts that other waves change in the same launch: past the CU's cache.
__device__ __forceinline__ int load_ref(const int32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// A request of the update, as it waits in LDS: length (below 0: unused), new rows and
// prompt rows, and the pages needed up to it.
struct PageReq {
  int len, fresh, prompt, upto;
};

// Its entries of new rows, [e0, e1), counted without signs as they are everywhere (a step of a
// group's lanes past the last of 2^31 - 1 has no place below 0); fits: it is in use, and its
// rows have entries.
struct PageSpan {
  uint32_t e0, e1;
  bool fits;
};
__device__ __forceinline__ PageSpan page_span(const PageUpdateArgs& a, const PageReq& r) {
  const int64_t end = static_cast<int64_t>(r.len) + r.fresh;
  PageSpan s;
  s.fits = r.len >= 0 && end <= static_cast<int64_t>(a.M) << a.lg;
  const bool some = s.fits && r.fresh > 0;
  s.e0 = some ? r.len >> a.lg : 0;
  s.e1 = some ? static_cast<uint32_t>((end + (1 << a.lg) - 1) >> a.lg) : 0;
  return s;
}

__device__ __forceinline__ bool in_pool(int page, int pool) {
  return static_cast<unsigned>(page) < static_cast<unsigned>(pool);
}

// One workgroup, LANES lanes to a request.  Its parts, with a barrier after each:
//   1. lengths, new and prompt rows into LDS
//   2. pages that ended or fell behind go back
//   3. the pages that the new rows need are counted; an entry whose page is shared
//      becomes -2 - page until part 6
//   4. running sums of the needs
//   5. free pages from the cursor on, 4096 looked at a time; the k-th goes to
//      the request whose share of the sums k lies in, and waits in its slots
//      (a request has a new row for every page that it needs)
//   6. they go into the table, and slots come out; more than a group's lanes of them
//      in a part of their own, a wave to a request
// Bound by the way to memory and back, some 0.5 us for each part but 4: 3.2 us for one
// request; then by the rounds of groups: a new row each for 64, 128, 256, 1024 and 4096
// requests takes 6.0, 6.2, 6.5, 13 and 39 us (with 16 lanes to each 6.0, 7.9, 12, 35 and
// 127), so fewer lanes where there are many.
template <int LANES>
__global__ __launch_bounds__(kUpdateThreads) void page_update_kernel(PageUpdateArgs a) {
  constexpr uint32_t kAll = (1u << LANES) - 1;  // a group's lanes in its ballot
  extern __shared__ PageReq req[];
  __shared__ int part[kLook][kUpdateWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t sub = tid % LANES;
  const int group = tid / LANES;
  const int shift = lane - static_cast<int>(sub);  // of the group's ballot
  const int rows = 1 << a.lg;

  for (int b = tid; b < a.B; b += kUpdateThreads) {
    PageReq r;
    r.len = a.length[b];
    r.fresh = a.fresh ? a.fresh[b] : 1;
    r.prompt = a.prompt ? a.prompt[b] : a.Lp;
    r.fresh = min(max(r.fresh, 0), a.N);
    r.prompt = min(max(r.prompt, 0), a.Lp);
    r.upto = 0;
    req[b] = r;
  }
  __syncthreads();

  for (int b = group; b < a.B; b += kUpdateThreads / LANES) {
    const PageReq r = req[b];
    int32_t* row = a.table + static_cast<int64_t>(b) * a.M;
    uint32_t lo = 0, hi = r.len < 0 ? a.M : 0;
    if (r.len >= 0 && a.W > 0) {
      const int64_t front = static_cast<int64_t>(r.prompt) + a.S;
      const int64_t back = static_cast<int64_t>(r.len) - a.W + 1;
      lo = static_cast<uint32_t>(min((front + rows - 1) >> a.lg, static_cast<int64_t>(a.M)));
      hi = back > 0 ? static_cast<uint32_t>(min(back >> a.lg, static_cast<int64_t>(a.M))) : 0;
    }
    for (uint32_t i = lo + sub; i < hi; i += LANES) {
      const int page = row[i];
      if (in_pool(page, a.pool)) atomicSub(a.refs + page, 1);
      if (page != -1) row[i] = -1;
    }
  }
  // The counts have changed (in the L2, where all of them are read) before anyone
  // reads them.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();

  for (int b = group; b < a.B; b += kUpdateThreads / LANES) {
    const PageSpan s = page_span(a, req[b]);
    int32_t* row = a.table + static_cast<int64_t>(b) * a.M;
    int need = 0;
    for (uint32_t i = s.e0 + sub; i - sub < s.e1; i += LANES) {
      int want = 0;  // what the entry becomes, if anything
      if (i < s.e1) {
        const int page = row[i];
        if (!in_pool(page, a.pool))
          want = -1;
        else if (load_ref(a.refs + page) > 1)
          want = -2 - page;
        if (want && want != page) row[i] = want;
      }
      need += __popc(static_cast<uint32_t>(__ballot(want != 0) >> shift) & kAll);
    }
    if (sub == 0) req[b].upto = need;
  }
  __syncthreads();

  int total = 0;
  for (int b0 = 0; b0 < a.B; b0 += kUpdateThreads) {
    const int b = b0 + tid;
    const int x = wave_scan(b < a.B ? req[b].upto : 0);
    if (lane == 63) part[0][wave] = x;
    __syncthreads();
    int before = total;
    for (int w = 0; w < kUpdateWaves; ++w) {
      before += w < wave ? part[0][w] : 0;
      total += part[0][w];
    }
    if (b < a.B) req[b].upto = before + x;
    __syncthreads();
  }

  int found = 0;
  if (total > 0) {
    // Unsigned: a place on from the cursor is below twice the pool, so below 2^32.
    const uint32_t pool = a.pool;
    const int c = a.cursor[0] % a.pool;
    const uint32_t start = c < 0 ? c + a.pool : c;
    for (uint32_t i0 = 0; i0 < pool && found < total; i0 += kLook * kUpdateThreads) {
      int page[kLook], rank[kLook];
      bool free[kLook];
#pragma unroll
      for (int k = 0; k < kLook; ++k) {
        const uint32_t i = i0 + k * kUpdateThreads + tid, at = start + min(i, pool - 1);
        page[k] = static_cast<int>(at >= pool ? at - pool : at);
        free[k] = load_ref(a.refs + page[k]) == 0 && i < pool;
      }
#pragma unroll
      for (int k = 0; k < kLook; ++k) {
        const uint64_t mask = __ballot(free[k]);
        rank[k] = __popcll(mask & ((uint64_t(1) << lane) - 1));
        if (lane == 0) part[k][wave] = __popcll(mask);
      }
      __syncthreads();
      // The counts of 16 waves four times over, a lane each, and their sums up to it.
      const int mine = part[lane >> 4][lane & 15];
      const int sums = wave_scan(mine);
#pragma unroll
      for (int k = 0; k < kLook; ++k) {
        const int at = 16 * k + wave;
        rank[k] += found + __shfl(sums - mine, at, 64);
        if (free[k] && rank[k] < total) {
          int lo = 0, hi = a.B - 1;  // the first request whose sum passes the rank
          while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (req[mid].upto > rank[k]) hi = mid; else lo = mid + 1;
          }
          a.slots[static_cast<int64_t>(lo) * a.N + rank[k] - (lo ? req[lo - 1].upto : 0)] = page[k];
        }
      }
      found += __shfl(sums, 63, 64);
      __syncthreads();
    }
  }
  found = min(found, total);

  for (int b = group; b < a.B; b += kUpdateThreads / LANES) {
    const PageReq r = req[b];
    const PageSpan s = page_span(a, r);
    const int need = r.upto - (b ? req[b - 1].upto : 0);
    const bool pages = need == 0 || r.upto <= found, ok = s.fits && pages;
    int32_t* row = a.table + static_cast<int64_t>(b) * a.M;
    int32_t* slots = a.slots + static_cast<int64_t>(b) * a.N;
    int x = -1, y = -1;  // the first entry's old and new page, where rows are copied
    int last = 0;        // the last page that the request is given
    int got = -1;        // page of entry e0 + sub
    int rank = 0;
    for (uint32_t i = s.e0 + sub; i - sub < s.e1; i += LANES) {
      int now = i < s.e1 ? row[i] : 0;
      const uint32_t mask = static_cast<uint32_t>(__ballot(now < 0) >> shift) & kAll;
      if (now < 0) {
        const int old = -2 - now;  // the shared page, or -1
        now = old;
        if (ok) {
          now = slots[rank + __popc(mask & ((1u << sub) - 1))];
          atomicExch(a.refs + now, 1);
          if (old >= 0) atomicSub(a.refs + old, 1);
          if (i == s.e0 && old >= 0 && (r.len & (rows - 1))) {
            x = old;
            y = now;
          }
        }
        row[i] = now;
      }
      if (mask) last = __shfl(now, shift + 31 - __clz(mask), 64);
      rank += __popc(mask);
      if (i - sub == s.e0) got = now;
    }
    if (sub == 0) {
      // The last page that anyone was given?
      bool end = ok && need > 0;
      if (found == total) {
        end &= r.upto == total;
      } else {
        for (int f = b + 1; f < a.B && end; ++f) {
          if (req[f].upto == req[f - 1].upto) continue;  // needs none
          end = req[f].upto > found;
          break;
        }
      }
      if (end) a.cursor[0] = last + 1 == a.pool ? 0 : last + 1;
      a.flags[b] = r.len < 0 ? 0
                             : (s.fits ? (pages ? 0 : DSA_PAGE_FLAG_NO_PAGES)
                                       : DSA_PAGE_FLAG_TOO_LONG);
      const int64_t pos = static_cast<int64_t>(r.len) + r.fresh - 1 - r.prompt;
      a.pos[b] = ok && pos >= 0 ? static_cast<int>(pos) : -1;
      int32_t* told = a.copies + 3 * static_cast<int64_t>(b);
      told[0] = x;
      told[1] = y;
      told[2] = x >= 0 ? r.len & (rows - 1) : -1;
    }
    // What waited in the slots has been read: they become the rows' places.
    const int n = ok ? r.fresh : 0;
    if (a.N > LANES) {
      if (sub == 0) req[b].fresh = n;
      continue;
    }
    fence_wave();
    const uint32_t at = (n ? r.len : 0) + sub, e = at >> a.lg;
    const int held = __shfl(got, shift + static_cast<int>((e - s.e0) & (LANES - 1)), 64);
    if (static_cast<int>(sub) < a.N)
      slots[sub] = static_cast<int>(sub) < n ? (held << a.lg) + static_cast<int>(at & (rows - 1)) : -1;
  }
  if (a.N <= LANES) return;
  __syncthreads();
  for (int b = wave; b < a.B; b += kUpdateWaves) {
    const int len = req[b].len, n = req[b].fresh;
    const int32_t* row = a.table + static_cast<int64_t>(b) * a.M;
    int32_t* slots = a.slots + static_cast<int64_t>(b) * a.N;
    for (int64_t i = lane; i < a.N; i += 64) {
      int slot = -1;
      if (i < n) {
        const int at = len + static_cast<int>(i);
        slot = (row[at >> a.lg] << a.lg) + (at & (rows - 1));
      }
      slots[i] = slot;
    }
  }
}

constexpr int kReorderThreads = 512;
constexpr int kReorderMost = 2048;  // entries that a workgroup holds, about
constexpr uint32_t kReorderGroups = 1 << 20;  // of a launch, whose threads are below 2^32

// A workgroup takes some columns of the table: all their entries into LDS, then
// every row its parent's; then others, where there are more of them than workgroups.  Bound by
// the way to memory and back: 2.2 us for four rows of 53 entries, 4.5 for 256.
__global__ __launch_bounds__(kReorderThreads) void page_reorder_kernel(PageReorderArgs a,
                                                                      int lg_cols, uint32_t groups) {
  extern __shared__ int32_t held[];  // [B][cols]
  const int cols = 1 << lg_cols;
  const uint32_t M = a.M;  // columns are below M + cols, so below 2^32
  const int n = a.B << lg_cols;
  for (uint32_t group = blockIdx.x;;) {
    const uint32_t first = group << lg_cols;
    for (int e = threadIdx.x; e < n; e += kReorderThreads) {
      const uint32_t i = first + (e & (cols - 1));
      held[e] = i < M ? a.table[static_cast<int64_t>(e >> lg_cols) * a.M + i] : -1;
    }
    int parent = threadIdx.x < n ? a.parent[threadIdx.x >> lg_cols] : 0;
    __syncthreads();
    for (int e = threadIdx.x; e < n; e += kReorderThreads) {
      const int b = e >> lg_cols;
      const uint32_t i = first + (e & (cols - 1));
      if (e != static_cast<int>(threadIdx.x)) parent = a.parent[b];
      if (i >= M || parent == b) continue;
      const int old = held[e];
      const bool there = static_cast<unsigned>(parent) < static_cast<unsigned>(a.B);
      const int page = there ? held[(parent << lg_cols) + (e & (cols - 1))] : -1;
      if (page == old) continue;
      if (in_pool(page, a.pool)) atomicAdd(a.refs + page, 1);
      if (in_pool(old, a.pool)) atomicSub(a.refs + old, 1);
      a.table[static_cast<int64_t>(b) * a.M + i] = page;
    }
    group += gridDim.x;
    if (group >= groups) return;
    __syncthreads();  // all have read what the next columns replace
  }
}

// bf16 values over a scale, within +-448 (NaN stays NaN), in three operations where the
// compiler's division takes ten: Markstein's correction.  With y the rounded reciprocal of s and
// q = x * y rounded, q + (x - q * s) * y by fma is x / s rounded to nearest, unless that lies
// within 2^-21 of a unit in the last place of the middle between two fp32 values (q is off by
// 1.5 units at most; nothing is below 2^-138).  E4M3 codes could differ where, besides, one of
// the two is a border between codes, of five bits: with integers X, S and b of 8, 24 and 5 bits
// that is |X 2^k - S (b 2^20 +- 1)| <= 16 with k >= 39, which leaves S = 2^24 - 1 and b = 16,
// the border 2^-10, and there the steps round as the quotient does.  So the codes are the
// division's.  Quotients past 1024 end at 448 by either, those below 2^-12 at a zero of their
// sign; scales far from 1 are divided by.
__device__ __forceinline__ void over_scale(const uint4& x, float s, float (&f)[8]) {
  unpack8(x, f);
  const float y = 1.f / s, size = fabsf(s);
  if (size > 0x1p-80f && size < 0x1p80f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float q = f[i] * y;
      f[i] = fabsf(q) < 1024.f && fabsf(q) > 0x1p-12f ? fmaf(fmaf(-q, s, f[i]), y, q) : q;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] /= s;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = f[i] != f[i] ? f[i] : fminf(fmaxf(f[i], -448.f), 448.f);
}

__device__ __forceinline__ uint4 fp8_codes(const uint4& a, const uint4& b, float scale) {
  uint32_t w[4];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float f[8];
    over_scale(h ? b : a, scale, f);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      int c = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i], f[4 * i + 1], 0, false);
      c = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2], f[4 * i + 3], c, true);
      w[2 * h + i] = static_cast<uint32_t>(c);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// 16 bytes of a K row and of its V row in the cache per thread.  The first `blocks`
// workgroups of a (layer, request) take new rows, the others rows of its copy.  Bound by
// memory: 32 prompts of 256 rows at most in 8 layers of 8 heads, d = 128, bf16 to fp8,
// 66.5 us or 4.6 TB/s of a copy's 5.0; a row and half a page copied for 32 requests in 30
// layers of 32 heads, 42 us or 4.1 TB/s.  Two or four rows a thread, or a workgroup's
// copies row by row, were within 2%.
template <bool FP8, int D>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedAppendArgs a, int blocks,
                                                           int copy_blocks) {
  constexpr int chunks = D * (FP8 ? 1 : 2) / 16;
  const int per = blocks + copy_blocks;
  const uint32_t group = a.first + blockIdx.x;
  const int lb = group / per, b = lb % a.B, layer = lb / a.B;
  const int block = group % per;
  const int rows = 1 << a.lg;
  const unsigned at = (block < blocks ? block : block - blocks) * 256u + threadIdx.x;
  const int c = at % chunks, h = at / chunks % static_cast<unsigned>(a.Hkv);
  const int i = at / chunks / static_cast<unsigned>(a.Hkv);
  const int64_t cache = layer * a.sl + h * a.sh + c * 16;
  if (block < blocks) {
    if (i >= a.N) return;
    const int slot = a.slots[static_cast<int64_t>(b) * a.N + i];
    if (!in_pool(slot >> a.lg, a.pool)) return;  // a negative slot is of no page
    const int64_t from = layer * a.nsl + b * a.nsb + i * a.nsn + h * a.nsh + c * (FP8 ? 16 : 8);
    const int64_t to = cache + (slot >> a.lg) * a.sp + (slot & (rows - 1)) * a.sr;
    uint4 k = load_stream16(a.kn + from), v = load_stream16(a.vn + from);
    if constexpr (FP8) {
      const uint4 k1 = load_stream16(a.kn + from + 8), v1 = load_stream16(a.vn + from + 8);
      const int s = layer * a.Hkv + h;
      k = fp8_codes(k, k1, a.ks ? a.ks[s] : 1.f);
      v = fp8_codes(v, v1, a.vs ? a.vs[s] : 1.f);
    }
    *reinterpret_cast<uint4*>(a.k + to) = k;
    *reinterpret_cast<uint4*>(a.v + to) = v;
    return;
  }
  const int32_t* told = a.copies + 3 * static_cast<int64_t>(b);
  const int x = told[0], y = told[1], n = min(told[2], rows);
  if (!in_pool(x, a.pool) || !in_pool(y, a.pool) || x == y || i >= n) return;
  const int64_t in = cache + i * a.sr;
  const uint4 k = *reinterpret_cast<const uint4*>(a.k + in + x * a.sp);
  const uint4 v = *reinterpret_cast<const uint4*>(a.v + in + x * a.sp);
  *reinterpret_cast<uint4*>(a.k + in + y * a.sp) = k;
  *reinterpret_cast<uint4*>(a.v + in + y * a.sp) = v;
}

template <bool FP8, int D>
hipError_t append_grid(PagedAppendArgs a, hipStream_t st) {
  const int64_t row = static_cast<int64_t>(a.Hkv) * (D * (FP8 ? 1 : 2) / 16);
  const int blocks = static_cast<int>((a.N * row + 255) / 256);
  const int copies = a.copies ? static_cast<int>(((row << a.lg) + 255) / 256) : 0;
  const int64_t groups = (int64_t{blocks} + copies) * a.layers * a.B;
  return launch_parts(groups, 256, [&](uint32_t first, dim3 grid) {
    a.first = first;
    paged_append_kernel<FP8, D><<<grid, dim3(256), 0, st>>>(a, blocks, copies);
  });
}

}  // namespace

hipError_t launch_page_update(const PageUpdateArgs& a, hipStream_t st) {
  const dim3 one(1), block(kUpdateThreads);
  const size_t lds = a.B * sizeof(PageReq);
  if (a.B <= kUpdateThreads / 16)
    page_update_kernel<16><<<one, block, lds, st>>>(a);
  else if (a.B <= kUpdateThreads / 8)
    page_update_kernel<8><<<one, block, lds, st>>>(a);
  else
    page_update_kernel<4><<<one, block, lds, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_page_reorder(const PageReorderArgs& a, hipStream_t st) {
  int lg = 0;
  while (lg < 4 && (a.B << (lg + 1)) <= kReorderMost && (1 << lg) < a.M) ++lg;
  const uint32_t groups = (static_cast<uint32_t>(a.M) + (1 << lg) - 1) >> lg;
  const dim3 grid(std::min(groups, kReorderGroups));
  page_reorder_kernel<<<grid, dim3(kReorderThreads), (a.B << lg) * 4, st>>>(a, lg, groups);
  return hipGetLastError();
}

hipError_t launch_paged_append(const PagedAppendArgs& a, int dtype, hipStream_t st) {
  if (dtype == DSA_KV_FP8_E4M3)
    return a.D == 64 ? append_grid<true, 64>(a, st) : append_grid<true, 128>(a, st);
  return a.D == 64 ? append_grid<false, 64>(a, st) : append_grid<false, 128>(a, st);
}

}  // namespace dsa
