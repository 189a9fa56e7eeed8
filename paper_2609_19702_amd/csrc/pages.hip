// Page tables: pages for new rows and back, requests that go on from others'
// pages, and the new K/V rows' way into their slots.
#include <type_traits>

#include "device.h"
#include "paged.h"

namespace dsa {
namespace {

constexpr int kUpdateThreads = 1024;
constexpr int kUpdateWaves = kUpdateThreads / 64;

// Counts that other waves change in the same launch: past the CU's cache.
__device__ __forceinline__ int load_ref(const int32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// A request of the update.
struct PageReq {
  int64_t end;  // rows after the call
  int len, fresh, prompt;
  int e0, e1;   // entries of the new rows
  bool fits;    // in use, and its rows in the table
};

__device__ __forceinline__ PageReq page_request(const PageUpdateArgs& a, int b) {
  PageReq r;
  r.len = a.length[b];
  r.fresh = a.fresh ? min(max(a.fresh[b], 0), a.N) : 1;
  r.prompt = a.prompt ? min(max(a.prompt[b], 0), a.Lp) : a.Lp;
  r.end = static_cast<int64_t>(r.len) + r.fresh;
  r.fits = r.len >= 0 && r.end <= static_cast<int64_t>(a.M) << a.lg;
  const bool some = r.fits && r.fresh > 0;
  r.e0 = some ? r.len >> a.lg : 0;
  r.e1 = some ? static_cast<int>((r.end + (1 << a.lg) - 1) >> a.lg) : 0;
  return r;
}

__device__ __forceinline__ bool in_pool(int page, int pool) {
  return static_cast<unsigned>(page) < static_cast<unsigned>(pool);
}

// One workgroup.  Its parts, with a barrier after each:
//   1. a wave per request gives back the pages that ended or fell behind
//   2. a wave per request counts the pages that its new rows need; an entry whose
//      page is shared becomes -2 - page until part 5
//   3. running sums of the needs
//   4. free pages from the cursor on, 1024 looked at a time; the k-th goes to
//      the request whose share of the sums k lies in, and waits in its slots
//      (a request has a new row for every page that it needs)
//   5. a wave per request puts them into the table
//   6. slots
__global__ __launch_bounds__(kUpdateThreads) void page_update_kernel(PageUpdateArgs a) {
  __shared__ int upto[DSA_MAX_PAGED_BATCH];  // needs, then their running sums
  __shared__ int part[kUpdateWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int rows = 1 << a.lg;

  for (int b = wave; b < a.B; b += kUpdateWaves) {
    const PageReq r = page_request(a, b);
    int32_t* row = a.table + static_cast<int64_t>(b) * a.M;
    int lo = 0, hi = r.len < 0 ? a.M : 0;
    if (r.len >= 0 && a.W > 0) {
      const int64_t front = static_cast<int64_t>(r.prompt) + a.S;
      const int64_t back = static_cast<int64_t>(r.len) - a.W + 1;
      lo = static_cast<int>(min((front + rows - 1) >> a.lg, static_cast<int64_t>(a.M)));
      hi = back > 0 ? static_cast<int>(min(back >> a.lg, static_cast<int64_t>(a.M))) : 0;
    }
    for (int i = lo + lane; i < hi; i += 64) {
      const int page = row[i];
      if (in_pool(page, a.pool)) atomicSub(a.refs + page, 1);
      if (page != -1) row[i] = -1;
    }
  }
  __threadfence();  // the counts have changed before anyone reads them
  __syncthreads();

  for (int b = wave; b < a.B; b += kUpdateWaves) {
    const PageReq r = page_request(a, b);
    int32_t* row = a.table + static_cast<int64_t>(b) * a.M;
    int need = 0;
    for (int i0 = r.e0; i0 < r.e1; i0 += 64) {
      const int i = i0 + lane;
      int want = 0;  // what the entry becomes, if anything
      if (i < r.e1) {
        const int page = row[i];
        if (!in_pool(page, a.pool))
          want = -1;
        else if (load_ref(a.refs + page) > 1)
          want = -2 - page;
        if (want && want != page) row[i] = want;
      }
      need += __popcll(__ballot(want != 0));
    }
    if (lane == 0) upto[b] = need;
  }
  __syncthreads();

  int total = 0;
  for (int b0 = 0; b0 < a.B; b0 += kUpdateThreads) {
    const int b = b0 + tid;
    const int x = wave_scan(b < a.B ? upto[b] : 0);
    if (lane == 63) part[wave] = x;
    __syncthreads();
    int before = total;
    for (int w = 0; w < kUpdateWaves; ++w) {
      before += w < wave ? part[w] : 0;
      total += part[w];
    }
    if (b < a.B) upto[b] = before + x;
    __syncthreads();
  }

  int found = 0;
  if (total > 0) {
    const int c = a.cursor[0] % a.pool, start = c < 0 ? c + a.pool : c;
    for (int i0 = 0; i0 < a.pool && found < total; i0 += kUpdateThreads) {
      int page = start + min(i0 + tid, a.pool - 1);
      page = page >= a.pool ? page - a.pool : page;
      const bool free = i0 + tid < a.pool && load_ref(a.refs + page) == 0;
      const uint64_t mask = __ballot(free);
      if (lane == 0) part[wave] = __popcll(mask);
      __syncthreads();
      int rank = found + __popcll(mask & ((uint64_t(1) << lane) - 1));
      for (int w = 0; w < kUpdateWaves; ++w) {
        rank += w < wave ? part[w] : 0;
        found += part[w];
      }
      if (free && rank < total) {
        int lo = 0, hi = a.B - 1;  // the first request whose sum passes the rank
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          if (upto[mid] > rank) hi = mid; else lo = mid + 1;
        }
        a.slots[static_cast<int64_t>(lo) * a.N + rank - (lo ? upto[lo - 1] : 0)] = page;
      }
      __syncthreads();
    }
  }
  found = min(found, total);

  for (int b = wave; b < a.B; b += kUpdateWaves) {
    const PageReq r = page_request(a, b);
    const int before = b ? upto[b - 1] : 0, need = upto[b] - before;
    const bool pages = need == 0 || upto[b] <= found, ok = r.fits && pages;
    int32_t* row = a.table + static_cast<int64_t>(b) * a.M;
    const int32_t* got = a.slots + static_cast<int64_t>(b) * a.N;
    int x = -1, y = -1;  // the first entry's old and new page, where rows are copied
    int rank = 0;
    if (need > 0) {
      for (int i0 = r.e0; i0 < r.e1; i0 += 64) {
        const int i = i0 + lane;
        const int old = i < r.e1 ? row[i] : 0;
        const uint64_t mask = __ballot(old < 0);
        const int page = -2 - old;  // the shared one, or -1
        if (old < 0 && ok) {
          const int mine = got[rank + __popcll(mask & ((uint64_t(1) << lane) - 1))];
          row[i] = mine;
          atomicExch(a.refs + mine, 1);
          if (page >= 0) atomicSub(a.refs + page, 1);
          if (i == r.e0 && page >= 0 && (r.len & (rows - 1))) {
            x = page;
            y = mine;
          }
        } else if (old < -1) {
          row[i] = page;
        }
        rank += __popcll(mask);
      }
      // The last page that anyone was given.
      if (ok && lane == 0) {
        bool last = true;
        if (found == total) {
          last = upto[b] == total;
        } else {
          for (int f = b + 1; f < a.B && last; ++f) {
            if (upto[f] == upto[f - 1]) continue;  // needs none
            last = upto[f] > found;
            break;
          }
        }
        if (last) {
          const int next = got[need - 1] + 1;
          a.cursor[0] = next == a.pool ? 0 : next;
        }
      }
    }
    if (lane == 0) {
      a.flags[b] = r.len < 0 ? 0
                             : (r.fits ? (pages ? 0 : DSA_PAGE_FLAG_NO_PAGES)
                                       : DSA_PAGE_FLAG_TOO_LONG);
      const int64_t pos = r.end - 1 - r.prompt;
      a.pos[b] = ok && pos >= 0 ? static_cast<int>(pos) : -1;
      int32_t* told = a.copies + 3 * static_cast<int64_t>(b);
      told[0] = x;  // lane 0 holds the first entry
      told[1] = y;
      told[2] = x >= 0 ? r.len & (rows - 1) : -1;
    }
    // What waited in the slots has been read: they become the rows' places.
    fence_wave();
    int32_t* to = a.slots + static_cast<int64_t>(b) * a.N;
    for (int i = lane; i < a.N; i += 64) {
      int slot = -1;
      if (ok && i < r.fresh) {
        const int at = r.len + i;
        slot = (row[at >> a.lg] << a.lg) + (at & (rows - 1));
      }
      to[i] = slot;
    }
  }
}

constexpr int kReorderThreads = 512;
constexpr int kReorderLds = 32768;  // bytes of the columns that a workgroup holds

// A workgroup takes `cols` columns of the table: all their entries into LDS, then
// every row its parent's.
__global__ __launch_bounds__(kReorderThreads) void page_reorder_kernel(PageReorderArgs a,
                                                                      int lg_cols) {
  extern __shared__ int32_t held[];  // [B][cols]
  const int cols = 1 << lg_cols, first = blockIdx.x << lg_cols;
  const int n = a.B << lg_cols;
  for (int e = threadIdx.x; e < n; e += kReorderThreads) {
    const int i = first + (e & (cols - 1));
    held[e] = i < a.M ? a.table[static_cast<int64_t>(e >> lg_cols) * a.M + i] : -1;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < n; e += kReorderThreads) {
    const int b = e >> lg_cols, i = first + (e & (cols - 1));
    const int parent = a.parent[b];
    if (i >= a.M || parent == b) continue;
    const int old = held[e];
    const bool there = static_cast<unsigned>(parent) < static_cast<unsigned>(a.B);
    const int page = there ? held[(parent << lg_cols) + (e & (cols - 1))] : -1;
    if (page == old) continue;
    if (in_pool(page, a.pool)) atomicAdd(a.refs + page, 1);
    if (in_pool(old, a.pool)) atomicSub(a.refs + old, 1);
    a.table[static_cast<int64_t>(b) * a.M + i] = page;
  }
}

// bf16 values to E4M3 codes of value / scale.
__device__ __forceinline__ uint2 fp8_codes(const uint4& x, float scale) {
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
}

// Eight elements of a K row and of its V row per thread.  The first `blocks`
// workgroups of a (layer, request) take new rows, the others rows of its copy.
template <bool FP8>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedAppendArgs a, int chunks,
                                                           int blocks, int copy_blocks) {
  const int per = blocks + copy_blocks;
  const int64_t lb = blockIdx.x / per;
  const int b = static_cast<int>(lb % a.B), layer = static_cast<int>(lb / a.B);
  const int block = blockIdx.x % per;
  const int rows = 1 << a.lg;
  if (block < blocks) {
    const int at = block * 256 + threadIdx.x;
    const int c = at % chunks, h = at / chunks % a.Hkv, i = at / chunks / a.Hkv;
    if (i >= a.N) return;
    const int slot = a.slots[static_cast<int64_t>(b) * a.N + i];
    if (!in_pool(slot >> a.lg, a.pool)) return;  // a negative slot is of no page
    const int64_t from = layer * a.nsl + b * a.nsb + i * a.nsn + h * a.nsh + c * 8;
    const int64_t to = layer * a.sl + (slot >> a.lg) * a.sp + h * a.sh +
                       (slot & (rows - 1)) * a.sr + c * (FP8 ? 8 : 16);
    const uint4 xk = *reinterpret_cast<const uint4*>(a.kn + from);
    const uint4 xv = *reinterpret_cast<const uint4*>(a.vn + from);
    if constexpr (FP8) {
      const int s = layer * a.Hkv + h;
      *reinterpret_cast<uint2*>(a.k + to) = fp8_codes(xk, a.ks ? a.ks[s] : 1.f);
      *reinterpret_cast<uint2*>(a.v + to) = fp8_codes(xv, a.vs ? a.vs[s] : 1.f);
    } else {
      *reinterpret_cast<uint4*>(a.k + to) = xk;
      *reinterpret_cast<uint4*>(a.v + to) = xv;
    }
    return;
  }
  const int32_t* told = a.copies + 3 * static_cast<int64_t>(b);
  const int x = told[0], y = told[1], n = min(told[2], rows);
  if (!in_pool(x, a.pool) || !in_pool(y, a.pool) || x == y) return;
  const int at = (block - blocks) * 256 + threadIdx.x;
  const int c = at % chunks, h = at / chunks % a.Hkv, i = at / chunks / a.Hkv;
  if (i >= n) return;
  using Raw = std::conditional_t<FP8, uint2, uint4>;
  const int64_t in = layer * a.sl + h * a.sh + i * a.sr + c * static_cast<int>(sizeof(Raw));
  const Raw rk = *reinterpret_cast<const Raw*>(a.k + in + x * a.sp);
  const Raw rv = *reinterpret_cast<const Raw*>(a.v + in + x * a.sp);
  *reinterpret_cast<Raw*>(a.k + in + y * a.sp) = rk;
  *reinterpret_cast<Raw*>(a.v + in + y * a.sp) = rv;
}

}  // namespace

hipError_t launch_page_update(const PageUpdateArgs& a, hipStream_t st) {
  page_update_kernel<<<dim3(1), dim3(kUpdateThreads), 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_page_reorder(const PageReorderArgs& a, hipStream_t st) {
  int lg = 0;
  while (lg < 4 && (static_cast<int64_t>(a.B) << (lg + 1)) * 4 <= kReorderLds && (1 << lg) < a.M)
    ++lg;
  const int groups = (a.M + (1 << lg) - 1) >> lg;
  page_reorder_kernel<<<dim3(groups), dim3(kReorderThreads), (a.B << lg) * 4, st>>>(a, lg);
  return hipGetLastError();
}

hipError_t launch_paged_append(const PagedAppendArgs& a, int dtype, hipStream_t st) {
  const int chunks = a.D / 8;
  const int64_t row = static_cast<int64_t>(a.Hkv) * chunks;
  const int blocks = static_cast<int>((a.N * row + 255) / 256);
  const int copies = a.copies ? static_cast<int>(((row << a.lg) + 255) / 256) : 0;
  const dim3 grid(static_cast<uint32_t>(static_cast<int64_t>(blocks + copies) * a.layers * a.B));
  if (dtype == DSA_KV_FP8_E4M3)
    paged_append_kernel<true><<<grid, dim3(256), 0, st>>>(a, chunks, blocks, copies);
  else
    paged_append_kernel<false><<<grid, dim3(256), 0, st>>>(a, chunks, blocks, copies);
  return hipGetLastError();
}

}  // namespace dsa
