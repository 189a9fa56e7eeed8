// Host side of the calls over a cache in pages and of the beam selection: argument
// checks and launch shapes.
#include <algorithm>
#include <cmath>

#include "paged.h"

namespace dsa {
namespace {

dsa_status hip_status(hipError_t e) { return e == hipSuccess ? DSA_OK : DSA_ERR_HIP; }

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

constexpr int64_t kInt = (int64_t{1} << 31) - 1;

// log2 of the rows of a page, or -1.
int log_rows(int page_rows) {
  for (int lg = 0; lg <= 10; ++lg)
    if (page_rows == 1 << lg) return lg;
  return -1;
}

dsa_status check_pages(const dsa_pages* pages, bool pool) {
  if (!pages || !pages->d_table || log_rows(pages->page_rows) < 0 || pages->max_pages < 1)
    return DSA_ERR_INVALID_ARG;
  if (int64_t{pages->max_pages} * pages->page_rows > kInt) return DSA_ERR_INVALID_ARG;
  if (!pool) return DSA_OK;
  if (!pages->d_refs || pages->num_pages < 1) return DSA_ERR_INVALID_ARG;
  if (int64_t{pages->num_pages} * pages->page_rows > kInt) return DSA_ERR_INVALID_ARG;
  return DSA_OK;
}

// Elements of 16 bytes, less one: rows are read 16 bytes at a time.
int64_t align_mask(const dsa_page_layout* l) { return l->dtype == DSA_KV_BF16 ? 7 : 15; }

dsa_status check_layout(const dsa_page_layout* l) {
  if (!l || log_rows(l->page_rows) < 0 || l->num_pages < 1) return DSA_ERR_INVALID_ARG;
  if (int64_t{l->num_pages} * l->page_rows > kInt) return DSA_ERR_INVALID_ARG;
  if (l->stride_page < 0 || l->stride_head < 0 || l->stride_row < 0) return DSA_ERR_INVALID_ARG;
  if (l->dtype != DSA_KV_BF16 && l->dtype != DSA_KV_FP8_E4M3) return DSA_ERR_INVALID_ARG;
  if ((l->stride_page | l->stride_head | l->stride_row) & align_mask(l))
    return DSA_ERR_INVALID_ARG;
  if (l->dtype == DSA_KV_BF16 && (l->d_k_scale || l->d_v_scale)) return DSA_ERR_INVALID_ARG;
  return DSA_OK;
}

dsa_status paged_derive(const dsa_params* p, const dsa_shape* s, Derived* d, PagedLaunch* l) {
  const dsa_status st = derive(p, s, d);
  if (st != DSA_OK) return st;
  *l = paged_launch(*d);
  return l->workgroups > kInt || int64_t{d->B} * d->Hq > kInt - 4 ? DSA_ERR_INVALID_ARG : DSA_OK;
}

}  // namespace

// Eight waves to a workgroup.  Up to 896 rows, three or four tiles per wave, are not
// split: the second kernel costs more (per layer, replayed: 20 pairs, 696 rows, d = 64, 7.0
// us whole and 8.3 in three; 160 such 9.0 and 10.7; 512 pairs, 832 rows, d = 128, 28.4 and
// 30.4; but 32 of these 10.5 and 9.8).  Longer ones are split into 256 to 768 rows, as many
// as give each CU a workgroup: few pairs get more (at 256, 512 and 128 workgroups in all:
// four requests of 8 heads and 4300 rows at most, fp8, d = 128, 13.2, 15.2 and 15.0 us; one
// of 9472 11.7, 11.7 and 12.9).  From 512 rows on in whole tiles for all waves (the four
// requests 13.2 in splits of 512 rows, 13.8 in those of 576), but halves stay halves (24
// requests of 4 heads and 1105 rows, 19.2 in two, 20.5 in three; 16 of 8 heads 19.7 and
// 20.7; though 12 of 8, d = 64, 18.8 and 17.4).  With 768 rows two workgroups share a CU,
// and requests of other lengths end together (16 requests of 32 heads, 200 to 4300 rows,
// d = 128, in 512, 768, 1024, 2048 and 4096 rows: 100, 101, 103, 108 and 117 us; fp8 59,
// 56, 57, 60 and 66; 32 of 8 heads with four queries each 71, 69, 78, 81 and 77).  All of
// 2304 rows, 56 us for the whole requests' 55; 8 of 8 heads with eight queries each, up to
// 9472 rows, 48 for the 45 of 2048 rows.
PagedLaunch paged_launch(const Derived& d) {
  constexpr int64_t kWhole = 14, kLeast = 4, kMost = 12;  // units of 64 rows
  PagedLaunch l{};
  const int64_t pairs = static_cast<int64_t>(d.B) * d.Hkv;
  const int64_t units = (int64_t{d.rows_max} + 63) / 64;
  const int64_t want = std::max<int64_t>(1, 256 / pairs);
  int64_t per = (units + want - 1) / want;
  if (per >= 8 && want > 2) per &= ~int64_t{3};
  per = units <= kWhole ? units : std::clamp<int64_t>(per, kLeast, kMost);
  l.C = static_cast<int>(per * 64);
  l.S = static_cast<int>((units + per - 1) / per);
  l.waves = 8;
  l.workgroups = pairs * l.S;
  l.ws_bytes = l.S > 1 ? static_cast<size_t>(l.workgroups) * d.G * (d.D + 2) * 4 : 0;
  return l;
}

}  // namespace dsa

using dsa::Derived;
using dsa::PagedLaunch;

extern "C" {

DSA_API dsa_status dsa_get_paged_launch_info(const dsa_params* p, const dsa_shape* s,
                                             dsa_paged_launch_info* out) {
  Derived d;
  PagedLaunch l;
  const dsa_status st = dsa::paged_derive(p, s, &d, &l);
  if (st != DSA_OK) return st;
  if (!out) return DSA_ERR_INVALID_ARG;
  out->rows_per_split = l.C;
  out->max_splits = l.S;
  out->waves_per_group = l.waves;
  out->workgroups = static_cast<int32_t>(l.workgroups);
  out->workspace_bytes = l.ws_bytes;
  return DSA_OK;
}

DSA_API size_t dsa_paged_workspace_bytes(const dsa_params* p, const dsa_shape* s) {
  Derived d;
  PagedLaunch l;
  return dsa::paged_derive(p, s, &d, &l) == DSA_OK ? l.ws_bytes : 0;
}

DSA_API dsa_status dsa_page_update(const dsa_params* p, int32_t batch, const dsa_pages* pages,
                                   const int32_t* d_length, const int32_t* d_new,
                                   int32_t most_new, int32_t* d_slots, int32_t* d_pos,
                                   int32_t* d_copies, int32_t* d_flags, hipStream_t stream) {
  Derived d;
  const dsa_shape one = {1, 1, 1, 64};  // parameters are checked as by every call
  dsa_status st = dsa::derive(p, &one, &d);
  if (st != DSA_OK) return st;
  if ((st = dsa::check_pages(pages, true)) != DSA_OK) return st;
  if (!pages->d_cursor || !d_length || !d_slots || !d_pos || !d_copies || !d_flags)
    return DSA_ERR_INVALID_ARG;
  if (batch < 1 || most_new < 1 || int64_t{batch} * most_new > dsa::kInt)
    return DSA_ERR_INVALID_ARG;
  if (batch > DSA_MAX_PAGED_BATCH) return DSA_ERR_UNSUPPORTED;
  dsa::PageUpdateArgs a{};
  a.length = d_length;
  a.fresh = d_new;
  a.prompt = pages->d_prompt;
  a.table = pages->d_table;
  a.refs = pages->d_refs;
  a.cursor = pages->d_cursor;
  a.slots = d_slots;
  a.pos = d_pos;
  a.copies = d_copies;
  a.flags = d_flags;
  a.B = batch;
  a.M = pages->max_pages;
  a.N = most_new;
  a.pool = pages->num_pages;
  a.lg = dsa::log_rows(pages->page_rows);
  a.Lp = d.Lp;
  a.S = d.Ns;
  a.W = d.mode == DSA_MODE_DENSE ? 0 : d.Nr;
  return dsa::hip_status(dsa::launch_page_update(a, stream));
}

DSA_API dsa_status dsa_page_reorder(int32_t batch, const dsa_pages* pages,
                                    const int32_t* d_parent, hipStream_t stream) {
  const dsa_status st = dsa::check_pages(pages, true);
  if (st != DSA_OK) return st;
  if (batch < 1 || !d_parent) return DSA_ERR_INVALID_ARG;
  if (batch > DSA_MAX_PAGED_BATCH) return DSA_ERR_UNSUPPORTED;
  dsa::PageReorderArgs a{d_parent, pages->d_table, pages->d_refs, batch, pages->max_pages,
                         pages->num_pages};
  return dsa::hip_status(dsa::launch_page_reorder(a, stream));
}

DSA_API dsa_status dsa_paged_append(const dsa_shape* s, int32_t most_new, const int32_t* d_slots,
                                    const void* d_k_new, const void* d_v_new,
                                    const dsa_node_rows* new_rows, int32_t layers, void* d_k,
                                    void* d_v, const dsa_page_layout* layout,
                                    int64_t stride_layer, const int32_t* d_copies,
                                    hipStream_t stream) {
  const dsa_params any = {0, 1, 1, 1, 1, DSA_MODE_DENSE, 0};
  Derived d;
  dsa_status st = dsa::derive(&any, s, &d);
  if (st != DSA_OK) return st;
  if ((st = dsa::check_layout(layout)) != DSA_OK) return st;
  if (!d_slots || !d_k_new || !d_v_new || !new_rows || !d_k || !d_v) return DSA_ERR_INVALID_ARG;
  if (most_new < 1 || layers < 1 || stride_layer < 0 ||
      (stride_layer & dsa::align_mask(layout)))
    return DSA_ERR_INVALID_ARG;
  const int64_t strides[] = {new_rows->stride_batch, new_rows->stride_node, new_rows->stride_head,
                             new_rows->stride_layer};
  for (int64_t x : strides)
    if (x < 0 || (x & 7)) return DSA_ERR_INVALID_ARG;
  for (const void* x : {d_k_new, d_v_new, static_cast<const void*>(d_k),
                        static_cast<const void*>(d_v)})
    if (!dsa::aligned16(x)) return DSA_ERR_INVALID_ARG;
  const int64_t chunks = int64_t{d.Hkv} * (d.D / 8);
  const int64_t most = int64_t{1} << 40;  // the products below stay in 64 bits
  if (chunks * most_new > dsa::kInt - 512 || chunks * layout->page_rows > dsa::kInt - 512 ||
      int64_t{layers} * d.B > most / chunks)
    return DSA_ERR_INVALID_ARG;
  const int64_t blocks = (chunks * most_new + 255) / 256 +
                         (d_copies ? (chunks * layout->page_rows + 255) / 256 : 0);
  if (blocks > dsa::kInt / (int64_t{layers} * d.B)) return DSA_ERR_INVALID_ARG;

  const int64_t esz = layout->dtype == DSA_KV_BF16 ? 2 : 1;
  dsa::PagedAppendArgs a{};
  a.slots = d_slots;
  a.copies = d_copies;
  a.kn = static_cast<const uint16_t*>(d_k_new);
  a.vn = static_cast<const uint16_t*>(d_v_new);
  a.nsl = new_rows->stride_layer;
  a.nsb = new_rows->stride_batch;
  a.nsn = new_rows->stride_node;
  a.nsh = new_rows->stride_head;
  a.k = static_cast<uint8_t*>(d_k);
  a.v = static_cast<uint8_t*>(d_v);
  a.sl = stride_layer * esz;
  a.sp = layout->stride_page * esz;
  a.sh = layout->stride_head * esz;
  a.sr = layout->stride_row * esz;
  a.ks = layout->d_k_scale;
  a.vs = layout->d_v_scale;
  a.layers = layers;
  a.B = d.B;
  a.N = most_new;
  a.Hkv = d.Hkv;
  a.D = d.D;
  a.pool = layout->num_pages;
  a.lg = dsa::log_rows(layout->page_rows);
  return dsa::hip_status(dsa::launch_paged_append(a, layout->dtype, stream));
}

DSA_API dsa_status dsa_paged_attention(const dsa_params* p, const dsa_shape* s,
                                       const dsa_pages* pages, const void* d_q, const void* d_k,
                                       const void* d_v, const dsa_page_layout* layout,
                                       const int32_t* d_decode_pos, const void* d_plan,
                                       float sm_scale, void* d_out, int32_t out_type,
                                       float* d_window_logits, void* d_ws, size_t ws_bytes,
                                       hipStream_t stream) {
  Derived d;
  PagedLaunch l;
  dsa_status st = dsa::paged_derive(p, s, &d, &l);
  if (st != DSA_OK) return st;
  if ((st = dsa::check_pages(pages, false)) != DSA_OK) return st;
  if ((st = dsa::check_layout(layout)) != DSA_OK) return st;
  if (layout->page_rows != pages->page_rows) return DSA_ERR_INVALID_ARG;
  if (!d_q || !d_k || !d_v || !d_decode_pos || !d_out) return DSA_ERR_INVALID_ARG;
  if (out_type != DSA_OUT_FP32 && out_type != DSA_OUT_BF16) return DSA_ERR_INVALID_ARG;
  if (!(std::fabs(sm_scale) <= 0x1p126f)) return DSA_ERR_INVALID_ARG;  // times log2(e), too
  const bool diagonal = d.mode == DSA_MODE_DIAGONAL;
  if (diagonal ? !d_plan : d_window_logits != nullptr) return DSA_ERR_INVALID_ARG;
  for (const void* x : {d_q, d_k, d_v, static_cast<const void*>(d_out)})
    if (!dsa::aligned16(x)) return DSA_ERR_INVALID_ARG;
  if (l.ws_bytes && (!d_ws || ws_bytes < l.ws_bytes)) return DSA_ERR_WORKSPACE;
  if (l.ws_bytes && !dsa::aligned16(d_ws)) return DSA_ERR_INVALID_ARG;

  const int64_t esz = layout->dtype == DSA_KV_BF16 ? 2 : 1;
  dsa::PagedArgs a{};
  a.q = static_cast<const uint16_t*>(d_q);
  a.k = static_cast<const uint8_t*>(d_k);
  a.v = static_cast<const uint8_t*>(d_v);
  a.sp = layout->stride_page * esz;
  a.sh = layout->stride_head * esz;
  a.sr = layout->stride_row * esz;
  a.ks = layout->d_k_scale;
  a.vs = layout->d_v_scale;
  a.table = pages->d_table;
  a.prompt = pages->d_prompt;
  a.pos = d_decode_pos;
  if (diagonal) {
    const char* pb = static_cast<const char*>(d_plan);
    a.count = reinterpret_cast<const int32_t*>(pb + d.plan.count_offset);
    a.idx = reinterpret_cast<const int32_t*>(pb + d.plan.indices_offset);
  }
  a.scale = sm_scale;
  a.scale_log2 = sm_scale * 1.4426950408889634f;
  a.out = d_out;
  a.wlog = d_window_logits;
  a.part = static_cast<float*>(d_ws);
  a.B = d.B;
  a.Hq = d.Hq;
  a.Hkv = d.Hkv;
  a.G = d.G;
  a.Lp = d.Lp;
  a.Ldec = d.Ldec;
  a.mode = d.mode;
  a.Ns = d.Ns;
  a.W = d.Nr;
  a.cap = d.mode == DSA_MODE_DENSE ? d.Ldec : d.plan_cap;
  a.M = pages->max_pages;
  a.pool = layout->num_pages;
  a.lg = dsa::log_rows(pages->page_rows);
  a.C = l.C;
  a.f32 = out_type == DSA_OUT_FP32;
  return dsa::hip_status(layout->dtype == DSA_KV_FP8_E4M3 ? dsa::launch_paged_fp8(d, l, a, stream)
                                                          : dsa::launch_paged_bf16(d, l, a, stream));
}

DSA_API size_t dsa_beam_workspace_bytes(int32_t batch, int32_t beams, int32_t vocab) {
  if (batch < 1 || beams < 1 || beams > DSA_MAX_BEAMS || vocab < 1 || vocab > 1 << 24 ||
      int64_t{batch} * beams >= 1 << 22)
    return 0;
  return std::max(dsa::beam_launch(batch, beams, vocab, false).bytes,
                  dsa::beam_launch(batch, beams, vocab, true).bytes);
}

DSA_API dsa_status dsa_beam_select(int32_t batch, int32_t beams, int32_t vocab,
                                   const void* d_logits, int64_t stride_row, int32_t logits_type,
                                   const float* d_score, float* d_next_score, int32_t* d_parent,
                                   int32_t* d_token, void* d_ws, size_t ws_bytes,
                                   hipStream_t stream) {
  const size_t need = dsa_beam_workspace_bytes(batch, beams, vocab);
  if (!need) return DSA_ERR_INVALID_ARG;
  if (!d_logits || !d_score || !d_next_score || !d_parent || !d_token) return DSA_ERR_INVALID_ARG;
  if (logits_type != DSA_OUT_FP32 && logits_type != DSA_OUT_BF16) return DSA_ERR_INVALID_ARG;
  if (stride_row < vocab) return DSA_ERR_INVALID_ARG;
  if (!d_ws || ws_bytes < need) return DSA_ERR_WORKSPACE;
  if (!dsa::aligned16(d_ws)) return DSA_ERR_INVALID_ARG;
  const bool bf16 = logits_type == DSA_OUT_BF16;
  const dsa::BeamLaunch l = dsa::beam_launch(batch, beams, vocab, bf16);
  if (int64_t{batch} * beams * l.chunks > dsa::kInt) return DSA_ERR_INVALID_ARG;
  char* ws = static_cast<char*>(d_ws);
  dsa::BeamArgs a{};
  a.x = d_logits;
  a.stride = stride_row;
  a.score = d_score;
  a.next = d_next_score;
  a.parent = d_parent;
  a.token = d_token;
  a.sums = reinterpret_cast<double*>(ws + l.sums);
  a.tops = reinterpret_cast<float*>(ws + l.tops);
  a.cands = reinterpret_cast<uint64_t*>(ws + l.cands);
  a.B = batch;
  a.W = beams;
  a.V = vocab;
  a.chunks = l.chunks;
  a.per = l.per;
  a.bf16 = bf16;
  a.many = l.many;
  return dsa::hip_status(dsa::launch_beam(a, stream));
}

}  // extern "C"
