// Host side of the calls that take several tokens per request: argument
// checks, the tree plan's layout and the launch of the attention.
#include <algorithm>
#include <cmath>

#include "tree.h"

namespace dsa {
namespace {

constexpr int kMostNodes = 1 << 20;
constexpr int64_t kMostGrid = (int64_t(1) << 31) - 1;

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

dsa_status hip_status(hipError_t e) { return e == hipSuccess ? DSA_OK : DSA_ERR_HIP; }

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

dsa_status tree_plan_layout(int batch, int nodes, dsa_tree_plan_layout* l) {
  if (batch < 1 || nodes < 1 || nodes > DSA_MAX_TREE_NODES) return DSA_ERR_INVALID_ARG;
  if (static_cast<int64_t>(batch) * nodes > (int64_t(1) << 30)) return DSA_ERR_INVALID_ARG;
  const size_t b = batch, bn = b * nodes;
  l->words = (nodes + 31) / 32;
  l->flags_offset = 0;
  l->max_depth_offset = align256(4 * b);
  l->depth_offset = l->max_depth_offset + align256(4 * b);
  l->parent_offset = l->depth_offset + align256(4 * bn);
  l->ancestors_offset = l->parent_offset + align256(4 * bn);
  l->bytes = l->ancestors_offset + align256(4 * bn * l->words);
  return DSA_OK;
}

dsa_status check_tree(const dsa_tree* t, int batch, int most) {
  if (!t || t->nodes < 1 || t->nodes > most) return DSA_ERR_INVALID_ARG;
  if (t->d_plan && (t->nodes > DSA_MAX_TREE_NODES || !aligned16(t->d_plan)))
    return DSA_ERR_INVALID_ARG;
  if (static_cast<int64_t>(batch) * t->nodes > (int64_t(1) << 30)) return DSA_ERR_INVALID_ARG;
  return DSA_OK;
}

dsa_status check_rows(const dsa_node_rows* r) {
  if (!r || r->stride_batch < 0 || r->stride_node < 0 || r->stride_head < 0)
    return DSA_ERR_INVALID_ARG;
  if ((r->stride_batch | r->stride_node | r->stride_head) & 7) return DSA_ERR_INVALID_ARG;
  return DSA_OK;
}

// derive() for the calls that need no plan of kept rows, so that their modes
// and nodes bound nothing but their own launch.
dsa_status tree_derive(const dsa_params* p, const dsa_shape* s, int nodes, Derived* d,
                       TreeLaunch* l) {
  const dsa_status st = derive(p, s, d);
  if (st != DSA_OK) return st;
  if (nodes < 1 || nodes > kMostNodes) return DSA_ERR_INVALID_ARG;
  if (d->mode == DSA_MODE_DIAGONAL) return DSA_ERR_UNSUPPORTED;
  *l = tree_launch(*d, nodes);
  // pairs rounded up to eight (tree_grid)
  if (l->workgroups / d->B / d->Hkv * (static_cast<int64_t>(d->B) * d->Hkv + 8) > kMostGrid ||
      static_cast<int64_t>(d->B) * nodes > (int64_t(1) << 30))
    return DSA_ERR_INVALID_ARG;
  return DSA_OK;
}

}  // namespace

// Two kernels.  Up to 64 query rows per (request, KV head), and more of them where
// the chip holds all their tiles at once (two workgroups on each of 256 CUs), stream
// the keys for 32 rows at a time (tree_stream_kernel).  32 heads over 8, d = 128, bf16
// outputs, streamed and through LDS: 512 nodes after 2256 keys 57 and 94 us; 30
// nodes of 16 requests (512 tiles) after 256 to 802 keys 26 and 37, after 256 to 4322 77
// and 140; of 32 requests 46 and 41, 137 and 143, of 48 67 and 49, 206 and 161; 13
// nodes of 32 requests (two row tiles) 89 and 141, fp8 67 and 151.  The others go
// through LDS for 128 rows at a time (tree_tile_kernel).
//
// The keys of a streaming row tile are split where the row tiles alone would leave
// CUs without a workgroup: into about eight, a tile per wave or more (40 tiles of
// d = 128, 32 heads: 14.1 us; at two tiles per wave 15.4), and more of them at two tiles
// per wave (139 tiles, 8 heads: 17.5 us; at one 19.3, at four 21.3, unsplit 48.5).
//
// A split costs a row of partial results and a second kernel: 2.9 us more for a call
// from the host (19.8 us whole and 22.7 split, up to 40 tiles), and on replays what two
// tiles per wave take.  One more tile per wave costs a replay 1.0 us at d = 64 and 2.3
// at d = 128, the next one as much again; so up to three stay whole at d = 64, where
// that is a third of a launch, and up to two at d = 128.  Replayed, 20 heads, whole and
// split: d = 64, 16 tiles 8.9 and 9.1 us, 18 to 24 9.8 to 10.5 and 9.1 to 9.3, 26 11.5
// and 9.2; d = 128, 10 to 16 tiles 10.9 to 11.6 and 10.7 to 11.5, 18 13.5 and 11.3.
// (4, 32 and 64 heads, and 8 with four query heads each, step at the same places.)
TreeLaunch tree_launch(const Derived& d, int nodes) {
  TreeLaunch l{};
  const int64_t rows = static_cast<int64_t>(nodes) * d.G;
  const int64_t pairs = static_cast<int64_t>(d.B) * d.Hkv;
  const bool stream = rows <= 64 || pairs * ((rows + 31) / 32) <= 512;
  l.rows = stream ? 32 : 128;
  l.row_tiles = static_cast<int>((rows + l.rows - 1) / l.rows);
  l.splits = 1;
  l.workgroups = pairs * l.row_tiles;
  if (!stream) return l;
  // Twice the waves on the keys where at most one workgroup per CU has work (32
  // heads, d = 128, 552 keys, 16 nodes, whole: 14.6 us with eight waves, 15.2 with four);
  // with more, what a CU holds at a time decides (32 such requests: 62.3 and 57.3).
  l.waves = l.workgroups <= 256 ? 8 : 4;
  const int64_t keys = d.Lp + (d.mode == DSA_MODE_WINDOW ? std::min(d.Natt, d.Ldec) : d.Ldec) +
                       int64_t{nodes};
  const int64_t tiles = (keys + 31) / 32 + 2;
  const int64_t want = std::max<int64_t>(1, 256 / l.workgroups);
  const int64_t per_wave = (tiles + l.waves - 1) / l.waves;
  const int64_t least = (per_wave - 2) * d.D <= 64
                            ? tiles
                            : std::clamp<int64_t>(tiles / 8, l.waves, 2 * l.waves);
  l.split_tiles = static_cast<int>(std::max(least, (tiles + want - 1) / want));
  l.splits = static_cast<int>((tiles + l.split_tiles - 1) / l.split_tiles);
  l.workgroups *= l.splits;
  l.ws_bytes = l.splits > 1 ? static_cast<size_t>(l.workgroups) * l.rows * (d.D + 4) * 4 : 0;
  return l;
}

}  // namespace dsa

using dsa::Derived;
using dsa::TreeLaunch;

extern "C" {

DSA_API dsa_status dsa_get_tree_plan_layout(int32_t batch, int32_t nodes,
                                            dsa_tree_plan_layout* out) {
  dsa_tree_plan_layout l;
  const dsa_status st = dsa::tree_plan_layout(batch, nodes, &l);
  if (st != DSA_OK) return st;
  if (!out) return DSA_ERR_INVALID_ARG;
  *out = l;
  return DSA_OK;
}

DSA_API size_t dsa_tree_plan_bytes(int32_t batch, int32_t nodes) {
  dsa_tree_plan_layout l;
  return dsa::tree_plan_layout(batch, nodes, &l) == DSA_OK ? l.bytes : 0;
}

DSA_API dsa_status dsa_get_tree_launch_info(const dsa_params* p, const dsa_shape* s, int32_t nodes,
                                            dsa_tree_launch_info* out) {
  Derived d;
  TreeLaunch l;
  const dsa_status st = dsa::tree_derive(p, s, nodes, &d, &l);
  if (st != DSA_OK) return st;
  if (!out) return DSA_ERR_INVALID_ARG;
  out->rows_per_tile = l.rows;
  out->row_tiles = l.row_tiles;
  out->splits = l.splits;
  out->workgroups = static_cast<int32_t>(l.workgroups);
  out->workspace_bytes = l.ws_bytes;
  return DSA_OK;
}

DSA_API size_t dsa_tree_workspace_bytes(const dsa_params* p, const dsa_shape* s, int32_t nodes) {
  Derived d;
  TreeLaunch l;
  return dsa::tree_derive(p, s, nodes, &d, &l) == DSA_OK ? l.ws_bytes : 0;
}

DSA_API dsa_status dsa_tree_plan(int32_t batch, int32_t nodes, const int32_t* d_parent,
                                 const int32_t* d_count, void* d_plan, size_t plan_bytes,
                                 hipStream_t stream) {
  dsa_tree_plan_layout l;
  const dsa_status st = dsa::tree_plan_layout(batch, nodes, &l);
  if (st != DSA_OK) return st;
  if (!d_parent || !d_plan || !dsa::aligned16(d_plan)) return DSA_ERR_INVALID_ARG;
  if (plan_bytes < l.bytes) return DSA_ERR_WORKSPACE;
  char* pb = static_cast<char*>(d_plan);
  dsa::TreePlanArgs a{};
  a.parent = d_parent;
  a.count = d_count;
  a.flags = reinterpret_cast<int32_t*>(pb + l.flags_offset);
  a.max_depth = reinterpret_cast<int32_t*>(pb + l.max_depth_offset);
  a.depth = reinterpret_cast<int32_t*>(pb + l.depth_offset);
  a.out_parent = reinterpret_cast<int32_t*>(pb + l.parent_offset);
  a.anc = reinterpret_cast<uint32_t*>(pb + l.ancestors_offset);
  a.B = batch;
  a.N = nodes;
  a.words = l.words;
  return dsa::hip_status(dsa::launch_tree_plan(a, stream));
}

DSA_API dsa_status dsa_tree_attention(const dsa_params* p, const dsa_shape* s,
                                      const dsa_tree* tree, const void* d_q,
                                      const dsa_node_rows* q_rows, const void* d_k_new,
                                      const void* d_v_new, const dsa_node_rows* new_rows,
                                      const void* d_k, const void* d_v, const dsa_kv_layout* kv,
                                      float sm_scale, void* d_out, int32_t out_type, void* d_ws,
                                      size_t ws_bytes, hipStream_t stream) {
  Derived d;
  TreeLaunch l;
  dsa_status st = dsa::derive(p, s, &d);
  if (st != DSA_OK) return st;
  if ((st = dsa::check_tree(tree, d.B, dsa::kMostNodes)) != DSA_OK) return st;
  if ((st = dsa::tree_derive(p, s, tree->nodes, &d, &l)) != DSA_OK) return st;
  if (!tree->d_base || !d_q || !d_k_new || !d_v_new || !d_k || !d_v || !kv || !d_out)
    return DSA_ERR_INVALID_ARG;
  if ((st = dsa::check_rows(q_rows)) != DSA_OK) return st;
  if ((st = dsa::check_rows(new_rows)) != DSA_OK) return st;
  if (!std::isfinite(sm_scale)) return DSA_ERR_INVALID_ARG;
  if (out_type != DSA_OUT_FP32 && out_type != DSA_OUT_BF16) return DSA_ERR_INVALID_ARG;
  if ((st = dsa::check_kv(kv, d)) != DSA_OK) return st;
  for (const void* x : {d_q, d_k_new, d_v_new, d_k, d_v, static_cast<const void*>(d_out)})
    if (!dsa::aligned16(x)) return DSA_ERR_INVALID_ARG;
  if (l.ws_bytes && (!d_ws || ws_bytes < l.ws_bytes)) return DSA_ERR_WORKSPACE;
  if (l.ws_bytes && !dsa::aligned16(d_ws)) return DSA_ERR_INVALID_ARG;

  const int64_t esz = kv->dtype == DSA_KV_BF16 ? 2 : 1;
  dsa::TreeArgs a{};
  a.q = static_cast<const uint16_t*>(d_q);
  a.kn = static_cast<const uint16_t*>(d_k_new);
  a.vn = static_cast<const uint16_t*>(d_v_new);
  a.k = static_cast<const uint8_t*>(d_k);
  a.v = static_cast<const uint8_t*>(d_v);
  a.qsb = q_rows->stride_batch;
  a.qsn = q_rows->stride_node;
  a.qsh = q_rows->stride_head;
  a.nsb = new_rows->stride_batch;
  a.nsn = new_rows->stride_node;
  a.nsh = new_rows->stride_head;
  a.row_base = kv->d_row_base;
  a.sb = kv->stride_batch * esz;
  a.sh = kv->stride_head * esz;
  a.sr = kv->stride_row * esz;
  a.ks = kv->d_k_scale;
  a.vs = kv->d_v_scale;
  a.base = tree->d_base;
  a.count = tree->d_count;
  if (tree->d_plan) {
    dsa_tree_plan_layout pl;
    dsa::tree_plan_layout(d.B, tree->nodes, &pl);
    const char* pb = static_cast<const char*>(tree->d_plan);
    a.max_depth = reinterpret_cast<const int32_t*>(pb + pl.max_depth_offset);
    a.depth = reinterpret_cast<const int32_t*>(pb + pl.depth_offset);
    a.anc = reinterpret_cast<const uint32_t*>(pb + pl.ancestors_offset);
    a.words = pl.words;
  }
  a.scale_log2 = std::max(std::fabs(sm_scale) * 1.4426950408889634f, dsa::kTreeMinScale);
  a.q_sign = std::signbit(sm_scale) ? 0x80008000u : 0u;
  a.out = d_out;
  a.part = static_cast<float*>(d_ws);
  a.B = d.B;
  a.Hq = d.Hq;
  a.Hkv = d.Hkv;
  a.G = d.G;
  a.N = tree->nodes;
  a.Lp = d.Lp;
  a.Ldec = d.Ldec;
  a.S = d.Ns;
  a.W = d.mode == DSA_MODE_WINDOW ? d.Nr : dsa::kTreeNone;
  a.ring = dsa::ring_slots(kv, d);
  a.row_tiles = l.row_tiles;
  a.splits = l.splits;
  a.split_tiles = l.split_tiles;
  const bool f32 = out_type == DSA_OUT_FP32;
  return dsa::hip_status(kv->dtype == DSA_KV_BF16 ? dsa::launch_tree_bf16(d, l, a, f32, stream)
                                                  : dsa::launch_tree_fp8(d, l, a, f32, stream));
}

DSA_API dsa_status dsa_tree_verify(int32_t batch, int32_t vocab, const dsa_tree* tree,
                                   const int32_t* d_tokens, const float* d_target,
                                   const float* d_draft, const float* d_uniform, int32_t* d_path,
                                   int32_t* d_accepted, int32_t* d_next, hipStream_t stream) {
  if (batch < 1 || vocab < 1 || vocab > (1 << 24)) return DSA_ERR_INVALID_ARG;
  const dsa_status st = dsa::check_tree(tree, batch, DSA_MAX_TREE_NODES);
  if (st != DSA_OK) return st;
  if (!d_tokens || !d_target || !d_uniform || !d_path || !d_accepted || !d_next)
    return DSA_ERR_INVALID_ARG;
  dsa::VerifyArgs a{};
  a.count = tree->d_count;
  if (tree->d_plan) {
    dsa_tree_plan_layout pl;
    dsa::tree_plan_layout(batch, tree->nodes, &pl);
    a.parent = reinterpret_cast<const int32_t*>(static_cast<const char*>(tree->d_plan) +
                                                pl.parent_offset);
  }
  a.tokens = d_tokens;
  a.target = d_target;
  a.draft = d_draft;
  a.uniform = d_uniform;
  a.path = d_path;
  a.accepted = d_accepted;
  a.next = d_next;
  a.N = tree->nodes;
  a.V = vocab;
  return dsa::hip_status(dsa::launch_verify(a, batch, stream));
}

DSA_API dsa_status dsa_kv_append(const dsa_params* p, const dsa_shape* s, const dsa_tree* tree,
                                 const void* d_k_new, const void* d_v_new,
                                 const dsa_node_rows* new_rows, const int32_t* d_path,
                                 const int32_t* d_accepted, int32_t layers, void* d_k, void* d_v,
                                 const dsa_kv_layout* kv, int64_t stride_layer,
                                 hipStream_t stream) {
  Derived d;
  dsa_status st = dsa::derive(p, s, &d);
  if (st != DSA_OK) return st;
  if ((st = dsa::check_tree(tree, d.B, dsa::kMostNodes)) != DSA_OK) return st;
  if (!tree->d_base || !d_k_new || !d_v_new || !d_k || !d_v || !kv) return DSA_ERR_INVALID_ARG;
  if ((st = dsa::check_rows(new_rows)) != DSA_OK) return st;
  if (layers < 1 || stride_layer < 0 || new_rows->stride_layer < 0 ||
      ((stride_layer | new_rows->stride_layer) & 7))
    return DSA_ERR_INVALID_ARG;
  if ((st = dsa::check_kv(kv, d)) != DSA_OK) return st;
  for (const void* x : {d_k_new, d_v_new, static_cast<const void*>(d_k),
                        static_cast<const void*>(d_v)})
    if (!dsa::aligned16(x)) return DSA_ERR_INVALID_ARG;
  const int64_t per = (static_cast<int64_t>(tree->nodes) * d.Hkv * (d.D / 8) + 255) / 256;
  // (a thread's place among a request's rows is counted in 31 bits)
  if (per > std::min(dsa::kMostGrid / 256, dsa::kMostGrid / layers / d.B))
    return DSA_ERR_INVALID_ARG;
  const int64_t esz = kv->dtype == DSA_KV_BF16 ? 2 : 1;
  dsa::AppendArgs a{};
  a.kn = static_cast<const uint16_t*>(d_k_new);
  a.vn = static_cast<const uint16_t*>(d_v_new);
  a.nsl = new_rows->stride_layer;
  a.nsb = new_rows->stride_batch;
  a.nsn = new_rows->stride_node;
  a.nsh = new_rows->stride_head;
  a.base = tree->d_base;
  a.count = tree->d_count;
  a.path = d_path;
  a.accepted = d_accepted;
  a.k = static_cast<uint8_t*>(d_k);
  a.v = static_cast<uint8_t*>(d_v);
  a.row_base = kv->d_row_base;
  a.sl = stride_layer * esz;
  a.sb = kv->stride_batch * esz;
  a.sh = kv->stride_head * esz;
  a.sr = kv->stride_row * esz;
  a.ks = kv->d_k_scale;
  a.vs = kv->d_v_scale;
  a.layers = layers;
  a.B = d.B;
  a.Hkv = d.Hkv;
  a.N = tree->nodes;
  a.Lp = d.Lp;
  a.Ldec = d.Ldec;
  a.S = d.Ns;
  a.ring = dsa::ring_slots(kv, d);
  return dsa::hip_status(dsa::launch_append(a, d.D, kv->dtype, stream));
}

}  // extern "C"
