// C ABI of attention over whole histories: argument checks and launches of the windowed attention, of
// the paged 8-bit cache, and of the beams that continue its sequences.  No allocation, no synchronisation.
#include "common.h"
#include "internal.h"

using namespace tav2;

namespace {

constexpr size_t WS_ALIGN = 256;
constexpr int64_t MAX_ROWS = (int64_t(1) << 31) - 1;
constexpr int64_t MAX_GROUPS = (int64_t(1) << 24) - 1;   // of 256 threads: a launch has fewer than 2^32
constexpr int MAX_HEADS = 65535;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

tav2_status hip_status(hipError_t e) { return e == hipSuccess ? TAV2_OK : TAV2_ERR_HIP; }

bool head_dim_ok(int d) { return d == 32 || d == 64 || d == 128; }

// A scale of 0 stands for 1 / sqrt(head_dim).  The kernels multiply by log2(e): the bound leaves that
// finite.
bool scale_ok(float s) { return s >= 0.f && s <= 2.3e38f; }

// Rows of `heads` heads at least, `per` elements in 16 bytes.
bool stride_ok(int64_t ld, int heads, int head_dim, int per) {
  return ld >= int64_t(heads) * head_dim && ld % per == 0 && ld <= (1 << 24);
}

tav2_status check_kv(const tav2_kv* c) {
  if (!c) return TAV2_ERR_NULL;
  if (!c->k || !c->v || !c->k_scale || !c->v_scale || !c->k_tail || !c->v_tail || !c->table ||
      !c->len || !c->fresh || !c->refs)
    return TAV2_ERR_NULL;
  if (c->num_seqs < 1 || c->layers < 1 || c->pages < 1 || c->max_blocks < 1 || c->kv_heads < 1 ||
      c->max_len < 0)
    return TAV2_ERR_SHAPE;
  if (c->num_seqs > TAV2_KV_SEQS_MAX || c->max_blocks > (1 << 20) || c->kv_heads > MAX_HEADS ||
      !head_dim_ok(c->head_dim) || int64_t(c->layers) * c->kv_heads > 65535)
    return TAV2_ERR_UNSUPPORTED;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_tail, 16) || !aligned(c->v_tail, 16))
    return TAV2_ERR_SHAPE;
  return TAV2_OK;
}

tav2_status check_layer(const tav2_kv* c, int32_t layer) {
  return layer >= 0 && layer < c->layers ? TAV2_OK : TAV2_ERR_SHAPE;
}

tav2_status check_query_sizes(const tav2_kv* c, const tav2_kv_queries* q) {
  if (!q) return TAV2_ERR_NULL;
  if (q->total < 0 || q->max_count < 0 || q->max_count > q->total) return TAV2_ERR_SHAPE;
  if (q->total > 0 && q->max_count == 0) return TAV2_ERR_SHAPE;
  if (q->heads < 1 || q->heads % c->kv_heads || q->window < 0 || q->sinks < 0 || !scale_ok(q->scale))
    return TAV2_ERR_SHAPE;
  if (q->heads > MAX_HEADS || q->total > MAX_ROWS / q->heads) return TAV2_ERR_UNSUPPORTED;
  if (!stride_ok(q->ld, q->heads, c->head_dim, 8)) return TAV2_ERR_SHAPE;
  return TAV2_OK;
}

tav2_status check_queries(const tav2_kv* c, const tav2_kv_queries* q) {
  if (const tav2_status st = check_query_sizes(c, q)) return st;
  if (q->total > 0 && kv_attend_groups(*c, *q) > MAX_GROUPS) return TAV2_ERR_UNSUPPORTED;
  return TAV2_OK;
}

tav2_status check_groups(const tav2_kv_groups* g, bool prefix) {
  if (!g) return TAV2_ERR_NULL;
  if (g->num_groups < 0 || g->max_members < 1 || g->max_members > TAV2_BEAMS_MAX || g->max_own < 0)
    return TAV2_ERR_SHAPE;
  if (g->num_groups > TAV2_KV_SEQS_MAX) return TAV2_ERR_UNSUPPORTED;
  if (g->num_groups > 0 && (!g->offset || (prefix && !g->prefix))) return TAV2_ERR_NULL;
  return TAV2_OK;
}

// The queries over groups of members, besides their sizes.
tav2_status check_prefix(const tav2_kv* c, const tav2_kv_groups* g, const tav2_kv_queries* q) {
  if (q->total > 0 && g->num_groups > 0 && kv_prefix_workgroups(*c, *g, *q) > double(MAX_GROUPS))
    return TAV2_ERR_UNSUPPORTED;
  return TAV2_OK;
}

tav2_status check_beams(const tav2_beams* b, int32_t keep) {
  if (!b) return TAV2_ERR_NULL;
  if (b->dtype != TAV2_F32 && b->dtype != TAV2_BF16) return TAV2_ERR_DTYPE;
  if (b->num_requests < 0 || b->beams < 1 || b->beams > TAV2_BEAMS_MAX || b->vocab < 1 ||
      b->vocab > TAV2_VOCAB_MAX || keep < 1 || keep > TAV2_K_MAX || b->ld < b->vocab ||
      b->eos >= b->vocab)
    return TAV2_ERR_SHAPE;
  if (b->allowed && b->allowed_ld != 0 && b->allowed_ld < (int64_t(b->vocab) + 7) / 8) return TAV2_ERR_SHAPE;
  if (!aligned(b->logits, b->dtype == TAV2_BF16 ? 2 : 4)) return TAV2_ERR_SHAPE;
  const int64_t rows = int64_t(b->num_requests) * b->beams, most = int64_t(1) << 60;
  if (int64_t(b->beams) * b->vocab > MAX_ROWS || rows > MAX_ROWS) return TAV2_ERR_UNSUPPORTED;
  if (rows > 0 && (b->ld > most / rows || (b->allowed && b->allowed_ld > most / rows)))
    return TAV2_ERR_UNSUPPORTED;
  if (beam_select_groups(*b, keep) > MAX_GROUPS) return TAV2_ERR_UNSUPPORTED;
  return TAV2_OK;
}

tav2_status check_ws(const void* ws, size_t ws_bytes, size_t need) {
  if (need == 0) return TAV2_OK;
  return ws && ws_bytes >= need && aligned(ws, WS_ALIGN) ? TAV2_OK : TAV2_ERR_WORKSPACE;
}

}  // namespace

extern "C" {

tav2_status tav2_attend_window(const tav2_window* a, void* stream) {
  if (!a) return TAV2_ERR_NULL;
  if (a->dtype != TAV2_F32 && a->dtype != TAV2_BF16) return TAV2_ERR_DTYPE;
  if (a->num_requests < 0 || a->max_len < 0 || a->heads < 1 || a->kv_heads < 1 ||
      a->heads % a->kv_heads || a->window < 0 || a->sinks < 0 || !scale_ok(a->scale))
    return TAV2_ERR_SHAPE;
  if (!head_dim_ok(a->head_dim) || a->heads > MAX_HEADS) return TAV2_ERR_UNSUPPORTED;
  const int per = a->dtype == TAV2_BF16 ? 8 : 4;
  if (!stride_ok(a->q_ld, a->heads, a->head_dim, per) ||
      !stride_ok(a->k_ld, a->kv_heads, a->head_dim, per) ||
      !stride_ok(a->v_ld, a->kv_heads, a->head_dim, per))
    return TAV2_ERR_SHAPE;
  if (a->num_requests == 0 || a->max_len == 0) return TAV2_OK;
  if (!a->q || !a->k || !a->v || !a->out || !a->offset || !a->len) return TAV2_ERR_NULL;
  if (!aligned(a->q, 16) || !aligned(a->k, 16) || !aligned(a->v, 16) || !aligned(a->out, 16))
    return TAV2_ERR_SHAPE;
  if (int64_t(a->max_len) * (a->heads / a->kv_heads) > (int64_t(1) << 30) ||
      int64_t(a->num_requests) * a->kv_heads > MAX_GROUPS || attend_window_groups(*a) > MAX_GROUPS)
    return TAV2_ERR_UNSUPPORTED;
  return hip_status(launch_attend_window(*a, static_cast<hipStream_t>(stream)));
}

tav2_status tav2_kv_extend(const tav2_kv* c, const int32_t* count, void* stream) {
  tav2_status st;
  if ((st = check_kv(c))) return st;
  if (!count) return TAV2_ERR_NULL;
  return hip_status(launch_kv_extend(*c, count, static_cast<hipStream_t>(stream)));
}

tav2_status tav2_kv_append(const tav2_kv* c, int32_t layer, const void* k, int64_t k_ld,
                           const void* v, int64_t v_ld, const int64_t* offset, int32_t max_count,
                           void* stream) {
  tav2_status st;
  if ((st = check_kv(c)) || (st = check_layer(c, layer))) return st;
  if (max_count < 0) return TAV2_ERR_SHAPE;
  if (!stride_ok(k_ld, c->kv_heads, c->head_dim, 8) || !stride_ok(v_ld, c->kv_heads, c->head_dim, 8))
    return TAV2_ERR_SHAPE;
  if (max_count == 0) return TAV2_OK;
  if (!k || !v || !offset) return TAV2_ERR_NULL;
  if (!aligned(k, 16) || !aligned(v, 16)) return TAV2_ERR_SHAPE;
  if (kv_append_groups(*c, max_count) > MAX_GROUPS) return TAV2_ERR_UNSUPPORTED;
  return hip_status(launch_kv_append(*c, layer, k, k_ld, v, v_ld, offset, max_count,
                                     static_cast<hipStream_t>(stream)));
}

size_t tav2_kv_attend_workspace(const tav2_kv* c, const tav2_kv_queries* q) {
  if (check_kv(c) || check_queries(c, q) || q->total == 0) return 0;
  return kv_attend_bytes(*c, *q);
}

tav2_status tav2_kv_attend(const tav2_kv* c, int32_t layer, const tav2_kv_queries* q,
                           uint32_t flags, void* out, float* lse, void* ws, size_t ws_bytes,
                           void* stream) {
  tav2_status st;
  if ((st = check_kv(c)) || (st = check_layer(c, layer)) || (st = check_queries(c, q))) return st;
  if (flags != TAV2_MASK_CAUSAL && flags != TAV2_MASK_NONE) return TAV2_ERR_SHAPE;
  if (q->total == 0) return TAV2_OK;
  if (!q->q || !q->offset || !out) return TAV2_ERR_NULL;
  if (!aligned(q->q, 16) || !aligned(out, 16)) return TAV2_ERR_SHAPE;
  if ((st = check_ws(ws, ws_bytes, kv_attend_bytes(*c, *q)))) return st;
  return hip_status(launch_kv_attend(*c, layer, *q, flags == TAV2_MASK_CAUSAL, out, lse, ws,
                                     static_cast<hipStream_t>(stream)));
}

tav2_status tav2_kv_fork(const tav2_kv* c, const int32_t* parent, void* stream) {
  tav2_status st;
  if ((st = check_kv(c))) return st;
  if (!parent) return TAV2_ERR_NULL;
  return hip_status(launch_kv_fork(*c, parent, static_cast<hipStream_t>(stream)));
}

tav2_status tav2_kv_free(const tav2_kv* c, const uint8_t* drop, void* stream) {
  tav2_status st;
  if ((st = check_kv(c))) return st;
  if (!drop) return TAV2_ERR_NULL;
  return hip_status(launch_kv_free(*c, drop, static_cast<hipStream_t>(stream)));
}

tav2_status tav2_kv_trim(const tav2_kv* c, int32_t window, int32_t sinks, void* stream) {
  tav2_status st;
  if ((st = check_kv(c))) return st;
  if (window < 1 || sinks < 0) return TAV2_ERR_SHAPE;
  return hip_status(launch_kv_trim(*c, window, sinks, static_cast<hipStream_t>(stream)));
}

size_t tav2_kv_compact_workspace(const tav2_kv* c) { return check_kv(c) ? 0 : kv_plan_bytes(*c); }

tav2_status tav2_kv_compact(const tav2_kv* c, int32_t* used, void* ws, size_t ws_bytes,
                            void* stream) {
  tav2_status st;
  if ((st = check_kv(c))) return st;
  if (!used) return TAV2_ERR_NULL;
  if ((st = check_ws(ws, ws_bytes, kv_plan_bytes(*c)))) return st;
  return hip_status(launch_kv_compact(*c, used, ws, static_cast<hipStream_t>(stream)));
}

tav2_status tav2_kv_reorder(const tav2_kv* c, const tav2_kv_groups* g, const int32_t* parent,
                            int32_t members, void* stream) {
  tav2_status st;
  if ((st = check_kv(c)) || (st = check_groups(g, false))) return st;
  if (members < 0) return TAV2_ERR_SHAPE;
  if (members == 0 || g->num_groups == 0) return TAV2_OK;
  if (!parent) return TAV2_ERR_NULL;
  if (kv_reorder_parts(*c) * g->num_groups > MAX_GROUPS) return TAV2_ERR_UNSUPPORTED;
  return hip_status(launch_kv_reorder(*c, *g, parent, members, static_cast<hipStream_t>(stream)));
}

size_t tav2_kv_attend_prefix_workspace(const tav2_kv* c, const tav2_kv_groups* g,
                                       const tav2_kv_queries* q) {
  if (check_kv(c) || check_groups(g, true) || check_query_sizes(c, q) || check_prefix(c, g, q) ||
      q->total == 0 || g->num_groups == 0)
    return 0;
  return kv_prefix_bytes(*c, *g, *q);
}

tav2_status tav2_kv_attend_prefix(const tav2_kv* c, int32_t layer, const tav2_kv_groups* g,
                                  const tav2_kv_queries* q, uint32_t flags, void* out, float* lse,
                                  void* ws, size_t ws_bytes, void* stream) {
  tav2_status st;
  if ((st = check_kv(c)) || (st = check_layer(c, layer)) || (st = check_groups(g, true)) ||
      (st = check_query_sizes(c, q)) || (st = check_prefix(c, g, q)))
    return st;
  if (flags != TAV2_MASK_CAUSAL && flags != TAV2_MASK_NONE) return TAV2_ERR_SHAPE;
  if (q->total == 0 || g->num_groups == 0) return TAV2_OK;
  if (!q->q || !q->offset || !out) return TAV2_ERR_NULL;
  if (!aligned(q->q, 16) || !aligned(out, 16)) return TAV2_ERR_SHAPE;
  if ((st = check_ws(ws, ws_bytes, kv_prefix_bytes(*c, *g, *q)))) return st;
  return hip_status(launch_kv_prefix(*c, layer, *g, *q, flags == TAV2_MASK_CAUSAL, out, lse, ws,
                                     static_cast<hipStream_t>(stream)));
}

size_t tav2_beam_select_workspace(const tav2_beams* b, int32_t keep) {
  return check_beams(b, keep) || b->num_requests == 0 ? 0 : beam_select_bytes(*b, keep);
}

tav2_status tav2_beam_select(const tav2_beams* b, int32_t keep, uint32_t flags, int32_t* out_parent,
                             int32_t* out_token, float* out_score, uint8_t* out_done, void* ws,
                             size_t ws_bytes, void* stream) {
  tav2_status st;
  if ((st = check_beams(b, keep))) return st;
  if (flags != TAV2_BEAM_RANKED && flags != TAV2_BEAM_IN_PLACE) return TAV2_ERR_SHAPE;
  if (flags == TAV2_BEAM_IN_PLACE && keep != b->beams) return TAV2_ERR_SHAPE;
  if (b->num_requests == 0) return TAV2_OK;
  if (!b->logits || !out_parent || !out_token || !out_score) return TAV2_ERR_NULL;
  if ((st = check_ws(ws, ws_bytes, beam_select_bytes(*b, keep)))) return st;
  return hip_status(launch_beam_select(*b, keep, flags == TAV2_BEAM_IN_PLACE, out_parent, out_token,
                                       out_score, out_done, ws, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
