// One decoder layer as a sequence of the library's launches
// (include/ssa_layer.h): host code only.  All sizes, pointers, positions and
// the workspace are checked before the first launch.
#include <stddef.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "../../include/ssa_evict.h"
#include "../../include/ssa_layer.h"
#include "../../include/ssa_sparse.h"
#include "ssa_evict_format.h"
#include "ssa_layer_internal.h"
#include "ssa_plan_format.h"
#include "ssa_sparse_format.h"

namespace ssa {
int check_plan(const ssa_shape* s, const void* plan_host, const PlanHeader** out);
}

namespace {
using namespace ssa;

constexpr double kPi = 3.14159265358979323846;

size_t align256(size_t b) { return (b + 255) / 256 * 256; }

// Byte offsets of the regions of the layer workspace.  Where the split tickets
// of attention and of the linear layers lie depends on the plan, so another
// plan's call may have left records or activations there: the first launch
// clears them.  The attention workspace comes first, so its launch counters and
// status word lie at the same place for every plan, and are left alone.
struct LayerWs {
  size_t attn, gemm, xn, qkv, q, a, h, act, total;
  size_t attn_bytes, gemm_bytes;
};

int layer_ws(const ssa_shape* shape, const void* plan_host, const ssa_layer_weights* w,
             const PlanHeader** hdr, LayerWs* l) {
  if (!shape || !plan_host || !w || !hdr || !l) return SSA_ERR_NULL;
  const PlanHeader* h = nullptr;
  int rc = check_plan(shape, plan_host, &h);
  if (rc) return rc;
  const int64_t t = h->num_tokens;
  const int64_t qd = (int64_t)h->hq * h->head_dim;
  const int64_t nqkv = (int64_t)(h->hq + 2 * h->hkv) * h->head_dim;
  if (w->hidden <= 0 || w->hidden % 128 || w->hidden > 8192 || w->inter <= 0 || w->inter % 64 ||
      nqkv % 128 || !(w->eps >= 0.f) || w->max_position < 0)
    return SSA_ERR_ARG;
  size_t g = 0, b = 0;
  const int32_t m = (int32_t)t;
  if ((rc = ssa_linear_workspace_size(m, (int32_t)nqkv, w->hidden, &b))) return rc;
  g = std::max(g, b);
  if ((rc = ssa_linear_workspace_size(m, w->hidden, (int32_t)qd, &b))) return rc;
  g = std::max(g, b);
  if ((rc = ssa_linear_workspace_size(m, 2 * w->inter, w->hidden, &b))) return rc;
  g = std::max(g, b);
  if ((rc = ssa_linear_workspace_size(m, w->hidden, w->inter, &b))) return rc;
  g = std::max(g, b);
  l->attn_bytes = (size_t)h->ws_bytes;
  l->gemm_bytes = g;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off += align256(bytes);
    return o;
  };
  l->attn = take(l->attn_bytes);
  l->gemm = take(l->gemm_bytes);
  l->xn = take((size_t)t * w->hidden * 2);
  l->qkv = take((size_t)t * nqkv * 2);
  l->q = take((size_t)t * qd * 2);
  l->a = take((size_t)t * qd * 2);
  l->h = take((size_t)t * w->hidden * 2);
  l->act = take((size_t)t * w->inter * 2);
  l->total = off;
  *hdr = h;
  return SSA_OK;
}

// e: the parts of ssa_layer_forward_evicting, sp: of ssa_layer_forward_sparse; or null.
int layer_forward(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                  const ssa_layer_weights* w, const ssa_layer_eviction* e,
                  const ssa_layer_sparse* sp, const uint16_t* x, uint16_t* out, uint16_t* k_cache,
                  uint16_t* v_cache, const int32_t* block_table, void* workspace, size_t ws_bytes,
                  void* stream) {
  const PlanHeader* h = nullptr;
  LayerWs l;
  int rc = layer_ws(shape, plan_host, w, &h, &l);
  if (rc) return rc;
  if (!plan_dev) return SSA_ERR_NULL;
  const ReqEntry* reqs =
      reinterpret_cast<const ReqEntry*>(static_cast<const uint8_t*>(plan_host) + h->off_reqs);
  const int32_t* shift = e ? e->shift_host : sp ? sp->shift_host : nullptr;
  const int32_t* shift_dev = e ? e->shift_dev : sp ? sp->shift_dev : nullptr;
  const void* const score_plan = e ? e->score_plan_host : nullptr;
  const void* const sparse_plan = sp ? sp->plan_host : nullptr;
  if (!shift != !shift_dev) return SSA_ERR_NULL;
  if (sp && sp->rope && !rope_form_ok(*sp->rope, h->head_dim)) return SSA_ERR_ARG;
  for (int32_t i = 0; i < h->num_reqs; ++i) {
    if (reqs[i].q_len <= 0) continue;
    const int64_t s = shift ? shift[i] : 0;
    if (s < 0 || s + reqs[i].ctx_len + reqs[i].q_len > w->max_position) return SSA_ERR_ARG;
  }
  const int32_t t = h->num_tokens;
  if (score_plan) {
    const ScoreHeader* sh = nullptr;
    if ((rc = check_score_plan(shape, score_plan, &sh))) return rc;
    if (sh->num_reqs != h->num_reqs) return SSA_ERR_PLAN_MISMATCH;
    const ScoreReq* scored = reinterpret_cast<const ScoreReq*>(
        static_cast<const uint8_t*>(score_plan) + sizeof(ScoreHeader));
    for (int32_t i = 0; i < h->num_reqs; ++i)
      if (scored[i].q_len != reqs[i].q_len || scored[i].ctx_len != reqs[i].ctx_len)
        return SSA_ERR_PLAN_MISMATCH;
  }
  if (sparse_plan) {
    const SparseHeader* sh = nullptr;
    if ((rc = check_sparse_plan(shape, sparse_plan, &sh))) return rc;
    if (sh->num_reqs != h->num_reqs) return SSA_ERR_PLAN_MISMATCH;
    const SparseReq* of = reinterpret_cast<const SparseReq*>(
        static_cast<const uint8_t*>(sparse_plan) + sizeof(SparseHeader));
    for (int32_t i = 0; i < h->num_reqs; ++i)
      if (of[i].q_len != reqs[i].q_len || of[i].ctx_len != reqs[i].ctx_len)
        return SSA_ERR_PLAN_MISMATCH;
    if (!sp->summary) return SSA_ERR_NULL;
    if (sp->block_keys != sh->block_keys) return SSA_ERR_ARG;
  }
  if (t == 0) return SSA_OK;
  if (!x || !out || !k_cache || !v_cache || !block_table || !w->attn_norm || !w->w_qkv ||
      !w->w_o || !w->mlp_norm || !w->w_gate_up || !w->w_down || !w->cos_sin)
    return SSA_ERR_NULL;
  if (!workspace || ws_bytes < l.total) return SSA_ERR_WORKSPACE;
  if (score_plan &&
      (rc = check_key_scores(shape, score_plan, e->score_plan_dev,
                             reinterpret_cast<const uint16_t*>(static_cast<char*>(workspace) + l.q),
                             k_cache, block_table, e->scores_in, e->decay, e->scores_out,
                             e->score_workspace, e->score_ws_bytes)))
    return rc;
  if (sp && sp->summary &&
      (rc = check_block_summary(shape, plan_host, plan_dev, sp->block_keys, k_cache, block_table,
                                sp->summary)))
    return rc;
  if (sparse_plan) {
    const char* const of = static_cast<const char*>(workspace);
    if ((rc = check_sparse_calls(shape, sparse_plan, sp->plan_dev,
                                 reinterpret_cast<const uint16_t*>(of + l.q), k_cache, v_cache,
                                 sp->summary, block_table, sp->scores, sp->blocks,
                                 reinterpret_cast<const uint16_t*>(of + l.a), sp->workspace,
                                 sp->ws_bytes)))
      return rc;
  }
  char* ws = static_cast<char*>(workspace);
  auto at = [&](size_t off) { return reinterpret_cast<uint16_t*>(ws + off); };
  uint16_t *xn = at(l.xn), *qkv = at(l.qkv), *q = at(l.q), *a = at(l.a), *hb = at(l.h),
           *act = at(l.act);
  void* gws = ws + l.gemm;
  const int32_t hid = w->hidden, qd = h->hq * h->head_dim;
  const int32_t nqkv = (h->hq + 2 * h->hkv) * h->head_dim;

  const size_t counters = kLaunchCounters * sizeof(uint32_t);
  const ClearWords tickets = {
      {reinterpret_cast<uint32_t*>(ws + l.attn + counters), static_cast<uint32_t*>(gws)},
      {((int64_t)h->ws_partials_off - (int64_t)counters) / 4,
       l.gemm_bytes > 0 ? (int64_t)(kLinearTicketBytes / 4) : 0}};
  if ((rc = rms_norm(t, hid, x, w->attn_norm, w->eps, xn, tickets, stream))) return rc;
  if ((rc = ssa_linear(t, nqkv, hid, SSA_EPILOGUE_NONE, xn, w->w_qkv, nullptr, qkv, gws,
                       l.gemm_bytes, stream)))
    return rc;
  if (sp && sp->rope)
    rc = ssa_rope_append_as(shape, plan_host, plan_dev, sp->rope, qkv, w->cos_sin, w->max_position,
                            shift, shift_dev, q, k_cache, v_cache, block_table, stream);
  else
    rc = shift ? ssa_rope_append_shifted(shape, plan_host, plan_dev, qkv, w->cos_sin,
                                         w->max_position, shift, shift_dev, q, k_cache, v_cache,
                                         block_table, stream)
               : ssa_rope_append(shape, plan_host, plan_dev, qkv, w->cos_sin, w->max_position, q,
                                 k_cache, v_cache, block_table, stream);
  if (rc) return rc;
  if (sp && sp->summary &&
      (rc = ssa_block_summary(shape, plan_host, plan_dev, sp->block_keys, k_cache, block_table,
                              sp->summary, stream)))
    return rc;
  if (score_plan &&
      (rc = ssa_key_scores(shape, score_plan, e->score_plan_dev, q, k_cache, block_table,
                           e->scores_in, e->decay, e->scores_out, e->score_workspace,
                           e->score_ws_bytes, stream)))
    return rc;
  if (sparse_plan) {
    if ((rc = ssa_block_scores(shape, sparse_plan, sp->plan_dev, q, sp->summary, block_table,
                               sp->scores, stream)) ||
        (rc = ssa_block_select(shape, sparse_plan, sp->plan_dev, sp->scores, sp->blocks, stream)) ||
        (rc = ssa_sparse_attention(shape, sparse_plan, sp->plan_dev, q, k_cache, v_cache,
                                   block_table, sp->blocks, a, sp->workspace, sp->ws_bytes,
                                   stream)))
      return rc;
  } else if ((rc = ssa_mixed_attention(shape, plan_host, plan_dev, q, k_cache, v_cache,
                                       block_table, a, ws + l.attn, l.attn_bytes, stream))) {
    return rc;
  }
  if ((rc = ssa_linear(t, hid, qd, SSA_EPILOGUE_RESIDUAL, a, w->w_o, x, hb, gws, l.gemm_bytes,
                       stream)))
    return rc;
  if ((rc = ssa_rms_norm(t, hid, hb, w->mlp_norm, w->eps, xn, stream))) return rc;
  if ((rc = ssa_linear(t, 2 * w->inter, hid, SSA_EPILOGUE_SWIGLU, xn, w->w_gate_up, nullptr, act,
                       gws, l.gemm_bytes, stream)))
    return rc;
  return ssa_linear(t, hid, w->inter, SSA_EPILOGUE_RESIDUAL, act, w->w_down, hb, out, gws,
                    l.gemm_bytes, stream);
}

}  // namespace

extern "C" {

int ssa_rope_table(int32_t max_position, int32_t d, double base, float* out) {
  const ssa_rope_scaling none = {SSA_ROPE_SCALE_NONE, 0, 1.0, 0.0, 0.0, 1.0};
  return ssa_rope_table_scaled(max_position, d, base, &none, out);
}

int ssa_rope_table_scaled(int32_t max_position, int32_t d, double base,
                          const ssa_rope_scaling* scaling, float* out) {
  if (!out || !scaling) return SSA_ERR_NULL;
  if (max_position < 1 || d < 2 || d % 2 || !std::isfinite(base) || !(base > 1.0)) return SSA_ERR_ARG;
  const ssa_rope_scaling& s = *scaling;
  if (s.kind < SSA_ROPE_SCALE_NONE || s.kind > SSA_ROPE_SCALE_PARTS || !std::isfinite(s.magnitude) ||
      !(s.magnitude > 0.0))
    return SSA_ERR_ARG;
  if (s.kind != SSA_ROPE_SCALE_NONE && (!std::isfinite(s.factor) || !(s.factor >= 1.0)))
    return SSA_ERR_ARG;
  if (s.kind == SSA_ROPE_SCALE_BASE) {
    if (d <= 2) return SSA_ERR_ARG;
    base *= std::pow(s.factor, (double)d / (d - 2));
    if (!std::isfinite(base)) return SSA_ERR_ARG;
  }
  if (s.kind == SSA_ROPE_SCALE_PARTS &&
      (s.trained_positions < 1 || !std::isfinite(s.high) || !(s.low >= 0.0) || !(s.low < s.high)))
    return SSA_ERR_ARG;
  const int half = d / 2;
  for (int i = 0; i < half; ++i) {
    double t = std::pow(base, -2.0 * i / d);
    if (s.kind == SSA_ROPE_SCALE_LINEAR) {
      t /= s.factor;
    } else if (s.kind == SSA_ROPE_SCALE_PARTS) {
      const double turns = s.trained_positions * t / (2.0 * kPi);
      const double w = std::min(1.0, std::max(0.0, (turns - s.low) / (s.high - s.low)));
      t = w * t + (1.0 - w) * t / s.factor;
    }
    for (int64_t p = 0; p < max_position; ++p) {
      const double a = (double)p * t;
      out[p * d + i] = (float)(s.magnitude * std::cos(a));
      out[p * d + half + i] = (float)(s.magnitude * std::sin(a));
    }
  }
  return SSA_OK;
}

int ssa_layer_workspace_size(const ssa_shape* shape, const void* plan_host,
                             const ssa_layer_weights* w, size_t* ws_bytes) {
  if (!ws_bytes) return SSA_ERR_NULL;
  const PlanHeader* h = nullptr;
  LayerWs l;
  const int rc = layer_ws(shape, plan_host, w, &h, &l);
  if (rc) return rc;
  *ws_bytes = l.total;
  return SSA_OK;
}

int ssa_layer_forward(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                      const ssa_layer_weights* w, const uint16_t* x, uint16_t* out,
                      uint16_t* k_cache, uint16_t* v_cache, const int32_t* block_table,
                      void* workspace, size_t ws_bytes, void* stream) {
  return layer_forward(shape, plan_host, plan_dev, w, nullptr, nullptr, x, out, k_cache, v_cache,
                       block_table, workspace, ws_bytes, stream);
}

int ssa_layer_forward_evicting(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                               const ssa_layer_weights* w, const ssa_layer_eviction* eviction,
                               const uint16_t* x, uint16_t* out, uint16_t* k_cache,
                               uint16_t* v_cache, const int32_t* block_table, void* workspace,
                               size_t ws_bytes, void* stream) {
  if (!eviction) return SSA_ERR_NULL;
  return layer_forward(shape, plan_host, plan_dev, w, eviction, nullptr, x, out, k_cache, v_cache,
                       block_table, workspace, ws_bytes, stream);
}

int ssa_layer_forward_sparse(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                             const ssa_layer_weights* w, const ssa_layer_sparse* sparse,
                             const uint16_t* x, uint16_t* out, uint16_t* k_cache, uint16_t* v_cache,
                             const int32_t* block_table, void* workspace, size_t ws_bytes,
                             void* stream) {
  if (!sparse) return SSA_ERR_NULL;
  return layer_forward(shape, plan_host, plan_dev, w, nullptr, sparse, x, out, k_cache, v_cache,
                       block_table, workspace, ws_bytes, stream);
}

}  // extern "C"
