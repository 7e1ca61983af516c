// What ssa_layer_forward uses of the dense kernels beyond include/ssa_layer.h.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include "../../include/ssa.h"
#include "../../include/ssa_layer.h"

namespace ssa {

// Split tickets at the start of a linear workspace.
constexpr size_t kLinearTicketBytes = 256;

// Two runs of words to set to zero (n[i] = 0: none).
struct ClearWords {
  uint32_t* at[2];
  int64_t n[2];
};

// ssa_rms_norm whose launch also clears words; the buffers must not overlap.
int rms_norm(int32_t m, int32_t n, const uint16_t* x, const uint16_t* weight, float eps,
             uint16_t* out, const ClearWords& clear, void* stream);

// The checks of ssa_key_scores, without its launches.
int check_key_scores(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                     const uint16_t* q, const uint16_t* k_cache, const int32_t* block_table,
                     const float* scores_in, float decay, float* scores_out, void* workspace,
                     size_t ws_bytes);
// The checks of ssa_block_summary, and of the three calls with a sparse plan, without their
// launches; and those of a rotary form.
int check_block_summary(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                        int32_t block_keys, const uint16_t* k_cache, const int32_t* block_table,
                        const uint16_t* summary);
int check_sparse_calls(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                       const uint16_t* q, const uint16_t* k_cache, const uint16_t* v_cache,
                       const uint16_t* summary, const int32_t* block_table, const float* scores,
                       const int32_t* blocks, const uint16_t* out, const void* workspace,
                       size_t ws_bytes);
bool rope_form_ok(const ssa_rope_form& form, int32_t head_dim);
struct SparseHeader;
int check_sparse_plan(const ssa_shape* s, const void* plan_host, const SparseHeader** out);

struct ScoreHeader;
int check_score_plan(const ssa_shape* s, const void* plan_host, const ScoreHeader** out);

}  // namespace ssa
