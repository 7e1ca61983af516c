// Plan blob of include/ssa_sparse.h: written by the host planner (ssa_sparse_plan.cpp),
// read unchanged by the kernels.
//
//   [SparseHeader][SparseReq x num_reqs][SparseRows x (num_groups + num_singles)]
//   [SparseScore x num_scores]
//
// A workgroup runs one row (or score item) for one kv head; a request's fields are copied
// into its records, so that a workgroup reads one before it starts.
#pragma once
#include <stdint.h>

namespace ssa {

// Kind and, in the last character, version of the layout.
constexpr uint32_t kSparseMagic = 0x31505353u;  // "SSP1"
constexpr int kSparseThreads = 256;      // four waves (summaries, scores, attention)
constexpr int kRowGroup = 16;            // rows of a chunk's SparseRows, at most
constexpr int kSparseMaxBlocks = 32768;  // blocks of a request
// Blocks of one pass of a score workgroup: two 16-block tiles for each of four waves.
constexpr int kScorePass = 128;
constexpr int kSparseTickets = 1024;     // int32 words at the start of the workspace

struct SparseHeader {
  uint32_t magic;
  int32_t block_keys;
  uint64_t hash;
  int32_t num_reqs, num_tokens;
  int32_t hq, hkv, head_dim, page_size, max_pages_per_req, num_pages;
  float softmax_scale;
  int32_t top, sink, recent;
  int32_t max_blocks;   // stride of the scores
  int32_t most_blocks;  // blocks that the longest row sees
  int32_t num_groups, num_singles, num_scores;
  int32_t off_rows, off_scores;
  int32_t score_tiles;    // 16-column tiles of a chunk's score item
  int32_t nsplit;         // pieces that a row's list is cut into
  int32_t split_entries;  // entries of a piece
  int64_t plan_bytes, ws_bytes;
};
static_assert(sizeof(SparseHeader) == 120, "sparse header size");

// The batch that the plan is of; host side only.
struct SparseReq {
  int32_t q_len, ctx_len;
};

// Consecutive new rows of one request: up to kRowGroup of a chunk (the first num_groups
// records), or a decode's single one.
struct SparseRows {
  int32_t req;
  int32_t row0;  // token row of the first
  int32_t pos0;  // its position
  int32_t n;
};
static_assert(sizeof(SparseRows) == 16, "rows size");

// Scores of rows row0 .. row0 + n - 1 (positions pos0 ..) in blocks [blk0, blk1).
struct SparseScore {
  int32_t req, row0, pos0, n;
  int32_t blk0, blk1, pad0, pad1;
};
static_assert(sizeof(SparseScore) == 32, "score item size");

// Rows of a chunk record that an attention workgroup takes, 32 columns (row, head of the
// group) at most, and workgroups of a record.
constexpr int sparse_tokens(int g) { return 32 / g < kRowGroup ? 32 / g : kRowGroup; }
constexpr int sparse_subs(int g) { return (kRowGroup + sparse_tokens(g) - 1) / sparse_tokens(g); }
// One piece's record of a workgroup's rows and kv head: m and l for `cols` columns (row,
// head of the group), padded to four floats, then o [cols][D].
constexpr int sparse_rec_o(int cols) { return (2 * cols + 3) / 4 * 4; }
constexpr int sparse_rec_floats(int cols, int d) { return sparse_rec_o(cols) + cols * d; }

}  // namespace ssa
