// Plan blobs of include/ssa_evict.h: written by the host planner
// (ssa_evict_plan.cpp), read unchanged by the kernels.
//
//   score plan  [ScoreHeader][ScoreReq x num_reqs][ScoreItem x (the five lists)]
//   evict plan  [EvictHeader][EvictReq x num_reqs][EvictShort x num_short]
//               [EvictSeg x num_segs][EvictItem x num_items]
//
// A workgroup runs one item for one kv head; a request's fields are copied into
// its items, so that a workgroup reads one record before it starts.
#pragma once
#include <stdint.h>

namespace ssa {

// Kind and, in the last character, version of the layout.
constexpr uint32_t kScoreMagic = 0x32435353u;  // "SSC2"
constexpr uint32_t kEvictMagic = 0x31565353u;  // "SSV1"
constexpr int kScoreThreads = 256;             // four waves
constexpr int kScoreWaveCols = 64;             // stationary vectors of a wave (chunk kernels)
constexpr int kSumKeys = 4 * kScoreWaveCols;   // keys of a tile of the second chunk pass
constexpr int kJoinKeys = 1024;                // keys of one item of the decode join
constexpr int kWholeLogits = 8192;             // logits of a decode row that one workgroup holds
constexpr int kColsPad = 256;                  // a chunk request's columns are padded to this
constexpr int kEvictSlots = 64;                // kept keys of one compaction item
constexpr int kShortList = 8192;               // keys of a list that one workgroup selects from
constexpr int kSegKeys = 8192;                 // keys of a segment of a longer one
constexpr int kSegBins = 4096;                 // its first histogram: 12 bits
// Columns (row, head in group) of a request: index arithmetic by a 32-bit reciprocal.
constexpr int64_t kMaxScoreCols = (int64_t)1 << 28;

// The item lists of a score plan, in this order.
enum ScoreList : int32_t {
  kListLse = 0,    // chunk requests: log-sum-exp of columns over a key range
  kListDecode,     // one counted row: logits (and attention) over a key range
  kListLseJoin,    // log-sum-exps over the pieces of a cut key range
  kListSum,        // chunk requests: a key tile's weights over all columns
  kListDecodeJoin, // one counted row: a key range's weights, and the joined attention
  kNumScoreLists
};

struct ScoreHeader {
  uint32_t magic;
  int32_t last_rows;
  uint64_t hash;
  int32_t num_reqs, num_tokens;
  int32_t hq, hkv, head_dim, page_size, max_pages_per_req, num_pages;
  float softmax_scale;
  int32_t max_q_len;
  int32_t lse_groups;   // waves side by side over the columns in the first chunk pass
  int32_t sum_cols;     // columns of an item of the second, a multiple of 32
  int32_t off_items;
  int32_t num_tickets;  // of the second: int32 words at the start of the workspace
  int32_t count[kNumScoreLists], first[kNumScoreLists];  // items of each list
  int64_t plan_bytes, ws_bytes;
};
static_assert(sizeof(ScoreHeader) == 128, "score header size");

// The batch that the plan is of; host side only.
struct ScoreReq {
  int32_t q_len, ctx_len;
};

struct ScoreItem {
  int32_t req;
  int32_t q_row;    // token row of the first counted row
  int32_t ticket;   // kListSum, of several pieces: the tile's ticket for kv head 0
  int32_t rows;     // counted rows; row j sees keys 0 .. len - rows + j
  int32_t len;      // keys, u + c
  int32_t ctx_len;  // u
  int32_t col0;     // first column (row * G + head in group) of the item
  int32_t cols_pad; // columns of the request, padded; decode lists: its padded length
  int32_t key0, key1;
  int32_t split, nsplit;  // kListDecode: split -1, the whole row (no join)
  // float offsets in the workspace for kv head 0:
  //   chunk lists:   off0 = (m 32 times, 1 / l 32 times) [Hkv][cols_pad / 32][2][32],
  //                  off1 = (m, l) [Hkv][nsplit][cols_pad][2],
  //                  kListSum: sums [pieces][Hkv][len, padded to kSumKeys]
  //   decode lists:  off0 = logits [Hkv][G][cols_pad], off1 = records [Hkv][nsplit][record]
  int64_t off0, off1;
};
static_assert(sizeof(ScoreItem) == 64, "score item size");

// One key range's record of a decode row: m and l for G heads, padded to four floats,
// then o [G][D].
constexpr int score_rec_o(int g) { return (2 * g + 3) / 4 * 4; }
constexpr int score_rec_floats(int g, int d) { return score_rec_o(g) + g * d; }

struct EvictHeader {
  uint32_t magic;
  int32_t sink, recent;
  int32_t num_reqs;
  uint64_t hash;
  int32_t hq, hkv, head_dim, page_size, max_pages_per_req, num_pages;
  float softmax_scale;
  int32_t num_short, num_segs, num_items;           // selection: short lists, segments; compaction
  int32_t off_short, off_segs, off_items, num_long;  // num_long: requests of more than kShortList keys
  int64_t num_keep;  // kept keys of one kv head over all requests
  int64_t plan_bytes, ws_bytes;
  int64_t ws_counts, ws_cands;  // byte offsets in the workspace
  int64_t pad;
};
static_assert(sizeof(EvictHeader) == 128, "evict header size");

struct EvictReq {
  int32_t len, kept;
  int64_t keep_off;  // n_0 + ... + n_{i-1}
};

// A request of at most kShortList keys: one workgroup a kv head.
struct EvictShort {
  int32_t req, len, kept, pad;
  int64_t keep_off;
};
static_assert(sizeof(EvictShort) == 24, "short list size");

// kSegKeys keys of a longer one.  Workspace, for list = long_index * Hkv + kv head:
//   int32 [lists][kSegBins]   histogram of the scores' first 12 bits, at 0
//   SegState [lists]          after it
//   int32 [segments][Hkv]     kept for sure, at ws_counts
//   uint64 candidates         at ws_cands: list's from Hkv * cand_off + kv head * len on
struct EvictSeg {
  int32_t req, len, kept;
  int32_t key0;        // the segment's first key
  int32_t seg0;        // index of the request's first segment in the plan
  int32_t long_index;  // of the request among those of more than kShortList keys
  int64_t keep_off;
  int64_t cand_off;    // keys of the long requests before
};
static_assert(sizeof(EvictSeg) == 40, "segment size");

struct SegState {
  int32_t num_cands;  // scores whose first 12 bits are the threshold's
  int32_t bin, need;  // those bits, and how many candidates stay
  int32_t pad;
};

// kept keys slot0 .. slot0 + n - 1 of every kv head of a request that loses keys
struct EvictItem {
  int32_t req, slot0, n, len;
  int32_t kept, pad;
  int64_t keep_off;
};
static_assert(sizeof(EvictItem) == 32, "evict item size");

}  // namespace ssa
