// Host side of include/ssa_sparse.h: argument checks and the plan.  Pure host code (no
// HIP call), so it is testable without a GPU.
#include <algorithm>
#include <cstring>
#include <new>
#include <vector>

#include "../../include/ssa_sparse.h"
#include "ssa_sparse_format.h"

namespace ssa {

int validate_shape(const ssa_shape* s);

namespace {

constexpr int64_t kMaxLen = 1 << 30;
// A token's queries: 32-bit byte offsets within a few rows of them.
constexpr int64_t kMaxQueryRow = 1 << 24;
// Workgroups that a launch should have, at least: four on each of 256 compute units.
constexpr int64_t kFillGroups = 1024;
// And of attention: two on each, which its registers allow.  (32 decode rows of 4096 keys, 64/8
// heads: 116, 105, 117 and 109 us in lists cut for 256, 512, 768 and 1024 workgroups, 8
// such rows 28, 32 and 35 in those for 512, 768 and 1024.)
constexpr int64_t kAttentionGroups = 512;
// Keys of a piece of a row's list, at least: 32 for each of four waves, twice.  (A row of 2048
// keys, 32/8 heads: 12.1, 12.1 and 14.6 us in pieces of 128, 256 and 512, of 4096, 64/8: 14.9,
// 13.3 and 14.5.)
constexpr int64_t kPieceKeys = 256;
constexpr int64_t kMaxScoreRow = 1 << 24;
constexpr int kMaxScoreTiles = 16;
constexpr int64_t kMaxSplits = 64;  // pieces of a list: one workgroup joins them

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }

uint64_t fnv1a(uint64_t h, const void* p, size_t n) {
  const unsigned char* b = static_cast<const unsigned char*>(p);
  for (size_t i = 0; i < n; ++i) {
    h ^= b[i];
    h *= 1099511628211ull;
  }
  return h;
}

struct SparsePlan {
  SparseHeader hdr;
  std::vector<SparseRows> groups, singles;
  std::vector<SparseScore> scores;
};

int build(const ssa_shape* s, const ssa_sparse_config* cfg, const int32_t* q_len,
          const int32_t* ctx_len, int32_t n, SparsePlan* p) {
  const int rc = validate_shape(s);
  if (rc) return rc;
  if (!cfg) return SSA_ERR_NULL;
  if (n < 0) return SSA_ERR_LENGTH;
  if (n > 0 && (!q_len || !ctx_len)) return SSA_ERR_NULL;
  const int64_t bk = cfg->block_keys, top = cfg->top_blocks;
  if (bk != 16 && bk != 32 && bk != 64 && bk != 128) return SSA_ERR_ARG;
  if (cfg->sink_blocks < 0 || cfg->recent_blocks < 1 || top > kSparseMaxBlocks ||
      (int64_t)cfg->sink_blocks + cfg->recent_blocks > top)
    return SSA_ERR_ARG;
  const int hkv = s->num_kv_heads, g = s->num_q_heads / hkv, d = s->head_dim;
  if ((int64_t)s->num_q_heads * d > kMaxQueryRow) return SSA_ERR_SHAPE;
  int64_t tokens = 0, keys = 0, most = 0, groups = 0, singles = 0, single_passes = 0;
  for (int32_t i = 0; i < n; ++i) {
    const int64_t c = q_len[i], u = ctx_len[i];
    if (c < 0 || u < 0) return SSA_ERR_LENGTH;
    tokens += c;
    keys += c + u;
    if (tokens > kMaxLen || keys > kMaxLen) return SSA_ERR_LENGTH;
    if (ceil_div(c + u, SSA_PAGE_SIZE) > s->max_pages_per_req) return SSA_ERR_PAGES;
    if (c == 0) continue;
    const int64_t blocks = ceil_div(c + u, bk);
    if (blocks > kSparseMaxBlocks) return SSA_ERR_LENGTH;
    most = std::max(most, blocks);
    if (c == 1) {
      ++singles;
      single_passes += ceil_div(blocks, kScorePass);
    } else {
      groups += ceil_div(c, kRowGroup);
    }
  }
  if ((groups + singles) * (int64_t)sizeof(SparseRows) > INT32_MAX) return SSA_ERR_LENGTH;

  // Score items: a chunk's are 128 blocks by as many 16-column tiles (tokens x heads of
  // a group) as leave enough workgroups; a decode row's as many passes of 128 blocks.
  int64_t tokens_per_tile = 16;
  while (tokens_per_tile * g > 16) tokens_per_tile /= 2;  // heads padded to a power of two
  auto chunk_items = [&](int64_t tiles) {
    int64_t items = 0;
    for (int32_t i = 0; i < n; ++i)
      if (q_len[i] > 1)
        for (int64_t r = 0; r < q_len[i]; r += tiles * tokens_per_tile) {
          const int64_t last = std::min<int64_t>(q_len[i], r + tiles * tokens_per_tile) - 1;
          items += ceil_div((ctx_len[i] + last) / bk + 1, kScorePass);
        }
    return items;
  };
  int64_t tiles = kMaxScoreTiles;
  while (tiles > 1 && groups > 0 && chunk_items(tiles) * hkv < kFillGroups / 2) tiles /= 2;
  const int64_t passes = std::max<int64_t>(1, single_passes * hkv / (2 * kFillGroups));
  // nothing is built that would not fit
  const int64_t max_scores = (groups > 0 ? chunk_items(tiles) : 0) + single_passes;
  const int64_t off_rows = round_up(
      (int64_t)sizeof(SparseHeader) + (int64_t)sizeof(SparseReq) * n, sizeof(SparseRows));
  const int64_t off_scores =
      round_up(off_rows + (groups + singles) * (int64_t)sizeof(SparseRows), sizeof(SparseScore));
  if (off_scores + max_scores * (int64_t)sizeof(SparseScore) > INT32_MAX) return SSA_ERR_LENGTH;

  int64_t row = 0;
  p->groups.reserve(groups);
  p->singles.reserve(singles);
  for (int32_t i = 0; i < n; ++i) {
    const int32_t c = q_len[i], u = ctx_len[i];
    if (c == 0) continue;
    const int32_t step = c == 1 ? 1 : (int32_t)(tiles * tokens_per_tile);
    const int64_t blocks = c == 1 ? passes * kScorePass : kScorePass;
    for (int32_t r = 0; r < c; r += step) {
      const int32_t rows = std::min(step, c - r);
      const int64_t last = ((int64_t)u + r + rows - 1) / bk + 1;
      for (int64_t b = 0; b < last; b += blocks)
        p->scores.push_back({i, (int32_t)row + r, u + r, rows, (int32_t)b,
                             (int32_t)std::min(last, b + blocks), 0, 0});
    }
    if (c == 1)
      p->singles.push_back({i, (int32_t)row, u, 1});
    else
      for (int32_t r = 0; r < c; r += kRowGroup)
        p->groups.push_back({i, (int32_t)row + r, u + r, std::min(kRowGroup, c - r)});
    row += c;
  }

  SparseHeader& h = p->hdr;
  std::memset(&h, 0, sizeof h);
  // The lists are cut only where the workgroups are too few for the compute units, so that
  // the tickets of cut lists always fit.
  const int64_t units = (int64_t)p->groups.size() * sparse_subs(g) + (int64_t)p->singles.size();
  const int64_t lists = units * hkv;
  int64_t entries = top;
  if (lists > 0 && lists < kAttentionGroups)
    entries = std::min(top, std::max(std::max(ceil_div(kPieceKeys, bk), ceil_div(top, kMaxSplits)),
                                     ceil_div(top * lists, kAttentionGroups)));
  h.split_entries = (int32_t)entries;
  h.nsplit = (int32_t)ceil_div(top, entries);
  h.magic = kSparseMagic;
  h.block_keys = cfg->block_keys;
  h.num_reqs = n;
  h.num_tokens = (int32_t)tokens;
  h.hq = s->num_q_heads;
  h.hkv = hkv;
  h.head_dim = d;
  h.page_size = s->page_size;
  h.max_pages_per_req = s->max_pages_per_req;
  h.num_pages = s->num_pages;
  h.softmax_scale = s->softmax_scale;
  h.top = cfg->top_blocks;
  h.sink = cfg->sink_blocks;
  h.recent = cfg->recent_blocks;
  h.most_blocks = (int32_t)most;
  h.max_blocks = (int32_t)std::max<int64_t>(4, round_up(most, 4));
  h.num_groups = (int32_t)p->groups.size();
  h.num_singles = (int32_t)p->singles.size();
  h.num_scores = (int32_t)p->scores.size();
  h.off_rows = (int32_t)off_rows;
  h.off_scores = (int32_t)off_scores;
  h.score_tiles = (int32_t)tiles;
  h.plan_bytes = off_scores + (int64_t)p->scores.size() * (int64_t)sizeof(SparseScore);
  // 16 rows of scores are within a 32-bit byte offset
  if ((int64_t)hkv * h.max_blocks > kMaxScoreRow) return SSA_ERR_LENGTH;
  // workgroups of a launch
  const int64_t rows = (int64_t)h.num_groups * kRowGroup + h.num_singles;
  if ((int64_t)h.num_scores * hkv > INT32_MAX ||
      std::max(rows * hkv, lists * h.nsplit) > INT32_MAX)
    return SSA_ERR_LENGTH;
  h.ws_bytes = kSparseTickets * 4;
  if (h.nsplit > 1)
    h.ws_bytes += lists * h.nsplit * (int64_t)sparse_rec_floats(sparse_tokens(g) * g, d) * 4;
  uint64_t hv = 1469598103934665603ull;
  const int32_t f[10] = {s->num_q_heads,         s->num_kv_heads, s->head_dim,     s->page_size,
                         s->num_pages,           s->max_pages_per_req, cfg->block_keys,
                         cfg->top_blocks,        cfg->sink_blocks, cfg->recent_blocks};
  hv = fnv1a(hv, f, sizeof f);
  hv = fnv1a(hv, &s->softmax_scale, sizeof(float));
  if (n > 0) {
    hv = fnv1a(hv, q_len, sizeof(int32_t) * n);
    hv = fnv1a(hv, ctx_len, sizeof(int32_t) * n);
  }
  // how the work is cut is this planner's own
  const int64_t cut[4] = {h.num_scores, h.score_tiles, h.nsplit, h.ws_bytes};
  h.hash = fnv1a(hv, cut, sizeof cut);
  return SSA_OK;
}

}  // namespace

// Check that plan_host is a plan of its kind for this shape; used by the launchers.
int check_sparse_plan(const ssa_shape* s, const void* plan_host, const SparseHeader** out) {
  const int rc = validate_shape(s);
  if (rc) return rc;
  if (!plan_host) return SSA_ERR_NULL;
  const SparseHeader* h = static_cast<const SparseHeader*>(plan_host);
  if (h->magic != kSparseMagic || h->hq != s->num_q_heads || h->hkv != s->num_kv_heads ||
      h->head_dim != s->head_dim || h->page_size != s->page_size ||
      h->num_pages != s->num_pages || h->max_pages_per_req != s->max_pages_per_req ||
      std::memcmp(&h->softmax_scale, &s->softmax_scale, sizeof(float)) != 0)
    return SSA_ERR_PLAN_MISMATCH;
  *out = h;
  return SSA_OK;
}

}  // namespace ssa

extern "C" {

int ssa_sparse_plan_size(const ssa_shape* shape, const ssa_sparse_config* config,
                         const int32_t* q_len_host, const int32_t* ctx_len_host, int32_t num_reqs,
                         size_t* plan_bytes, size_t* ws_bytes, int32_t* max_blocks) {
  if (!plan_bytes || !ws_bytes || !max_blocks) return SSA_ERR_NULL;
  try {
    ssa::SparsePlan p;
    const int rc = ssa::build(shape, config, q_len_host, ctx_len_host, num_reqs, &p);
    if (rc) return rc;
    *plan_bytes = (size_t)p.hdr.plan_bytes;
    *ws_bytes = (size_t)p.hdr.ws_bytes;
    *max_blocks = p.hdr.max_blocks;
    return SSA_OK;
  } catch (const std::bad_alloc&) {
    return SSA_ERR_LENGTH;
  }
}

int ssa_sparse_plan(const ssa_shape* shape, const ssa_sparse_config* config,
                    const int32_t* q_len_host, const int32_t* ctx_len_host, int32_t num_reqs,
                    void* plan_host, size_t plan_bytes) {
  if (!plan_host) return SSA_ERR_NULL;
  try {
    ssa::SparsePlan p;
    const int rc = ssa::build(shape, config, q_len_host, ctx_len_host, num_reqs, &p);
    if (rc) return rc;
    if (plan_bytes < (size_t)p.hdr.plan_bytes) return SSA_ERR_PLAN_SIZE;
    char* b = static_cast<char*>(plan_host);
    std::memset(b, 0, (size_t)p.hdr.plan_bytes);
    std::memcpy(b, &p.hdr, sizeof p.hdr);
    for (int32_t i = 0; i < num_reqs; ++i) {
      const ssa::SparseReq r = {q_len_host[i], ctx_len_host[i]};
      std::memcpy(b + sizeof p.hdr + sizeof r * (size_t)i, &r, sizeof r);
    }
    char* rows = b + p.hdr.off_rows;
    if (!p.groups.empty())
      std::memcpy(rows, p.groups.data(), sizeof(ssa::SparseRows) * p.groups.size());
    if (!p.singles.empty())
      std::memcpy(rows + sizeof(ssa::SparseRows) * p.groups.size(), p.singles.data(),
                  sizeof(ssa::SparseRows) * p.singles.size());
    if (!p.scores.empty())
      std::memcpy(b + p.hdr.off_scores, p.scores.data(),
                  sizeof(ssa::SparseScore) * p.scores.size());
    return SSA_OK;
  } catch (const std::bad_alloc&) {
    return SSA_ERR_LENGTH;
  }
}

}  // extern "C"
