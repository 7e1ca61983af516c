// Host side of include/ssa_evict.h: argument checks, the score plan and the
// eviction plan.  Pure host code (no HIP call), so it is testable without a GPU.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "../../include/ssa_evict.h"
#include "ssa_evict_format.h"

namespace ssa {

int validate_shape(const ssa_shape* s);

namespace {

constexpr int64_t kMaxLen = 1 << 30;
// Workgroups that the decode rows are cut into, at least: four on each of 256 compute
// units.
constexpr int64_t kFillGroups = 1024;
// Records of all lists: the blob's size stays within its 32-bit offsets.
constexpr int64_t kMaxScoreItems = (INT32_MAX - 4096) / (int64_t)sizeof(ScoreItem);
// A token's queries: 32-bit byte offsets within a few rows of them.
constexpr int64_t kMaxQueryRow = 1 << 24;
// A decode row's key range is cut into pieces of a multiple of 128 keys (one
// 32-key block for each of four waves), at most kDecodeMaxKeys: a piece costs a
// record of G (D + 2) floats, and long ones leave compute units idle at the end (32
// rows of 8k to 33k keys, 64/8 heads: 596 us in pieces of 2048, 585 of 1024, 592 of
// 512).
constexpr int64_t kDecodeStepKeys = 128;
constexpr int64_t kDecodeMaxKeys = 1024;
// A piece of a chunk column tile's key range, at least, and pieces of one, at most.
constexpr int64_t kLseMinKeys = 256;
constexpr int64_t kMaxPieces = 64;
// The chunk passes' estimate, in 32-row tiles: starting an item of the first and of the
// second pass, and a compute unit with one workgroup.  (Of 2, 3, 5 and 8 for the second,
// 5 chose best: 31, 28, 27 and 28 us of a mixed batch, 105, 106, 104 and 116 of four
// chunks.)
constexpr int64_t kCus = 256;
constexpr double kItemTiles = 3;
constexpr double kSumItemTiles = 5;
constexpr double kAlone = 1.2;
constexpr double kGroupCost[3] = {1.3, 1.15, 1.0};  // a tile's, in 1, 2 and 4 column groups

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

uint64_t hash_shape(const ssa_shape* s, const int32_t* more, int n_more) {
  uint64_t h = 1469598103934665603ull;
  const int32_t f[6] = {s->num_q_heads, s->num_kv_heads,     s->head_dim,
                        s->page_size,   s->num_pages,        s->max_pages_per_req};
  h = fnv1a(h, f, sizeof f);
  h = fnv1a(h, &s->softmax_scale, sizeof(float));
  return fnv1a(h, more, sizeof(int32_t) * n_more);
}

struct ScorePlan {
  ScoreHeader hdr;
  std::vector<ScoreReq> reqs;
  std::vector<ScoreItem> list[kNumScoreLists];
};

int build_score(const ssa_shape* s, const int32_t* q_len, const int32_t* ctx_len, int32_t n,
                int32_t last_rows, ScorePlan* p) {
  const int rc = validate_shape(s);
  if (rc) return rc;
  if (n < 0) return SSA_ERR_LENGTH;
  if (n > 0 && (!q_len || !ctx_len)) return SSA_ERR_NULL;
  if (last_rows < 0) return SSA_ERR_ARG;
  const int hkv = s->num_kv_heads, g = s->num_q_heads / hkv, d = s->head_dim;
  if ((int64_t)s->num_q_heads * d > kMaxQueryRow) return SSA_ERR_SHAPE;
  int64_t tokens = 0, keys = 0, decode_keys = 0, decode_rows = 0, max_q = 0;
  struct Chunk {
    int64_t cols, span;
  };
  std::vector<Chunk> chunks;
  for (int32_t i = 0; i < n; ++i) {
    const int64_t c = q_len[i], u = ctx_len[i];
    if (c < 0 || u < 0) return SSA_ERR_LENGTH;
    tokens += c;
    keys += c + u;
    if (tokens > kMaxLen || keys > kMaxLen) return SSA_ERR_LENGTH;
    if (ceil_div(c + u, SSA_PAGE_SIZE) > s->max_pages_per_req) return SSA_ERR_PAGES;
    if (c == 0) continue;
    max_q = std::max(max_q, c);
    const int64_t r = last_rows ? std::min<int64_t>(c, last_rows) : c;
    if (r * g > kMaxScoreCols) return SSA_ERR_LENGTH;
    if (r == 1) {
      decode_keys += c + u;
      ++decode_rows;
    } else
      chunks.push_back({r * g, c + u});
  }
  ScoreHeader& h = p->hdr;
  std::memset(&h, 0, sizeof h);

  // The first chunk pass's column groups and pieces of the key ranges.  Waves side by
  // side (column groups) share the keys that go through LDS, waves one behind the other
  // take different ones: four groups read LDS and cache least (kGroupCost), fewer fill
  // narrow requests better and are done sooner where there are few workgroups.  Both
  // are cut for the shortest estimate: the workgroups of the busiest compute unit times
  // their 32-row tiles, kItemTiles for starting one, and kAlone more where there are not
  // two to a unit to fill each other's waits.  (200 rows on 200 to 4000 keys, 8/8 heads of
  // 64: 18 to 21 us with the groups that pad the fewest columns, 15 to 19 so; 32 rows on
  // 200 keys, 64/8 of 128: 19 and 15.)
  auto estimate = [&](int64_t wgs, double tiles) {
    const int64_t per_cu = std::max<int64_t>(1, ceil_div(wgs, kCus));
    return (double)per_cu * (tiles + kItemTiles) * (per_cu == 1 ? kAlone : 1.0);
  };
  int64_t longest = 0, widest = 0;
  for (const Chunk& c : chunks) {
    longest = std::max(longest, c.span);
    widest = std::max(widest, c.cols);
  }
  int lse_k = 2;
  int64_t piece = 0;
  double best = 0;
  for (int k = 2; k >= 0 && !chunks.empty(); --k)
    for (int64_t n = 1; n <= kMaxPieces; ++n) {
      const int64_t p = std::max(kLseMinKeys, round_up(ceil_div(longest, n), 128));
      int64_t wgs = 0;
      double tiles = 0;
      for (const Chunk& c : chunks) {
        const int64_t w = ceil_div(c.cols, (int64_t)kScoreWaveCols << k) * ceil_div(c.span, p) * hkv;
        wgs += w;
        tiles += (double)w * std::min(p, c.span) / (32 * (4 >> k));
      }
      const double cost = estimate(wgs, tiles / wgs * kGroupCost[k]);
      if (best == 0 || cost < best) {
        best = cost;
        piece = p;
        lse_k = k;
      }
      if (p == kLseMinKeys) break;
    }
  const int64_t lse_cols = (int64_t)kScoreWaveCols << lse_k;
  // The second pass: 256 keys stay in registers, columns go through LDS.  Its column
  // ranges, by the same estimate over tiles of equal length and one item's time for
  // the end.
  int64_t sum_cols = 32;
  best = 0;
  for (int64_t n = 1; n <= kMaxPieces && !chunks.empty(); ++n) {
    const int64_t p = round_up(ceil_div(widest, n), 32);
    double wgs = 0, tiles = 0;
    for (const Chunk& c : chunks) {
      const double k = (double)ceil_div(c.span, kSumKeys) * hkv;
      wgs += k * ceil_div(c.cols, p);
      tiles += k * c.cols / 32;
    }
    const double cost = std::max(1.0, std::ceil(wgs / kCus) * kCus / wgs) * (tiles + wgs * kSumItemTiles) / kCus +
                        p / 32 + kSumItemTiles;
    if (best == 0 || cost < best) {
      best = cost;
      sum_cols = p;
    }
  }
  h.lse_groups = 1 << lse_k;
  h.sum_cols = (int32_t)sum_cols;
  // nothing is built that would not fit
  int64_t records = ceil_div(decode_keys, kDecodeStepKeys) * 2 + 2 * decode_rows;
  for (const Chunk& c : chunks) {
    const int64_t pieces = ceil_div(c.span, piece), tiles = ceil_div(c.span, kSumKeys);
    records += ceil_div(c.cols, lse_cols) * pieces + ceil_div(c.cols, kScoreThreads) + 1 +
               tiles * ceil_div(c.cols, sum_cols);
    if (records > kMaxScoreItems) return SSA_ERR_LENGTH;
  }
  const int64_t decode_piece =
      std::min(std::min(kDecodeMaxKeys, kWholeLogits / g / kDecodeStepKeys * kDecodeStepKeys),
               std::max(kDecodeStepKeys,
                        round_up(ceil_div(decode_keys * hkv, kFillGroups), kDecodeStepKeys)));

  // Rows that one workgroup does, at once and without a second launch: as long as its
  // LDS holds the logits where there are enough rows for every compute unit, shorter
  // ones where there are not.  Attention and scores in us, in pieces and whole (heads
  // of 128, 32/8): 128 rows of 2048 keys 245 and 206, of 256 42 and 39; 8 rows of 2048 35
  // and 33, of 512 25 and 17; 1 row of 2048 20 and 26, of 1024 16.5 and 16.9, of 512 15 and
  // 12.  (8/8 heads of 64: 8 rows of 4096 32 and 38, 32 of 4096 60 and 57.)
  // Beside chunk rows, which have a second launch anyway, only short ones (64 decodes
  // of 512 to 4096 keys and a chunk: 98 us with rows of 2048 whole, 92 in pieces).
  const int64_t decode_groups = decode_rows * hkv;
  const int64_t whole_keys = std::min<int64_t>(
      kWholeLogits / g, !chunks.empty()              ? 512
                        : decode_groups >= kCus      ? kWholeLogits
                        : decode_groups >= kCus / 4  ? 2048
                                                     : 1024);

  int64_t ws = 0, row = 0;  // floats; token row
  std::vector<ScoreItem> sums;  // a chunk request's fields each
  auto take = [&](int64_t floats) {
    const int64_t at = ws;
    ws += round_up(floats, 64);
    return at;
  };
  for (int32_t i = 0; i < n; ++i) {
    const int64_t c = q_len[i], u = ctx_len[i], len = c + u;
    if (c == 0) continue;
    const int64_t r = last_rows ? std::min<int64_t>(c, last_rows) : c;
    ScoreItem it{};
    it.req = i;
    it.q_row = (int32_t)(row + c - r);
    it.rows = (int32_t)r;
    it.len = (int32_t)len;
    it.ctx_len = (int32_t)u;
    row += c;
    if (r == 1) {
      const int64_t padded = round_up(len, 32);
      it.cols_pad = (int32_t)padded;
      if (padded <= whole_keys) {
        it.nsplit = 1;
        it.split = -1;
        it.key1 = it.len;
        p->list[kListDecode].push_back(it);
        continue;
      }
      it.nsplit = (int32_t)ceil_div(len, decode_piece);
      it.off0 = take(padded * g * hkv);
      it.off1 = take((int64_t)hkv * it.nsplit * score_rec_floats(g, d));
      for (int32_t k = 0; k < it.nsplit; ++k) {
        ScoreItem x = it;
        x.split = k;
        x.key0 = (int32_t)(k * decode_piece);
        x.key1 = (int32_t)std::min(len, (k + 1) * decode_piece);
        p->list[kListDecode].push_back(x);
      }
      for (int64_t k = 0; k < len; k += kJoinKeys) {
        ScoreItem x = it;
        x.key0 = (int32_t)k;
        x.key1 = (int32_t)std::min(len, k + kJoinKeys);
        p->list[kListDecodeJoin].push_back(x);
      }
      continue;
    }
    const int64_t cols = r * g, padded = round_up(cols, kColsPad);
    it.cols_pad = (int32_t)padded;
    it.nsplit = (int32_t)ceil_div(len, piece);
    it.off0 = take(padded * hkv * 2);
    it.off1 = it.nsplit > 1 ? take(padded * hkv * it.nsplit * 2) : 0;
    for (int64_t col = 0; col < cols; col += lse_cols)
      for (int32_t k = 0; k < it.nsplit; ++k) {
        ScoreItem x = it;
        x.col0 = (int32_t)col;
        x.split = k;
        x.key0 = (int32_t)(k * piece);
        x.key1 = (int32_t)std::min(len, (k + 1) * piece);
        p->list[kListLse].push_back(x);
      }
    if (it.nsplit > 1)
      for (int64_t col = 0; col < padded; col += kScoreThreads) {
        ScoreItem x = it;
        x.col0 = (int32_t)col;
        p->list[kListLseJoin].push_back(x);
      }
    sums.push_back(it);
  }
  std::stable_sort(sums.begin(), sums.end(),
                   [](const ScoreItem& a, const ScoreItem& b) { return a.rows > b.rows; });
  int64_t tickets = 0;
  for (const ScoreItem& it : sums) {
    // tiles from the first key on (the most rows see those), each column range that
    // sees some of the tile
    const int64_t cols = (int64_t)it.rows * g, pieces = ceil_div(cols, sum_cols);
    const int64_t off = pieces > 1 ? take(pieces * hkv * round_up(it.len, kSumKeys)) : 0;
    for (int64_t k = 0; k < it.len; k += kSumKeys) {
      const int64_t first = std::max<int64_t>(0, k - (it.len - it.rows)) * g / sum_cols;
      for (int64_t c = first; c < pieces; ++c) {
        ScoreItem x = it;
        x.key0 = (int32_t)k;
        x.key1 = (int32_t)std::min<int64_t>(it.len, k + kSumKeys);
        x.col0 = (int32_t)(c * sum_cols);
        x.split = (int32_t)(c - first);
        x.nsplit = (int32_t)(pieces - first);
        x.off1 = off;
        if (x.nsplit > 1) x.ticket = (int32_t)tickets;
        p->list[kListSum].push_back(x);
      }
      if (pieces - first > 1) tickets += hkv;
      if (tickets > INT32_MAX / 4) return SSA_ERR_LENGTH;
    }
  }
  h.num_tickets = (int32_t)tickets;
  // the tickets come first in the workspace
  const int64_t shift = round_up(tickets, 64);
  ws += shift;
  for (auto& l : p->list)
    for (ScoreItem& x : l) {
      x.off0 += shift;
      x.off1 += shift;
    }
  h.magic = kScoreMagic;
  h.last_rows = last_rows;
  h.num_reqs = n;
  h.num_tokens = (int32_t)tokens;
  h.hq = s->num_q_heads;
  h.hkv = hkv;
  h.head_dim = d;
  h.page_size = s->page_size;
  h.max_pages_per_req = s->max_pages_per_req;
  h.num_pages = s->num_pages;
  h.softmax_scale = s->softmax_scale;
  h.max_q_len = (int32_t)max_q;
  const int64_t off_items =
      round_up((int64_t)sizeof(ScoreHeader) + (int64_t)sizeof(ScoreReq) * n, sizeof(ScoreItem));
  int64_t items = 0;
  for (int l = 0; l < kNumScoreLists; ++l) {
    const int64_t count = (int64_t)p->list[l].size();
    if ((items + count) * hkv > INT32_MAX) return SSA_ERR_LENGTH;  // workgroups of a launch
    h.first[l] = (int32_t)items;
    h.count[l] = (int32_t)count;
    items += count;
  }
  h.plan_bytes = off_items + items * (int64_t)sizeof(ScoreItem);
  if (h.plan_bytes > INT32_MAX) return SSA_ERR_LENGTH;
  h.off_items = (int32_t)off_items;
  p->reqs.reserve(n);
  for (int32_t i = 0; i < n; ++i) p->reqs.push_back({q_len[i], ctx_len[i]});
  h.ws_bytes = std::max<int64_t>(256, ws * 4);
  uint64_t hv = hash_shape(s, &last_rows, 1);
  if (n > 0) {
    hv = fnv1a(hv, q_len, sizeof(int32_t) * n);
    hv = fnv1a(hv, ctx_len, sizeof(int32_t) * n);
  }
  // how the lists are cut is this planner's own
  const int64_t cut[4] = {items, h.ws_bytes, h.lse_groups, h.sum_cols};
  h.hash = fnv1a(hv, cut, sizeof cut);
  return SSA_OK;
}

struct EvictPlan {
  EvictHeader hdr;
  std::vector<EvictReq> reqs;
  std::vector<EvictShort> shorts;
  std::vector<EvictSeg> segs;
  std::vector<EvictItem> items;
};

int build_evict(const ssa_shape* s, const int32_t* kv_len, const int32_t* budget, int32_t n,
                int32_t sink, int32_t recent, EvictPlan* p) {
  const int rc = validate_shape(s);
  if (rc) return rc;
  if (n < 0) return SSA_ERR_LENGTH;
  if (n > 0 && (!kv_len || !budget)) return SSA_ERR_NULL;
  if (sink < 0 || recent < 0) return SSA_ERR_ARG;
  EvictHeader& h = p->hdr;
  std::memset(&h, 0, sizeof h);
  int64_t keys = 0, keep = 0, cands = 0;
  for (int32_t i = 0; i < n; ++i) {
    const int64_t len = kv_len[i], kept = std::min(kv_len[i], budget[i]);
    if (len < 0 || budget[i] < 0) return SSA_ERR_LENGTH;
    keys += len;
    if (keys > kMaxLen) return SSA_ERR_LENGTH;
    if (ceil_div(len, SSA_PAGE_SIZE) > s->max_pages_per_req) return SSA_ERR_PAGES;
    if (kept < len && (int64_t)sink + recent > kept) return SSA_ERR_ARG;
    p->reqs.push_back({(int32_t)len, (int32_t)kept, keep});
    if (kept > 0 && (len <= kShortList || kept == len)) {
      p->shorts.push_back({i, (int32_t)len, (int32_t)kept, 0, keep});
    } else if (kept > 0) {
      const int32_t seg0 = (int32_t)p->segs.size();
      for (int64_t k = 0; k < len; k += kSegKeys)
        p->segs.push_back({i, (int32_t)len, (int32_t)kept, (int32_t)k, seg0, h.num_long, keep, cands});
      ++h.num_long;
      cands += len;
    }
    if (kept < len)
      for (int64_t k = 0; k < kept; k += kEvictSlots)
        p->items.push_back({i, (int32_t)k, (int32_t)std::min<int64_t>(kEvictSlots, kept - k),
                            (int32_t)len, (int32_t)kept, 0, keep});
    keep += kept;
  }
  h.magic = kEvictMagic;
  h.sink = sink;
  h.recent = recent;
  h.num_reqs = n;
  h.hq = s->num_q_heads;
  h.hkv = s->num_kv_heads;
  h.head_dim = s->head_dim;
  h.page_size = s->page_size;
  h.max_pages_per_req = s->max_pages_per_req;
  h.num_pages = s->num_pages;
  h.softmax_scale = s->softmax_scale;
  h.num_keep = keep;
  const int64_t items = (int64_t)p->items.size(), shorts = (int64_t)p->shorts.size(),
                segs = (int64_t)p->segs.size();
  const int64_t off_short = sizeof(EvictHeader) + (int64_t)sizeof(EvictReq) * n;
  const int64_t off_segs = off_short + (int64_t)sizeof(EvictShort) * shorts;
  const int64_t off_items = off_segs + (int64_t)sizeof(EvictSeg) * segs;
  h.plan_bytes = off_items + items * (int64_t)sizeof(EvictItem);
  if (h.plan_bytes > INT32_MAX || (items + segs + shorts) * h.hkv > INT32_MAX)
    return SSA_ERR_LENGTH;
  h.num_items = (int32_t)items;
  h.num_short = (int32_t)shorts;
  h.num_segs = (int32_t)segs;
  h.off_short = (int32_t)off_short;
  h.off_segs = (int32_t)off_segs;
  h.off_items = (int32_t)off_items;
  const int64_t lists = (int64_t)h.num_long * h.hkv;
  h.ws_counts = lists * (kSegBins * 4 + (int64_t)sizeof(SegState));
  h.ws_cands = round_up(h.ws_counts + segs * h.hkv * 4, 256);
  h.ws_bytes = std::max<int64_t>(256, h.ws_cands + cands * h.hkv * 8);
  const int32_t more[2] = {sink, recent};
  uint64_t hv = hash_shape(s, more, 2);
  if (n > 0) {
    hv = fnv1a(hv, kv_len, sizeof(int32_t) * n);
    hv = fnv1a(hv, budget, sizeof(int32_t) * n);
  }
  const int64_t cut[3] = {items, segs, h.ws_bytes};
  h.hash = fnv1a(hv, cut, sizeof cut);
  return SSA_OK;
}

template <class H>
int check_header(const ssa_shape* s, const void* plan_host, uint32_t magic, const H** out) {
  const int rc = validate_shape(s);
  if (rc) return rc;
  if (!plan_host) return SSA_ERR_NULL;
  const H* h = static_cast<const H*>(plan_host);
  if (h->magic != magic || h->hq != s->num_q_heads || h->hkv != s->num_kv_heads ||
      h->head_dim != s->head_dim || h->page_size != s->page_size ||
      h->num_pages != s->num_pages || h->max_pages_per_req != s->max_pages_per_req ||
      std::memcmp(&h->softmax_scale, &s->softmax_scale, sizeof(float)) != 0)
    return SSA_ERR_PLAN_MISMATCH;
  *out = h;
  return SSA_OK;
}

}  // namespace

// Check that plan_host is a plan of its kind for this shape; used by the launchers.
int check_score_plan(const ssa_shape* s, const void* plan_host, const ScoreHeader** out) {
  return check_header(s, plan_host, kScoreMagic, out);
}
int check_evict_plan(const ssa_shape* s, const void* plan_host, const EvictHeader** out) {
  return check_header(s, plan_host, kEvictMagic, out);
}

}  // namespace ssa

extern "C" {

int ssa_score_plan_size(const ssa_shape* shape, const int32_t* q_len_host,
                        const int32_t* ctx_len_host, int32_t num_reqs, int32_t last_rows,
                        size_t* plan_bytes, size_t* ws_bytes) {
  if (!plan_bytes || !ws_bytes) return SSA_ERR_NULL;
  try {
    ssa::ScorePlan p;
    const int rc = ssa::build_score(shape, q_len_host, ctx_len_host, num_reqs, last_rows, &p);
    if (rc) return rc;
    *plan_bytes = (size_t)p.hdr.plan_bytes;
    *ws_bytes = (size_t)p.hdr.ws_bytes;
    return SSA_OK;
  } catch (const std::bad_alloc&) {
    return SSA_ERR_LENGTH;
  }
}

int ssa_score_plan(const ssa_shape* shape, const int32_t* q_len_host, const int32_t* ctx_len_host,
                   int32_t num_reqs, int32_t last_rows, void* plan_host, size_t plan_bytes) {
  if (!plan_host) return SSA_ERR_NULL;
  try {
    ssa::ScorePlan p;
    const int rc = ssa::build_score(shape, q_len_host, ctx_len_host, num_reqs, last_rows, &p);
    if (rc) return rc;
    if (plan_bytes < (size_t)p.hdr.plan_bytes) return SSA_ERR_PLAN_SIZE;
    char* b = static_cast<char*>(plan_host);
    std::memcpy(b, &p.hdr, sizeof p.hdr);
    std::memset(b + sizeof p.hdr, 0, p.hdr.off_items - sizeof p.hdr);
    if (!p.reqs.empty())
      std::memcpy(b + sizeof p.hdr, p.reqs.data(), sizeof(ssa::ScoreReq) * p.reqs.size());
    char* at = b + p.hdr.off_items;
    for (const auto& l : p.list) {
      if (!l.empty()) std::memcpy(at, l.data(), sizeof(ssa::ScoreItem) * l.size());
      at += sizeof(ssa::ScoreItem) * l.size();
    }
    return SSA_OK;
  } catch (const std::bad_alloc&) {
    return SSA_ERR_LENGTH;
  }
}

int ssa_evict_plan_size(const ssa_shape* shape, const int32_t* kv_len_host,
                        const int32_t* budget_host, int32_t num_reqs, int32_t sink,
                        int32_t recent, size_t* plan_bytes, size_t* ws_bytes) {
  if (!plan_bytes || !ws_bytes) return SSA_ERR_NULL;
  try {
    ssa::EvictPlan p;
    const int rc = ssa::build_evict(shape, kv_len_host, budget_host, num_reqs, sink, recent, &p);
    if (rc) return rc;
    *plan_bytes = (size_t)p.hdr.plan_bytes;
    *ws_bytes = (size_t)p.hdr.ws_bytes;
    return SSA_OK;
  } catch (const std::bad_alloc&) {
    return SSA_ERR_LENGTH;
  }
}

int ssa_evict_plan(const ssa_shape* shape, const int32_t* kv_len_host, const int32_t* budget_host,
                   int32_t num_reqs, int32_t sink, int32_t recent, void* plan_host,
                   size_t plan_bytes) {
  if (!plan_host) return SSA_ERR_NULL;
  try {
    ssa::EvictPlan p;
    const int rc = ssa::build_evict(shape, kv_len_host, budget_host, num_reqs, sink, recent, &p);
    if (rc) return rc;
    if (plan_bytes < (size_t)p.hdr.plan_bytes) return SSA_ERR_PLAN_SIZE;
    char* b = static_cast<char*>(plan_host);
    std::memcpy(b, &p.hdr, sizeof p.hdr);
    if (!p.reqs.empty())
      std::memcpy(b + sizeof p.hdr, p.reqs.data(), sizeof(ssa::EvictReq) * p.reqs.size());
    if (!p.shorts.empty())
      std::memcpy(b + p.hdr.off_short, p.shorts.data(), sizeof(ssa::EvictShort) * p.shorts.size());
    if (!p.segs.empty())
      std::memcpy(b + p.hdr.off_segs, p.segs.data(), sizeof(ssa::EvictSeg) * p.segs.size());
    if (!p.items.empty())
      std::memcpy(b + p.hdr.off_items, p.items.data(), sizeof(ssa::EvictItem) * p.items.size());
    return SSA_OK;
  } catch (const std::bad_alloc&) {
    return SSA_ERR_LENGTH;
  }
}

int ssa_check_evict_tables(const ssa_shape* shape, const void* plan_host,
                           const int32_t* block_table_host, const int32_t* new_table_host) {
  const ssa::EvictHeader* h = nullptr;
  const int rc = ssa::check_evict_plan(shape, plan_host, &h);
  if (rc) return rc;
  if (h->num_reqs > 0 && !block_table_host) return SSA_ERR_NULL;
  const ssa::EvictReq* reqs = reinterpret_cast<const ssa::EvictReq*>(
      static_cast<const char*>(plan_host) + sizeof(ssa::EvictHeader));
  try {
    std::vector<bool> taken((size_t)h->num_pages, false);
    for (int32_t i = 0; i < h->num_reqs; ++i) {
      const int32_t* row = block_table_host + (size_t)i * h->max_pages_per_req;
      for (int64_t k = 0; k < ssa::ceil_div(reqs[i].len, SSA_PAGE_SIZE); ++k) {
        if (row[k] < 0 || row[k] >= h->num_pages) return SSA_ERR_PAGES;
        taken[row[k]] = true;
      }
    }
    for (int32_t i = 0; new_table_host && i < h->num_reqs; ++i) {
      if (reqs[i].kept == reqs[i].len) continue;
      const int32_t* row = new_table_host + (size_t)i * h->max_pages_per_req;
      for (int64_t k = 0; k < ssa::ceil_div(reqs[i].kept, SSA_PAGE_SIZE); ++k) {
        if (row[k] < 0 || row[k] >= h->num_pages || taken[row[k]]) return SSA_ERR_PAGES;
        taken[row[k]] = true;
      }
    }
    return SSA_OK;
  } catch (const std::bad_alloc&) {
    return SSA_ERR_LENGTH;
  }
}

}  // extern "C"
