// HIP kernels for gfx950 of include/ssa_sparse.h: block summaries, their scores, the
// selection, attention over the selected blocks.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>
#include <initializer_list>
#include <type_traits>

#include "../../include/ssa_sparse.h"
#include "ssa_device.h"
#include "ssa_layer_internal.h"
#include "ssa_plan_format.h"
#include "ssa_sparse_format.h"

namespace ssa {
int check_plan(const ssa_shape* s, const void* plan_host, const PlanHeader** out);
}  // namespace ssa

namespace {
using namespace ssa;
using namespace ssa_dev;

constexpr float kInf = __builtin_huge_valf();
constexpr int kGridRow = 1 << 16;  // workgroups in a row of the grid (2^32 threads at most)

__device__ __forceinline__ int workgroup_id() {
  return (int)(blockIdx.y * gridDim.x + blockIdx.x);
}

// ---------------------------------------------------------------------------
// Summaries.  A wave takes one kv head of one block: 16 bytes of a key row a lane, the
// block's rows dealt to groups of D / 8 lanes, all loads before the first use.  bf16 values
// are compared as 16-bit integers (negative ones with their other bits inverted), two an
// instruction, so that the extremes are the keys' own bits.  Of the plan's append segments (a
// page of new tokens each) the first one in a block stands for it.  A chunk has one such in
// BLOCK / 16 of its segments: a wave looks at as many, so that every workgroup has work (with
// a workgroup a segment, those with work fell to two of the eight dies).  Memory bounds it:
// 33768 tokens of 8 heads in blocks of 64, 71 MB, take 15 us, 4.7 TB/s (29.5 so); the blocks of
// 64 decodes 4.1 us, three dependent loads and the launch.
struct SummaryArgs {
  const uint8_t* plan;
  uint64_t hash;
  int32_t off_segments, off_reqs;
  int32_t num_runs;  // runs of a block's pages among the chunks' segments
  int32_t num_chunk_segments;
  int32_t workgroups, head_groups;
  int32_t hkv, maxp, block_keys;
  const uint16_t* kc;
  const int32_t* bt;
  uint16_t* summary;
};

typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
// All ones in the halves of x whose sign is set.  (A function of its own: the cast of a
// vector's element in place reads its first one.)
__device__ __forceinline__ uint32_t negative_halves(uint32_t x) {
  return __builtin_bit_cast(uint32_t, __builtin_bit_cast(i16x2, x) >> 15);
}
// bf16 pairs to integers in the same order, and back.
__device__ __forceinline__ uint32_t ordered(uint32_t x) {
  return x ^ (negative_halves(x) & 0x7FFF7FFFu);
}
__device__ __forceinline__ uint32_t pair_max(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(i16x2, a),
                                                                __builtin_bit_cast(i16x2, b)));
}
__device__ __forceinline__ uint32_t pair_min(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_bit_cast(i16x2, a),
                                                                __builtin_bit_cast(i16x2, b)));
}

// Block of request `req` from position `first` on.
template <int D, int BLOCK>
__device__ __forceinline__ void summarise(const SummaryArgs& a, int req, int first, int len,
                                          int kvh, int lane) {
  constexpr int CPR = D / 8, ROWS = 64 / CPR;  // lanes a row, rows a load
  constexpr int LOADS = BLOCK / ROWS, PER_PAGE = 16 / ROWS;
  const auto row = as_uniform<int32_t>(a.bt + (size_t)req * a.maxp);
  // rows past the last key read that one again
  const int last = min(first + BLOCK, len) - 1;
  u32x4 k[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int page = row[min(first / 16 + i / PER_PAGE, last / 16)];
    const int t = min(first + i * ROWS + lane / CPR, last);
    k[i] = ld16(a.kc + (((size_t)page * a.hkv + kvh) * 16 + t % 16) * D + lane % CPR * 8);
  }
  u32x4 hi, lo;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    hi[w] = lo[w] = ordered(k[0][w]);
#pragma unroll
    for (int i = 1; i < LOADS; ++i) {
      const uint32_t x = ordered(k[i][w]);
      hi[w] = pair_max(hi[w], x);
      lo[w] = pair_min(lo[w], x);
    }
#pragma unroll
    for (int o = CPR; o < 64; o *= 2) {
      hi[w] = pair_max(hi[w], __shfl_xor(hi[w], o, 64));
      lo[w] = pair_min(lo[w], __shfl_xor(lo[w], o, 64));
    }
    hi[w] = ordered(hi[w]);
    lo[w] = ordered(lo[w]);
  }
  uint16_t* to = a.summary + ((size_t)row[first / 16] * a.hkv + kvh) * 2 * D + lane % CPR * 8;
  if (lane < CPR) st16(to, hi);
  else if (lane < 2 * CPR) st16(to + D, lo);
}

template <int D, int BLOCK>
__global__ __launch_bounds__(kSparseThreads) void block_summary_kernel(SummaryArgs a) {
  const int wg = workgroup_id();
  if (wg >= a.workgroups) return;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int kvh = wg % a.head_groups * 4 + wave;
  if (kvh >= a.hkv) return;
  const int unit = wg / a.head_groups;
  const auto h = as_uniform<PlanHeader>(a.plan);
  if (h->magic != kPlanMagic || h->hash != a.hash) return;
  int seg = a.num_chunk_segments + (unit - a.num_runs), end = seg + 1;
  if (unit < a.num_runs) {
    seg = unit * (BLOCK / 16);
    end = min(seg + BLOCK / 16, a.num_chunk_segments);
  }
  for (; seg < end; ++seg) {
    const auto sg = as_uniform<AppendSeg>(a.plan + a.off_segments) + seg;
    const int req = sg->req, pos0 = sg->pos0;
    const auto rq = as_uniform<ReqEntry>(a.plan + a.off_reqs) + req;
    if (pos0 % BLOCK == 0 || pos0 == rq->ctx_len)
      summarise<D, BLOCK>(a, req, pos0 / BLOCK * BLOCK, rq->ctx_len + rq->q_len, kvh, lane);
  }
}

// ---------------------------------------------------------------------------
// Launches with a sparse plan.
struct SparseArgs {
  const uint8_t* plan;
  uint64_t hash;
  int32_t workgroups;
  int32_t hq, hkv, g, maxp;
  int32_t num_groups, off_rows, off_scores;
  int32_t log_block;
  int32_t top, sink, recent, max_blocks;
  int32_t nsplit, split_entries;
  int32_t tokens, subs, g_magic;  // rows of an attention workgroup, workgroups of a record of rows
  float c;  // softmax_scale * log2(e)
  const uint16_t* q;
  const uint16_t* kc;
  const uint16_t* vc;
  const uint16_t* summary;
  const int32_t* bt;
  const float* scores_in;
  float* scores;
  const int32_t* blocks_in;
  int32_t* blocks;
  uint16_t* out;
  int32_t* tickets;
  float* records;
};

// Before any record is read: another plan may be a shorter one.  Both words are read before
// either is looked at.
__device__ __forceinline__ bool plan_ok(const SparseArgs& a) {
  const auto h = as_uniform<SparseHeader>(a.plan);
  return (h->magic == kSparseMagic) & (h->hash == a.hash);
}

// A record's fields in one load.  (Left alone, the row count is loaded, waited for and branched
// on before the rest.)
struct Rows {
  int req, row0, pos0, n;
  __device__ __forceinline__ Rows(const SparseArgs& a, int record) {
    const auto x = as_uniform<SparseRows>(a.plan + a.off_rows) + record;
    req = x->req, row0 = x->row0, pos0 = x->pos0, n = x->n;
    asm volatile("" ::"s"(req), "s"(row0), "s"(pos0), "s"(n));
  }
};

// One row: `unit` counts kRowGroup rows of every chunk record, then the single ones.
struct Row {
  int req, row, pos;
};
__device__ __forceinline__ bool take_row(const SparseArgs& a, int unit, Row* r) {
  const bool single = unit >= a.num_groups * kRowGroup;
  const int record = single ? a.num_groups + (unit - a.num_groups * kRowGroup) : unit / kRowGroup;
  const int j = single ? 0 : unit % kRowGroup;
  if (!plan_ok(a)) return false;
  const Rows x(a, record);
  r->req = x.req;
  r->row = x.row0 + j;
  r->pos = x.pos0 + j;
  return j < x.n;
}

// ---------------------------------------------------------------------------
// Scores.  [max(q, 0), min(q, 0)] times [high, low]: a matrix product over 2 D, exact in its
// bf16 factors.  A 16x16x32 product has (token, head) rows, the kv head's heads padded to a
// power of two with its last one, and 16 blocks as columns, so that a token's heads lie in
// the registers of a lane and, from eight on, in 2 or 4 lanes.  A wave keeps two tiles of
// blocks.  The queries of four tiles at a time go through LDS, split into their two parts, a
// tile by each wave, the next four on their way meanwhile: read and split by every wave for
// itself they bounded the kernel (512 rows on 32768 keys in blocks of 32, 32/8 heads: 33 us,
// 21 so).  A tile's last reads from LDS are the next one's, on their way while its sums are
// looked at, and which blocks a row sees is one comparison a store (with reads before each
// product and the rows' conditions apart 23.8 us beside 16 decodes, 21.5 so).  What is left
// there is the way to the first products, 6 us of plan, table and summaries, then queries, products
// and stores, none of which alone is half of it.  Every four tiles begin with a wait for all that
// is on its way, stores included: the loop over the tiles has a count that the compiler does not
// know, so it cannot tell the queries' loads from the stores behind them.  A decode's scores wait
// for memory (64 rows of 8000 to 30000 keys in blocks of 16: 273 MB in 48 us, 5.7 TB/s).
template <int D, int LOG_G>  // heads of a group: more than 2^(LOG_G - 1), up to 2^LOG_G
__global__ __launch_bounds__(kSparseThreads, 3) void block_scores_kernel(SparseArgs a) {
  constexpr int KS = D / 32, TOKENS = 16 >> LOG_G;  // tokens of a tile
  __shared__ u32x4 s_query[4][2 * KS][64];  // tile, part of the product, lane
  const int wg = workgroup_id();
  if (wg >= a.workgroups) return;
  const int kvh = wg % a.hkv;
  const auto it = as_uniform<SparseScore>(a.plan + a.off_scores) + wg / a.hkv;
  if (!plan_ok(a)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int r16 = lane & 15, quad = lane >> 4;
  const int token = r16 >> LOG_G, head = min(r16 & ((1 << LOG_G) - 1), a.g - 1);
  const int32_t* row = a.bt + (size_t)it->req * a.maxp;
  const int n = it->n, row0 = it->row0, pos0 = it->pos0, blk1 = it->blk1;
  const uint16_t* const queries = a.q + ((size_t)row0 * a.hq + kvh * a.g + head) * D + quad * 8;
  u32x4 ahead[KS];
  auto load_queries = [&](int j0) {  // rows past the last one read it again
    const uint16_t* from = queries + (size_t)min(j0 + wave * TOKENS + token, n - 1) * a.hq * D;
#pragma unroll
    for (int k = 0; k < KS; ++k) ahead[k] = ld16(from + k * 32);
  };
  for (int p0 = it->blk0; p0 < blk1; p0 += kScorePass) {
    const int b0 = p0 + wave * 32;
    load_queries(0);
    bf16x8 s[2][2 * KS];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      // blocks past the last one read that one again
      const int b = min(b0 + t * 16 + r16, blk1 - 1);
      const int page = row[(size_t)b << (a.log_block - 4)];
      const uint16_t* from = a.summary + ((size_t)page * a.hkv + kvh) * 2 * D + quad * 8;
#pragma unroll
      for (int k = 0; k < 2 * KS; ++k) s[t][k] = as_bf16x8(ld16(from + k * 32));
    }
    // a row's scores from block b0 on; rows j0 .. j0 + TOKENS - 1 are `step` floats apart
    const int step = a.hkv * a.max_blocks;  // at most 2^24
    float* to = a.scores + ((size_t)row0 * a.hkv + kvh) * a.max_blocks + b0;
    // Block b0 + 16 t + r16 has a score in rows first[t] .. n - 1.
    int first[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int b = b0 + t * 16 + r16;
      first[t] = b < blk1 ? min(max((b << a.log_block) - pos0, 0), n) : n;
    }
    for (int g0 = 0; g0 < n; g0 += 4 * TOKENS) {
      __syncthreads();  // the tiles before have been read
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        u32x4 plus, minus;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t m = negative_halves(ahead[k][w]);
          plus[w] = ahead[k][w] & ~m;
          minus[w] = ahead[k][w] & m;
        }
        s_query[wave][k][lane] = plus;
        s_query[wave][KS + k][lane] = minus;
      }
      if (g0 + 4 * TOKENS < n) load_queries(g0 + 4 * TOKENS);
      __syncthreads();
      if (b0 >= blk1) continue;
      u32x4 query[2 * KS];
      auto read_tile = [&](int i) {
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          query[k] = s_query[i][k][lane];
          query[KS + k] = s_query[i][KS + k][lane];
        }
      };
      read_tile(0);
      const int end = min(n, g0 + 4 * TOKENS);
      for (int j0 = g0; j0 < end; j0 += TOKENS, to += (size_t)TOKENS * step) {
        // the products with the high and with the low values apart: half as many terms in a
        // row, and no product waits for the one before
        f32x4 x[2], y[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) x[t] = y[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            x[t] = mfma(as_bf16x8(query[k]), s[t][k], x[t]);
            y[t] = mfma(as_bf16x8(query[KS + k]), s[t][KS + k], y[t]);
          }
        // the next tile (after the last one any), while this one's sums are looked at
        __builtin_amdgcn_sched_barrier(0);
        read_tile(((j0 - g0) / TOKENS + 1) & 3);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int t = 0; t < 2; ++t) x[t] += y[t];
        // Lanes without a score store outside the buffer's range, which drops it: no branch
        // stands between a tile's stores and the next tile's products.
        const PartWriter tile(to);
        auto put = [&](int token, int t, float x, bool mine = true) {
          const int from = t ? first[1] : first[0];
          const bool ok = mine && (uint32_t)(j0 + token - from) < (uint32_t)(n - from);
          const uint32_t at = ok ? (uint32_t)(token * step + t * 16 + r16) * 4 : 0x80000000u;
          __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(x), tile.rsrc, (int)at, 0, 0);
        };
        if constexpr (LOG_G == 0) {
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) put(quad * 4 + i, t, x[t][i]);
        } else if constexpr (LOG_G == 1) {
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i) put(quad * 2 + i, t, fmaxf(x[t][2 * i], x[t][2 * i + 1]));
        } else {
          float m[2];
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            m[t] = fmaxf(fmaxf(x[t][0], x[t][1]), fmaxf(x[t][2], x[t][3]));
            if constexpr (LOG_G > 2) m[t] = fmaxf(m[t], __shfl_xor(m[t], 16, 64));
            if constexpr (LOG_G > 3) m[t] = fmaxf(m[t], __shfl_xor(m[t], 32, 64));
          }
          const int token = quad >> (LOG_G - 2);
          if constexpr (LOG_G == 2) {
            put(token, 0, m[0]);
            put(token, 1, m[1]);
          } else {  // of the lanes that have it one a tile
            put(token, quad & 1, quad & 1 ? m[1] : m[0], LOG_G == 3 || quad < 2);
          }
        }
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Selection.  Scores map to 32-bit keys in the same order; what always stays has the
// highest key, what is not there the lowest.  WAVES waves hold a list in registers, 64 NR
// scores each, and find the key of the last one that stays bit by bit, from the highest
// bit in which the keys differ on: a count of the keys from a candidate on is a compare and
// a count of the lanes' mask per register, and it ends once the candidate parts as many as
// stay (some 12 to 18 counts of spread scores).  Lists in several waves meet at a barrier for
// every count, so one wave takes a list where there are lists for every compute unit (4224 of
// 1040 blocks: 30 us in four waves each, 16 so, 5 of them vector issue).  A wave holds 2048 blocks
// at most, and the longest request decides for all rows of the batch: beside one of 2063 blocks
// the same lists take 78 us in sixteen waves each, beside one of 2032 18.  The loads go as the
// counts do, four registers at a time: four scores are waited for before the next four are asked
// for, so that a list of 1040 blocks is five trips to memory, one of 512 two.  256 lists of 512
// blocks take 5.8 us, the launch, the plan, the scores and the search one after another.
__device__ __forceinline__ int lanes_below(uint64_t mask) {
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32),
                                        __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}
// NaN as +infinity, -0 as +0.
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) x = kInf;
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
constexpr uint32_t kAlways = 0xFFFFFFFFu, kAbsent = 0;

template <int WAVES, int NR>
__global__ __launch_bounds__(64 * WAVES) void block_select_kernel(SparseArgs a) {
  constexpr int THREADS = 64 * WAVES;
  __shared__ int s_count[2][WAVES];
  __shared__ uint32_t s_or[WAVES], s_and[WAVES];
  const int wg = workgroup_id();
  if (wg >= a.workgroups) return;
  Row r;
  if (!take_row(a, wg / a.hkv, &r)) return;
  const int kvh = wg % a.hkv, tid = threadIdx.x, lane = tid & 63;
  const int wave = WAVES == 1 ? 0 : __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = (r.pos >> a.log_block) + 1, need = min(n, a.top);
  const size_t list = (size_t)r.row * a.hkv + kvh;
  int32_t* out = a.blocks + list * a.top;
  for (int i = need + tid; i < a.top; i += THREADS) out[i] = -1;
  if (n <= a.top) {
    for (int i = tid; i < n; i += THREADS) out[i] = i;
    return;
  }
  const float* from = a.scores_in + list * a.max_blocks;
  const int first = wave * 64 * NR + lane;
  // registers that hold scores: the others are left out, a few at a time
  const int used = (n - wave * 64 * NR + 63) / 64;
  constexpr int STEP = NR < 4 ? NR : 4;
  auto each = [&](auto body) {
#pragma unroll
    for (int i0 = 0; i0 < NR; i0 += STEP)
      if (i0 < used) {
#pragma unroll
        for (int i = i0; i < i0 + STEP; ++i) body(i);
      }
  };
  uint32_t k[NR];
  uint32_t any = 0, all = ~0u;
#pragma unroll
  for (int i = 0; i < NR; ++i) k[i] = kAbsent;
  each([&](int i) {
    const int b = first + i * 64;
    const float x = from[min(b, n - 1)];
    uint32_t key = order_key(x);
    const bool other = b >= a.sink && b < n - a.recent;
    any |= other ? key : 0;
    all &= other ? key : ~0u;
    key = other ? key : kAlways;
    k[i] = b < n ? key : kAbsent;
  });
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    any |= __shfl_xor(any, o, 64);
    all &= __shfl_xor(all, o, 64);
  }
  if constexpr (WAVES > 1) {
    if (lane == 0) {
      s_or[wave] = any;
      s_and[wave] = all;
    }
    __syncthreads();
    any = s_or[0];
    all = s_and[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) {
      any |= s_or[w];
      all &= s_and[w];
    }
  }
  any = __builtin_amdgcn_readfirstlane(any);
  all = __builtin_amdgcn_readfirstlane(all);
  int turn = 0;
  auto count = [&](uint32_t t) {  // keys >= t of all waves
    int c = 0;
    each([&](int i) { c += (int)__popcll(__ballot(k[i] >= t)); });
    if constexpr (WAVES > 1) {
      turn ^= 1;
      if (lane == 0) s_count[turn][wave] = c;
      __syncthreads();
      c = 0;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) c += s_count[turn][w];
      c = __builtin_amdgcn_readfirstlane(c);
    }
    return c;
  };
  // every other score's key agrees above the highest bit of `differ`
  const uint32_t differ = any & ~all;
  int bit = differ ? 31 - __builtin_clz(differ) : -1;
  uint32_t t = bit == 31 ? 0 : all & (~0u << (bit + 1));
  bool exact = false;  // the keys from t on are `need`
  for (; bit >= 0 && !exact; --bit) {
    const int c = count(t | 1u << bit);
    if (c >= need) t |= 1u << bit;
    exact = c == need;
  }
  // keys above t stay, and of those equal to it the first ones
  const uint32_t above = exact ? t - 1 : t;  // t > 0: -infinity's key is
  int n_in = 0, n_eq = 0;
  if (WAVES > 1 || !exact) each([&](int i) { n_in += (int)__popcll(__ballot(k[i] > above)); });
  if (WAVES > 1 && !exact) each([&](int i) { n_eq += (int)__popcll(__ballot(k[i] == t)); });
  int before_in = 0, before_eq = 0, all_in = n_in;
  if constexpr (WAVES > 1) {
    __syncthreads();  // the last count has been read
    if (lane == 0) {
      s_count[0][wave] = n_in;
      s_count[1][wave] = n_eq;
    }
    __syncthreads();
    all_in = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      before_in += w < wave ? s_count[0][w] : 0;
      before_eq += w < wave ? s_count[1][w] : 0;
      all_in += s_count[0][w];
    }
  }
  if (exact) {
    each([&](int i) {
      const bool in = k[i] > above;
      const uint64_t mask = __ballot(in);
      if (in) out[before_in + lanes_below(mask)] = first + i * 64;
      before_in += (int)__popcll(mask);
    });
    return;
  }
  const int quota = need - all_in;
  each([&](int i) {
    const bool in = k[i] > above, eq = k[i] == t;
    const uint64_t mi = __ballot(in), me = __ballot(eq);
    const int eq_at = before_eq + lanes_below(me);
    if (in || (eq && eq_at < quota))
      out[before_in + lanes_below(mi) + min(eq_at, quota)] = first + i * 64;
    before_in += (int)__popcll(mi);
    before_eq += (int)__popcll(me);
  });
}

// ---------------------------------------------------------------------------
// 16-byte loads of what other workgroups of the launch have written past their caches;
// the base is wave-uniform, offsets are bytes from it.
struct PartReader {
  __amdgpu_buffer_rsrc_t rsrc;
  __device__ explicit PartReader(float* base) : rsrc(PartWriter(base).rsrc) {}
  __device__ f32x4 operator()(int byte_off) const {
    return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, byte_off, 0,
                                                                           kCachePolicySc1));
  }
};

// Attention.  One workgroup takes as many neighbouring rows of a request as fit in 32 columns
// (row, query head) of a kv head, and the union of their lists: neighbours mostly look at the
// same blocks, whose keys and values are then read once, and a block costs the matrix cores the
// same for one row as for 16 columns of them.  A mask per block says whose it is.  A row alone
// (a decode) goes by its list as it is, and so do rows, one after the other, whose lists name a
// block twice or whose masks would not fit in LDS.
//
// The pages (of no block left out) go to LDS; the four waves take two of them, 32 keys, in
// turn.  The 16x16x32 products have keys as rows; key r of a step is row (r & 3) + 4 (r >> 3)
// of product (r >> 2) & 1, so that the logits of a lane are those whose weights it multiplies
// with the values (dim-major pages) next.  Keys and values go from memory to registers, a step
// ahead; the steps' loads are what bounds it, and the registers for them leave two waves a SIMD
// (three waves had to spill, and were slower).  64/8 heads of 128, lists of 64 blocks of 64 keys:
//   32 decode rows     105 us  538 MB from memory, 5.1 TB/s (96 rows 5.9)
//   128 rows of a chunk 87 us  151 with a workgroup a row (2.1 GB through the caches at 14 TB/s),
//                              110 with 16 columns a workgroup, 144 with two waves for each 16
//   512 and 2048 rows   280 and 1070 us: it grows with the rows, as every four of them read their
//                              own union (59 and 235 us of products at the library's rate)
// Where rows of one workgroup see more than kMaskBlocks blocks there is no union, and it goes row by
// row: 128 rows, 32/8 heads, 256 blocks of 16, on 130800 keys 81 us, on 131072 224.
// One row of 2048 keys, 11 us, is launch, plan, list, table, keys, join and the pieces' join.
constexpr int kPassPages = 512;     // pages in LDS at a time
constexpr int kMaskBlocks = 8192;   // blocks of a union, 16 bits each
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
// The highest x of a column: over the four lanes 16 apart.
__device__ __forceinline__ float max_over_quads(float x) {
  uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  u = __float_as_uint(x);
  const auto b = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
// Keeps the first n of 8 packed bf16 values.
__device__ __forceinline__ u32x4 first_values(int n) {
  u32x4 keep;
#pragma unroll
  for (int w = 0; w < 4; ++w)
    keep[w] = (n > 2 * w ? 0xFFFFu : 0u) | (n > 2 * w + 1 ? 0xFFFF0000u : 0u);
  return keep;
}

template <int D>
struct AttentionLds {
  int4 page[kPassPages + 2];        // page of the pool, its first position, the rows whose it is
  uint32_t mask[kMaskBlocks / 2];   // of two blocks each
  int part[2][4];
  int flag[2];
  int odd;                          // some sum is not finite
  float ml[2][4][16];
  float m[32], l[32];               // of the passes so far, and their sums
  __attribute__((aligned(16))) float sum[32][D];
  union {
    int2 block[kPassPages];         // block, the rows whose it is, until the pages are listed
    __attribute__((aligned(16))) float o[4][16][64];  // the waves' sums, 64 dims at a time
    float weight[64 * 2 * 32];      // m and l of a list's pieces
  };
};

template <int D>
__global__ __launch_bounds__(kSparseThreads, 2) void sparse_attention_kernel(SparseArgs a) {
  constexpr int KS = D / 32, DT = D / 16;
  // the joined sums: four dims of column c0 + i CSTEP a thread
  constexpr int NC = D / 32, CSTEP = 1024 / D;
  __shared__ AttentionLds<D> lds;
  const int wg = workgroup_id();
  if (wg >= a.workgroups) return;
  const int kvh = wg % a.hkv, split = wg / a.hkv % a.nsplit, unit = wg / a.hkv / a.nsplit;
  // the rows: `rows` of them from token row row0, position pos0 on
  const bool single = unit >= a.num_groups * a.subs;
  const int j0 = single ? 0 : unit % a.subs * a.tokens;
  if (!plan_ok(a)) return;
  const Rows record(a, single ? a.num_groups + (unit - a.num_groups * a.subs) : unit / a.subs);
  const int rows = min(single ? 1 : a.tokens, record.n - j0);
  if (rows <= 0) return;
  const int row0 = record.row0 + j0, pos0 = record.pos0 + j0, last = pos0 + rows - 1;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int columns = rows * a.g;
  const int32_t* const table = a.bt + (size_t)record.req * a.maxp;
  const int log_pages = a.log_block - 4;
  auto token_of = [&](int column) { return (column * a.g_magic) >> 16; };
  auto list_of = [&](int t) { return a.blocks_in + ((size_t)(row0 + t) * a.hkv + kvh) * a.top; };
  // (row, query head) of a column
  auto row_of = [&](int column) {
    const int t = token_of(column);
    return ((size_t)(row0 + t) * a.hq + kvh * a.g + (column - t * a.g)) * D;
  };
  // The thread's own number, and its first column and dim of the joined sums, made anew where
  // they are used: what the compiler knows to be the same all along it keeps in registers all
  // along, and the products need those.
  auto anew = [](int x) {
    asm volatile("" : "+v"(x));
    return x;
  };
  struct Place {
    int c0, d0;
  };
  auto place = [&] {
    const int x = anew(tid) * 4;
    return Place{x / D, x % D};
  };
  uint32_t seen;  // rows of which a key counts
  bool fresh;     // no pass yet: LDS holds no sums
  // m, l and the sums of column c: between the passes they lie in LDS, so that they take no
  // registers from the products.
  struct State {
    float m, l;
    f32x4 sum;
  };
  const State nothing = {-kInf, 0.f, f32x4{0.f, 0.f, 0.f, 0.f}};
  auto load_state = [&](int c, int d0) {
    return State{lds.m[c], lds.l[c], *reinterpret_cast<const f32x4*>(&lds.sum[c][d0])};
  };
  auto store_state = [&](int c, int d0, const State& x) {
    *reinterpret_cast<f32x4*>(&lds.sum[c][d0]) = x.sum;
    if (d0 == 0) {
      lds.m[c] = x.m;
      lds.l[c] = x.l;
    }
  };

  // The first `total` pages of lds.page by the matrix cores, for one or two tiles of 16
  // columns; the waves' sums are joined and added to those of the passes before.
  auto multiply = [&](int total, auto tiles) __attribute__((always_inline)) {
    constexpr int NT = tiles;
    const int r16 = anew(lane) & 15, quad = anew(lane) >> 4;
    int token[NT];
    bf16x8 qf[NT][KS];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int column = min(r16 + n * 16, columns - 1);  // the others repeat the last
      token[n] = token_of(column);
#pragma unroll
      for (int s = 0; s < KS; ++s)
        qf[n][s] = as_bf16x8(ld16(a.q + row_of(column) + s * 32 + quad * 8));
    }
    float m[NT], l[NT];
    f32x4 o[NT][DT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      m[n] = -kInf;
      l[n] = 0.f;
#pragma unroll
      for (int t = 0; t < DT; ++t) o[n][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const int slot0 = 8 * ((r16 >> 2) & 1) + (r16 & 3);
    u32x4 kf[2][KS], vf[DT];
    auto load_keys = [&](int p0, int p1) {
      const uint16_t* kp =
          a.kc + ((size_t)(r16 >> 3 ? p1 : p0) * a.hkv + kvh) * 16 * D + slot0 * D + quad * 8;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int s = 0; s < KS; ++s) kf[t][s] = ld16(kp + t * 4 * D + s * 32);
    };
    auto load_values = [&](int p0, int p1) {
      const uint16_t* vp =
          a.vc + ((size_t)(quad >> 1 ? p1 : p0) * a.hkv + kvh) * 16 * D + r16 * 16 + 8 * (quad & 1);
#pragma unroll
      for (int t = 0; t < DT; ++t) vf[t] = ld16(vp + t * 256);
    };
    const int steps = (total + 1) / 2;
    auto page_of = [&](int i) { return __builtin_amdgcn_readfirstlane(lds.page[i].x); };
    int p0 = 0, p1 = 0;
    if (wave < steps) {
      p0 = page_of(2 * wave);
      p1 = page_of(2 * wave + 1);
      load_keys(p0, p1);
      load_values(p0, p1);
    }
    // `more`: the wave has a step after this one.  (A condition known to the compiler: loads
    // that might not have been issued would be waited for with everything behind them.)
    auto step = [&](int s, auto more) __attribute__((always_inline)) {
      const int4 e0 = lds.page[2 * s], e1 = lds.page[2 * s + 1];
      if constexpr (more) {
        p0 = page_of(2 * s + 8);
        p1 = page_of(2 * s + 9);
      }
      // the lane's first key, and the last one of the step
      const int key0 = (quad >> 1 ? e1.y : e0.y) + 8 * (quad & 1);
      const uint32_t rows_of = quad >> 1 ? e1.z : e0.z;
      const int far = __builtin_amdgcn_readfirstlane(max(e0.y, e1.y)) + 15;
      f32x4 logits[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) logits[n][0] = logits[n][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int t = 0; t < 2; ++t)
            logits[n][t] = mfma(as_bf16x8(kf[t][k]), qf[n][k], logits[n][t]);
      if constexpr (more) load_keys(p0, p1);
      __builtin_amdgcn_sched_barrier(0);
      if (far > last) {
        // a slot that no row sees may hold anything, and 0 times NaN is NaN
        const u32x4 keep = first_values(last + 1 - key0);
#pragma unroll
        for (int t = 0; t < DT; ++t) vf[t] &= keep;
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = logits[n][i >> 2][i & 3];
        // Is the lane's page the column's row's?  Where it is not, its logits are left out of
        // the maximum, and their exponents are -infinity.
        const bool mine = rows_of >> token[n] & 1;
        if (far > pos0) {  // a row sees a part of it
          const int nv = pos0 + token[n] + 1 - key0;
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (i >= nv) x[i] = -kInf;
        }
        float mx = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])),
                         fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        mx = mine ? mx : -kInf;
        mx = max_over_quads(mx);
        const float mn = mx == -kInf ? m[n] : fmaxf(m[n], mx * a.c);
        const float ms = mn == -kInf ? 0.f : mn;
        const float alpha = exp2_fast(m[n] - ms), off = mine ? -ms : -kInf;
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = exp2_fast(__builtin_fmaf(x[i], a.c, off));
        if (far > pos0 && a.c == 0.f) {  // 0 times -infinity is NaN
          const int nv = mine ? pos0 + token[n] + 1 - key0 : 0;
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (i >= nv) p[i] = 0.f;
        }
        l[n] = l[n] * alpha + (((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7])));
        m[n] = mn;
        // A weight enters the matrix product as three bf16 values, the rounded one and what
        // that misses twice over: all of its 24 bits.
        u32x4 part[3];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          float x0 = p[2 * w], x1 = p[2 * w + 1];
#pragma unroll
          for (int i = 0; i < 3; ++i) {
            part[i][w] = pack2(x0, x1);
            x0 -= bf16_lo(part[i][w]);
            x1 -= bf16_hi(part[i][w]);
          }
        }
        if (__any(alpha != 1.f)) {
#pragma unroll
          for (int t = 0; t < DT; ++t) o[n][t] *= alpha;
        }
#pragma unroll
        for (int i = 0; i < 3; ++i)
#pragma unroll
          for (int t = 0; t < DT; ++t)
            o[n][t] = mfma(as_bf16x8(vf[t]), as_bf16x8(part[i]), o[n][t]);
        if (n + 1 < NT) __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (more) load_values(p0, p1);
      __builtin_amdgcn_sched_barrier(0);
    };
    int s = wave;
    for (; s + 4 < steps; s += 4) step(s, std::true_type{});
    if (s < steps) step(s, std::false_type{});
    const auto [c0, d0] = place();
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      l[n] += __shfl_xor(l[n], 16, 64);
      l[n] += __shfl_xor(l[n], 32, 64);
      if (n > 0) __syncthreads();
      if (quad == 0) {
        lds.ml[0][wave][r16] = m[n];
        lds.ml[1][wave][r16] = l[n];
      }
      constexpr int PER = NC / 2;  // of a thread's columns, 16 / CSTEP in a tile
      State x[PER];
#pragma unroll
      for (int h = 0; h < D / 64; ++h) {  // 64 dims at a time
        if (h > 0) __syncthreads();
#pragma unroll
        for (int t = 0; t < 4; ++t)
          *reinterpret_cast<f32x4*>(&lds.o[wave][r16][t * 16 + 4 * quad]) = o[n][h * 4 + t];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const int c = c0 + i * CSTEP;
          if (h == 0) x[i] = fresh ? nothing : load_state(n * 16 + c, d0);
          if (d0 / 64 != h) continue;
          float mm = x[i].m;
#pragma unroll
          for (int w = 0; w < 4; ++w) mm = fmaxf(mm, lds.ml[0][w][c]);
          const float ms = mm == -kInf ? 0.f : mm, scale = exp2_fast(x[i].m - ms);
          x[i].sum *= scale;
          x[i].l *= scale;
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const float f = exp2_fast(lds.ml[0][w][c] - ms);
            x[i].sum += *reinterpret_cast<const f32x4*>(&lds.o[w][c][d0 % 64]) * f;
            x[i].l += lds.ml[1][w][c] * f;
          }
          x[i].m = mm;
        }
      }
      __syncthreads();  // m and l have been read by all threads of a column
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        store_state(n * 16 + c0 + i * CSTEP, d0, x[i]);
        // 0 times what is not finite is NaN
        const float sums = (x[i].sum[0] + x[i].sum[1]) + (x[i].sum[2] + x[i].sum[3]);
        const float zero = (x[i].l + sums) * 0.f;
        if (__any(zero != 0.f) && lane == 0) lds.odd = 1;
      }
    }
    fresh = false;
  };
  // The same, key by key without the matrix cores, for values that are not finite: they reach
  // only the rows that see their keys, and with the whole weight.  (In the products above, 0
  // times an infinite value is NaN, for a row that does not see its key and for a part of a
  // weight.)  About 100 times slower.
  auto go_through = [&](int total) __attribute__((always_inline)) {
    const auto [c0, d0] = place();
    State x[NC];
#pragma unroll
    for (int n = 0; n < NC; ++n) x[n] = fresh ? nothing : load_state(c0 + n * CSTEP, d0);
    __syncthreads();
    for (int i = 0; i < total; ++i) {
      const int4 e = lds.page[i];
      const size_t base = ((size_t)e.x * a.hkv + kvh) * 16 * D;
      for (int s = 0; s < 16 && e.y + s <= last; ++s) {
        const u32x2 k = *reinterpret_cast<const u32x2*>(a.kc + base + s * D + d0);
        f32x4 v;
#pragma unroll
        for (int d = 0; d < 4; ++d) v[d] = bf16_lo(a.vc[base + (size_t)(d0 + d) * 16 + s]);
#pragma unroll
        for (int n = 0; n < NC; ++n) {
          const int c = c0 + n * CSTEP, t = token_of(c);
          u32x2 q = {0, 0};
          if (c < columns) q = *reinterpret_cast<const u32x2*>(a.q + row_of(c) + d0);
          float y = bf16_lo(q[0]) * bf16_lo(k[0]);
          y = __builtin_fmaf(bf16_hi(q[0]), bf16_hi(k[0]), y);
          y = __builtin_fmaf(bf16_lo(q[1]), bf16_lo(k[1]), y);
          y = __builtin_fmaf(bf16_hi(q[1]), bf16_hi(k[1]), y);
          for (int o = 1; o < D / 4; o *= 2) y += __shfl_xor(y, o, 64);
          if (c >= columns || !(e.z >> t & 1) || e.y + s > pos0 + t) continue;
          const float mn = y == -kInf ? x[n].m : fmaxf(x[n].m, y * a.c);
          const float ms = mn == -kInf ? 0.f : mn, scale = exp2_fast(x[n].m - ms);
          const float p = exp2_fast(__builtin_fmaf(y, a.c, -ms));
          if (scale != 1.f) {
            x[n].sum *= scale;
            x[n].l *= scale;
          }
          x[n].sum += v * p;
          x[n].l += p;
          x[n].m = mn;
        }
      }
    }
#pragma unroll
    for (int n = 0; n < NC; ++n) store_state(c0 + n * CSTEP, d0, x[n]);
    fresh = false;
  };
  // beside the last page of an odd number: the same one, of no row
  auto pad = [&](int total, int i, int4 e) {
    if (i == total - 1 && total & 1) lds.page[total] = int4{e.x, e.y, 0, 0};
  };
  // Pages base .. base + kPassPages - 1 of row t's list, up to page1; how many.
  auto list_pages = [&](int t, int base, int page1) {
    const int32_t* list = list_of(t);
    const int pos = pos0 + t;
    int4 mine[2];
    uint64_t mask[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int p = base + i * kSparseThreads + tid;
      mine[i] = int4{0, 0, 0, 0};
      if (p < page1) {
        const int b = list[p >> log_pages];
        if (b >= 0 && b <= pos >> a.log_block) {
          const int at = (b << log_pages) + (p & ((1 << log_pages) - 1));
          if (at * 16 <= pos) mine[i] = int4{table[at], at * 16, 1 << t, 0};
        }
      }
      mask[i] = __ballot(mine[i].z != 0);
      if (lane == 0) lds.part[i][wave] = (int)__popcll(mask[i]);
    }
    __syncthreads();
    int total = 0, at[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      at[i] = total + lanes_below(mask[i]);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        if (w < wave) at[i] += lds.part[i][w];
        total += lds.part[i][w];
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (mine[i].z) {
        lds.page[at[i]] = mine[i];
        pad(total, at[i], mine[i]);
      }
    if (total > 0) seen |= 1u << t;
    return __builtin_amdgcn_readfirstlane(total);
  };
  // The union's masks; a thread's words of them, how many blocks earlier threads have, and all
  // of its pages.  -1: a list names a block twice.
  int word0 = 0, word1 = 0, before = 0;
  auto make_union = [&] {
    const int blocks = (last >> a.log_block) + 1;
    if (tid < 2) lds.flag[tid] = 0;
    for (int i = tid; i < (blocks + 1) / 2; i += kSparseThreads) lds.mask[i] = 0;
    __syncthreads();
#pragma unroll 4
    for (int i = tid; i < rows * a.top; i += kSparseThreads) {
      const int t = i / a.top, b = list_of(t)[i - t * a.top];
      if (b < 0 || b > (pos0 + t) >> a.log_block) continue;
      const uint32_t bit = 1u << (t + 16 * (b & 1));
      if (atomicOr(&lds.mask[b >> 1], bit) & bit) lds.flag[0] = 1;
    }
    __syncthreads();
    if (lds.flag[0]) return -1;
    const int per = (blocks + 2 * kSparseThreads - 1) / (2 * kSparseThreads);
    word0 = tid * per;
    word1 = min(word0 + per, (blocks + 1) / 2);
    int n = 0;
    uint32_t mine = 0;
    for (int i = word0; i < word1; ++i) {
      const uint32_t x = lds.mask[i];
      n += ((x & 0xFFFFu) != 0) + (x >> 16 != 0);
      mine |= x | x >> 16;
    }
    before = n;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const int y = __shfl_up(before, d, 64);
      if (lane >= d) before += y;
      mine |= __shfl_xor(mine, d, 64);
    }
    if (lane == 63) {
      lds.part[0][wave] = before;
      atomicOr(&lds.flag[1], (int)(mine & 0xFFFFu));
    }
    __syncthreads();
    int total = 0;
    before -= n;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if (w < wave) before += lds.part[0][w];
      total += lds.part[0][w];
    }
    seen = lds.flag[1];  // whatever this workgroup's share
    return __builtin_amdgcn_readfirstlane(total) << log_pages;
  };
  // `pages` pages of the union from page `base` on.
  auto union_pages = [&](int base, int pages) {
    const int b0 = base >> log_pages, b1 = (base + pages - 1) >> log_pages;
    int at = before;
    for (int i = word0; i < word1; ++i) {
      const uint32_t x = lds.mask[i];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int rows_of = (int)(x >> (16 * h) & 0xFFFFu);
        if (!rows_of) continue;
        if (at >= b0 && at <= b1) lds.block[at - b0] = int2{2 * i + h, rows_of};
        ++at;
      }
    }
    __syncthreads();
    for (int i = tid; i < pages; i += kSparseThreads) {
      const int p = base + i;
      const int2 b = lds.block[(p >> log_pages) - b0];
      // a page behind the last row's position: that one's, of no row
      const int page = (b.x << log_pages) + (p & ((1 << log_pages) - 1));
      const bool here = page * 16 <= last;
      const int4 e = {table[here ? page : last / 16], (here ? page : last / 16) * 16,
                      here ? b.y : 0, 0};
      lds.page[i] = e;
      pad(pages, i, e);
    }
    return pages;
  };
  for (bool finite = true;; finite = false) {
    seen = 0;
    fresh = true;
    if (tid == 0) lds.odd = 0;
    // this workgroup's pages of the union, as many steps to every wave, or of each row's list
    int share = -1, base, end, t = rows - 1;
    if (rows > 1 && (last >> a.log_block) < kMaskBlocks) share = make_union();
    const bool joint = share >= 0;
    if (joint) {
      const int total = share;
      if (a.nsplit > 1) share = ((total + a.nsplit - 1) / a.nsplit + 7) / 8 * 8;
      base = min(total, split * share);
      end = min(total, base + share);
    } else {
      t = 0;
      base = split * a.split_entries << log_pages;
      end = min(a.top, (split + 1) * a.split_entries) << log_pages;
    }
    for (;;) {
      if (base >= end) {
        if (++t >= rows) break;
        base = split * a.split_entries << log_pages;
      }
      const int total =
          joint ? union_pages(base, min(kPassPages, end - base)) : list_pages(t, base, end);
      __syncthreads();
      if (finite && columns <= 16)
        multiply(total, std::integral_constant<int, 1>{});
      else if (finite)
        multiply(total, std::integral_constant<int, 2>{});
      else
        go_through(total);
      __syncthreads();  // the pages and sums have been read
      base += kPassPages;
    }
    // fresh: not one pass, all of whose barriers would lie behind here
    if (!finite || fresh || !lds.odd) break;
    __syncthreads();
  }
  if (fresh) {
    const auto [c0, d0] = place();
#pragma unroll
    for (int i = 0; i < NC; ++i) store_state(c0 + i * CSTEP, d0, nothing);
    __syncthreads();
  }

  const auto [c0, d0] = place();
  const int cols = a.tokens * a.g;  // of a record
  const int rec_floats = sparse_rec_floats(cols, D), rec_o = sparse_rec_o(cols);
  const int ticket = unit * a.hkv + kvh;
  auto store = [&, d0 = d0](int c, f32x4 v) {
    *reinterpret_cast<u32x2*>(a.out + row_of(c) + d0) = u32x2{pack2(v[0], v[1]), pack2(v[2], v[3])};
  };
  // no key: zeros; keys whose logits are all -infinity have no weights
  auto inverse = [&](float m, float l, bool any) {
    return m != -kInf ? 1.f / l : any ? __builtin_nanf("") : 0.f;
  };
  if (a.nsplit == 1) {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int c = c0 + i * CSTEP;
      const State x = load_state(c, d0);
      if (c < columns) store(c, x.sum * inverse(x.m, x.l, seen >> token_of(c) & 1));
    }
    return;
  }
  // A piece: its record goes past this die's cache (device scope) and has arrived before
  // the ticket is taken; the last piece to finish joins all of them in their order.
  float* const records = a.records + (size_t)ticket * a.nsplit * rec_floats;
  float* const rec = records + (int64_t)split * rec_floats;
  const PartWriter write(rec + rec_o);
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int c = c0 + i * CSTEP;
    if (c >= columns) continue;
    const State x = load_state(c, d0);
    write((c * D + d0) * 4, __builtin_bit_cast(u32x4, x.sum));
    if (d0 == 0) {
      const bool any = seen >> token_of(c) & 1;
      const float l = x.m != -kInf ? x.l : any ? 1.f : 0.f;
      __hip_atomic_store(rec + c, x.m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(rec + cols + c, l, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
  vm_wait<0>();
  __syncthreads();
  if (tid == 0) {
    const int earlier = __hip_atomic_fetch_add(a.tickets + ticket, 1, __ATOMIC_RELAXED,
                                               __HIP_MEMORY_SCOPE_AGENT);
    lds.flag[0] = earlier == a.nsplit - 1;
    if (lds.flag[0])
      __hip_atomic_store(a.tickets + ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!lds.flag[0]) return;
  // m and l of all pieces, their weights, then the sums
  for (int e = tid; e < a.nsplit * 2 * columns; e += kSparseThreads) {
    const int s = e / (2 * columns), i = e - s * 2 * columns;
    const float* from = records + (int64_t)s * rec_floats + (i < columns ? i : cols + i - columns);
    lds.weight[e] = __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  const PartReader read(records);
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int c = c0 + i * CSTEP;
    if (c >= columns) continue;
    const float* const w = lds.weight + c;
    float m = -kInf, l = 0.f, some = 0.f;
    for (int s = 0; s < a.nsplit; ++s) m = fmaxf(m, w[s * 2 * columns]);
    const float ms = m == -kInf ? 0.f : m;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int s = 0; s < a.nsplit; ++s) {
      const float f = exp2_fast(w[s * 2 * columns] - ms), ls = w[s * 2 * columns + columns];
      l += ls * f;
      some += ls;
      v += read((s * rec_floats + rec_o + c * D + d0) * 4) * f;
    }
    store(c, v * inverse(m, l, some > 0.f));
  }
}

// ---------------------------------------------------------------------------
// Launches.
template <class K, class A>
int launch(K kernel, const A& a, int threads, void* stream) {
  if (a.workgroups == 0) return SSA_OK;
  (void)hipGetLastError();
  const int64_t wgs = a.workgroups;
  const dim3 grid(wgs < kGridRow ? wgs : kGridRow, (wgs + kGridRow - 1) / kGridRow);
  hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, static_cast<hipStream_t>(stream), a);
  return hipGetLastError() == hipSuccess ? SSA_OK : SSA_ERR_HIP;
}

// Read and written 16 bytes at a time.
bool misaligned(std::initializer_list<const void*> pointers) {
  for (const void* p : pointers)
    if (reinterpret_cast<uintptr_t>(p) % 16) return true;
  return false;
}
bool misaligned_plan(const void* plan_dev) {  // it holds 64-bit fields
  return reinterpret_cast<uintptr_t>(plan_dev) % 8 != 0;
}

int log2_of(int32_t x) {
  int n = 0;
  while (x >> (n + 1)) ++n;
  return n;
}

SparseArgs sparse_args(const SparseHeader* h, const void* plan_dev) {
  SparseArgs a{};
  a.plan = static_cast<const uint8_t*>(plan_dev);
  a.hash = h->hash;
  a.hq = h->hq;
  a.hkv = h->hkv;
  a.g = h->hq / h->hkv;
  a.maxp = h->max_pages_per_req;
  a.num_groups = h->num_groups;
  a.off_rows = h->off_rows;
  a.off_scores = h->off_scores;
  a.log_block = log2_of(h->block_keys);
  a.top = h->top;
  a.sink = h->sink;
  a.recent = h->recent;
  a.max_blocks = h->max_blocks;
  a.nsplit = h->nsplit;
  a.split_entries = h->split_entries;
  a.tokens = sparse_tokens(a.g);
  a.subs = sparse_subs(a.g);
  a.g_magic = (65536 + a.g - 1) / a.g;  // x / g for x < 32: (x g_magic) >> 16
  a.c = h->softmax_scale * 1.44269504088896340736f;
  return a;
}

int32_t rows_of(const SparseHeader* h) { return h->num_groups * kRowGroup + h->num_singles; }

int32_t summary_runs(const PlanHeader* h, int32_t block_keys) {
  return (h->num_chunk_segments + block_keys / 16 - 1) / (block_keys / 16);
}
int64_t summary_workgroups(const PlanHeader* h, int32_t block_keys) {
  return ((int64_t)summary_runs(h, block_keys) + h->num_segments - h->num_chunk_segments) *
         ((h->hkv + 3) / 4);
}

template <int D>
int launch_summary(const SummaryArgs& a, void* stream) {
  switch (a.block_keys) {
    case 16: return launch(block_summary_kernel<D, 16>, a, kSparseThreads, stream);
    case 32: return launch(block_summary_kernel<D, 32>, a, kSparseThreads, stream);
    case 64: return launch(block_summary_kernel<D, 64>, a, kSparseThreads, stream);
    default: return launch(block_summary_kernel<D, 128>, a, kSparseThreads, stream);
  }
}

template <int D>
int launch_scores(const SparseArgs& a, void* stream) {
  switch (log2_of(2 * a.g - 1)) {
    case 0: return launch(block_scores_kernel<D, 0>, a, kSparseThreads, stream);
    case 1: return launch(block_scores_kernel<D, 1>, a, kSparseThreads, stream);
    case 2: return launch(block_scores_kernel<D, 2>, a, kSparseThreads, stream);
    case 3: return launch(block_scores_kernel<D, 3>, a, kSparseThreads, stream);
    default: return launch(block_scores_kernel<D, 4>, a, kSparseThreads, stream);
  }
}

}  // namespace

int ssa::check_block_summary(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                             int32_t block_keys, const uint16_t* k_cache,
                             const int32_t* block_table, const uint16_t* summary) {
  const PlanHeader* h = nullptr;
  const int rc = check_plan(shape, plan_host, &h);
  if (rc) return rc;
  if (block_keys != 16 && block_keys != 32 && block_keys != 64 && block_keys != 128)
    return SSA_ERR_ARG;
  if (!plan_dev) return SSA_ERR_NULL;
  if (h->num_segments == 0) return SSA_OK;
  if (!k_cache || !block_table || !summary) return SSA_ERR_NULL;
  if (misaligned({k_cache, summary}) || misaligned_plan(plan_dev)) return SSA_ERR_ARG;
  return summary_workgroups(h, block_keys) > INT32_MAX ? SSA_ERR_ARG : SSA_OK;
}

namespace {

int check_scores(const SparseHeader* h, const void* plan_dev, const uint16_t* q,
                 const uint16_t* summary, const int32_t* block_table, const float* scores) {
  if (!plan_dev) return SSA_ERR_NULL;
  if (h->num_tokens == 0) return SSA_OK;
  if (!q || !summary || !block_table || !scores) return SSA_ERR_NULL;
  return misaligned({q, summary, scores}) || misaligned_plan(plan_dev) ? SSA_ERR_ARG : SSA_OK;
}

int check_select(const SparseHeader* h, const void* plan_dev, const float* scores,
                 const int32_t* blocks) {
  if (!plan_dev) return SSA_ERR_NULL;
  if (h->num_tokens == 0) return SSA_OK;
  if (!scores || !blocks) return SSA_ERR_NULL;
  return misaligned({scores, blocks}) || misaligned_plan(plan_dev) ? SSA_ERR_ARG : SSA_OK;
}

int check_attention(const SparseHeader* h, const void* plan_dev, const uint16_t* q,
                    const uint16_t* k_cache, const uint16_t* v_cache, const int32_t* block_table,
                    const int32_t* blocks, const uint16_t* out, const void* workspace,
                    size_t ws_bytes) {
  if (!plan_dev) return SSA_ERR_NULL;
  if (!workspace || ws_bytes < (size_t)h->ws_bytes) return SSA_ERR_WORKSPACE;
  if (h->num_tokens == 0) return SSA_OK;
  if (!q || !k_cache || !v_cache || !block_table || !blocks || !out) return SSA_ERR_NULL;
  return misaligned({q, k_cache, v_cache, blocks, out, workspace}) || misaligned_plan(plan_dev)
             ? SSA_ERR_ARG
             : SSA_OK;
}

}  // namespace

int ssa::check_sparse_calls(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                            const uint16_t* q, const uint16_t* k_cache, const uint16_t* v_cache,
                            const uint16_t* summary, const int32_t* block_table,
                            const float* scores, const int32_t* blocks, const uint16_t* out,
                            const void* workspace, size_t ws_bytes) {
  const SparseHeader* h = nullptr;
  int rc = check_sparse_plan(shape, plan_host, &h);
  if (rc || (rc = check_scores(h, plan_dev, q, summary, block_table, scores)) ||
      (rc = check_select(h, plan_dev, scores, blocks)))
    return rc;
  return check_attention(h, plan_dev, q, k_cache, v_cache, block_table, blocks, out, workspace,
                         ws_bytes);
}

extern "C" {

int ssa_block_summary(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                      int32_t block_keys, const uint16_t* k_cache, const int32_t* block_table,
                      uint16_t* summary, void* stream) {
  const int rc =
      check_block_summary(shape, plan_host, plan_dev, block_keys, k_cache, block_table, summary);
  if (rc) return rc;
  const PlanHeader* h = static_cast<const PlanHeader*>(plan_host);
  SummaryArgs a{};
  a.plan = static_cast<const uint8_t*>(plan_dev);
  a.hash = h->hash;
  a.off_segments = h->off_segments;
  a.off_reqs = h->off_reqs;
  a.hkv = h->hkv;
  a.maxp = h->max_pages_per_req;
  a.block_keys = block_keys;
  a.kc = k_cache;
  a.bt = block_table;
  a.summary = summary;
  a.head_groups = (h->hkv + 3) / 4;
  a.num_chunk_segments = h->num_chunk_segments;
  a.num_runs = summary_runs(h, block_keys);
  a.workgroups = (int32_t)summary_workgroups(h, block_keys);
  return h->head_dim == 128 ? launch_summary<128>(a, stream) : launch_summary<64>(a, stream);
}

int ssa_block_scores(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                     const uint16_t* q, const uint16_t* summary, const int32_t* block_table,
                     float* scores, void* stream) {
  const SparseHeader* h = nullptr;
  int rc = check_sparse_plan(shape, plan_host, &h);
  if (rc || (rc = check_scores(h, plan_dev, q, summary, block_table, scores))) return rc;
  SparseArgs a = sparse_args(h, plan_dev);
  a.workgroups = h->num_scores * h->hkv;
  a.q = q;
  a.summary = summary;
  a.bt = block_table;
  a.scores = scores;
  return h->head_dim == 128 ? launch_scores<128>(a, stream) : launch_scores<64>(a, stream);
}

int ssa_block_select(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                     const float* scores, int32_t* blocks, void* stream) {
  const SparseHeader* h = nullptr;
  int rc = check_sparse_plan(shape, plan_host, &h);
  if (rc || (rc = check_select(h, plan_dev, scores, blocks))) return rc;
  SparseArgs a = sparse_args(h, plan_dev);
  a.workgroups = rows_of(h) * h->hkv;
  a.scores_in = scores;
  a.blocks = blocks;
  // the longest list's waves and registers: up to 2048 blocks one wave where the lists fill the
  // chip, several where there are few; past that sixteen, however many lists there are
  const bool many = (int64_t)h->num_tokens * h->hkv >= 1024;
  const int32_t most = h->most_blocks;
  if (most <= 512) return launch(block_select_kernel<1, 8>, a, 64, stream);
  if (most <= 1024 && many) return launch(block_select_kernel<1, 16>, a, 64, stream);
  if (most <= 1024) return launch(block_select_kernel<4, 4>, a, 256, stream);
  if (most <= 2048 && many) return launch(block_select_kernel<1, 32>, a, 64, stream);
  if (most <= 2048) return launch(block_select_kernel<4, 8>, a, 256, stream);
  if (most <= 8192) return launch(block_select_kernel<16, 8>, a, 1024, stream);
  return launch(block_select_kernel<16, 32>, a, 1024, stream);
}

int ssa_sparse_attention(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                         const uint16_t* q, const uint16_t* k_cache, const uint16_t* v_cache,
                         const int32_t* block_table, const int32_t* blocks, uint16_t* out,
                         void* workspace, size_t ws_bytes, void* stream) {
  const SparseHeader* h = nullptr;
  int rc = check_sparse_plan(shape, plan_host, &h);
  if (rc || (rc = check_attention(h, plan_dev, q, k_cache, v_cache, block_table, blocks, out,
                                  workspace, ws_bytes)))
    return rc;
  SparseArgs a = sparse_args(h, plan_dev);
  a.workgroups = (h->num_groups * a.subs + h->num_singles) * h->hkv * h->nsplit;
  a.q = q;
  a.kc = k_cache;
  a.vc = v_cache;
  a.bt = block_table;
  a.blocks_in = blocks;
  a.out = out;
  a.tickets = static_cast<int32_t*>(workspace);
  a.records = reinterpret_cast<float*>(static_cast<char*>(workspace) + kSparseTickets * 4);
  return h->head_dim == 128 ? launch(sparse_attention_kernel<128>, a, kSparseThreads, stream)
                            : launch(sparse_attention_kernel<64>, a, kSparseThreads, stream);
}

}  // extern "C"
