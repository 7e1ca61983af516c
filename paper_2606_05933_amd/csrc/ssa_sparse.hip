// HIP kernels for gfx950 of include/ssa_sparse.h: block summaries, their scores, the
// selection, attention over the selected blocks.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>
#include <initializer_list>

#include "../../include/ssa_sparse.h"
#include "ssa_device.h"
#include "ssa_plan_format.h"
#include "ssa_sparse_format.h"

namespace ssa {
int check_plan(const ssa_shape* s, const void* plan_host, const PlanHeader** out);
int check_sparse_plan(const ssa_shape* s, const void* plan_host, const SparseHeader** out);
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
// instruction, so that the extremes are the keys' own bits.
struct SummaryArgs {
  const uint8_t* plan;
  uint64_t hash;
  int32_t off_segments, off_reqs;
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

template <int D, int BLOCK>
__global__ __launch_bounds__(kSparseThreads) void block_summary_kernel(SummaryArgs a) {
  constexpr int CPR = D / 8, ROWS = 64 / CPR;  // lanes a row, rows a load
  constexpr int LOADS = BLOCK / ROWS;
  const int wg = workgroup_id();
  if (wg >= a.workgroups) return;
  const auto h = as_uniform<PlanHeader>(a.plan);
  const auto sg = as_uniform<AppendSeg>(a.plan + a.off_segments) + wg / a.head_groups;
  const int req = sg->req, pos0 = sg->pos0;
  if (h->magic != kPlanMagic || h->hash != a.hash) return;
  const auto rq = as_uniform<ReqEntry>(a.plan + a.off_reqs) + req;
  // of a block's segments the first one does it
  if (pos0 % BLOCK != 0 && pos0 != rq->ctx_len) return;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int kvh = wg % a.head_groups * 4 + wave;
  if (kvh >= a.hkv) return;
  const int first = pos0 / BLOCK * BLOCK, len = rq->ctx_len + rq->q_len;
  const auto row = as_uniform<int32_t>(a.bt + (size_t)req * a.maxp);
  // rows past the last key read that one again
  const int last = min(first + BLOCK, len) - 1;
  u32x4 k[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    constexpr int PER_PAGE = 16 / ROWS;  // loads of a page
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

// ---------------------------------------------------------------------------
// Launches with a sparse plan.
struct SparseArgs {
  const uint8_t* plan;
  uint64_t hash;
  int32_t workgroups;
  int32_t hq, hkv, g, maxp;
  int32_t num_groups, off_rows, off_scores;
  int32_t block_keys, log_block;
  int32_t top, sink, recent, max_blocks;
  int32_t nsplit, split_entries;
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

__device__ __forceinline__ bool plan_ok(const SparseArgs& a) {
  const auto h = as_uniform<SparseHeader>(a.plan);
  return h->magic == kSparseMagic && h->hash == a.hash;
}

// One row: `unit` counts kRowGroup rows of every chunk record, then the single ones.
struct Row {
  int req, row, pos;
};
__device__ __forceinline__ bool take_row(const SparseArgs& a, int unit, Row* r) {
  const bool single = unit >= a.num_groups * kRowGroup;
  const int record = single ? a.num_groups + (unit - a.num_groups * kRowGroup) : unit / kRowGroup;
  const int j = single ? 0 : unit % kRowGroup;
  const auto x = as_uniform<SparseRows>(a.plan + a.off_rows) + record;
  r->req = x->req;
  r->row = x->row0 + j;
  r->pos = x->pos0 + j;
  return plan_ok(a) && j < x->n;
}

// ---------------------------------------------------------------------------
// Scores.  [max(q, 0), min(q, 0)] times [high, low]: a matrix product over 2 D, exact in its
// bf16 factors.  Blocks are the rows of the 16x16x32 products, (token, head) pairs of a kv
// head the columns, whole tokens in a tile; the highest of a token's heads is taken over
// its lanes.  A wave keeps two tiles of 16 blocks and goes over the item's columns.
template <int D>
__global__ __launch_bounds__(kSparseThreads) void block_scores_kernel(SparseArgs a) {
  constexpr int KS = D / 32;
  const int wg = workgroup_id();
  if (wg >= a.workgroups) return;
  const int kvh = wg % a.hkv;
  const auto it = as_uniform<SparseScore>(a.plan + a.off_scores) + wg / a.hkv;
  if (!plan_ok(a)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int r16 = lane & 15, quad = lane >> 4;
  const int tokens = 16 / a.g;  // of a tile
  const int token = r16 / a.g, head = r16 - token * a.g;
  const bool column = token < tokens;
  const int32_t* row = a.bt + (size_t)it->req * a.maxp;
  const int n = it->n, row0 = it->row0, pos0 = it->pos0, blk1 = it->blk1;
  for (int b0 = it->blk0 + wave * 32; b0 < blk1; b0 += kScorePass) {
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
    for (int j0 = 0; j0 < n; j0 += tokens) {
      const int j = j0 + token;
      const bool here = column && j < n;
      bf16x8 qf[2 * KS];
      const uint16_t* from =
          a.q + ((size_t)(row0 + (here ? j : 0)) * a.hq + kvh * a.g + (here ? head : 0)) * D + quad * 8;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const u32x4 v = ld16(from + k * 32);
        u32x4 plus, minus;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t m = negative_halves(v[w]);
          plus[w] = v[w] & ~m;
          minus[w] = v[w] & m;
        }
        qf[k] = as_bf16x8(plus);
        qf[KS + k] = as_bf16x8(minus);
      }
      f32x4 x[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int k = 0; k < 2 * KS; ++k)
#pragma unroll
        for (int t = 0; t < 2; ++t) x[t] = mfma(s[t][k], qf[k], x[t]);
      // the highest of heads head .. head + 2^i - 1, as far as the group goes
#pragma unroll
      for (int o = 1; o < 16; o *= 2) {
        if (o < a.g) {
          const bool more = head + o < a.g;
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float y = __shfl_down(x[t][i], o, 16);
              x[t][i] = more ? fmaxf(x[t][i], y) : x[t][i];
            }
        }
      }
      if (here && head == 0) {
        const int seen = ((pos0 + j) >> a.log_block) + 1;
        float* to = a.scores + ((size_t)(row0 + j) * a.hkv + kvh) * a.max_blocks;
        const int end = min(seen, blk1);
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const int b = b0 + t * 16 + quad * 4;
          if (b + 4 <= end) {
            *reinterpret_cast<f32x4*>(to + b) = x[t];
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (b + i < end) to[b + i] = x[t][i];
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
// a count of the lanes' mask per register.
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
  uint32_t k[NR];
  uint32_t any = 0, all = ~0u;
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const int b = first + i * 64;
    k[i] = kAbsent;
    if (b < n) {
      k[i] = order_key(from[b]);
      if (b < a.sink || b >= n - a.recent) {
        k[i] = kAlways;
      } else {
        any |= k[i];
        all &= k[i];
      }
    }
  }
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
#pragma unroll
    for (int i = 0; i < NR; ++i) c += (int)__popcll(__ballot(k[i] >= t));
    if constexpr (WAVES > 1) {
      turn ^= 1;
      if (lane == 0) s_count[turn][wave] = c;
      __syncthreads();
      c = 0;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) c += s_count[turn][w];
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
  int n_in = 0, n_eq = 0;
  const uint32_t above = exact ? t - 1 : t;  // t > 0: -infinity's key is
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    n_in += (int)__popcll(__ballot(k[i] > above));
    n_eq += (int)__popcll(__ballot(k[i] == t));
  }
  if (exact) n_eq = 0;
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
  const int quota = exact ? 0 : need - all_in;
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const bool in = k[i] > above, eq = !exact && k[i] == t;
    const uint64_t mi = __ballot(in), me = __ballot(eq);
    const int eq_at = before_eq + lanes_below(me);
    if (in || (eq && eq_at < quota))
      out[before_in + lanes_below(mi) + min(eq_at, quota)] = first + i * 64;
    before_in += (int)__popcll(mi);
    before_eq += (int)__popcll(me);
  }
}

// ---------------------------------------------------------------------------
// Attention.  One workgroup takes a piece of a row's list for one kv head.  Its pages (and
// how many of each one's slots the row sees) go to LDS, those of no block left out; the four
// waves take two pages (32 keys) each in turn.  The 16x16x32 products have keys as rows and
// the group's query heads as columns, and key r of a step is row (r & 3) + 4 (r >> 3) of
// product (r >> 2) & 1, so that the logits of a lane are those whose weights it multiplies
// with the values (dim-major pages) next.  Keys and values go from memory to registers, a
// step ahead.
constexpr int kPassPages = 512;  // pages in LDS at a time
constexpr uint32_t kMagnitudes = 0x7FFF7FFFu, kInfBits = 0x7F80u;  // above it: NaN
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t max_halves(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a),
                                                                __builtin_bit_cast(u16x2, b)));
}
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

template <int D>
struct AttentionLds {
  int2 page[kPassPages + 2];  // page, slots that count
  int part[2][4];
  float ml[2][4][16];
  float m[16], inv[16];
  int last;
  __attribute__((aligned(16))) float o[4 * 16 * D];
};

template <int D>
__global__ __launch_bounds__(kSparseThreads, 2) void sparse_attention_kernel(SparseArgs a) {
  constexpr int KS = D / 32, DT = D / 16;
  __shared__ AttentionLds<D> lds;
  const int wg = workgroup_id();
  if (wg >= a.workgroups) return;
  const int kvh = wg % a.hkv, split = wg / a.hkv % a.nsplit;
  Row r;
  if (!take_row(a, wg / a.hkv / a.nsplit, &r)) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, quad = lane >> 4;
  const size_t list = (size_t)r.row * a.hkv + kvh;
  const int32_t* blocks = a.blocks_in + list * a.top;
  const int32_t* table = a.bt + (size_t)r.req * a.maxp;
  const int log_pages = a.log_block - 4;
  const int page0 = (split * a.split_entries) << log_pages;
  const int page1 = min(a.top, (split + 1) * a.split_entries) << log_pages;

  bf16x8 qf[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    u32x4 v = {0, 0, 0, 0};
    if (r16 < a.g) v = ld16(a.q + ((size_t)r.row * a.hq + kvh * a.g + r16) * D + s * 32 + quad * 8);
    qf[s] = as_bf16x8(v);
  }
  float m = -kInf, l = 0.f;
  bool any = false;  // a key counts
  f32x4 o[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};

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

  for (int base = page0; base < page1; base += kPassPages) {
    // the pages of this pass, in the list's order
    int2 mine[2];
    uint64_t mask[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int p = base + i * kSparseThreads + tid;
      mine[i] = int2{0, 0};
      if (p < page1) {
        const int b = blocks[p >> log_pages];
        if (b >= 0 && b <= r.pos >> a.log_block) {
          const int at = (b << log_pages) + (p & ((1 << log_pages) - 1));  // page of the request
          if (at * 16 <= r.pos) mine[i] = int2{table[at], min(16, r.pos + 1 - at * 16)};
        }
      }
      mask[i] = __ballot(mine[i].y > 0);
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
      if (mine[i].y > 0) {
        lds.page[at[i]] = mine[i];
        // beside the last one of an odd number: the same page, none of its slots
        if (at[i] == total - 1 && total & 1) lds.page[total] = int2{mine[i].x, 0};
      }
    __syncthreads();
    total = __builtin_amdgcn_readfirstlane(total);
    if (total == 0) continue;
    any = true;
    const int steps = (total + 1) / 2;
    auto pages = [&](int s, int* p0, int* p1) {
      *p0 = __builtin_amdgcn_readfirstlane(lds.page[2 * s].x);
      *p1 = __builtin_amdgcn_readfirstlane(lds.page[2 * s + 1].x);
    };
    int p0 = 0, p1 = 0;
    if (wave < steps) {
      pages(wave, &p0, &p1);
      load_keys(p0, p1);
      load_values(p0, p1);
    }
    for (int s = wave; s < steps; s += 4) {
      const bool more = s + 4 < steps;
      if (more) pages(s + 4, &p0, &p1);
      const int c0 = __builtin_amdgcn_readfirstlane(lds.page[2 * s].y);
      const int c1 = __builtin_amdgcn_readfirstlane(lds.page[2 * s + 1].y);
      f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        s0 = mfma(as_bf16x8(kf[0][k]), qf[k], s0);
        s1 = mfma(as_bf16x8(kf[1][k]), qf[k], s1);
      }
      if (more) load_keys(p0, p1);
      __builtin_amdgcn_sched_barrier(0);
      float x[8] = {s0[0], s0[1], s0[2], s0[3], s1[0], s1[1], s1[2], s1[3]};
      const bool cut = c0 + c1 < 32;
      const int nv = (quad >> 1 ? c1 : c0) - 8 * (quad & 1);  // this lane's keys that count
      if (cut) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i >= nv) x[i] = -kInf;
      }
      float mx = x[0];
#pragma unroll
      for (int i = 1; i < 8; ++i) mx = fmaxf(mx, x[i]);
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float mn = mx == -kInf ? m : fmaxf(m, mx * a.c);
      const float ms = mn == -kInf ? 0.f : mn;
      const float alpha = exp2_fast(m - ms);
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = exp2_fast(__builtin_fmaf(x[i], a.c, -ms));
      if (cut) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (i >= nv) p[i] = 0.f;  // scale 0 times -inf is NaN
      }
      l = l * alpha + (((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7])));
      m = mn;
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
        for (int t = 0; t < DT; ++t) o[t] *= alpha;
      }
      if (cut) {
        // a slot that does not count may hold anything, and 0 times NaN is NaN
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            if (2 * w >= nv) vf[t][w] = 0;
            else if (2 * w + 1 >= nv) vf[t][w] &= 0xFFFFu;
          }
      }
#pragma unroll
      for (int t = 0; t < DT; ++t) o[t] = mfma(as_bf16x8(vf[t]), as_bf16x8(part[0]), o[t]);
      // An infinite value times a part that is zero or negative is not what it is times
      // the weight: the rounded weight alone has it.
      uint32_t most = 0;
#pragma unroll
      for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int w = 0; w < 4; ++w) most = max_halves(most, vf[t][w] & kMagnitudes);
      if (__any((most & 0xFFFFu) >= kInfBits || most >> 16 >= kInfBits)) {
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t v = vf[t][w] & kMagnitudes;
            if ((v & 0xFFFFu) >= kInfBits) vf[t][w] &= 0xFFFF0000u;
            if (v >> 16 >= kInfBits) vf[t][w] &= 0xFFFFu;
          }
      }
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        o[t] = mfma(as_bf16x8(vf[t]), as_bf16x8(part[1]), o[t]);
        o[t] = mfma(as_bf16x8(vf[t]), as_bf16x8(part[2]), o[t]);
      }
      if (more) load_values(p0, p1);
      __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();  // the pages have been read
  }

  // join the waves
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (quad == 0) {
    lds.ml[0][wave][r16] = m;
    lds.ml[1][wave][r16] = l;
  }
#pragma unroll
  for (int t = 0; t < DT; ++t)
    *reinterpret_cast<f32x4*>(lds.o + (wave * 16 + r16) * D + t * 16 + 4 * quad) = o[t];
  __syncthreads();
  const int rec_floats = sparse_rec_floats(a.g, D), rec_o = sparse_rec_o(a.g);
  float* records = a.nsplit > 1 ? a.records + list * a.nsplit * rec_floats : nullptr;
  if (tid < 16) {
    float mm = -kInf, ll = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) mm = fmaxf(mm, lds.ml[0][w][tid]);
    const float ms = mm == -kInf ? 0.f : mm;
#pragma unroll
    for (int w = 0; w < 4; ++w) ll += lds.ml[1][w][tid] * exp2_fast(lds.ml[0][w][tid] - ms);
    // no key: zeros; keys whose logits are all -infinity have no weights
    lds.m[tid] = ms;
    lds.inv[tid] = mm != -kInf ? 1.f / ll : any ? __builtin_nanf("") : 0.f;
    if (a.nsplit > 1 && tid < a.g) {
      float* rec = records + (int64_t)split * rec_floats;
      if (mm == -kInf && any) ll = 1.f;
      __hip_atomic_store(rec + tid, mm, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(rec + a.g + tid, ll, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
  __syncthreads();
  auto joined = [&](int g, int d) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w)
      v += *reinterpret_cast<const f32x4*>(lds.o + (w * 16 + g) * D + d) *
           exp2_fast(lds.ml[0][w][g] - lds.m[g]);
    return v;
  };
  uint16_t* out = a.out + ((size_t)r.row * a.hq + kvh * a.g) * D;
  auto store = [&](int e, f32x4 v) {
    *reinterpret_cast<u32x2*>(out + e) = u32x2{pack2(v[0], v[1]), pack2(v[2], v[3])};
  };
  if (a.nsplit == 1) {
    for (int e = tid * 4; e < a.g * D; e += kSparseThreads * 4)
      store(e, joined(e / D, e % D) * lds.inv[e / D]);
    return;
  }
  // A piece: its record goes past this die's cache (device scope) and has arrived before
  // the ticket is taken; the last piece to finish joins all of them in their order.
  {
    const PartWriter write(records + (int64_t)split * rec_floats + rec_o);
    for (int e = tid * 4; e < a.g * D; e += kSparseThreads * 4)
      write(e * 4, __builtin_bit_cast(u32x4, joined(e / D, e % D)));
  }
  vm_wait<0>();
  __syncthreads();
  if (tid == 0) {
    const int before = __hip_atomic_fetch_add(a.tickets + list, 1, __ATOMIC_RELAXED,
                                              __HIP_MEMORY_SCOPE_AGENT);
    lds.last = before == a.nsplit - 1;
    if (lds.last)
      __hip_atomic_store(a.tickets + list, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  if (!lds.last) return;
  auto get = [&](int64_t at) {
    return __hip_atomic_load(records + at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  };
  // weights of the pieces, then their sums
  float* weight = lds.o;  // [G][nsplit]
  if (tid < a.g) {
    float mm = -kInf, ll = 0.f, some = 0.f;
    for (int s = 0; s < a.nsplit; ++s) mm = fmaxf(mm, get((int64_t)s * rec_floats + tid));
    const float ms = mm == -kInf ? 0.f : mm;
    for (int s = 0; s < a.nsplit; ++s) {
      const float w = exp2_fast(get((int64_t)s * rec_floats + tid) - ms);
      const float ls = get((int64_t)s * rec_floats + a.g + tid);
      weight[tid * a.nsplit + s] = w;
      ll += ls * w;
      some += ls;
    }
    lds.inv[tid] = mm != -kInf ? 1.f / ll : some > 0.f ? __builtin_nanf("") : 0.f;
  }
  __syncthreads();
  for (int e = tid * 4; e < a.g * D; e += kSparseThreads * 4) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < a.nsplit; ++s) {
      const float w = weight[e / D * a.nsplit + s];
      const int64_t at = (int64_t)s * rec_floats + rec_o + e;
      v += f32x4{get(at), get(at + 1), get(at + 2), get(at + 3)} * w;
    }
    store(e, v * lds.inv[e / D]);
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
  a.block_keys = h->block_keys;
  a.log_block = log2_of(h->block_keys);
  a.top = h->top;
  a.sink = h->sink;
  a.recent = h->recent;
  a.max_blocks = h->max_blocks;
  a.nsplit = h->nsplit;
  a.split_entries = h->split_entries;
  a.c = h->softmax_scale * 1.44269504088896340736f;
  return a;
}

int32_t rows_of(const SparseHeader* h) { return h->num_groups * kRowGroup + h->num_singles; }

template <int D>
int launch_summary(const SummaryArgs& a, void* stream) {
  switch (a.block_keys) {
    case 16: return launch(block_summary_kernel<D, 16>, a, kSparseThreads, stream);
    case 32: return launch(block_summary_kernel<D, 32>, a, kSparseThreads, stream);
    case 64: return launch(block_summary_kernel<D, 64>, a, kSparseThreads, stream);
    default: return launch(block_summary_kernel<D, 128>, a, kSparseThreads, stream);
  }
}

}  // namespace

extern "C" {

int ssa_block_summary(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                      int32_t block_keys, const uint16_t* k_cache, const int32_t* block_table,
                      uint16_t* summary, void* stream) {
  const PlanHeader* h = nullptr;
  const int rc = check_plan(shape, plan_host, &h);
  if (rc) return rc;
  if (block_keys != 16 && block_keys != 32 && block_keys != 64 && block_keys != 128)
    return SSA_ERR_ARG;
  if (!plan_dev) return SSA_ERR_NULL;
  if (h->num_segments == 0) return SSA_OK;
  if (!k_cache || !block_table || !summary) return SSA_ERR_NULL;
  if (misaligned({k_cache, summary}) || misaligned_plan(plan_dev)) return SSA_ERR_ARG;
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
  const int64_t wgs = (int64_t)h->num_segments * a.head_groups;
  if (wgs > INT32_MAX) return SSA_ERR_ARG;
  a.workgroups = (int32_t)wgs;
  return h->head_dim == 128 ? launch_summary<128>(a, stream) : launch_summary<64>(a, stream);
}

int ssa_block_scores(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                     const uint16_t* q, const uint16_t* summary, const int32_t* block_table,
                     float* scores, void* stream) {
  const SparseHeader* h = nullptr;
  const int rc = check_sparse_plan(shape, plan_host, &h);
  if (rc) return rc;
  if (!plan_dev) return SSA_ERR_NULL;
  if (h->num_scores == 0) return SSA_OK;
  if (!q || !summary || !block_table || !scores) return SSA_ERR_NULL;
  if (misaligned({q, summary, scores}) || misaligned_plan(plan_dev)) return SSA_ERR_ARG;
  SparseArgs a = sparse_args(h, plan_dev);
  a.workgroups = h->num_scores * h->hkv;
  a.q = q;
  a.summary = summary;
  a.bt = block_table;
  a.scores = scores;
  return h->head_dim == 128 ? launch(block_scores_kernel<128>, a, kSparseThreads, stream)
                            : launch(block_scores_kernel<64>, a, kSparseThreads, stream);
}

int ssa_block_select(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                     const float* scores, int32_t* blocks, void* stream) {
  const SparseHeader* h = nullptr;
  const int rc = check_sparse_plan(shape, plan_host, &h);
  if (rc) return rc;
  if (!plan_dev) return SSA_ERR_NULL;
  if (h->num_tokens == 0) return SSA_OK;
  if (!scores || !blocks) return SSA_ERR_NULL;
  if (misaligned({scores, blocks}) || misaligned_plan(plan_dev)) return SSA_ERR_ARG;
  SparseArgs a = sparse_args(h, plan_dev);
  a.workgroups = rows_of(h) * h->hkv;
  a.scores_in = scores;
  a.blocks = blocks;
  // the longest list's waves and registers
  if (h->most_blocks <= 512) return launch(block_select_kernel<1, 8>, a, 64, stream);
  if (h->most_blocks <= 2048) return launch(block_select_kernel<4, 8>, a, 256, stream);
  if (h->most_blocks <= 8192) return launch(block_select_kernel<16, 8>, a, 1024, stream);
  return launch(block_select_kernel<16, 32>, a, 1024, stream);
}

int ssa_sparse_attention(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                         const uint16_t* q, const uint16_t* k_cache, const uint16_t* v_cache,
                         const int32_t* block_table, const int32_t* blocks, uint16_t* out,
                         void* workspace, size_t ws_bytes, void* stream) {
  const SparseHeader* h = nullptr;
  const int rc = check_sparse_plan(shape, plan_host, &h);
  if (rc) return rc;
  if (!plan_dev) return SSA_ERR_NULL;
  if (!workspace || ws_bytes < (size_t)h->ws_bytes) return SSA_ERR_WORKSPACE;
  if (h->num_tokens == 0) return SSA_OK;
  if (!q || !k_cache || !v_cache || !block_table || !blocks || !out) return SSA_ERR_NULL;
  if (misaligned({q, k_cache, v_cache, blocks, out, workspace}) || misaligned_plan(plan_dev))
    return SSA_ERR_ARG;
  SparseArgs a = sparse_args(h, plan_dev);
  a.workgroups = rows_of(h) * h->hkv * h->nsplit;
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
