// HIP kernels for gfx950 of ssa_evict_select and ssa_evict_compact
// (include/ssa_evict.h): which keys of a request and kv head stay, and their move
// to new pages.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <initializer_list>

#include "../../include/ssa_evict.h"
#include "ssa_device.h"
#include "ssa_evict_format.h"

namespace ssa {
int check_evict_plan(const ssa_shape* s, const void* plan_host, const EvictHeader** out);
}

namespace {
using namespace ssa;
using namespace ssa_dev;

struct EvictArgs {
  const uint8_t* plan;
  uint64_t hash;
  int32_t workgroups, off_items;  // of the launch, and where its items lie in the plan
  int32_t lists;                  // long lists
  int32_t hkv, maxp, sink, recent;
  const float* scores;
  const int32_t* bt;
  int32_t* keep;
  uint8_t* ws;
  int64_t ws_counts, ws_cands;
  // compaction
  const int32_t* keep_in;
  const int32_t* nt;
  uint16_t* kc;
  uint16_t* vc;
  float* scores_io;
};

__device__ __forceinline__ bool plan_ok(const EvictArgs& a) {
  const EvictHeader* h = reinterpret_cast<const EvictHeader*>(a.plan);
  return h->magic == kEvictMagic && h->hash == a.hash;
}
__device__ __forceinline__ int workgroup_id() {
  return (int)(blockIdx.y * gridDim.x + blockIdx.x);
}

// ---------------------------------------------------------------------------
// Selection.  Scores map to 32-bit keys in the same order.  The candidates (all but
// the first `sink` and the last `recent`) are searched for the key T of the last score
// that stays, by histograms of its bits from the highest on, and for how many of T's
// equals do; an ordered pass writes the indexes.

// A total order of scores: NaN as -infinity, -0 as +0.
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) x = -__builtin_huge_valf();
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ int lanes_below(uint64_t mask) {
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32),
                                        __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}
// Four keys of one page from index i on.
__device__ __forceinline__ u32x4 read_keys(const EvictArgs& a, const int32_t* row, int kvh, int i) {
  const f32x4 x = *reinterpret_cast<const f32x4*>(
      a.scores + ((size_t)row[i / 16] * a.hkv + kvh) * 16 + i % 16);
  return u32x4{order_key(x[0]), order_key(x[1]), order_key(x[2]), order_key(x[3])};
}

// Inclusive sum over the lanes of a wave, within the vector registers.
template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_add(int x) {
  return x + __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xF, false);
}
__device__ __forceinline__ int wave_scan(int x) {
  x = dpp_add<0x111, 0xF>(x);  // from the lane 1, 2, 4, 8 before, in rows of 16
  x = dpp_add<0x112, 0xF>(x);
  x = dpp_add<0x114, 0xF>(x);
  x = dpp_add<0x118, 0xF>(x);
  x = dpp_add<0x142, 0xA>(x);  // the last lane of the row before, to rows 1 and 3
  return dpp_add<0x143, 0xC>(x);  // lane 31, to rows 2 and 3
}

struct Found {
  int bin, above, in_bin;  // the bin, and how many lie above and in it
};
template <int THREADS>
struct FindLds {
  int part[THREADS / 64];
  Found found;
};
// The bin of a histogram in LDS, counted from its top, that holds the need-th entry
// (1 <= need <= entries).  All threads call it; the histogram may be written again
// after it.
template <int THREADS, int BINS>
__device__ __forceinline__ Found find_bin(const int* hist, int need, FindLds<THREADS>& lds) {
  constexpr int PER = BINS / THREADS;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int mine[PER], total = 0;
#pragma unroll
  for (int b = 0; b < PER; ++b) {
    mine[b] = hist[BINS - 1 - (tid * PER + b)];
    total += mine[b];
  }
  const int scan = wave_scan(total);
  if (lane == 63) lds.part[wave] = scan;
  __syncthreads();
  int above = scan - total;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) above += w < wave ? lds.part[w] : 0;
#pragma unroll
  for (int b = 0; b < PER; ++b) {
    if (above < need && above + mine[b] >= need)
      lds.found = Found{BINS - 1 - (tid * PER + b), above, mine[b]};
    above += mine[b];
  }
  __syncthreads();
  return lds.found;
}

// The flags of four keys: kept for sure, and equal to T.
struct Flags {
  bool in[4], eq[4];
};
// Indexes before these four of the lane, in the wave's lane-major order.
__device__ __forceinline__ void count_before(const Flags& f, int* in, int* eq, int* all_in,
                                             int* all_eq) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint64_t bi = __ballot(f.in[j]), be = __ballot(f.eq[j]);
    *in += lanes_below(bi);
    *eq += lanes_below(be);
    *all_in += (int)__popcll(bi);
    *all_eq += (int)__popcll(be);
  }
}

// Short lists: one workgroup, four 4-key groups a thread in registers.  It is a chain of
// latencies (plan, table, scores, then histograms of 11, 11 and 10 bits, of which
// the last is left out where all of a bin stays): 512 lists of 600 to 4096 keys, of
// which 1000 stay, take 9.3 us (with a scan over the waves in a loop 15.8).
constexpr int kShortThreads = 512;
constexpr int kShortGroups = kShortList / 4 / kShortThreads;
constexpr int kShortBins = 2048;

__global__ __launch_bounds__(kShortThreads) void evict_select_kernel(EvictArgs a) {
  constexpr int THREADS = kShortThreads, WAVES = THREADS / 64, NG = kShortGroups;
  __shared__ int s_hist[kShortBins];
  __shared__ FindLds<THREADS> s_find;
  __shared__ int s_count[NG * WAVES];
  const int wg = workgroup_id();
  if (wg >= a.workgroups || !plan_ok(a)) return;
  const EvictShort rq = reinterpret_cast<const EvictShort*>(a.plan + a.off_items)[wg / a.hkv];
  const int kvh = wg % a.hkv, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int32_t* out = a.keep + rq.keep_off * a.hkv + (int64_t)kvh * rq.kept;
  const int len = rq.len;
  if (rq.kept == len) {
    for (int i = tid; i < len; i += THREADS) out[i] = i;
    return;
  }
  const int32_t* row = a.bt + (size_t)rq.req * a.maxp;
  const int lo = a.sink, hi = len - a.recent;  // candidates
  int need = rq.kept - a.sink - a.recent;      // of which this many stay
  const int groups = (len + THREADS * 4 - 1) / (THREADS * 4);  // that hold keys
  u32x4 k[NG];
#pragma unroll
  for (int n = 0; n < NG; ++n) {
    const int i = (n * THREADS + tid) * 4;
    k[n] = i < len ? read_keys(a, row, kvh, i) : u32x4{0, 0, 0, 0};
  }
  uint32_t t = 0xFFFFFFFFu;  // above every score's key
  if (need > 0) {
    t = 0;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
      const uint32_t digits = pass == 2 ? 1023u : 2047u;
      const uint32_t done = pass == 0 ? 0u : pass == 1 ? ~0u << 21 : ~0u << 10;
      for (int b = tid; b < kShortBins; b += THREADS) s_hist[b] = 0;
      __syncthreads();
#pragma unroll
      for (int n = 0; n < NG; ++n) {
        if (n >= groups) break;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int i = (n * THREADS + tid) * 4 + j;
          if (i >= lo && i < hi && (k[n][j] & done) == t)
            atomicAdd(&s_hist[(k[n][j] >> shift) & digits], 1);
        }
      }
      __syncthreads();
      const Found f = find_bin<THREADS, kShortBins>(s_hist, need, s_find);
      t |= (uint32_t)f.bin << shift;
      need -= f.above;
      if (f.in_bin == need) {  // the whole bin stays: every key above t - 1
        t -= 1;                // t is not 0: -infinity's key is not
        need = 0;
        break;
      }
    }
  }
  auto flags = [&](int n) {
    Flags f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = (n * THREADS + tid) * 4 + j;
      const bool cand = i >= lo && i < hi;
      f.in[j] = i < len && (!cand || k[n][j] > t);
      f.eq[j] = i < len && cand && k[n][j] == t;
    }
    return f;
  };
  // kept and equal ones before each wave's keys of each group, in one scan of the
  // NG x WAVES pairs (16 bits each hold a list's length)
  static_assert(NG * WAVES <= 64 && kShortList < 1 << 15, "one wave, one word");
  int before_in[NG], before_eq[NG];
#pragma unroll
  for (int n = 0; n < NG; ++n) {
    if (n >= groups) break;
    int all_in = 0, all_eq = 0;
    before_in[n] = before_eq[n] = 0;
    count_before(flags(n), &before_in[n], &before_eq[n], &all_in, &all_eq);
    if (lane == 0) s_count[n * WAVES + wave] = all_in | all_eq << 16;
  }
  __syncthreads();
  const int mine = lane < groups * WAVES ? s_count[lane] : 0, scan = wave_scan(mine) - mine;
#pragma unroll
  for (int n = 0; n < NG; ++n) {
    if (n >= groups) break;
    const int before = __builtin_amdgcn_readlane(scan, n * WAVES + wave);
    before_in[n] += before & 0xFFFF;
    before_eq[n] += before >> 16;
    const Flags f = flags(n);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (f.in[j] || (f.eq[j] && before_eq[n] < need))
        out[before_in[n] + min(before_eq[n], need)] = (n * THREADS + tid) * 4 + j;
      before_in[n] += f.in[j];
      before_eq[n] += f.eq[j];
    }
  }
}

// Long lists: segments of 8192 keys, four launches (clear, histogram, candidates, write),
// because one workgroup would read a list at one compute unit's rate (8 lists of 131072
// keys: 123 us in one workgroup each, 2.5 + 5 + 9 + 9 us in these).
//   histogram   of the first 12 bits, added up over the segments (integers: their
//               order does not matter);
//   candidates  every segment finds the threshold's bin, counts what lies above it
//               and lists the scores in it, (key, index) in one word that orders them;
//   write       every segment finds the last candidate that stays (few: about 1 in
//               200 where scores spread over a dozen octaves), and from the counts and
//               the candidates before it the place of its first index.  Segments times
//               candidates: 8 lists of 131072 take 28 us of spread scores, 80 of scores
//               from 1.0 to 1.2, 575 of equal ones.
constexpr int kSegThreads = 512;
constexpr int kSegGroups = kSegKeys / 4 / kSegThreads;
constexpr int kCandDigit = 10, kCandBins = 1 << kCandDigit;
constexpr int kCandHeld = 4096;  // candidates held in LDS; more are read again

__device__ __forceinline__ int* seg_hist(const EvictArgs& a, int list) {
  return reinterpret_cast<int*>(a.ws) + (int64_t)list * kSegBins;
}
__device__ __forceinline__ SegState* seg_state(const EvictArgs& a, int list) {
  return reinterpret_cast<SegState*>(a.ws + (int64_t)a.lists * kSegBins * 4) + list;
}
// (key, index), the higher the better: the lower index of equal keys first.
__device__ __forceinline__ uint64_t cand_word(uint32_t key, int i) {
  return (uint64_t)key << 32 | (uint32_t)~i;
}

__global__ __launch_bounds__(256) void evict_clear_kernel(EvictArgs a) {
  if (!plan_ok(a)) return;
  const int64_t words = (int64_t)a.lists * (kSegBins + sizeof(SegState) / 4);
  for (int64_t i = ((int64_t)workgroup_id() * 256 + threadIdx.x) * 4; i < words;
       i += (int64_t)a.workgroups * 1024)
    *reinterpret_cast<u32x4*>(a.ws + i * 4) = u32x4{0, 0, 0, 0};
}

struct SegWork {
  EvictSeg sg;
  int kvh, list, tid;
  int lo, hi, end;  // candidates are lo .. hi - 1; the segment's keys end before `end`
  u32x4 k[kSegGroups];
};
__device__ __forceinline__ int seg_index(const SegWork& w, int n) {
  return w.sg.key0 + (n * kSegThreads + w.tid) * 4;
}
__device__ __forceinline__ bool seg_work(const EvictArgs& a, SegWork* w) {
  const int wg = workgroup_id();
  if (wg >= a.workgroups || !plan_ok(a)) return false;
  w->sg = reinterpret_cast<const EvictSeg*>(a.plan + a.off_items)[wg / a.hkv];
  w->kvh = wg % a.hkv;
  w->list = w->sg.long_index * a.hkv + w->kvh;
  w->tid = threadIdx.x;
  w->lo = a.sink;
  w->hi = w->sg.len - a.recent;
  w->end = min(w->sg.len, w->sg.key0 + kSegKeys);
  const int32_t* row = a.bt + (size_t)w->sg.req * a.maxp;
#pragma unroll
  for (int n = 0; n < kSegGroups; ++n) {
    const int i = seg_index(*w, n);
    w->k[n] = i < w->end ? read_keys(a, row, w->kvh, i) : u32x4{0, 0, 0, 0};
  }
  return true;
}

__global__ __launch_bounds__(kSegThreads) void evict_histogram_kernel(EvictArgs a) {
  __shared__ int s_hist[kSegBins];
  SegWork w;
  if (!seg_work(a, &w)) return;
  for (int b = w.tid; b < kSegBins; b += kSegThreads) s_hist[b] = 0;
  __syncthreads();
#pragma unroll
  for (int n = 0; n < kSegGroups; ++n)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = seg_index(w, n) + j;
      if (i >= w.lo && i < w.hi && i < w.end) atomicAdd(&s_hist[w.k[n][j] >> 20], 1);
    }
  __syncthreads();
  int* hist = seg_hist(a, w.list);
  for (int b = w.tid; b < kSegBins; b += kSegThreads)
    if (s_hist[b]) atomicAdd(hist + b, s_hist[b]);
}

__global__ __launch_bounds__(kSegThreads) void evict_candidates_kernel(EvictArgs a) {
  constexpr int WAVES = kSegThreads / 64;
  __shared__ __attribute__((aligned(16))) int s_hist[kSegBins];
  __shared__ FindLds<kSegThreads> s_find;
  __shared__ int s_in[WAVES], s_eq[WAVES], s_base;
  SegWork w;
  if (!seg_work(a, &w)) return;
  const int* hist = seg_hist(a, w.list);
  for (int b = w.tid * 4; b < kSegBins; b += kSegThreads * 4)
    *reinterpret_cast<u32x4*>(s_hist + b) = ld16(hist + b);
  __syncthreads();
  const int need = w.sg.kept - a.sink - a.recent;
  Found f{kSegBins, 0, 0};  // nothing but sinks and recent keys stays: above every bin
  if (need > 0) f = find_bin<kSegThreads, kSegBins>(s_hist, need, s_find);
  SegState* state = seg_state(a, w.list);
  if (w.sg.key0 == 0 && w.tid == 0) {
    state->bin = f.bin;
    state->need = need - f.above;
  }
  const int lane = w.tid & 63, wave = w.tid >> 6;
  int n_in = 0, n_eq = 0, before[kSegGroups];
#pragma unroll
  for (int n = 0; n < kSegGroups; ++n) {
    before[n] = n_eq;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = seg_index(w, n) + j, bin = (int)(w.k[n][j] >> 20);
      const bool cand = i >= w.lo && i < w.hi;
      const uint64_t eq = __ballot(i < w.end && cand && bin == f.bin);
      n_in += (int)__popcll(__ballot(i < w.end && (!cand || bin > f.bin)));
      n_eq += (int)__popcll(eq);
    }
  }
  if (lane == 0) {
    s_in[wave] = n_in;
    s_eq[wave] = n_eq;
  }
  __syncthreads();
  if (w.tid == 0) {
    int in = 0, eq = 0;
    for (int x = 0; x < WAVES; ++x) {
      in += s_in[x];
      eq += s_eq[x];
    }
    reinterpret_cast<int*>(a.ws + a.ws_counts)[((int64_t)w.sg.seg0 + w.sg.key0 / kSegKeys) * a.hkv + w.kvh] =
        in;
    s_base = eq ? atomicAdd(&state->num_cands, eq) : 0;
  }
  __syncthreads();
  int base = s_base;
  for (int x = 0; x < wave; ++x) base += s_eq[x];
  uint64_t* cands = reinterpret_cast<uint64_t*>(a.ws + a.ws_cands) + w.sg.cand_off * a.hkv +
                    (int64_t)w.kvh * w.sg.len;
#pragma unroll
  for (int n = 0; n < kSegGroups; ++n) {
    int at = base + before[n];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = seg_index(w, n) + j;
      const bool eq = i < w.end && i >= w.lo && i < w.hi && (int)(w.k[n][j] >> 20) == f.bin;
      const uint64_t mask = __ballot(eq);
      if (eq) cands[at + lanes_below(mask)] = cand_word(w.k[n][j], i);
      at += (int)__popcll(mask);
    }
  }
}

__global__ __launch_bounds__(kSegThreads) void evict_write_kernel(EvictArgs a) {
  constexpr int WAVES = kSegThreads / 64, NG = kSegGroups;
  __shared__ uint64_t s_cand[kCandHeld];
  __shared__ int s_hist[kCandBins];
  __shared__ FindLds<kSegThreads> s_find;
  __shared__ int s_in[NG * WAVES], s_before;
  SegWork w;
  if (!seg_work(a, &w)) return;
  const SegState st = *seg_state(a, w.list);
  const uint64_t* cands = reinterpret_cast<const uint64_t*>(a.ws + a.ws_cands) +
                          w.sg.cand_off * a.hkv + (int64_t)w.kvh * w.sg.len;
  const int held = min(st.num_cands, kCandHeld);
  for (int c = w.tid; c < held; c += kSegThreads) s_cand[c] = cands[c];
  if (w.tid == 0) s_before = 0;
  // the word of the last candidate that stays: its 20 lower key bits, then the index
  uint64_t t = (uint64_t)st.bin << 52;
  int need = st.need;
  if (need > 0 && need < st.num_cands) {
    for (int shift = 52 - kCandDigit; shift > -kCandDigit; shift -= kCandDigit) {
      const int sh = max(shift, 0);
      const uint64_t done = ~0ull << (shift + kCandDigit);
      for (int b = w.tid; b < kCandBins; b += kSegThreads) s_hist[b] = 0;
      __syncthreads();
      for (int c = w.tid; c < st.num_cands; c += kSegThreads) {
        const uint64_t x = c < kCandHeld ? s_cand[c] : cands[c];
        // the last digit has fewer bits: those of the digit before it are t's
        if ((x & done) == (t & done)) atomicAdd(&s_hist[(x >> sh) & (kCandBins - 1)], 1);
      }
      __syncthreads();
      const Found f = find_bin<kSegThreads, kCandBins>(s_hist, need, s_find);
      t = (t & done) | (uint64_t)f.bin << sh;
      need -= f.above;
      if (f.in_bin == need) break;  // every candidate from t on stays
    }
  } else if (need <= 0) {
    t = ~0ull;  // no candidate does
  }
  // what stays before this segment
  __syncthreads();
  int n = 0;
  const int* counts = reinterpret_cast<const int*>(a.ws + a.ws_counts) + (int64_t)w.sg.seg0 * a.hkv + w.kvh;
  for (int s = w.tid; s < w.sg.key0 / kSegKeys; s += kSegThreads) n += counts[(int64_t)s * a.hkv];
  for (int c = w.tid; c < st.num_cands; c += kSegThreads) {
    const uint64_t x = c < kCandHeld ? s_cand[c] : cands[c];
    n += x >= t && (int)~(uint32_t)x < w.sg.key0;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
  const int lane = w.tid & 63, wave = __builtin_amdgcn_readfirstlane(w.tid >> 6);
  if (lane == 0 && n) atomicAdd(&s_before, n);
  int before[NG];
  auto keep = [&](int g, int j) {
    const int i = seg_index(w, g) + j, bin = (int)(w.k[g][j] >> 20);
    if (i >= w.end) return false;
    if (i < w.lo || i >= w.hi) return true;
    return bin > st.bin || (bin == st.bin && cand_word(w.k[g][j], i) >= t);
  };
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    int all = 0;
    before[g] = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint64_t mask = __ballot(keep(g, j));
      before[g] += lanes_below(mask);
      all += (int)__popcll(mask);
    }
    if (lane == 0) s_in[g * WAVES + wave] = all;
  }
  __syncthreads();
  static_assert(NG * WAVES <= 64, "one wave");
  int32_t* out = a.keep + w.sg.keep_off * a.hkv + (int64_t)w.kvh * w.sg.kept + s_before;
  const int mine = lane < NG * WAVES ? s_in[lane] : 0, scan = wave_scan(mine) - mine;
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    before[g] += __builtin_amdgcn_readlane(scan, g * WAVES + wave);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (keep(g, j)) out[before[g]++] = seg_index(w, g) + j;
  }
}

// ---------------------------------------------------------------------------
// Compaction: one workgroup moves 64 kept keys of a kv head (four new pages).
// Keys are whole 2 D-byte rows.  Values lie dim-major, so a kept key is one
// 2-byte element of each of a page's D rows: a thread gathers the 8 elements of one
// 16-byte piece of a new page's row, neighbours from the same old rows.  A page with
// one kept key is read whole (32-byte rows), so that cutting long contexts to a
// quarter reads most of the values: 32 contexts of 8k to 33k keys cut to 8192, 64/8
// heads, read 1.83 GB for 1.08 GB that stay and write those, in 517 to 590 us on
// different cards (4.9 to 5.6 TB/s; with loads and stores by turns 651 us).  Every load is issued before the first store; a
// slot that is not followed loads from the first page and stores nothing.
template <int D>
__global__ __launch_bounds__(256) void evict_compact_kernel(EvictArgs a) {
  constexpr int CPR = D / 8, PER = kEvictSlots * CPR / 256;
  __shared__ int s_page[kEvictSlots], s_slot[kEvictSlots];
  __shared__ uint64_t s_valid;
  const int wg = workgroup_id();
  if (wg >= a.workgroups || !plan_ok(a)) return;
  const EvictItem it = reinterpret_cast<const EvictItem*>(a.plan + a.off_items)[wg / a.hkv];
  const int kvh = wg % a.hkv, tid = threadIdx.x;
  const int32_t* old_row = a.bt + (size_t)it.req * a.maxp;
  const int32_t* new_row = a.nt + (size_t)it.req * a.maxp + it.slot0 / 16;
  float score = 0.f;
  if (tid < kEvictSlots) {  // the first wave
    int key = -1;
    if (tid < it.n)
      key = a.keep_in[it.keep_off * a.hkv + (int64_t)kvh * it.kept + it.slot0 + tid];
    const bool valid = key >= 0 && key < it.len;
    const int page = valid ? old_row[key / 16] : 0, slot = valid ? key % 16 : 0;
    s_page[tid] = page;
    s_slot[tid] = slot;
    const uint64_t mask = __ballot(valid);
    if (tid == 0) s_valid = mask;
    if (valid && a.scores_io) score = a.scores_io[((size_t)page * a.hkv + kvh) * 16 + slot];
  }
  __syncthreads();
  const uint64_t valid = s_valid;
  // keys: 16-byte piece p % CPR of slot p / CPR; values: piece p is dims p / 2 % D,
  // slots 8 (p & 1) .. + 7 of new page p / (2 D)
  u32x4 k[PER];
  uint16_t e[PER][8];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int p = tid + i * 256, s = p / CPR;
    k[i] = ld16(a.kc + (((size_t)s_page[s] * a.hkv + kvh) * 16 + s_slot[s]) * D + p % CPR * 8);
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int p = tid + i * 256, d = p / 2 % D, s0 = p / (2 * D) * 16 + (p & 1) * 8;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      e[i][j] = a.vc[((size_t)s_page[s0 + j] * a.hkv + kvh) * 16 * D + (size_t)d * 16 + s_slot[s0 + j]];
  }
  __builtin_amdgcn_sched_barrier(0);
  if (tid < kEvictSlots && (valid >> tid & 1) && a.scores_io)
    a.scores_io[((size_t)new_row[tid / 16] * a.hkv + kvh) * 16 + tid % 16] = score;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int p = tid + i * 256, s = p / CPR;
    if (valid >> s & 1)
      st16(a.kc + (((size_t)new_row[s / 16] * a.hkv + kvh) * 16 + s % 16) * D + p % CPR * 8, k[i]);
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int p = tid + i * 256, page = p / (2 * D), d = p / 2 % D;
    const uint32_t here = valid >> (page * 16 + (p & 1) * 8) & 0xFF;
    if (!here) continue;
    uint16_t* to = a.vc + ((size_t)new_row[page] * a.hkv + kvh) * 16 * D + (size_t)d * 16 + (p & 1) * 8;
    if (here == 0xFF) {
      u32x4 v;
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = e[i][2 * j] | (uint32_t)e[i][2 * j + 1] << 16;
      st16(to, v);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (here >> j & 1) to[j] = e[i][j];
    }
  }
}

constexpr int kGridRow = 1 << 16;  // workgroups in a row of the grid (2^32 threads at most)

template <class K>
int launch(K kernel, const EvictArgs& a, int threads, hipStream_t stream) {
  if (a.workgroups == 0) return SSA_OK;
  (void)hipGetLastError();
  const int64_t wgs = a.workgroups;
  const dim3 grid(wgs < kGridRow ? wgs : kGridRow, (wgs + kGridRow - 1) / kGridRow);
  hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, stream, a);
  return hipGetLastError() == hipSuccess ? SSA_OK : SSA_ERR_HIP;
}

// Pages are read and written 16 bytes at a time.
bool misaligned(std::initializer_list<const void*> pointers) {
  for (const void* p : pointers)
    if (reinterpret_cast<uintptr_t>(p) % 16) return true;
  return false;
}

// Items hold 64-bit fields.
bool misaligned_plan(const void* plan_dev) {
  return reinterpret_cast<uintptr_t>(plan_dev) % 8 != 0;
}

EvictArgs evict_args(const EvictHeader* h, const void* plan_dev, const int32_t* block_table) {
  EvictArgs a{};
  a.plan = static_cast<const uint8_t*>(plan_dev);
  a.hash = h->hash;
  a.off_items = h->off_items;
  a.hkv = h->hkv;
  a.maxp = h->max_pages_per_req;
  a.sink = h->sink;
  a.recent = h->recent;
  a.bt = block_table;
  return a;
}

}  // namespace

extern "C" {

int ssa_evict_select(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                     const float* scores, const int32_t* block_table, int32_t* keep,
                     void* workspace, size_t ws_bytes, void* stream) {
  const EvictHeader* h = nullptr;
  int rc = check_evict_plan(shape, plan_host, &h);
  if (rc) return rc;
  if (!plan_dev) return SSA_ERR_NULL;
  if (h->num_keep > 0 && (!scores || !block_table || !keep)) return SSA_ERR_NULL;
  if (!workspace || ws_bytes < (size_t)h->ws_bytes) return SSA_ERR_WORKSPACE;
  if (misaligned({scores, workspace})) return SSA_ERR_ARG;
  if (h->num_keep == 0) return SSA_OK;
  if (misaligned_plan(plan_dev)) return SSA_ERR_ARG;
  EvictArgs a = evict_args(h, plan_dev, block_table);
  a.scores = scores;
  a.keep = keep;
  a.ws = static_cast<uint8_t*>(workspace);
  a.ws_counts = h->ws_counts;
  a.ws_cands = h->ws_cands;
  a.lists = h->num_long * h->hkv;
  hipStream_t s = static_cast<hipStream_t>(stream);
  a.workgroups = h->num_short * h->hkv;
  a.off_items = h->off_short;
  rc = launch(evict_select_kernel, a, kShortThreads, s);
  if (rc || a.lists == 0) return rc;
  // 16 KB of histogram a list, in workgroups of 4 KB at a time
  a.workgroups = std::min(a.lists * 4, 1024);
  if ((rc = launch(evict_clear_kernel, a, 256, s))) return rc;
  a.workgroups = h->num_segs * h->hkv;
  a.off_items = h->off_segs;
  if ((rc = launch(evict_histogram_kernel, a, kSegThreads, s))) return rc;
  if ((rc = launch(evict_candidates_kernel, a, kSegThreads, s))) return rc;
  return launch(evict_write_kernel, a, kSegThreads, s);
}

int ssa_evict_compact(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                      const int32_t* keep, const int32_t* block_table, const int32_t* new_table,
                      uint16_t* k_cache, uint16_t* v_cache, float* scores, void* stream) {
  const EvictHeader* h = nullptr;
  const int rc = check_evict_plan(shape, plan_host, &h);
  if (rc) return rc;
  if (!plan_dev) return SSA_ERR_NULL;
  if (h->num_items == 0) return SSA_OK;
  if (!keep || !block_table || !new_table || !k_cache || !v_cache) return SSA_ERR_NULL;
  if (misaligned({k_cache, v_cache}) || misaligned_plan(plan_dev)) return SSA_ERR_ARG;
  EvictArgs a = evict_args(h, plan_dev, block_table);
  a.workgroups = h->num_items * h->hkv;
  a.keep_in = keep;
  a.nt = new_table;
  a.kc = k_cache;
  a.vc = v_cache;
  a.scores_io = scores;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return h->head_dim == 128 ? launch(evict_compact_kernel<128>, a, 256, s)
                            : launch(evict_compact_kernel<64>, a, 256, s);
}

}  // extern "C"
