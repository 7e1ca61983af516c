// HIP kernels for gfx950 of ssa_evict_select and ssa_evict_compact
// (include/ssa_evict.h): which keys of a request and kv head stay, and their move
// to new pages.
#include <hip/hip_runtime.h>
#include <stdint.h>

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
  int32_t workgroups, off_items;
  int32_t hkv, maxp, sink, recent;
  const float* scores;
  const int32_t* bt;
  int32_t* keep;
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
// Selection: one workgroup a list.  Scores map to 32-bit keys in the same order;
// three histogram passes (11, 11, 10 bits, highest first) find the key T of the
// last score that stays and how many of its equals do; one ordered pass writes the
// indexes.  Keys are held in LDS, up to CAP of them; longer lists read the others
// again from the cache.
constexpr int kBins = 2048;

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

template <int THREADS, int CAP>
__global__ __launch_bounds__(THREADS) void evict_select_kernel(EvictArgs a) {
  constexpr int WAVES = THREADS / 64, BPT = kBins / THREADS;
  __shared__ __attribute__((aligned(16))) uint32_t s_key[CAP];
  __shared__ int s_hist[kBins];
  __shared__ int s_part[WAVES], s_eq[WAVES];
  __shared__ int s_bin, s_above;
  const int wg = workgroup_id();
  if (wg >= a.workgroups || !plan_ok(a)) return;
  const EvictReq rq = reinterpret_cast<const EvictReq*>(a.plan + sizeof(EvictHeader))[wg / a.hkv];
  const int kvh = wg % a.hkv, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int32_t* out = a.keep + rq.keep_off * a.hkv + (int64_t)kvh * rq.kept;
  const int len = rq.len;
  if (rq.kept == len) {
    for (int i = tid; i < len; i += THREADS) out[i] = i;
    return;
  }
  const int32_t* row = a.bt + (size_t)(wg / a.hkv) * a.maxp;
  const int lo = a.sink, hi = len - a.recent;  // candidates
  int need = rq.kept - a.sink - a.recent;      // of which this many stay

  // four scores of one page
  auto read4 = [&](int i) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(
        a.scores + ((size_t)row[i / 16] * a.hkv + kvh) * 16 + i % 16);
    return u32x4{order_key(x[0]), order_key(x[1]), order_key(x[2]), order_key(x[3])};
  };
  auto keys4 = [&](int i) {
    return i < CAP ? *reinterpret_cast<const u32x4*>(s_key + i) : read4(i);
  };
  for (int i = tid * 4; i < len && i < CAP; i += THREADS * 4)
    *reinterpret_cast<u32x4*>(s_key + i) = read4(i);

  uint32_t prefix = 0;  // the bits of T found so far
  if (need > 0) {
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
      const uint32_t digit_mask = pass == 2 ? 1023u : 2047u;
      const uint32_t done = pass == 0 ? 0u : pass == 1 ? ~0u << 21 : ~0u << 10;
#pragma unroll
      for (int b = 0; b < BPT; ++b) s_hist[b * THREADS + tid] = 0;
      __syncthreads();
      for (int i = tid * 4; i < len; i += THREADS * 4) {
        const u32x4 k = keys4(i);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (i + j >= lo && i + j < hi && (k[j] & done) == prefix)
            atomicAdd(&s_hist[(k[j] >> shift) & digit_mask], 1);
      }
      __syncthreads();
      // thread t owns bins from the top: kBins - 1 - t BPT downwards
      int mine[BPT], total = 0;
#pragma unroll
      for (int b = 0; b < BPT; ++b) {
        mine[b] = s_hist[kBins - 1 - (tid * BPT + b)];
        total += mine[b];
      }
      int scan = total;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(scan, o, 64);
        if (lane >= o) scan += v;
      }
      if (lane == 63) s_part[wave] = scan;
      __syncthreads();
      int above = scan - total;
      for (int w = 0; w < wave; ++w) above += s_part[w];
#pragma unroll
      for (int b = 0; b < BPT; ++b) {
        if (above < need && above + mine[b] >= need) {
          s_bin = kBins - 1 - (tid * BPT + b);
          s_above = above;
        }
        above += mine[b];
      }
      __syncthreads();
      prefix |= (uint32_t)s_bin << shift;
      need -= s_above;
    }
  } else {
    prefix = 0xFFFFFFFFu;  // above every score's key: no candidate stays
    __syncthreads();
  }

  // Each wave takes a run of 256-key units, counts what stays above T and equal to
  // it, and after a scan over the waves writes its indexes in order.
  const int units = (len + 255) / 256, per = (units + WAVES - 1) / WAVES;
  const int u0 = wave * per, u1 = min(units, u0 + per);
  auto flags = [&](int i, bool* in, bool* eq) {
    u32x4 k = {0, 0, 0, 0};
    if (i < len) k = keys4(i);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int at = i + j;
      const bool cand = at >= lo && at < hi;
      in[j] = at < len && (!cand || k[j] > prefix);
      eq[j] = at < len && cand && k[j] == prefix;
    }
  };
  int n_in = 0, n_eq = 0;
  for (int u = u0; u < u1; ++u) {
    bool in[4], eq[4];
    flags(u * 256 + lane * 4, in, eq);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      n_in += (int)__popcll(__ballot(in[j]));
      n_eq += (int)__popcll(__ballot(eq[j]));
    }
  }
  if (lane == 0) {
    s_part[wave] = n_in;
    s_eq[wave] = n_eq;
  }
  __syncthreads();
  n_in = n_eq = 0;
  for (int w = 0; w < wave; ++w) {
    n_in += s_part[w];
    n_eq += s_eq[w];
  }
  for (int u = u0; u < u1; ++u) {
    const int i = u * 256 + lane * 4;
    bool in[4], eq[4];
    flags(i, in, eq);
    int before_in = n_in, before_eq = n_eq;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint64_t bi = __ballot(in[j]), be = __ballot(eq[j]);
      before_in += lanes_below(bi);
      before_eq += lanes_below(be);
      n_in += (int)__popcll(bi);
      n_eq += (int)__popcll(be);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (in[j] || (eq[j] && before_eq < need)) out[before_in + min(before_eq, need)] = i + j;
      before_in += in[j];
      before_eq += eq[j];
    }
  }
}

// ---------------------------------------------------------------------------
// Compaction: one workgroup moves 64 kept keys of a kv head (four new pages).
// Keys are whole 2 D-byte rows.  Values lie dim-major, so a kept key is one
// 2-byte element of each of a page's D rows: a thread gathers the 8 elements of one
// 16-byte piece of a new page's row, neighbours from the same old rows.
template <int D>
__global__ __launch_bounds__(256) void evict_compact_kernel(EvictArgs a) {
  constexpr int CPR = D / 8, PER = kEvictSlots * CPR / 256;
  __shared__ int s_page[kEvictSlots], s_slot[kEvictSlots];
  const int wg = workgroup_id();
  if (wg >= a.workgroups || !plan_ok(a)) return;
  const EvictItem it = reinterpret_cast<const EvictItem*>(a.plan + a.off_items)[wg / a.hkv];
  const int kvh = wg % a.hkv, tid = threadIdx.x;
  const int32_t* old_row = a.bt + (size_t)it.req * a.maxp;
  const int32_t* new_row = a.nt + (size_t)it.req * a.maxp + it.slot0 / 16;
  if (tid < kEvictSlots) {
    int page = -1, slot = 0;
    if (tid < it.n) {
      const int key = a.keep_in[it.keep_off * a.hkv + (int64_t)kvh * it.kept + it.slot0 + tid];
      if (key >= 0 && key < it.len) {
        page = old_row[key / 16];
        slot = key % 16;
      }
    }
    s_page[tid] = page;
    s_slot[tid] = slot;
    if (page >= 0 && a.scores_io) {
      const size_t to = ((size_t)new_row[tid / 16] * a.hkv + kvh) * 16 + tid % 16;
      a.scores_io[to] = a.scores_io[((size_t)page * a.hkv + kvh) * 16 + slot];
    }
  }
  __syncthreads();
  // keys: all loads, then all stores
  u32x4 v[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int p = tid + i * 256, s = p / CPR;
    if (s_page[s] >= 0)
      v[i] = ld16(a.kc + (((size_t)s_page[s] * a.hkv + kvh) * 16 + s_slot[s]) * D + p % CPR * 8);
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int p = tid + i * 256, s = p / CPR;
    if (s_page[s] >= 0)
      st16(a.kc + (((size_t)new_row[s / 16] * a.hkv + kvh) * 16 + s % 16) * D + p % CPR * 8, v[i]);
  }
  // values: piece p is dims p / 2 % D, slots 8 (p & 1) .. + 7 of new page p / (2 D)
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int p = tid + i * 256, page = p / (2 * D), d = p / 2 % D, s0 = page * 16 + (p & 1) * 8;
    uint32_t e[8];
    bool all = true, any = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int old = s_page[s0 + j];
      e[j] = 0;
      all &= old >= 0;
      any |= old >= 0;
      if (old >= 0)
        e[j] = a.vc[((size_t)old * a.hkv + kvh) * 16 * D + (size_t)d * 16 + s_slot[s0 + j]];
    }
    if (!any) continue;
    uint16_t* to = a.vc + ((size_t)new_row[page] * a.hkv + kvh) * 16 * D + (size_t)d * 16 + (p & 1) * 8;
    if (all) {
      st16(to, u32x4{e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16});
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (s_page[s0 + j] >= 0) to[j] = (uint16_t)e[j];
    }
  }
}

constexpr int kGridRow = 1 << 16;  // workgroups in a row of the grid (2^32 threads at most)
// Lists of at most this many keys run in small workgroups, several to a compute unit.
constexpr int kShortList = 4096;
constexpr int kLongCap = 32768;

template <class K>
int launch(K kernel, const EvictArgs& a, int threads, hipStream_t stream) {
  if (a.workgroups == 0) return SSA_OK;
  (void)hipGetLastError();
  const int64_t wgs = a.workgroups;
  const dim3 grid(wgs < kGridRow ? wgs : kGridRow, (wgs + kGridRow - 1) / kGridRow);
  hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, stream, a);
  return hipGetLastError() == hipSuccess ? SSA_OK : SSA_ERR_HIP;
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
  const int rc = check_evict_plan(shape, plan_host, &h);
  if (rc) return rc;
  if (!plan_dev) return SSA_ERR_NULL;
  if (h->num_keep > 0 && (!scores || !block_table || !keep)) return SSA_ERR_NULL;
  if (!workspace || ws_bytes < (size_t)h->ws_bytes) return SSA_ERR_WORKSPACE;
  if (h->num_keep == 0) return SSA_OK;
  EvictArgs a = evict_args(h, plan_dev, block_table);
  a.workgroups = h->num_reqs * h->hkv;
  a.scores = scores;
  a.keep = keep;
  hipStream_t s = static_cast<hipStream_t>(stream);
  return h->max_len <= kShortList ? launch(evict_select_kernel<256, kShortList>, a, 256, s)
                                  : launch(evict_select_kernel<1024, kLongCap>, a, 1024, s);
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
