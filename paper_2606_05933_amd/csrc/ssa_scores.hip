// HIP kernels for gfx950 of ssa_key_scores and ssa_decode_scored
// (include/ssa_evict.h): the attention weights of a batch, summed per key.
//
// With t = scale log2(e) <q, k>, row j's weight on key t is 2^(t - m_j) / l_j, m_j a
// maximum and l_j the sum of 2^(t - m_j) over the keys that it sees.  A key's score is a
// sum over rows, and l_j a sum over keys, so the weights need m and l first:
//
//   one counted row   The logits are few (Hq per key, against 2 D bytes of K per
//                     kv head): a first pass reads K, writes the logits (fp32)
//                     and each key range's maximum and sum; a second joins those
//                     and turns logits into weights.  K is read once.  With the
//                     attention output wanted, the first pass also reads V.
//   several rows      The logits do not fit; K goes through the matrix cores
//                     twice.  First pass: 64 columns (row, head) a wave stay in
//                     registers, keys stream through LDS, and every lane keeps a
//                     running maximum and sum of its two columns.  Second pass:
//                     64 keys a wave stay in registers, the columns with their m
//                     and 1 / l stream through LDS, and every lane sums the weights of its
//                     two keys.  Where there are few keys the columns are cut into
//                     ranges too, whose sums the last workgroup of a key tile adds
//                     in their order.
//
// Rows stream into LDS with their 16-byte pieces permuted within the row (piece c
// of row r lies at c ^ r), so that the 32 rows of a fragment read hit all banks.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>
#include <initializer_list>
#include <type_traits>

#include "../../include/ssa_evict.h"
#include "ssa_device.h"
#include "ssa_evict_format.h"

namespace ssa {
int check_score_plan(const ssa_shape* s, const void* plan_host, const ScoreHeader** out);
}

namespace {
using namespace ssa;
using namespace ssa_dev;

typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float kInf = __builtin_huge_valf();
constexpr float kLog2e = 1.44269504088896340736f;

struct ScoreArgs {
  const uint8_t* plan;
  uint64_t hash;
  // the launch's items: chunk items, then items of requests with one counted row
  int64_t off_chunk, off_decode;  // byte offsets of the lists
  int32_t chunk_groups, workgroups;
  int32_t sum_cols, num_tickets;
  int32_t hq, hkv, g, maxp;
  uint32_t g_magic;   // ceil(2^32 / g)
  int32_t g_magic12;  // ceil(2^12 / g): exact for x < 32
  float c;            // softmax scale times log2(e)
  float decay;
  const uint16_t* q;
  const uint16_t* kc;
  const uint16_t* vc;
  const int32_t* bt;
  const float* scores_in;
  float* scores_out;
  uint16_t* out;
  float* ws;
};

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
// x < 2^28 over g <= 16
__device__ __forceinline__ int div_g(const ScoreArgs& a, int x) {
  return a.g == 1 ? x : (int)__umulhi((uint32_t)x, a.g_magic);
}

// The workgroup's item and kv head; false: nothing to do (past the grid's end, or
// another plan than the host's lies at plan_dev).
struct Work {
  ScoreItem it;
  int kvh;
  bool chunk;
};
__device__ __forceinline__ bool take_item(const ScoreArgs& a, Work* w) {
  int wg = (int)(blockIdx.y * gridDim.x + blockIdx.x);
  if (wg >= a.workgroups) return false;
  w->chunk = wg < a.chunk_groups;
  if (!w->chunk) wg -= a.chunk_groups;
  w->kvh = wg % a.hkv;
  const auto h = as_uniform<ScoreHeader>(a.plan);
  const auto it = as_uniform<ScoreItem>(a.plan + (w->chunk ? a.off_chunk : a.off_decode)) + wg / a.hkv;
  w->it = ScoreItem{it->req,      it->q_row, it->ticket, it->rows,  it->len,    it->ctx_len, it->col0,
                    it->cols_pad, it->key0,  it->key1,   it->split, it->nsplit, it->off0,    it->off1};
  return h->magic == kScoreMagic && h->hash == a.hash;
}

// Four keys' new scores (keys k0 .. k0 + 3 of one page); w: their weights.
__device__ __forceinline__ void add_scores4(const ScoreArgs& a, const ScoreItem& it, int kvh, int k0,
                                            int key1, f32x4 w) {
  const int page = a.bt[(size_t)it.req * a.maxp + k0 / 16];
  const size_t at = ((size_t)page * a.hkv + kvh) * 16 + k0 % 16;
  if (k0 + 4 <= key1) {
    if (a.scores_in && k0 + 4 <= it.ctx_len) {
      const f32x4 old = *reinterpret_cast<const f32x4*>(a.scores_in + at);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] += old[i] * a.decay;
    } else if (a.scores_in) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (k0 + i < it.ctx_len) w[i] += a.scores_in[at + i] * a.decay;
    }
    *reinterpret_cast<f32x4*>(a.scores_out + at) = w;
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (k0 + i < key1) {
      float x = w[i];
      if (a.scores_in && k0 + i < it.ctx_len) x += a.scores_in[at + i] * a.decay;
      a.scores_out[at + i] = x;
    }
}

// ---------------------------------------------------------------------------
// One counted row: logits over a key range.  Memory bounds it: 32 rows of 8k to 33k
// keys, 64/8 heads of 128, with the output: 2.46 GB of keys and values and 0.17 GB of
// logits in 527 us, 5.0 TB/s where a copy of 4 GiB reaches 4.8 and the attention launch's
// reads 6.5 (without the logits' stores 435 us), and 48 us for the join; 622 us together before a block's loads were
// issued a step ahead and the pieces cut to 1024 keys.  The non-temporal hint changes
// nothing.
//
// Each wave takes every fourth 32-key block (two pages).  S^T = K Q^T in 16x16
// tiles: the A rows of the two tiles are dealt so that a lane ends up with 8
// consecutive keys of one column (head), which is also the layout of the B operand
// of the P V product: no data moves between lanes but the block's maximum.  Logits are
// stored as they lie, [G][32 keys][tile][quarter][4 keys]: a store instruction writes
// 64 bytes of each head, and 8 threads of the join read 128.
//
// A row whose logits fit in LDS is one item: the workgroup turns them into scores and
// writes the output itself.
struct JoinLds {
  float m[16], inv[16];
  __attribute__((aligned(16))) f32x4 part[kScoreThreads];
};
template <int D, bool OUT>
struct DecodeLds {
  static constexpr int kO = OUT ? 4 * 16 * D : 0;
  float ml[2][4][16];
  float m[16], inv[16];
  __attribute__((aligned(16))) float big[kO > kWholeLogits ? kO : kWholeLogits];  // logits, then o
};

// Four keys' weights from their logits, x[g * stride .. + 3] for head g.
__device__ __forceinline__ f32x4 weights4(const ScoreArgs& a, const float* x, int stride,
                                          const float* m, const float* inv) {
  f32x4 w = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int g = 0; g < a.g; ++g) {
    const f32x4 v = *reinterpret_cast<const f32x4*>(x + (int64_t)g * stride);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] += exp2_fast(__builtin_fmaf(v[i], a.c, -m[g])) * inv[g];
  }
  return w;
}
// Where the logits of keys k0 .. k0 + 3 lie in a head's: quarter k0 / 8 % 4 of tile
// k0 / 4 % 2 of their 32 keys.
__device__ __forceinline__ int logits_at(int k0) {
  return k0 / 32 * 32 + (k0 / 4 % 2) * 16 + k0 / 8 % 4 * 4;
}
// Two bf16 values without their signs, and the larger of each of two such pairs.
constexpr uint32_t kMagnitudes = 0x7FFF7FFFu, kInfBits = 0x7F80u;  // above it: NaN
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t max_halves(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a),
                                                                __builtin_bit_cast(u16x2, b)));
}
__device__ __forceinline__ u32x2 pack4(f32x4 v) {
  return u32x2{pack2(v[0], v[1]), pack2(v[2], v[3])};
}

template <int D, bool OUT>
__device__ __forceinline__ void decode_item(const ScoreArgs& a, const ScoreItem& it, int kvh,
                                            DecodeLds<D, OUT>& lds) {
  constexpr int KS = D / 32, DT = D / 16;
  auto& s_ml = lds.ml;
  float* const s_o = lds.big;
  const bool whole = it.split < 0;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, quad = lane >> 4;
  const auto row = as_uniform<int32_t>(a.bt + (size_t)it.req * a.maxp);
  const int last_page = (it.len - 1) / 16;

  bf16x8 qf[KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    u32x4 v = {0, 0, 0, 0};
    if (r16 < a.g)
      v = ld16(a.q + ((size_t)it.q_row * a.hq + kvh * a.g + r16) * D + s * 32 + quad * 8);
    qf[s] = as_bf16x8(v);
  }
  // the item's logits, in LDS until it has read its keys
  const int stride = (it.key1 - it.key0 + 31) / 32 * 32;
  float* held = lds.big + r16 * stride + quad * 4 - it.key0;
  float m = -kInf, l = 0.f;
  f32x4 o[OUT ? DT : 1];
#pragma unroll
  for (int t = 0; t < (OUT ? DT : 1); ++t) o[t] = f32x4{0.f, 0.f, 0.f, 0.f};

  // A block's keys go into registers while the block before is at its softmax, its
  // values while that one's products run: loads are always in flight.
  const int slot0 = 8 * ((r16 >> 2) & 1) + (r16 & 3);
  u32x4 kf[2][KS], vf[OUT ? DT : 1];
  auto load_keys = [&](int p0, int p1) {
    const uint16_t* kp =
        a.kc + ((size_t)(r16 >> 3 ? p1 : p0) * a.hkv + kvh) * 16 * D + slot0 * D + quad * 8;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int s = 0; s < KS; ++s) kf[t][s] = ld16(kp + t * 4 * D + s * 32);
  };
  auto load_values = [&](int p0, int p1) {
    if constexpr (OUT) {
      const uint16_t* vp =
          a.vc + ((size_t)(quad >> 1 ? p1 : p0) * a.hkv + kvh) * 16 * D + r16 * 16 + 8 * (quad & 1);
#pragma unroll
      for (int t = 0; t < DT; ++t) vf[t] = ld16(vp + t * 256);
    }
  };
  const int first = it.key0 + wave * 32;
  int p0 = 0, p1 = 0;
  if (first < it.key1) {
    p0 = row[first / 16];
    p1 = row[min(first / 16 + 1, last_page)];
    load_keys(p0, p1);
    load_values(p0, p1);
  }
  for (int kb = first; kb < it.key1; kb += 128) {
    const bool more = kb + 128 < it.key1;
    if (more) {
      p0 = row[(uint32_t)(kb + 128) / 16];
      p1 = row[min((kb + 128) / 16 + 1, last_page)];
    }
    f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      s0 = mfma(as_bf16x8(kf[0][s]), qf[s], s0);
      s1 = mfma(as_bf16x8(kf[1][s]), qf[s], s1);
    }
    if (more) load_keys(p0, p1);
    __builtin_amdgcn_sched_barrier(0);
    float x[8] = {s0[0], s0[1], s0[2], s0[3], s1[0], s1[1], s1[2], s1[3]};
    if (r16 < a.g) {
      *reinterpret_cast<f32x4*>(held + kb) = s0;
      *reinterpret_cast<f32x4*>(held + kb + 16) = s1;
    }
    const int nv = it.key1 - kb - 8 * quad;  // this lane's keys that exist
    if (kb + 32 > it.key1) {
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
    float p[8], sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = exp2_fast(__builtin_fmaf(x[i], a.c, -ms));
    if (kb + 32 > it.key1) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i >= nv) p[i] = 0.f;  // scale 0 times -inf is NaN
    }
    sum = ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
    l = l * alpha + sum;
    m = mn;
    if constexpr (OUT) {
      // A weight enters the matrix product as three bf16 values, the rounded one and what
      // that misses twice over: all of its 24 bits.  Memory bounds this loop, and they
      // cost no time.  (One alone put as much error into the output as its own rounding
      // to bf16.)
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
      if (kb + 32 > it.key1) {
        // a slot past the last key may hold anything, and 0 times NaN is NaN
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
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (quad == 0) {
    s_ml[0][wave][r16] = m;
    s_ml[1][wave][r16] = l;
  }
  __syncthreads();
  float* rec = a.ws + it.off1 + ((int64_t)kvh * it.nsplit + it.split) * score_rec_floats(a.g, D);
  if (tid < a.g) {
    float mm = -kInf, ll = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) mm = fmaxf(mm, s_ml[0][w][tid]);
    const float ms = mm == -kInf ? 0.f : mm;
#pragma unroll
    for (int w = 0; w < 4; ++w) ll += s_ml[1][w][tid] * exp2_fast(s_ml[0][w][tid] - ms);
    lds.m[tid] = ms;
    lds.inv[tid] = 1.f / ll;
    if (!whole) {
      rec[tid] = mm;
      rec[a.g + tid] = ll;
    }
  }
  if (whole) {
    __syncthreads();
    for (int k0 = tid * 4; k0 < it.len; k0 += kScoreThreads * 4)
      add_scores4(a, it, kvh, k0, it.len, weights4(a, lds.big + logits_at(k0), stride, lds.m, lds.inv));
  } else {
    float* to = a.ws + it.off0 + (int64_t)kvh * a.g * it.cols_pad + it.key0;
    for (int g = wave; g < a.g; g += 4)
      for (int k = lane * 4; k < stride; k += 256)
        *reinterpret_cast<f32x4*>(to + (int64_t)g * it.cols_pad + k) =
            *reinterpret_cast<const f32x4*>(lds.big + g * stride + k);
  }
  if constexpr (OUT) {
    __syncthreads();
#pragma unroll
    for (int t = 0; t < DT; ++t)
      *reinterpret_cast<f32x4*>(s_o + (wave * 16 + r16) * D + t * 16 + 4 * quad) = o[t];
    __syncthreads();
    float* ro = rec + score_rec_o(a.g);
    for (int e = tid * 4; e < a.g * D; e += kScoreThreads * 4) {
      const int g = e / D, d = e % D;
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < 4; ++w)
        v += *reinterpret_cast<const f32x4*>(s_o + (w * 16 + g) * D + d) *
             exp2_fast(s_ml[0][w][g] - lds.m[g]);
      if (whole)
        *reinterpret_cast<u32x2*>(a.out + ((size_t)it.q_row * a.hq + kvh * a.g + g) * D + d) =
            pack4(v * lds.inv[g]);
      else
        *reinterpret_cast<f32x4*>(ro + e) = v;
    }
  }
}

// One counted row: join the key ranges' sums, turn a range's logits into scores.  The
// row's items share out its output, a few 4-dim pieces each, whose records all
// threads read.
template <int D, bool OUT>
__device__ __forceinline__ void decode_join_item(const ScoreArgs& a, const ScoreItem& it, int kvh,
                                                 JoinLds& lds) {
  auto &s_m = lds.m, &s_inv = lds.inv;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int stride = score_rec_floats(a.g, D);
  const float* recs = a.ws + it.off1 + (int64_t)kvh * it.nsplit * stride;
  for (int g = wave; g < a.g; g += 4) {
    float m = -kInf;
    for (int s = lane; s < it.nsplit; s += 64) m = fmaxf(m, recs[(int64_t)s * stride + g]);
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor(m, x, 64));
    const float ms = m == -kInf ? 0.f : m;
    float l = 0.f;
    for (int s = lane; s < it.nsplit; s += 64) {
      const float* r = recs + (int64_t)s * stride;
      l += r[a.g + g] * exp2_fast(r[g] - ms);
    }
#pragma unroll
    for (int x = 32; x > 0; x >>= 1) l += __shfl_xor(l, x, 64);
    if (lane == 0) {
      s_m[g] = ms;
      s_inv[g] = 1.f / l;
    }
  }
  __syncthreads();
  const int k0 = it.key0 + tid * 4;
  if (k0 < it.key1) {
    const float* lg = a.ws + it.off0 + (int64_t)kvh * a.g * it.cols_pad + logits_at(k0);
    add_scores4(a, it, kvh, k0, it.key1, weights4(a, lg, it.cols_pad, s_m, s_inv));
  }
  if constexpr (OUT) {
    const int items = (it.len + kJoinKeys - 1) / kJoinKeys, pieces = a.g * D / 4;
    const int per = (pieces + items - 1) / items;  // pieces of an item, at most 512
    const int first = it.key0 / kJoinKeys * per, mine = min(per, pieces - first);
    for (int p0 = 0; p0 < mine; p0 += kScoreThreads) {
      const int n = min(kScoreThreads, mine - p0);   // pieces of this round ...
      const int lanes = kScoreThreads / n;           // ... and the threads of each
      const int p = tid % n, lane0 = tid / n, e = (first + p0 + p) * 4, g = e / D;
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
      if (lane0 < lanes)
#pragma unroll 4
        for (int s = lane0; s < it.nsplit; s += lanes) {
          const float* r = recs + (int64_t)s * stride;
          v += *reinterpret_cast<const f32x4*>(r + score_rec_o(a.g) + e) * exp2_fast(r[g] - s_m[g]);
        }
      lds.part[tid] = v;
      __syncthreads();
      if (tid < n) {
        for (int x = 1; x < lanes; ++x) v += lds.part[x * n + tid];
        *reinterpret_cast<u32x2*>(a.out + ((size_t)it.q_row * a.hq + kvh * a.g + g) * D + e % D) =
            pack4(v * s_inv[g]);
      }
      __syncthreads();
    }
  }
}

// ---------------------------------------------------------------------------
// Several rows: both passes.  The issue of matrix and vector instructions bounds them:
// per 32 x 64 scores a wave runs 16 products (512 cycles), 32 exponentials (half
// rate), 32 multiply-adds and 32 additions (second pass: 64 and 8).  Four chunks of 64
// to 1024 rows, 267 M scores of 28/4 heads: 83 us and 104 us; of the first pass's cycles
// the matrix unit is busy 0.35, and 0.46 of those have a vector instruction beside.
// Waves of 32 vectors (twice as many resident) took 97 and 108 us when the second pass
// took 101.  A wave holds 64 stationary vectors (columns in the first pass, keys in the
// second) as B operands of the 32x32x16 product and runs the streamed rows (keys,
// columns) past them in 32-row tiles; NC waves lie side by side over the same rows, 4 /
// NC one behind the other.  Lane n of a 32x32 result owns stationary vector n % 32 and,
// of the tile, the 16 rows (r & 3) + 8 (r >> 2) + 4 (n / 32): sums over rows stay in the
// lane to the end.
__device__ __forceinline__ f32x16 mfma32(bf16x8 x, bf16x8 y, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, c, 0, 0, 0);
}

constexpr int kTiles = kScoreWaveCols / 32;

template <int D, int NC, int TILES = 1>
struct ChunkCfg {
  static constexpr int RG = 4 / NC;             // row groups
  static constexpr int TPS = TILES;             // 32-row tiles of a wave in a stage
  static constexpr int ROWS = 32 * RG * TPS;    // streamed rows of a stage
  static constexpr int ROWB = D * 2;
  static constexpr int CPR = D / 8;             // 16-byte pieces of a row
  static constexpr int RPD = 64 / CPR;          // rows of one copy instruction
  static constexpr int STAGE = ROWS * ROWB;
  static constexpr int NB = NC == 1 ? 2 : 3;    // stages in LDS
  static constexpr int LOADS = ROWS * CPR / kScoreThreads;  // copies of a wave per stage
  static constexpr int KS = D / 16;
  static constexpr int COLS = kScoreWaveCols * NC;  // stationary vectors of a workgroup
};

// A wave copies LOADS x RPD rows of a stage, RPD at a time: copy i starts at the
// stage's row copy_row(wave, i).  Lane n takes piece n % CPR of row n / CPR, from the
// permuted place; copy_offset is its byte offset from the first row where rows lie one
// after the other.
template <class C>
__device__ __forceinline__ int copy_row(int wave, int i) {
  return (wave * C::LOADS + i) * C::RPD;
}
template <class C>
__device__ __forceinline__ uint32_t copy_offset(int lane, int row0) {
  const int row = lane / C::CPR;
  const uint32_t first = row * C::ROWB + ((lane % C::CPR) ^ (row & (C::CPR - 1))) * 16;
  return first ^ (uint32_t)((row0 & (C::CPR - 1)) * 16);  // row0 is a multiple of RPD
}

// Where a lane reads the fragments of its row of the first stage.
template <class C, int D>
__device__ __forceinline__ void fragment_addresses(const char* buf, int rg, int lane,
                                                   const char* (&at)[D / 16]) {
#pragma unroll
  for (int s = 0; s < C::KS; ++s)
    at[s] = buf + (rg * 32 * C::TPS + (lane & 31)) * C::ROWB +
            ((2 * s + (lane >> 5)) ^ (lane & (C::CPR - 1))) * 16;
}

// Run `stage(k, buffer)` for k = 0 .. stages - 1, the buffer k % NB a constant of each
// copy of the body: LDS addresses are then a register and an immediate.
template <int NB, class F>
__device__ __forceinline__ void for_stages(int stages, F stage) {
  for (int k = 0; k < stages; k += NB) {
    stage(k, std::integral_constant<int, 0>{});
    if (k + 1 >= stages) break;
    stage(k + 1, std::integral_constant<int, 1>{});
    if constexpr (NB == 3) {
      if (k + 2 >= stages) break;
      stage(k + 2, std::integral_constant<int, 2>{});
    }
  }
}

// One 32-row tile's products with the wave's 64 vectors.  All of the tile's
// fragments are on their way before the first product.
template <class C, int D>
__device__ __forceinline__ void tile_products(const char* const (&at)[D / 16], int offset,
                                              const bf16x8 (*st)[D / 16], f32x16* acc) {
  bf16x8 x[C::KS];
#pragma unroll
  for (int s = 0; s < C::KS; ++s) x[s] = as_bf16x8(ld16(at[s] + offset));
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_setprio(1);
#pragma unroll
  for (int t = 0; t < kTiles; ++t) acc[t] = f32x16{};
#pragma unroll
  for (int s = 0; s < C::KS; ++s)
#pragma unroll
    for (int t = 0; t < kTiles; ++t) acc[t] = mfma32(x[s], st[t][s], acc[t]);
  __builtin_amdgcn_s_setprio(0);
}

__device__ __forceinline__ float sum16(float* p) {
#pragma unroll
  for (int w = 8; w > 0; w >>= 1)
#pragma unroll
    for (int i = 0; i < w; ++i) p[i] += p[i + w];
  return p[0];
}
// A column's m and 1 / l for the second pass, in blocks of 32 columns: 32 of the one,
// then 32 of the other.  They stay apart, so that a row's weights add up to 1: as one
// number, m + log2(l), they were off by half a step of it, 1e-5 for logits of deviation
// 64.  Where no weight is a number (l is 0 or NaN), m is NaN and 1 / l is 1: keys that the
// row does not see then still get nothing.
__device__ __forceinline__ int norm_at(int n) { return (n & ~31) * 2 + (n & 31); }
__device__ __forceinline__ void put_norm(float* norms, int n, float m, float l) {
  const bool weighs = l > 0.f;
  norms[norm_at(n)] = weighs ? m : __builtin_nanf("");
  norms[norm_at(n) + 32] = weighs ? 1.f / l : 1.f;
}
// a column that only pads
__device__ __forceinline__ void put_no_norm(float* norms, int n) {
  norms[norm_at(n)] = kInf;
  norms[norm_at(n) + 32] = 0.f;
}

// row of a tile that register i of a lane holds, less 4 (lane / 32)
__device__ __forceinline__ constexpr int tile_row(int i) { return (i & 3) + 8 * (i >> 2); }

// The first guess at a tile's exponentials may be this much over 1 (the sum of them
// is far from overflow); past it the column's reference is raised.
constexpr float kRaise = 0x1p40f;

// A column's reference m and the sum l of 2^(t - m) over one more tile.  m is a
// maximum over some of the keys, not all: exponentials are formed against it as it
// is, which saves the maximum over the tile, and only a tile that has one of over
// 2^40 raises it.  2^(t - m) / l does not depend on m.
__device__ __forceinline__ void lse_add(const f32x16& x, float c, float* m, float* l) {
  float v[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = exp2_fast(__builtin_fmaf(x[i], c, -*m));
  const float sum = sum16(v);
  if (__any(!(sum < kRaise))) {
    float mx = x[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, x[i]);
    const float mn = fmaxf(*m, mx * c), ms = mn == -kInf ? 0.f : mn;  // -inf: all logits so far
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = exp2_fast(__builtin_fmaf(x[i], c, -ms));
    *l = *l * exp2_fast(*m - ms) + sum16(v);
    *m = mn;
  } else {
    *l += sum;
  }
}

// The same with the maximum taken first, for the first tile and for MASK: rows past
// `limit` are not seen.
__device__ __forceinline__ void lse_update(const f32x16& x, float c, int limit, float* m, float* l) {
  float v[16], mx = -kInf;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    v[i] = tile_row(i) > limit ? -kInf : x[i];
    mx = fmaxf(mx, v[i]);
  }
  // nothing seen: the maximum stays, and may be -inf
  const float mn = mx == -kInf ? *m : fmaxf(*m, mx * c);
  const float ms = mn == -kInf ? 0.f : mn;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    v[i] = exp2_fast(__builtin_fmaf(v[i], c, -ms));
    if (tile_row(i) > limit) v[i] = 0.f;  // scale 0 times -inf is NaN
  }
  *l = *l * exp2_fast(*m - ms) + sum16(v);
  *m = mn;
}

// Two tiles a stage where four waves share them (half the barriers; 85.7 us of the
// chunks above, 82.5 with).  The second pass was slower with two (105 us, 111 with).
template <int D, int NC>
using LseCfg = ChunkCfg<D, NC, NC == 4 ? 2 : 1>;
template <int D, int NC>
struct LseLds {
  using C = LseCfg<D, NC>;
  __attribute__((aligned(16))) char buf[C::NB * C::STAGE];
  float m[C::RG][C::COLS], l[C::RG][C::COLS];
};
template <int D, int NC>
__device__ __forceinline__ void lse_item(const ScoreArgs& a, const ScoreItem& it, int kvh,
                                         LseLds<D, NC>& lds) {
  using C = LseCfg<D, NC>;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int cg = wave % NC, rg = wave / NC, half = lane >> 5;
  const int ncols = it.rows * a.g, limit0 = it.len - it.rows;
  const int first_limit = limit0 + div_g(a, it.col0);
  const int last_limit = limit0 + div_g(a, min(it.col0 + C::COLS, ncols) - 1);
  const int kend = min(it.key1, last_limit + 1);  // keys past it are seen by no column

  bf16x8 st[kTiles][C::KS];
  int limit[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const int n = min(it.col0 + cg * kScoreWaveCols + t * 32 + (lane & 31), ncols - 1);
    const int j = div_g(a, n);
    limit[t] = min(limit0 + j, kend - 1) - 4 * half;
    const uint16_t* p =
        a.q + ((size_t)(it.q_row + j) * a.hq + kvh * a.g + (n - j * a.g)) * D + half * 8;
#pragma unroll
    for (int s = 0; s < C::KS; ++s) st[t][s] = as_bf16x8(ld16(p + s * 16));
  }
  float m[kTiles], l[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    m[t] = -kInf;
    l[t] = 0.f;
  }

  const int stages = kend > it.key0 ? (kend - it.key0 + C::ROWS - 1) / C::ROWS : 0;
  // Rows past kend are copied as they lie in the last page (and are not seen): whole
  // pages are there to read.
  const auto row = as_uniform<int32_t>(a.bt + (size_t)it.req * a.maxp);
  // A wave's rows of a stage lie in NP pages, named one stage ahead.
  constexpr int RPW = C::LOADS * C::RPD, NP = RPW < 16 ? 1 : RPW / 16;
  const int page0 = it.key0 / 16 + wave * RPW / 16, last_page = (kend - 1) / 16;
  int page[NP];
  auto name_pages = [&](int k) {
#pragma unroll
    for (int i = 0; i < NP; ++i) page[i] = row[min(page0 + k * (C::ROWS / 16) + i, last_page)];
  };
  auto issue = [&](int k) {
    char* buf = lds.buf + (k % C::NB) * C::STAGE;
#pragma unroll
    for (int i = 0; i < C::LOADS; ++i) {
      const int row0 = copy_row<C>(wave, i);
      dma16_base(a.kc + (((size_t)page[i * C::RPD / 16] * a.hkv + kvh) * 16 + row0 % 16) * D,
                 copy_offset<C>(lane, row0), buf + row0 * C::ROWB);
    }
    name_pages(k + 1);
  };
  if (stages > 0) name_pages(0);
  vm_wait<0>();  // the stationary vectors have landed: the waits below count copies only
#pragma unroll
  for (int k = 0; k < C::NB - 1; ++k)
    if (k < stages) issue(k);
  const char* at[C::KS];
  fragment_addresses<C, D>(lds.buf, rg, lane, at);
  for_stages<C::NB>(stages, [&](int k, auto buffer) {
    if (C::NB == 3 && k + 1 < stages)
      vm_wait<C::LOADS>();
    else
      vm_wait<0>();
    __syncthreads();
    if (k + C::NB - 1 < stages) issue(k + C::NB - 1);
#pragma unroll
    for (int tile = 0; tile < C::TPS; ++tile) {
      const int kb = it.key0 + k * C::ROWS + (rg * C::TPS + tile) * 32;
      if (tile > 0 && kb >= kend) break;
      f32x16 acc[kTiles];
      tile_products<C, D>(at, buffer() * C::STAGE + tile * 32 * C::ROWB, st, acc);
      if (k > 0 && kb + 31 <= first_limit && kb + 32 <= kend) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) lse_add(acc[t], a.c, &m[t], &l[t]);
      } else {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) lse_update(acc[t], a.c, limit[t] - kb, &m[t], &l[t]);
      }
    }
  });
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    const float m2 = __shfl_xor(m[t], 32, 64), l2 = __shfl_xor(l[t], 32, 64);
    const float mm = fmaxf(m[t], m2), ms = mm == -kInf ? 0.f : mm;
    if (half == 0) {
      lds.m[rg][cg * kScoreWaveCols + t * 32 + lane] = mm;
      lds.l[rg][cg * kScoreWaveCols + t * 32 + lane] = l[t] * exp2_fast(m[t] - ms) + l2 * exp2_fast(m2 - ms);
    }
  }
  __syncthreads();
  if (tid < C::COLS) {
    float mm = -kInf, ll = 0.f;
#pragma unroll
    for (int r = 0; r < C::RG; ++r) mm = fmaxf(mm, lds.m[r][tid]);
    const float ms = mm == -kInf ? 0.f : mm;
#pragma unroll
    for (int r = 0; r < C::RG; ++r) ll += lds.l[r][tid] * exp2_fast(lds.m[r][tid] - ms);
    const int n = it.col0 + tid;
    float* norms = a.ws + it.off0 + (int64_t)kvh * it.cols_pad * 2;
    if (it.nsplit > 1) {
      if (n < it.cols_pad) {
        float* to = a.ws + it.off1 + (((int64_t)kvh * it.nsplit + it.split) * it.cols_pad + n) * 2;
        *reinterpret_cast<f32x2*>(to) = f32x2{mm, ll};
      }
    } else if (n < ncols) {
      put_norm(norms, n, ms, ll);
    }
  }
  // columns that only pad: their weights are zero
  if (it.nsplit == 1 && it.col0 + C::COLS >= ncols)
    for (int n = ncols + tid; n < it.cols_pad; n += kScoreThreads)
      put_no_norm(a.ws + it.off0 + (int64_t)kvh * it.cols_pad * 2, n);
}

// m and l of 256 columns from the pieces of a cut key range.
__device__ __forceinline__ void lse_join_item(const ScoreArgs& a, const ScoreItem& it, int kvh) {
  const int n = it.col0 + (int)threadIdx.x;  // < cols_pad, a multiple of 256
  float* norms = a.ws + it.off0 + (int64_t)kvh * it.cols_pad * 2;
  if (n >= it.rows * a.g) {
    put_no_norm(norms, n);
    return;
  }
  const float* r = a.ws + it.off1 + ((int64_t)kvh * it.nsplit * it.cols_pad + n) * 2;
  float m = -kInf, l = 0.f;
#pragma unroll 8
  for (int s = 0; s < it.nsplit; ++s) {
    const f32x2 v = *reinterpret_cast<const f32x2*>(r + (int64_t)s * it.cols_pad * 2);
    const float mn = fmaxf(m, v[0]), ms = mn == -kInf ? 0.f : mn;
    l = l * exp2_fast(m - ms) + v[1] * exp2_fast(v[0] - ms);
    m = mn;
  }
  put_norm(norms, n, m, l);
}

template <int D>
struct SumLds {
  using C = ChunkCfg<D, 4>;
  __attribute__((aligned(16))) char buf[C::NB * C::STAGE];
  __attribute__((aligned(16))) float norm[C::NB][4][2 * C::ROWS];  // m, 1 / l: one copy a wave
  __attribute__((aligned(16))) float sum[C::COLS];
  int last;
};
template <int D>
__device__ __forceinline__ void sum_item(const ScoreArgs& a, const ScoreItem& it, int kvh,
                                         SumLds<D>& lds) {
  constexpr int NC = 4;  // tiles of 64 or 128 keys put too few products between copies
  using C = ChunkCfg<D, NC>;
  static_assert(C::RG == 1 && C::COLS == kSumKeys && C::ROWS == 32, "one row group of 32");
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5;
  const int ncols = min(it.rows * a.g, it.col0 + a.sum_cols), limit0 = it.len - it.rows;
  // columns of earlier rows see none of these keys
  const int n0 = max(it.col0, max(0, it.key0 - limit0) * a.g / C::ROWS * C::ROWS);
  const int stages = (ncols - n0 + C::ROWS - 1) / C::ROWS;

  // columns from here on see the whole tile
  const int64_t n_whole = (int64_t)(it.key0 + C::COLS - 1 - limit0) * a.g;
  // sums of 16 tiles, then the sums of those: few terms that differ much in size
  float sum[kTiles] = {}, total[kTiles] = {};
  const float* norms = a.ws + it.off0 + (int64_t)kvh * it.cols_pad * 2;
  // Copy i of a stage starts at column n[i], head at[i] of its group, row from[i]:
  // stepped from stage to stage, since dividing by G for each would cost a wave more
  // scalar instructions than its products.
  const uint16_t* from[C::LOADS];
  int head[C::LOADS];
#pragma unroll
  for (int i = 0; i < C::LOADS; ++i) {
    const int n = min(n0 + copy_row<C>(wave, i), ncols - 1), j = div_g(a, n);
    head[i] = n - j * a.g;
    from[i] = a.q + ((size_t)(it.q_row + j) * a.hq + kvh * a.g + head[i]) * D;
  }
  const int step_rows = div_g(a, C::ROWS), step_heads = C::ROWS - step_rows * a.g;
  const int64_t step = ((int64_t)step_rows * a.hq + step_heads) * D, wrap_step = (int64_t)(a.hq - a.g) * D;
  // The request's last column, which sees every key, stands in for columns past it: what
  // of it is not a number is so in every key's score already.
  const uint16_t* last_col =
      a.q + ((size_t)(it.q_row + it.rows - 1) * a.hq + kvh * a.g + a.g - 1) * D;
  auto issue = [&](int k) {
    const int nb = n0 + k * C::ROWS;
    char* buf = lds.buf + (k % C::NB) * C::STAGE;
#pragma unroll
    for (int i = 0; i < C::LOADS; ++i) {
      const int at = copy_row<C>(wave, i), left = ncols - 1 - (nb + at);
      if (left >= 0) {
        // a lane's row is `more` heads on, or in a later token
        const int more = min(lane / C::CPR, left);
        const int wrap = ((head[i] + more) * a.g_magic12) >> 12;
        dma16_base(from[i], copy_offset<C>(lane, at) + (more - lane / C::CPR + wrap * (a.hq - a.g)) * C::ROWB,
                   buf + at * C::ROWB);
      } else {
        dma16_base(last_col, copy_offset<C>(lane, at) % C::ROWB, buf + at * C::ROWB);
      }
      from[i] += step;
      head[i] += step_heads;
      if (head[i] >= a.g) {
        head[i] -= a.g;
        from[i] += wrap_step;
      }
    }
    if (lane < C::ROWS / 2)
      dma16(norms + norm_at(nb) + lane * 4,
            reinterpret_cast<const char*>(&lds.norm[k % C::NB][wave][0]));
  };
#pragma unroll
  for (int k = 0; k < C::NB - 1; ++k)
    if (k < stages) issue(k);
  bf16x8 st[kTiles][C::KS];
  int key[kTiles];
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    key[t] = it.key0 + wave * kScoreWaveCols + t * 32 + (lane & 31);
    const int k = min(key[t], it.len - 1);
    const int page = a.bt[(size_t)it.req * a.maxp + k / 16];
    const uint16_t* p = a.kc + (((size_t)page * a.hkv + kvh) * 16 + k % 16) * D + half * 8;
#pragma unroll
    for (int s = 0; s < C::KS; ++s) st[t][s] = as_bf16x8(ld16(p + s * 16));
  }
  vm_wait<0>();  // all of it has landed: the waits below count later copies only
  const char* at[C::KS];
  fragment_addresses<C, D>(lds.buf, 0, lane, at);
  const float* norm = &lds.norm[0][wave][4 * half];
  for_stages<C::NB>(stages, [&](int k, auto buffer) {
    if (C::NB == 3 && k + 1 < stages)
      vm_wait<C::LOADS + 1>();
    else
      vm_wait<0>();
    __syncthreads();
    if (k + C::NB - 1 < stages) issue(k + C::NB - 1);
    const int nb = n0 + k * C::ROWS;
    f32x16 acc[kTiles];
    f32x4 mv[4], rv[4];  // m and 1 / l of the lane's 16 columns
#pragma unroll
    for (int i = 0; i < 4; ++i)
      mv[i] = *reinterpret_cast<const f32x4*>(norm + buffer() * 8 * C::ROWS + 8 * i);
    tile_products<C, D>(at, buffer() * C::STAGE, st, acc);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      rv[i] = *reinterpret_cast<const f32x4*>(norm + buffer() * 8 * C::ROWS + C::ROWS + 8 * i);
#pragma unroll
    for (int t = 0; t < kTiles; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        acc[t][i] = exp2_fast(__builtin_fmaf(acc[t][i], a.c, -mv[i >> 2][i & 3]));
    if (nb < n_whole) {  // some row does not see some key
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int limit = limit0 + div_g(a, nb + tile_row(i) + 4 * half);
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
          if (limit < key[t]) acc[t][i] = 0.f;
      }
    }
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
      float p[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        p[j] = acc[t][j] * rv[0][j];
#pragma unroll
        for (int i = 1; i < 4; ++i) p[j] = __builtin_fmaf(acc[t][4 * i + j], rv[i][j], p[j]);
      }
      sum[t] += (p[0] + p[1]) + (p[2] + p[3]);
    }
    if ((k & 15) == 15) {
#pragma unroll
      for (int t = 0; t < kTiles; ++t) {
        total[t] += sum[t];
        sum[t] = 0.f;
      }
    }
  });
#pragma unroll
  for (int t = 0; t < kTiles; ++t) {
    float x = total[t] + sum[t];
    x += __shfl_xor(x, 32, 64);
    if (half == 0) lds.sum[wave * kScoreWaveCols + t * 32 + lane] = x;
  }
  __syncthreads();
  f32x4 w = *reinterpret_cast<const f32x4*>(&lds.sum[tid * 4 % C::COLS]);
  if (it.nsplit > 1) {
    // One of several column ranges: the last workgroup of the tile to finish adds all
    // of them in their order.  The sums go past this die's cache (device scope), and
    // have arrived before the ticket is taken.
    const int pad = (it.len + C::COLS - 1) / C::COLS * C::COLS;
    float* part = a.ws + it.off1 + (int64_t)kvh * pad + it.key0 + tid;
    const int64_t stride = (int64_t)a.hkv * pad;
    __hip_atomic_store(part + it.split * stride, lds.sum[tid], __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
    vm_wait<0>();
    __syncthreads();
    if (tid == 0)
      lds.last = __hip_atomic_fetch_add(reinterpret_cast<int*>(a.ws) + it.ticket + kvh, 1,
                                        __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == it.nsplit - 1;
    __syncthreads();
    if (!lds.last) return;
    float x = 0.f;
    for (int k = 0; k < it.nsplit; ++k)
      x += __hip_atomic_load(part + k * stride, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    lds.sum[tid] = x;
    __syncthreads();
    w = *reinterpret_cast<const f32x4*>(&lds.sum[tid * 4 % C::COLS]);
  }
  if (tid * 4 < C::COLS && it.key0 + tid * 4 < it.key1)
    add_scores4(a, it, kvh, it.key0 + tid * 4, it.key1, w);
}

// ---------------------------------------------------------------------------
// The launches.  A hybrid batch's decode rows, which wait for memory, run beside its
// chunk tiles, which wait for the matrix and vector units.

template <int D, bool OUT>
__global__ __launch_bounds__(kScoreThreads, OUT ? 3 : 4) void score_decode_kernel(ScoreArgs a) {
  __shared__ DecodeLds<D, OUT> lds;
  Work w;
  if (take_item(a, &w)) decode_item<D, OUT>(a, w.it, w.kvh, lds);
}

template <int D, bool OUT>
__global__ __launch_bounds__(kScoreThreads) void score_decode_join_kernel(ScoreArgs a) {
  __shared__ JoinLds lds;
  Work w;
  if (take_item(a, &w)) decode_join_item<D, OUT>(a, w.it, w.kvh, lds);
}

template <int D, int NC>
__global__ __launch_bounds__(kScoreThreads, 2) void score_first_kernel(ScoreArgs a) {
  __shared__ union {
    LseLds<D, NC> lse;
    DecodeLds<D, false> decode;
  } lds;
  Work w;
  if (!take_item(a, &w)) return;
  // tickets of the second pass
  for (int64_t i = (int64_t)(blockIdx.y * gridDim.x + blockIdx.x) * kScoreThreads + threadIdx.x;
       i < a.num_tickets; i += (int64_t)a.workgroups * kScoreThreads)
    reinterpret_cast<int*>(a.ws)[i] = 0;
  if (w.chunk)
    lse_item<D, NC>(a, w.it, w.kvh, lds.lse);
  else
    decode_item<D, false>(a, w.it, w.kvh, lds.decode);
}

__global__ __launch_bounds__(kScoreThreads) void score_lse_join_kernel(ScoreArgs a) {
  Work w;
  if (take_item(a, &w)) lse_join_item(a, w.it, w.kvh);
}

template <int D>
__global__ __launch_bounds__(kScoreThreads, 2) void score_second_kernel(ScoreArgs a) {
  __shared__ union {
    SumLds<D> sum;
    JoinLds join;
  } lds;
  Work w;
  if (!take_item(a, &w)) return;
  if (w.chunk)
    sum_item<D>(a, w.it, w.kvh, lds.sum);
  else
    decode_join_item<D, false>(a, w.it, w.kvh, lds.join);
}

// ---------------------------------------------------------------------------

// Workgroups go in rows of this many: one row of more than 2^24 workgroups would
// pass the 2^32 threads of a grid's x dimension.
constexpr int kGridRow = 1 << 16;

template <class K>
int launch(K kernel, ScoreArgs a, const ScoreHeader* h, int chunk_list, int decode_list,
           hipStream_t stream) {
  const int64_t chunks = chunk_list < 0 ? 0 : (int64_t)h->count[chunk_list] * h->hkv;
  const int64_t decodes = decode_list < 0 ? 0 : (int64_t)h->count[decode_list] * h->hkv;
  const int64_t wgs = chunks + decodes;
  if (wgs == 0) return SSA_OK;
  auto offset = [&](int list) {
    return list < 0 ? 0 : h->off_items + (int64_t)h->first[list] * (int64_t)sizeof(ScoreItem);
  };
  a.off_chunk = offset(chunk_list);
  a.off_decode = offset(decode_list);
  a.chunk_groups = (int32_t)chunks;
  a.workgroups = (int32_t)wgs;
  const dim3 grid(wgs < kGridRow ? wgs : kGridRow, (wgs + kGridRow - 1) / kGridRow);
  hipLaunchKernelGGL(kernel, grid, dim3(kScoreThreads), 0, stream, a);
  return hipGetLastError() == hipSuccess ? SSA_OK : SSA_ERR_HIP;
}

template <int D, bool OUT>
int launch_decodes(const ScoreArgs& a, const ScoreHeader* h, hipStream_t s) {
  const int rc = launch(score_decode_kernel<D, OUT>, a, h, -1, kListDecode, s);
  return rc ? rc : launch(score_decode_join_kernel<D, OUT>, a, h, -1, kListDecodeJoin, s);
}

template <int D>
int launch_scores(const ScoreArgs& a, const ScoreHeader* h, hipStream_t s) {
  if (h->count[kListSum] == 0) return launch_decodes<D, false>(a, h, s);
  auto first = h->lse_groups == 4   ? score_first_kernel<D, 4>
               : h->lse_groups == 2 ? score_first_kernel<D, 2>
                                    : score_first_kernel<D, 1>;
  int rc = launch(first, a, h, kListLse, kListDecode, s);
  if (rc) return rc;
  if ((rc = launch(score_lse_join_kernel, a, h, kListLseJoin, -1, s))) return rc;
  return launch(score_second_kernel<D>, a, h, kListSum, kListDecodeJoin, s);
}

// Rows, pages and records are read and written 16 bytes at a time.
bool misaligned(std::initializer_list<const void*> pointers) {
  for (const void* p : pointers)
    if (reinterpret_cast<uintptr_t>(p) % 16) return true;
  return false;
}

// The scalar loads of the plan's header drop the low bits of its address: the kernel would
// find another plan there and do nothing.
bool misaligned_plan(const ScoreHeader* h, const void* plan_dev) {
  return h->max_q_len > 0 && reinterpret_cast<uintptr_t>(plan_dev) % 8;
}

int score_args(const ssa_shape* shape, const ScoreHeader* h, const void* plan_dev,
               const uint16_t* q, const uint16_t* k_cache, const int32_t* block_table,
               const float* scores_in, float decay, float* scores_out, void* workspace,
               size_t ws_bytes, ScoreArgs* a) {
  if (!std::isfinite(decay) || decay < 0.f) return SSA_ERR_ARG;
  if (!plan_dev) return SSA_ERR_NULL;
  if (h->max_q_len > 0 && (!q || !k_cache || !block_table || !scores_out)) return SSA_ERR_NULL;
  if (!workspace || ws_bytes < (size_t)h->ws_bytes) return SSA_ERR_WORKSPACE;
  if (misaligned({q, k_cache, scores_in, scores_out, workspace})) return SSA_ERR_ARG;
  *a = ScoreArgs{};
  a->plan = static_cast<const uint8_t*>(plan_dev);
  a->hash = h->hash;
  a->hq = h->hq;
  a->hkv = h->hkv;
  a->g = h->hq / h->hkv;
  a->maxp = h->max_pages_per_req;
  a->g_magic = (uint32_t)((((uint64_t)1 << 32) + a->g - 1) / a->g);
  a->g_magic12 = (4096 + a->g - 1) / a->g;
  a->c = (float)((double)shape->softmax_scale * (double)kLog2e);
  a->decay = decay;
  a->sum_cols = h->sum_cols;
  a->num_tickets = h->num_tickets;
  a->q = q;
  a->kc = k_cache;
  a->bt = block_table;
  a->scores_in = scores_in;
  a->scores_out = scores_out;
  a->ws = static_cast<float*>(workspace);
  return SSA_OK;
}

}  // namespace

namespace ssa {

int check_key_scores(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                     const uint16_t* q, const uint16_t* k_cache, const int32_t* block_table,
                     const float* scores_in, float decay, float* scores_out, void* workspace,
                     size_t ws_bytes) {
  const ScoreHeader* h = nullptr;
  const int rc = check_score_plan(shape, plan_host, &h);
  if (rc) return rc;
  ScoreArgs a;
  const int args = score_args(shape, h, plan_dev, q, k_cache, block_table, scores_in, decay,
                              scores_out, workspace, ws_bytes, &a);
  return args ? args : misaligned_plan(h, plan_dev) ? SSA_ERR_ARG : SSA_OK;
}

}  // namespace ssa

extern "C" {

int ssa_key_scores(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                   const uint16_t* q, const uint16_t* k_cache, const int32_t* block_table,
                   const float* scores_in, float decay, float* scores_out, void* workspace,
                   size_t ws_bytes, void* stream) {
  const ScoreHeader* h = nullptr;
  int rc = check_score_plan(shape, plan_host, &h);
  if (rc) return rc;
  ScoreArgs a;
  if ((rc = score_args(shape, h, plan_dev, q, k_cache, block_table, scores_in, decay, scores_out,
                       workspace, ws_bytes, &a)))
    return rc;
  if (misaligned_plan(h, plan_dev)) return SSA_ERR_ARG;
  (void)hipGetLastError();
  hipStream_t s = static_cast<hipStream_t>(stream);
  return h->head_dim == 128 ? launch_scores<128>(a, h, s) : launch_scores<64>(a, h, s);
}

int ssa_decode_scored(const ssa_shape* shape, const void* plan_host, const void* plan_dev,
                      const uint16_t* q, const uint16_t* k_cache, const uint16_t* v_cache,
                      const int32_t* block_table, const float* scores_in, float decay,
                      float* scores_out, uint16_t* out, void* workspace, size_t ws_bytes,
                      void* stream) {
  const ScoreHeader* h = nullptr;
  int rc = check_score_plan(shape, plan_host, &h);
  if (rc) return rc;
  if (h->max_q_len > 1) return SSA_ERR_ARG;
  ScoreArgs a;
  if ((rc = score_args(shape, h, plan_dev, q, k_cache, block_table, scores_in, decay, scores_out,
                       workspace, ws_bytes, &a)))
    return rc;
  if (h->max_q_len > 0 && (!v_cache || !out)) return SSA_ERR_NULL;
  if (misaligned({v_cache, out}) || misaligned_plan(h, plan_dev)) return SSA_ERR_ARG;
  a.vc = v_cache;
  a.out = out;
  (void)hipGetLastError();
  hipStream_t s = static_cast<hipStream_t>(stream);
  return h->head_dim == 128 ? launch_decodes<128, true>(a, h, s)
                            : launch_decodes<64, true>(a, h, s);
}

}  // extern "C"
