// HIP kernel for gfx950 of ssa_pages_resize (include/ssa_pages.h).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "../../include/ssa_pages.h"

namespace ssa {
int validate_shape(const ssa_shape* s);
}

namespace {

constexpr int kPage = SSA_PAGE_SIZE;
constexpr int kMaxReqs = 65536;
constexpr int kMaxTokens = 1 << 30;  // of a request
constexpr int kWavesPerGroup = 4;
constexpr int kWholeWaves = 512;  // requests that have a wave (and its pieces) to themselves

struct PagesArgs {
  int32_t n, per, pieces;  // requests: all, of a wave; pieces of a request
  int32_t num_pages, maxp, most;  // most: of a request's tokens
  const int32_t* old_len;
  const int32_t* new_len;
  int32_t* table;
  int32_t* ring;
  const int32_t* state;
  int32_t* state_out;
  int32_t* row_start;
  int64_t* slots;
  int64_t max_rows;
};

// Sums that stay at 2^32 - 1 instead of passing it: what is left of valid ones is below
// 2^31.
__device__ __forceinline__ uint32_t add(uint32_t a, uint32_t b) {
  return __builtin_elementwise_add_sat(a, b);
}
__device__ __forceinline__ uint32_t wave_sum(uint32_t x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x = add(x, (uint32_t)__shfl_xor((int)x, o, 64));
  return x;
}
struct Sums {
  uint32_t taken, given, rows;
  __device__ __forceinline__ void count(int from, int to) {
    const int p = pages_of(from), q = pages_of(to);
    taken = add(taken, max(q - p, 0));
    given = add(given, max(p - q, 0));
    rows = add(rows, max(to - from, 0));
  }
  __device__ __forceinline__ Sums over_wave() const {
    return Sums{wave_sum(taken), wave_sum(given), wave_sum(rows)};
  }
  static __device__ __forceinline__ int pages_of(int len) { return (len + kPage - 1) / kPage; }
};

// A wave takes one piece of each of `per` requests.  It adds up what all requests take, give
// and add itself, those before its own apart: one launch, and no workgroup waits for another.
// The lengths are read by every wave that has something to write (64 requests 512 bytes), so
// latency bounds it as long as the requests are some thousands: the lengths, then the ring
// or the table.  (64 decodes 3.1 us; 504 requests with 58804 new rows 8.7; with waves
// that had nothing to write adding up too 18.)  More than 512 requests share waves, which
// would read too much between them otherwise: 1000 decodes take 10 us (with a wave each 16),
// 5000 30 (178).
__global__ __launch_bounds__(64 * kWavesPerGroup) void pages_resize_kernel(PagesArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t)blockIdx.x * kWavesPerGroup +
                       __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int req0 = (int)(unit / a.pieces) * a.per, piece = (int)(unit % a.pieces);
  if (req0 > 0 && req0 >= a.n) return;  // no requests: one wave copies the state
  const int count_own = min(a.per, a.n - req0);
  // lane i: lengths of request req0 + i
  const int own_from = lane < count_own ? a.old_len[req0 + lane] : 0;
  const int own_to = lane < count_own ? a.new_len[req0 + lane] : 0;
  // has the piece anything to write?  (Whatever lengths that are none say: the first piece is
  // there, and the others write nothing then.)
  const int64_t tokens = (int64_t)own_to - own_from;
  if (piece > 0 && !__any(tokens > piece * 64 || -tokens / kPage >= piece * 64)) return;
  const int head = a.state[0], count = a.state[1];
  Sums before{0, 0, 0}, all{0, 0, 0};
  bool bad = false;
#pragma unroll 4
  for (int i = lane; i < a.n; i += 64) {
    const int f = a.old_len[i], t = a.new_len[i];
    if (f < 0 || t < 0 || f > a.most || t > a.most) {
      bad = true;
      continue;
    }
    all.count(f, t);
    if (i < req0) before.count(f, t);
  }
  all = all.over_wave();
  before = before.over_wave();
  int status = __any(bad) ? SSA_PAGES_LENGTH : 0;
  uint32_t missing = 0;
  if (head < 0 || head >= a.num_pages || count < 0 || count > a.num_pages) {
    status |= SSA_PAGES_RING;
  } else if (!status) {
    if (all.taken > (uint32_t)count) {
      status |= SSA_PAGES_SHORT;
      missing = all.taken - (uint32_t)count;
    }
    if ((int64_t)count + all.given > a.num_pages) status |= SSA_PAGES_RING;
  }
  if (all.rows > (a.slots ? min(a.max_rows, (int64_t)INT32_MAX) : INT32_MAX))
    status |= SSA_PAGES_ROWS;
  if (unit == 0 && lane == 0) {
    a.state_out[0] = status ? head : (int)(((int64_t)head + all.taken) % a.num_pages);
    a.state_out[1] = status ? count : (int)(count - (int64_t)all.taken + all.given);
    a.state_out[2] = status;
    a.state_out[3] = (int)min(missing, (uint32_t)INT32_MAX);
    if (!status && a.row_start) a.row_start[0] = 0;
  }
  if (status) return;
  auto wrapped = [&](uint32_t at) {
    return at < (uint32_t)a.num_pages ? at : at - (uint32_t)a.num_pages;
  };
  const int step = a.pieces * 64, mine = piece * 64 + lane;
  for (int i = 0; i < count_own; ++i) {
    const int from = __shfl(own_from, i, 64), to = __shfl(own_to, i, 64), req = req0 + i;
    const int p = Sums::pages_of(from), q = Sums::pages_of(to);
    int32_t* row = a.table + (size_t)req * a.maxp;
    // entry k >= p takes ring entry (head + before.taken + k - p) mod num_pages
    const uint32_t take0 = wrapped((uint32_t)head + before.taken);
    const uint32_t give0 = wrapped(wrapped((uint32_t)head + count) + before.given);
    int64_t* slots = a.slots + before.rows;
    before.count(from, to);
    if (piece == 0 && lane == 0 && a.row_start) a.row_start[req + 1] = (int32_t)before.rows;
#pragma unroll 4
    for (int k = p + mine; k < q; k += step) row[k] = a.ring[wrapped(take0 + (uint32_t)(k - p))];
#pragma unroll 4
    for (int k = q + mine; k < p; k += step) a.ring[wrapped(give0 + (uint32_t)(k - q))] = row[k];
    if (!a.slots) continue;
#pragma unroll 4
    for (int t = from + mine; t < to; t += step) {
      const int k = t / kPage;
      // a page taken by this call from the ring, one of before from the table
      const int32_t* at = k < p ? row + k : a.ring + wrapped(take0 + (uint32_t)(k - p));
      slots[t - from] = (int64_t)*at * kPage + t % kPage;
    }
  }
}

}  // namespace

extern "C" int ssa_pages_resize(const ssa_shape* shape, int32_t num_reqs, const int32_t* old_len,
                                const int32_t* new_len, int32_t* block_table, int32_t* free_pages,
                                const int32_t* state, int32_t* state_out, int32_t* row_start,
                                int64_t* slots, int64_t max_rows, void* stream) {
  const int rc = ssa::validate_shape(shape);
  if (rc) return rc;
  if (num_reqs < 0 || num_reqs > kMaxReqs) return SSA_ERR_LENGTH;
  if (!state || !state_out) return SSA_ERR_NULL;
  const int32_t* const written = state_out;
  if (max_rows < 0 || std::max(state, written) < std::min(state, written) + 4) return SSA_ERR_ARG;
  if (num_reqs > 0 && (!old_len || !new_len || !block_table || !free_pages)) return SSA_ERR_NULL;
  PagesArgs a{};
  a.n = num_reqs;
  a.num_pages = shape->num_pages;
  a.maxp = shape->max_pages_per_req;
  a.most = std::min(shape->max_pages_per_req, kMaxTokens / kPage) * kPage;
  a.old_len = old_len;
  a.new_len = new_len;
  a.table = block_table;
  a.ring = free_pages;
  a.state = state;
  a.state_out = state_out;
  a.row_start = row_start;
  a.slots = slots;
  a.max_rows = max_rows;
  a.pieces = 32;
  a.per = std::min(64, std::max(1, (num_reqs + kWholeWaves - 1) / kWholeWaves));  // one a lane
  const int64_t units = std::max<int64_t>(1, (num_reqs + a.per - 1) / a.per) * a.pieces;
  (void)hipGetLastError();
  hipLaunchKernelGGL(pages_resize_kernel, dim3((units + kWavesPerGroup - 1) / kWavesPerGroup),
                     dim3(64 * kWavesPerGroup), 0, static_cast<hipStream_t>(stream), a);
  return hipGetLastError() == hipSuccess ? SSA_OK : SSA_ERR_HIP;
}
