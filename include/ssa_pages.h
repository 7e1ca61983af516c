/*
 * ssa_pages.h - block tables, free pages and slot maps of the paged KV cache, kept on
 * the device from the requests' lengths.
 *
 * Conventions and error codes as in ssa.h.  The pages that no request holds are a ring:
 *   free_pages  int32 [num_pages]: `count` page indexes from entry `head` on, past the
 *               last entry again from the first
 *   state       int32 [4]: head, count, the status of the call that wrote it, and how
 *               many pages that call was short of
 * A page belongs to one request: the ring knows no sharing.  If two requests' rows named the
 * same page (a common prefix), each that shrank past it would give it back, and it would be
 * handed out twice later: a request must not shrink past a page that another one holds.
 * A program starts with all pages free: free_pages = 0 .. num_pages - 1, state =
 * {0, num_pages, 0, 0}.
 */
#ifndef SSA_PAGES_H
#define SSA_PAGES_H

#include <stddef.h>
#include <stdint.h>

#include "ssa.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Status bits (state[2]); with any of them the call changed nothing else. */
#define SSA_PAGES_SHORT 1  /* fewer free pages than the requests need: state[3] are missing */
#define SSA_PAGES_LENGTH 2 /* a length below 0, above 2^30 or of over max_pages_per_req pages */
#define SSA_PAGES_ROWS 4   /* more than max_rows new rows (slots NULL: 2^31 - 1) */
#define SSA_PAGES_RING 8   /* head or count outside the ring, or more pages given back than
                              the ring has room for */

/*
 * Requests go from old_len[i] to new_len[i] cached tokens (one launch).  With p(n) =
 * ceil(n / P):
 *   growing requests   entries p(old) .. p(new) - 1 of block_table's row i take the free
 *                      pages from the ring's head on, in order of request and entry
 *   shrinking ones     (rejected tokens, a cut context, 0: the request ended) entries
 *                      p(new) .. p(old) - 1 go to the ring's end, in that order, and stay
 *                      as they are in the table; they can be taken from the next call on
 *   row_start  int32 [num_reqs + 1] or NULL: row_start[i] is the sum over earlier
 *              requests of max(new_len - old_len, 0), the row of request i's first new
 *              token (q_start of ssa.h); the last entry is their number
 *   slots      int64 [max_rows] or NULL: for row row_start[i] + j, the token at position
 *              t = old_len[i] + j, block_table[i][t / P] * P + t % P.  Rows behind the
 *              last one are left as they are.
 *   state      what the last call wrote (read only); state_out must be another buffer:
 *              a program takes two by turns
 * Lengths, table, ring and states are device memory.  What only the device knows is
 * checked there: state_out[2] says what was wrong (then head and count are those of
 * state, and table, ring, rows and slots stay as they were); it is not an error code.
 * Made for some thousands of requests: 500 take 8 us, 5000 30 us, 65536 0.7 ms.
 * Errors: NULL; SHAPE, HEAD_DIM, PAGE_SIZE, PAGES, SCALE of the shape; LENGTH (num_reqs
 * below 0 or above 65536); ARG (max_rows < 0, or state_out overlaps state); HIP.
 */
int ssa_pages_resize(const ssa_shape* shape, int32_t num_reqs, const int32_t* old_len,
                     const int32_t* new_len, int32_t* block_table, int32_t* free_pages,
                     const int32_t* state, int32_t* state_out, int32_t* row_start, int64_t* slots,
                     int64_t max_rows, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* SSA_PAGES_H */
