/*
 * kvr_tables.h -- block tables and slot maps built on the GPU.
 *
 * The rebuild and the decode step take block tables from the host.  A serving
 * step that never leaves the device (one captured into a HIP graph, say) grows
 * them there: kv_tables_grow gives every request the blocks its new positions
 * need, from a list of free blocks, and lists those positions' arena slots, as
 * kv_packed_store and kv_packed_attention (kvr_packed.h) read them.  Same
 * conventions as kvr.h (status codes, void* streams, host-side validation before
 * any device work, thread-compatible).
 */
#ifndef KVR_TABLES_H
#define KVR_TABLES_H

#include <stdint.h>

#include "kvr.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Grow the block tables of a request set and list the new positions.  With
 * held_r positions placed so far and len_r wanted, request r needs the table
 * entries ceil(held_r/B) .. min(ceil(len_r/B), max_blocks_per_req) - 1; requests
 * take them in order from the front of free_blocks.
 *   held           device int32 [num_requests], positions that have slots
 *                  already (NULL: none); a negative one counts as 0
 *   lens           device int32 [num_requests]; a request with len <= held
 *                  grows nothing.  The sum of the new positions stays below 2^31
 *   free_blocks    device int32 [num_free] block ids, handed out as they are.  A
 *                  negative one counts as a block: it is written to its table entry,
 *                  whose rows get slot -1 without being among counts[3]
 *   block_tables   device int32 [num_requests][max_blocks_per_req], in and out:
 *                  the needed entries are written (-1 where the free list has
 *                  ended), all others keep their bits
 *   max_rows       entries of slots and positions (0 .. 2^31 - 1)
 *   row_offsets    device int32 [num_requests + 1], written: request r's new
 *                  positions held_r .. len_r - 1 are rows row_offsets[r] ..
 *                  row_offsets[r+1] - 1
 *   slots          device int64 [max_rows], written: per row its arena slot
 *                  block * B + position % B; -1 where the request has no block
 *                  there (free list ended, table full, a negative entry) and in
 *                  every row behind the last.  Rows past max_rows are not listed;
 *                  their table entries are written all the same
 *   positions      optional device int32 [max_rows] (NULL = none), written: per
 *                  row its position, -1 behind the last row
 *   counts         device int32 [4], written: blocks taken from the list, blocks
 *                  it lacked, rows, rows without a slot (for lack of a block, of
 *                  room in the table, or in a negative entry held before)
 * No host synchronisation, no workspace; the same call again writes the same.
 *   KV_EINVAL  null arrays, num_requests, num_free, max_blocks_per_req or
 *              max_rows < 0, num_requests above 2^30, block_size <= 0, an array not
 *              on its elements' boundary
 *   KV_EDEVICE device not selectable, or a device error */
kv_status kv_tables_grow(const int32_t* held, const int32_t* lens, int32_t num_requests,
                         int32_t block_size, const int32_t* free_blocks, int32_t num_free,
                         int32_t* block_tables, int32_t max_blocks_per_req, int64_t max_rows,
                         int32_t* row_offsets, int64_t* slots, int32_t* positions, int32_t* counts,
                         int32_t device, void* stream);

#ifdef __cplusplus
}
#endif
#endif
