/*
 * kvr_attention.h -- attention over the retained arena, a shared prefix read once.
 *
 * A trainer samples several answers to one prompt, and agents share a system prompt:
 * their requests' block tables name the same blocks for a common prefix, as
 * kv_rebuild_from (kvr_reuse.h) fills them.  kv_group_attention attends over the arena
 * through such tables and reads a group's common positions once for many of its requests,
 * not once for each: for up to 128 pairs of a query row and a q head of one kv head in bf16, 32
 * in fp32 (16 with head_dim 128).  It is 16 in bf16 too where the arena does not start on a
 * boundary of 16 bytes or block_size is no multiple of 4, and in both types where the call's
 * groups have 16 such pairs or fewer on the average.  Calls so short that reading is not what
 * they wait for read them for each request.
 * kv_append (kvr_append.h) stores the rows it reads.  Without groups it is attention over
 * the arena, one or several query rows a request.  Same conventions as kvr.h (status codes,
 * host/device pointers, void* streams, host-side validation before any device work,
 * thread-compatible: calls that only read one arena may overlap).
 */
#ifndef KVR_ATTENTION_H
#define KVR_ATTENTION_H

#include <stdint.h>

#include "kvr.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Workspace bytes of kv_group_attention for up to num_requests requests in up to num_groups
 * groups, `rows` query rows in all, at most max_query of one request, lengths up to max_len,
 * enough for every smaller call too; 0 for an invalid description (kvr.h's rules, head_dim
 * % 32 == 0, at most 16 q heads per kv head) or sizes that no call takes (requests and rows
 * are 1 .. 2^24, groups 0 .. 2^24, max_len below 2^31). */
uint64_t kv_group_attention_workspace_bytes(const kv_model_desc* desc, int32_t num_requests,
                                            int64_t rows, int32_t num_groups, int32_t max_query,
                                            int64_t max_len);

/* Attention of one layer over the arena: one new token of each request, or several (drafted
 * tokens to be checked, a prompt's next piece).
 *   q            device [rows][nq][d], model dtype, rows q_stride elements apart
 *   q_offsets    device int32 [num_requests + 1]: request r's query rows are
 *                q_offsets[r] .. q_offsets[r+1] - 1; NULL: row r is request r's only
 *                one, rows == num_requests
 *   lens         device int32 [num_requests]: positions of request r in the arena,
 *                its query rows' own included (stored before the call); of m query
 *                rows, row i is at position lens[r] - m + i
 *   block_tables device int32 [num_requests][max_blocks_per_req]
 *   group_offsets  device int32 [num_groups + 1]: group g's requests are
 *                group_offsets[g] .. group_offsets[g+1] - 1; requests in none share nothing
 *   prefix_lens  device int32 [num_groups]: the positions 0 .. prefix_lens[g] - 1 of every
 *                request of group g are the same ones.  They are read through the table
 *                of the group's first request alone; any number goes, also one that ends
 *                inside a block (of which requests then have their own copies).  A row whose
 *                position lies before the prefix's end sees the positions up to its own
 *   num_groups   0: group_offsets and prefix_lens are not read
 *   max_query, max_len  host bounds of a request's query rows and length: its rows and
 *                positions past them are left out (row i stays at lens[r] - m + i).
 *                The workspace and the work of a call are sized by them;
 *                (num_requests + num_groups + rows * nq/nkv / 8) * (max_len / 8 + 16)
 *                below 2^31 always goes
 *   out          device [rows][nq][d], model dtype, rows out_stride elements apart
 *   workspace    device scratch, on a boundary of 16 bytes; calls in flight at once
 *                need one each
 * Row i attends positions 0 .. its own: out = sum_j p_j v_j, p the softmax of q . k_j / sqrt(d),
 * q head h reading kv head h / (nq/nkv).  Scores, softmax and sums are fp32 (in bf16 models a
 * weight enters the product with V as two bf16 numbers, which with its exponent's rounding are
 * off by 2^-16 of it), the output is rounded once; values next to the largest number do not
 * overflow on the way (below 2^-86 they may count as 0).  Positions in a block whose table entry
 * is outside the arena, and those past max_len or max_blocks_per_req, are left out; a row that
 * is left with no position, or with none whose score is above -infinity, is zero.  What lies at
 * positions that a row does not see changes nothing in it; a key that is not finite makes NaN of
 * the rows that see it (or, with a score of -infinity, nothing), a value that is not finite
 * makes NaN or an infinity of its dim in them.
 * Requests may share blocks, not query rows: q_offsets and group_offsets do not decrease.
 * Nothing but the requests' rows of out is written; q and out may be the same memory only as
 * the same rows, with the same stride.  Results do not depend on timing.  The arrays on the
 * device are read when the call runs there, so a captured call follows their contents.
 *   KV_EINVAL  null arrays, a layer outside the model, negative sizes, rows, num_requests
 *              or num_groups above 2^24, a stride below nq * d, a pointer or stride not on its
 *              boundary (4 bytes), several rows of out over q with another stride, more
 *              than 16 q heads per kv head, head_dim % 32 != 0, an arena of 2^31 slots or
 *              more, rows != num_requests without q_offsets, max_query or max_len < 1, more
 *              work than 2^31 units
 *   KV_ENOMEM  workspace smaller than kv_group_attention_workspace_bytes
 *   KV_ESTATE  unknown handle
 *   KV_EDEVICE device not selectable, or a device error */
kv_status kv_group_attention(kv_arena_t arena, int32_t layer, const void* q, int64_t q_stride,
                             const int32_t* q_offsets, int64_t rows, const int32_t* lens,
                             const int32_t* block_tables, int32_t num_requests,
                             int32_t max_blocks_per_req, const int32_t* group_offsets,
                             const int32_t* prefix_lens, int32_t num_groups, int32_t max_query,
                             int64_t max_len, void* out, int64_t out_stride, void* workspace,
                             uint64_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif
