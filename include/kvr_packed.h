/*
 * kvr_packed.h -- K/V held in 4 bits: a packed arena beside the retained one.
 *
 * The replacement worker keeps K/V in a retained arena (kvr.h).  A packed arena
 * holds the same rows in 17/64 of the bf16 bytes: interrupted or waiting requests
 * are parked in it and brought back, and generation can attend (and resume) over
 * it directly.  Same conventions as kvr.h (status codes, host/device pointers,
 * void* streams, host-side validation before any device work, thread-compatible:
 * calls on one packed arena must not overlap where one of them writes it).
 *
 * Values.  The head dim's elements are taken 32 at a time.  A group's scale is the
 * least power of two 2^e, -120 <= e <= 125, with max|x| <= 6 * 2^e; each x is held
 * as a sign and the nearest of {0, 0.5, 1, 1.5, 2, 3, 4, 6} to |x| / 2^e, ties to
 * the even code (0, 1, 2, 4).  A group with a value that is not finite reads as NaN
 * in all 32.
 *
 * Layout.  Per layer, block, kv head and tile of 16 slots one record of 17 d bytes:
 *   record(l, b, h, t) = (((l*num_blocks + b)*nkv + h)*(block_size/16) + t) * 17 d
 *   K values  at 0        [16 slots][d/2]
 *   V values  at 8 d      [4][16][4][d/32]: slots 4i .. 4i+3, sixteenth of the dims, slot
 *   K scales  at 16 d     [16 slots][d/32]
 *   V scales  at 16.5 d   [4][d/32][4]: slots 4i .. 4i+3, group, slot
 * A byte of values holds two of them, the even dim in the low four bits: 8 for the
 * sign and 0 .. 7 for the magnitudes above.  A scale byte holds e + 127, 255 for NaN.
 * (A record is what one wave of the attention reads in one go: a tile's K and V
 * values are two contiguous loads of 16 bytes a lane at d = 128, each lane's bytes
 * already those of its matrix operand.)
 */
#ifndef KVR_PACKED_H
#define KVR_PACKED_H

#include <stdint.h>

#include "kvr.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct kv_packed* kv_packed_t;

/* Bytes of a packed arena; 0 for an invalid description (kvr.h's rules, and
 * head_dim % 32 == 0), a block_size that is not a positive multiple of 16, or
 * num_blocks <= 0. */
uint64_t kv_packed_bytes(const kv_model_desc* desc, int32_t block_size, int64_t num_blocks);

/* Bind a packed arena: `base` is device memory on `device`, on a boundary of 16
 * bytes, of at least kv_packed_bytes bytes.  Checked like kv_arena_bind's, health
 * probe included; never written.  *out receives the handle. */
kv_status kv_packed_bind(void* base, uint64_t bytes, const kv_model_desc* desc,
                         int32_t block_size, int64_t num_blocks, int32_t device,
                         kv_packed_t* out);
/* Drop a handle.  Never frees or writes `base`. */
kv_status kv_packed_release(kv_packed_t packed);

/* Store K/V rows of one layer.
 *   k, v        device [rows][nkv][d] in the model dtype, rows k_stride / v_stride
 *               elements apart (even ones in bf16)
 *   slots       device int64 [rows]: row i goes to slot slots[i] = block *
 *               block_size + position % block_size (as kv_tables_grow lists them);
 *               rows whose slot lies outside the arena (-1, say) are passed over.
 *               A slot listed more than once holds undefined values afterwards.
 * Writes exactly the listed slots of the layer. */
kv_status kv_packed_store(kv_packed_t packed, int32_t layer, const void* k, int64_t k_stride,
                          const void* v, int64_t v_stride, const int64_t* slots, int64_t rows,
                          void* stream);
/* The way back: row i of k, v receives the values slot slots[i] holds, in the
 * model dtype (exactly: every one of them is a bf16 number).  Rows whose slot lies
 * outside the arena keep their bits. */
kv_status kv_packed_load(kv_packed_t packed, int32_t layer, void* k, int64_t k_stride, void* v,
                         int64_t v_stride, const int64_t* slots, int64_t rows, void* stream);

/* Park: every layer's K/V of the retained arena's slots arena_slots[i] (device
 * int64 [rows]) into the packed arena's slots packed_slots[i].  Restore: the way
 * back.  The two arenas describe the same model on one device; block sizes and
 * tables are their own.  Pairs with a slot outside its arena are passed over, a
 * destination listed more than once holds undefined values afterwards.
 * For these four:
 *   KV_EINVAL  null arrays, rows outside 0 .. 2^31 - 1, a layer outside the model, a
 *              stride below nkv * d, a pointer or stride not on its boundary
 *   KV_ESTATE  unknown handle, arenas of different models or devices */
kv_status kv_packed_park(kv_arena_t arena, const int64_t* arena_slots, kv_packed_t packed,
                         const int64_t* packed_slots, int64_t rows, void* stream);
kv_status kv_packed_restore(kv_packed_t packed, const int64_t* packed_slots, kv_arena_t arena,
                            const int64_t* arena_slots, int64_t rows, void* stream);

/* Workspace bytes of kv_packed_attention for up to num_requests requests, `rows`
 * query rows in all, at most max_query of one request, lengths up to max_len; 0 for
 * an invalid description (kv_packed_bytes's, at most 16 q heads per kv head) or
 * sizes that no call takes (requests and rows are 1 .. 2^24, max_len below 2^31). */
uint64_t kv_packed_attention_workspace_bytes(const kv_model_desc* desc, int32_t num_requests,
                                             int64_t rows, int32_t max_query, int64_t max_len);

/* Attention of one layer over a packed arena: one new token of each request, or
 * several (drafted tokens to be checked, a prompt's next piece).
 *   q            device [rows][nq][d], model dtype, rows q_stride elements apart
 *   q_offsets    device int32 [num_requests + 1]: request r's query rows are
 *                q_offsets[r] .. q_offsets[r+1] - 1; NULL: row r is request r's only
 *                one, rows == num_requests
 *   lens         device int32 [num_requests]: positions of request r in the arena,
 *                its query rows' own included (stored before the call); of m query
 *                rows, row i is at position lens[r] - m + i
 *   block_tables device int32 [num_requests][max_blocks_per_req]
 *   max_query, max_len  host bounds of a request's query rows and length: its rows and
 *                positions past them are left out (row i stays at lens[r] - m + i).
 *                The workspace and the work of a call are sized by them;
 *                (num_requests + rows * nq/nkv / 16) * (max_len / 32 + 5) below 2^31
 *                always goes
 *   out          device [rows][nq][d], model dtype, rows out_stride elements apart
 *   workspace    device scratch, on a boundary of 16 bytes; calls in flight at once
 *                need one each
 * Row i attends positions 0 .. its own: out = sum_j p_j v_j, p the softmax of
 * q . k_j / sqrt(d), q head h reading kv head h / (nq/nkv).  Scores, softmax and sums
 * are fp32, the output is rounded once; values next to the largest number do not overflow
 * on the way (below 2^-86 they may count as 0 beside values of 2^65 and more).  Positions
 * in a block whose table entry is outside the arena, and those past max_len or
 * max_blocks_per_req, are left out; a row that is left with no position, or with none whose
 * score is above -infinity, is zero.
 * Requests may share blocks, not query rows: q_offsets does not decrease.  Nothing but
 * the requests' rows of out is written; q and out may be the same memory only as the
 * same rows.  The arrays on the device are read when the call runs there, so a captured
 * call follows their contents.
 *   KV_EINVAL  null arrays, a layer outside the model, negative sizes, rows or
 *              num_requests above 2^24, a stride below nq * d, a pointer or stride not
 *              on its boundary (4 bytes), more than 16 q heads per kv head, rows !=
 *              num_requests without q_offsets, max_query or max_len < 1, more work
 *              than 2^31 units
 *   KV_ENOMEM  workspace smaller than kv_packed_attention_workspace_bytes
 *   KV_ESTATE  unknown handle */
kv_status kv_packed_attention(kv_packed_t packed, int32_t layer, const void* q, int64_t q_stride,
                              const int32_t* q_offsets, int64_t rows, const int32_t* lens,
                              const int32_t* block_tables, int32_t num_requests,
                              int32_t max_blocks_per_req, int32_t max_query, int64_t max_len,
                              void* out, int64_t out_stride, void* workspace,
                              uint64_t workspace_bytes, void* stream);

/* Workspace bytes of kv_packed_decode_step for up to num_requests requests whose
 * positions are all < max_position; 0 for an invalid description or sizes. */
uint64_t kv_packed_decode_workspace_bytes(const kv_model_desc* desc, int32_t num_requests,
                                          int64_t max_position);

/* One greedy decode step over a packed arena: kv_decode_step (kvr_decode.h) with the
 * context's K/V in a packed arena, the new position's K/V stored there in every layer
 * before that layer's attention reads it.  Arguments, outputs and status codes are
 * kv_decode_step's; besides, KV_EINVAL where kv_packed_attention would not take the step's
 * attention: above 2^24 requests, a position of 2^31 - 1, or more work than 2^31 units. */
kv_status kv_packed_decode_step(const kv_weights* w, const void* final_norm, const void* lm_head,
                                const int32_t* tokens, const int32_t* positions,
                                int32_t num_requests, const int32_t* block_tables,
                                int32_t max_blocks_per_req, kv_packed_t packed, void* workspace,
                                uint64_t workspace_bytes, void* stream, int32_t* next_tokens,
                                float* logits);

#ifdef __cplusplus
}
#endif
#endif
