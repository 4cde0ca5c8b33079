/*
 * kvr_append.h -- rows of a layer's q, k and v products into the retained arena.
 *
 * kv_rebuild and kv_decode_step run a whole model and put its K/V into the arena
 * on the way.  A worker that runs its own layers (drafted tokens to be checked, a
 * prompt's next piece, another sampler) puts them there with kv_append: bias,
 * per-head norm, rotation, rounding and the way into the slots in one pass over the
 * products.  kv_tables_grow (kvr_tables.h) lists the slots and positions,
 * kv_group_attention (kvr_attention.h) reads what was stored.  Same conventions as
 * kvr.h (status codes, host/device pointers, void* streams, host-side validation
 * before any device work, thread-compatible).
 */
#ifndef KVR_APPEND_H
#define KVR_APPEND_H

#include <stdint.h>

#include "kvr.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Rows of one layer.
 *   weights     host, the layer's: q_norm and k_norm are read where the arena's
 *               model has qk_norm, bq, bk and bv where it has qkv_bias (device
 *               pointers, as in kvr.h); NULL goes for a model with neither
 *   q, k, v     device [rows][nq or nkv][d] in the model dtype, the plain products,
 *               rows q_stride / k_stride / v_stride elements apart (even ones in
 *               bf16), so that the three may lie side by side in the rows of one
 *               product; q NULL: k and v alone
 *   positions   device int32 [rows]; a row whose position is negative is passed over
 *   slots       device int64 [rows]: row i's K and V go to slot slots[i] = block *
 *               block_size + position % block_size; where it lies outside the arena
 *               (-1, say) neither is stored.  A slot listed more than once holds
 *               undefined values afterwards
 *   q_out       device [rows][nq][d], model dtype, rows q_out_stride elements apart:
 *               the rotated q, in any row whose position is not negative; may be q
 *               itself with the same stride.  NULL exactly where q is
 * Each head x of q and k: x + bias; with qk_norm times its gain over sqrt(mean x^2 +
 * rms_eps); then the pairs (x_i, x_{i + d/2}) turned by the angle position *
 * rope_theta^(-2i/d), taken in fp64 and its cosine and sine rounded once to fp32.  V:
 * v + bias.  All of it in fp32, rounded once on the way out; values that are not finite
 * take the way that arithmetic gives them, and nothing else is affected by them.
 * Writes exactly the listed slots of the layer and those rows of q_out.  The arrays on the
 * device are read when the call runs there, so a captured call follows their contents.
 *   KV_EINVAL  null arrays, rows outside 0 .. 2^31 - 1, a layer outside the model, a stride
 *              below its row, a pointer or stride not on its boundary (4 bytes; weights
 *              too; slots 8), weights that the model needs missing
 *   KV_ESTATE  unknown handle
 *   KV_EDEVICE device not selectable, or a device error */
kv_status kv_append(kv_arena_t arena, int32_t layer, const kv_layer_weights* weights, const void* q,
                    int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                    int64_t v_stride, const int32_t* positions, const int64_t* slots, int64_t rows,
                    void* q_out, int64_t q_out_stride, void* stream);

#ifdef __cplusplus
}
#endif
#endif
