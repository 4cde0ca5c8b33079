// Addresses inside a packed arena (layout: kvr_packed.h) and its kernels' launches.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kvr.h"

struct kv_packed;

namespace kvr {

constexpr int PK_TILE = 16;    // slots of a record
constexpr int PK_GROUP = 32;   // values that share a scale
constexpr int PK_NAN = 255;    // scale byte of a group that reads as NaN
constexpr int PK_LOW = 7, PK_HIGH = 252;  // scale bytes of finite groups: 2^-120 .. 2^125

// One layer of a packed arena.
struct PackedLayer {
  char* base;
  int64_t slots;      // num_blocks * block_size
  int block_size, nkv;
};

// The record of slot `slot`'s tile of kv head h, d its head dim.
__device__ __forceinline__ char* packed_record(const PackedLayer& p, int64_t slot, int h, int d) {
  const int64_t blk = slot / p.block_size;
  const int t = (int)(slot - blk * p.block_size) / PK_TILE;
  return p.base + ((blk * p.nkv + h) * (p.block_size / PK_TILE) + t) * (17 * (int64_t)d);
}

// Rows between plain K/V and a packed arena, `layers` layers at once.
struct PackedMoveParams {
  PackedLayer packed;          // layer 0 of the call
  int64_t packed_layer;        // bytes from layer to layer
  char* k;                     // plain rows of layer 0
  char* v;
  int64_t k_stride, v_stride;  // bytes from row to row
  int64_t plain_layer;         // bytes from layer to layer
  const int64_t* plain_slots;  // plain row of row i (null: i)
  int64_t plain_rows;          // rows there are
  const int64_t* packed_slots;
  int64_t rows;
  int layers;
};
void launch_packed_move(int dtype, int d, bool to_packed, const PackedMoveParams& p, hipStream_t s);

// Whether the attention takes a call of R requests, `rows` query rows in all, at most
// max_query of one, and lengths up to max_len (all positive): their numbers and the work.
bool packed_attention_takes(const kv_model_desc& d, int64_t R, int64_t rows, int64_t max_query, int64_t max_len);

// What a decode step does with a packed arena: its new rows, dense [rows][nkv][d],
// into their slots, and the attention of one query row a request.
void packed_store_rows(const kv_packed* a, int32_t layer, const void* k, const void* v, const int64_t* slots,
                       int64_t rows, hipStream_t s);
void packed_attention_step(const kv_packed* a, int32_t layer, const void* q, const int32_t* lens,
                           const int32_t* tables, int R, int max_blocks, int64_t max_len, void* out,
                           void* workspace, hipStream_t s);

}  // namespace kvr
