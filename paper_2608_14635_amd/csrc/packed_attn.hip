// Attention over a packed arena (kvr_packed.h).
//
// The plain form: one wave a (query row, q head), a key per lane, online softmax in
// the exp2 domain; P.V with the dims over the lanes.
#include <algorithm>

#include "common.h"
#include "host.h"
#include "kvr_packed.h"
#include "launch.h"
#include "packed.h"

namespace kvr {
namespace {

__constant__ float MAGNITUDE[8] = {0.0f, 0.5f, 1.0f, 1.5f, 2.0f, 3.0f, 4.0f, 6.0f};

__device__ __forceinline__ float code_value(uint32_t c, uint32_t byte) {
  const float m = MAGNITUDE[c & 7];
  return (c & 8 ? -m : m) * __uint_as_float(byte == PK_NAN ? 0x7fc00000u : byte << 23);
}

template <typename T, int D>
__global__ __launch_bounds__(64) void packed_attn_plain_kernel(PackedAttnParams p) {
  __shared__ float s_q[D], s_p[64];
  __shared__ int64_t s_rec[64];
  const int lane = threadIdx.x;
  const int64_t row = blockIdx.x;
  const int h = blockIdx.y, nkv = p.packed.nkv, g = p.nq / nkv, kvh = h / g, B = p.packed.block_size;
  int r = (int)row, m = 1, i = 0;
  if (p.q_offsets) {
    int a = 0, b = p.R - 1;  // the last request whose first row is not past `row`
    while (a < b) {
      const int c = (a + b + 1) / 2;
      if (p.q_offsets[c] <= row) a = c;
      else b = c - 1;
    }
    r = a;
    i = (int)(row - p.q_offsets[r]);
    m = p.q_offsets[r + 1] - p.q_offsets[r];
    if (i < 0 || i >= m) return;
  }
  const int64_t len = min((int64_t)p.lens[r], (int64_t)p.max_blocks * B);
  const int64_t end = min(len, (int64_t)p.lens[r] - m + i + 1);
  for (int e = lane; e < D; e += 64)
    s_q[e] = Elem<T>::load(reinterpret_cast<const T*>(p.q + row * p.q_stride), (int64_t)h * D + e);
  __syncthreads();
  float mx = -INFINITY, l = 0.0f, o[(D + 63) / 64] = {};
  const float scale = 1.4426950408889634f / sqrtf((float)D);
  for (int64_t k0 = 0; k0 < end; k0 += 64) {
    const int64_t j = k0 + lane;
    float s = -INFINITY;
    s_rec[lane] = -1;
    if (j < end) {
      const int64_t blk = p.tables[(int64_t)r * p.max_blocks + j / B];
      if (blk >= 0 && blk < p.num_blocks) {
        const int64_t slot = blk * B + j % B;
        s_rec[lane] = slot;
        const char* rec = packed_record(p.packed, slot, kvh, D);
        const int c = (int)(slot % PK_TILE);
        s = 0.0f;
        for (int e = 0; e < D; ++e) {
          const uint32_t byte = (uint8_t)rec[c * (D / 2) + e / 2];
          s = fmaf(s_q[e], code_value(byte >> 4 * (e & 1), (uint8_t)rec[16 * D + c * (D / 32) + e / 32]), s);
        }
        s *= scale;
      }
    }
    float top = s;
#pragma unroll
    for (int w = 32; w > 0; w >>= 1) top = fmaxf(top, __shfl_xor(top, w, 64));
    const float m_new = fmaxf(mx, top);
    if (__all(s_rec[lane] < 0)) continue;
    const float alpha = mx == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mx - m_new);
    const float pr = s_rec[lane] < 0 ? 0.0f : __builtin_amdgcn_exp2f(s - m_new);
    l = l * alpha + wave_sum(pr);
    mx = m_new;
    s_p[lane] = pr;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < (D + 63) / 64; ++x) {
      const int e = x * 64 + lane;
      if (e < D) {
        o[x] *= alpha;
        for (int k = 0; k < 64; ++k)
          if (s_rec[k] >= 0) {
            const char* rec = packed_record(p.packed, s_rec[k], kvh, D);
            const int c = (int)(s_rec[k] % PK_TILE);
            const uint32_t byte = (uint8_t)rec[8 * D + (c / 4) * (2 * D) + (e / (D / 16)) * (D / 8) +
                                               (c % 4) * (D / 32) + e % (D / 16) / 2];
            const uint32_t sb = (uint8_t)rec[16 * D + D / 2 + (c / 4) * (D / 8) + (e / 32) * 4 + c % 4];
            o[x] = fmaf(s_p[k], code_value(byte >> 4 * (e & 1), sb), o[x]);
          }
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int x = 0; x < (D + 63) / 64; ++x) {
    const int e = x * 64 + lane;
    if (e < D)
      Elem<T>::store(reinterpret_cast<T*>(p.out + row * p.out_stride), (int64_t)h * D + e,
                     l == 0.0f ? 0.0f : o[x] / l);
  }
}

}  // namespace

void launch_packed_attention(int dtype, int d, const PackedAttnParams& p, hipStream_t s) {
  const dim3 grid((unsigned)p.rows, p.nq);
  if (dtype == KV_BF16)
    hipLaunchKernelGGL((packed_attn_plain_kernel<bf16_t, 128>), grid, dim3(64), 0, s, p);
  else if (d == 128)
    hipLaunchKernelGGL((packed_attn_plain_kernel<float, 128>), grid, dim3(64), 0, s, p);
  else if (d == 64)
    hipLaunchKernelGGL((packed_attn_plain_kernel<float, 64>), grid, dim3(64), 0, s, p);
  else
    hipLaunchKernelGGL((packed_attn_plain_kernel<float, 32>), grid, dim3(64), 0, s, p);
}

}  // namespace kvr

using namespace kvr;

namespace {

void run(const kv_packed* packed, int32_t layer, const void* q, int64_t q_stride, const int32_t* q_offsets,
         int64_t rows, const int32_t* lens, const int32_t* tables, int R, int max_blocks, int32_t max_query,
         int64_t max_len, void* out, int64_t out_stride, void* workspace, hipStream_t s) {
  const kv_model_desc& d = packed->desc;
  const int64_t e = elem_bytes(d.dtype);
  PackedAttnParams p{};
  p.packed = packed_layer(packed, layer);
  p.num_blocks = packed->num_blocks;
  p.q = static_cast<const char*>(q);
  p.out = static_cast<char*>(out);
  p.q_stride = q_stride * e;
  p.out_stride = out_stride * e;
  p.q_offsets = q_offsets;
  p.rows = rows;
  p.lens = lens;
  p.tables = tables;
  p.R = R;
  p.max_blocks = max_blocks;
  p.nq = d.num_q_heads;
  launch_packed_attention(d.dtype, d.head_dim, p, s);
}

}  // namespace

void kvr::packed_attention_step(const kv_packed* a, int32_t layer, const void* q, const int32_t* lens,
                                const int32_t* tables, int R, int max_blocks, int64_t max_len, void* out,
                                void* workspace, hipStream_t s) {
  const int64_t row = (int64_t)a->desc.num_q_heads * a->desc.head_dim;
  run(a, layer, q, row, nullptr, R, lens, tables, R, max_blocks, 1, max_len, out, row, workspace, s);
}

extern "C" {

uint64_t kv_packed_attention_workspace_bytes(const kv_model_desc* desc, int32_t num_requests, int64_t rows,
                                             int32_t max_query, int64_t max_len) {
  if (kv_packed_bytes(desc, PK_TILE, 1) == 0 || desc->num_q_heads / desc->num_kv_heads > 16) return 0;
  if (num_requests <= 0 || rows <= 0 || max_query <= 0 || max_len <= 0) return 0;
  return 256;
}

kv_status kv_packed_attention(kv_packed_t packed, int32_t layer, const void* q, int64_t q_stride,
                              const int32_t* q_offsets, int64_t rows, const int32_t* lens, const int32_t* tables,
                              int32_t R, int32_t max_blocks, int32_t max_query, int64_t max_len, void* out,
                              int64_t out_stride, void* workspace, uint64_t ws_bytes, void* stream) {
  if (!live_packed(packed)) return kvr_err::set(KV_ESTATE, "unknown or released packed arena handle");
  const kv_model_desc& d = packed->desc;
  const int64_t e = elem_bytes(d.dtype), row = (int64_t)d.num_q_heads * d.head_dim;
  if (d.num_q_heads / d.num_kv_heads > 16)
    return kvr_err::set(KV_EINVAL, "packed attention supports at most 16 q heads per kv head");
  if (layer < 0 || layer >= d.num_layers)
    return kvr_err::set(KV_EINVAL, "layer %d outside [0, %d)", layer, d.num_layers);
  if (R < 0 || rows < 0 || rows > INT32_MAX || max_blocks < 0)
    return kvr_err::set(KV_EINVAL, "num_requests, rows and max_blocks_per_req are 0 .. 2^31 - 1");
  if (!q_offsets && rows != R) return kvr_err::set(KV_EINVAL, "without q_offsets rows must equal num_requests");
  if (R == 0 || rows == 0) return kvr_err::clear();
  if (max_query < 1 || max_len < 1) return kvr_err::set(KV_EINVAL, "max_query and max_len must be positive");
  if (!q || !out || !lens || (max_blocks > 0 && !tables)) return kvr_err::set(KV_EINVAL, "null q, out, lens or block_tables");
  if (q_stride < row || out_stride < row)
    return kvr_err::set(KV_EINVAL, "a stride is below the row's %lld elements", (long long)row);
  if (((uintptr_t)q | (uintptr_t)out | (uintptr_t)(q_stride * e) | (uintptr_t)(out_stride * e) | (uintptr_t)q_offsets |
       (uintptr_t)lens | (uintptr_t)tables) % 4 != 0)
    return kvr_err::set(KV_EINVAL, "the arrays and the strides need boundaries of 4 bytes");
  if (!workspace || (uintptr_t)workspace % 16 != 0)
    return kvr_err::set(KV_EINVAL, "null workspace, or one not on a boundary of 16 bytes");
  const uint64_t need = kv_packed_attention_workspace_bytes(&d, R, rows, max_query, max_len);
  if (need > ws_bytes)
    return kvr_err::set(KV_ENOMEM, "workspace of %llu bytes < %llu needed", (unsigned long long)ws_bytes,
                        (unsigned long long)need);
  DeviceGuard dg(packed->device);
  const kv_status st = device_ready(dg, packed->device);
  if (st != KV_OK) return st;
  run(packed, layer, q, q_stride, q_offsets, rows, lens, tables, R, max_blocks, max_query, max_len, out, out_stride,
      workspace, reinterpret_cast<hipStream_t>(stream));
  return launched();
}

}  // extern "C"
