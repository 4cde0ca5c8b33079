// Rows between plain K/V and a packed arena (kvr_packed.h), and the entry points
// that move them.
//
// A lane holds 8 consecutive values of a row: 16 bytes of bf16 (two 16-byte loads
// of fp32) on one side, one 4-byte word of codes on the other; four neighbouring
// lanes make a group and agree on its scale with two exchanges.  gfx950 converts
// two values at a time with the scale's exponent applied, to the nearest code, ties
// to even (v_cvt_scalef32_pk_fp4_f32 and its inverse), which is the definition.
// A wave takes 4 consecutive rows of one kv head (8 or 16 of smaller heads) at a time,
// K and V; rows in consecutive slots fill whole lines of a record.  The four waves of a
// workgroup take neighbouring heads, so that together they read whole rows.  Bound by
// HBM: 2 bytes in and 17/32 out a value in bf16 (65K tokens of 4 layers: 1.27 GB each
// way at 4.2 TB/s in and 5.3 out; a plain copy reaches 4.8).
#include <algorithm>
#include <memory>
#include <mutex>
#include <new>
#include <set>

#include "common.h"
#include "host.h"
#include "kvr_packed.h"
#include "launch.h"
#include "packed.h"

namespace kvr {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_a4 __attribute__((aligned(4)));  // 16 bytes on any 4-byte boundary

// Eight values of a row as they lie in memory, as fp32, and back from codes.
template <typename T> struct Raw8;
template <> struct Raw8<bf16_t> {
  u32x4 u;
  __device__ __forceinline__ void load(const char* p) { u = *reinterpret_cast<const u32x4_a4*>(p); }
  __device__ __forceinline__ void values(float* v) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(u[i] << 16);
      v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
};
template <> struct Raw8<float> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const char* p) {
    a = reinterpret_cast<const f32x4_a4*>(p)[0];
    b = reinterpret_cast<const f32x4_a4*>(p)[1];
  }
  __device__ __forceinline__ void values(float* v) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = a[i];
      v[4 + i] = b[i];
    }
  }
};
__device__ __forceinline__ void put8(char* p, uint32_t codes, float scale, bf16_t) {
  u32x4 u;
  u[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0));
  u[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1));
  u[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2));
  u[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3));
  *reinterpret_cast<u32x4_a4*>(p) = u;
}
__device__ __forceinline__ void put8(char* p, uint32_t codes, float scale, float) {
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0);
  const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1);
  const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2);
  const auto d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
  reinterpret_cast<f32x4_a4*>(p)[0] = f32x4{a[0], a[1], b[0], b[1]};
  reinterpret_cast<f32x4_a4*>(p)[1] = f32x4{c[0], c[1], d[0], d[1]};
}

// The scale byte of a group whose largest |x| has these bits: with |x| = 1.m * 2^(E-127),
// 6 * 2^e = 1.5 * 2^(e+2) takes it from e + 127 = E - 2 on where 1.m <= 1.5, else from E - 1.
__device__ __forceinline__ uint32_t scale_byte(uint32_t most) {
  if (most >= 0x7f800000u) return PK_NAN;
  const int e = (int)(most >> 23) - ((most & 0x7fffff) <= 0x400000 ? 2 : 1);
  return (uint32_t)min(max(e, PK_LOW), PK_HIGH);
}

__device__ __forceinline__ uint32_t encode8(const float* v, uint32_t& byte) {
  uint32_t most = 0;  // of |x|'s bits: they order as the values do, infinities and NaN above all
#pragma unroll
  for (int i = 0; i < 8; ++i) most = max(most, __float_as_uint(v[i]) & 0x7fffffffu);
  most = max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0xb1, 0xf, 0xf, true));  // quad_perm 1 0 3 2
  most = max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0x4e, 0xf, 0xf, true));  // quad_perm 2 3 0 1
  byte = scale_byte(most);
  const float s = __uint_as_float(byte << 23);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], s, 3);
  return c;
}

// The addresses of a lane's word u (values 8u .. 8u+7) of slot c of a record, and of
// group w's scale.
template <int D>
__device__ __forceinline__ int k_word(int c, int u) { return c * (D / 2) + u * 4; }
template <int D>
__device__ __forceinline__ int k_scale(int c, int w) { return 16 * D + c * (D / 32) + w; }
template <int D>
__device__ __forceinline__ int v_scale(int c, int w) { return 16 * D + D / 2 + (c / 4) * (D / 8) + w * 4 + c % 4; }
// V: a word's values lie in 128 / D sixteenths of the dims, D / 16 values each
template <int D>
__device__ __forceinline__ void v_put(char* rec, int c, int u, uint32_t word) {
  constexpr int BYTES = D / 32, PIECES = 4 / BYTES;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    char* dst = rec + 8 * D + (c / 4) * (2 * D) + (u * PIECES + i) * (4 * BYTES) + (c % 4) * BYTES;
    if constexpr (BYTES == 4) *reinterpret_cast<uint32_t*>(dst) = word;
    if constexpr (BYTES == 2) *reinterpret_cast<uint16_t*>(dst) = (uint16_t)(word >> (16 * i));
    if constexpr (BYTES == 1) *reinterpret_cast<uint8_t*>(dst) = (uint8_t)(word >> (8 * i));
  }
}
template <int D>
__device__ __forceinline__ uint32_t v_get(const char* rec, int c, int u) {
  constexpr int BYTES = D / 32, PIECES = 4 / BYTES;
  uint32_t word = 0;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const char* src = rec + 8 * D + (c / 4) * (2 * D) + (u * PIECES + i) * (4 * BYTES) + (c % 4) * BYTES;
    if constexpr (BYTES == 4) word = *reinterpret_cast<const uint32_t*>(src);
    if constexpr (BYTES == 2) word |= (uint32_t)*reinterpret_cast<const uint16_t*>(src) << (16 * i);
    if constexpr (BYTES == 1) word |= (uint32_t)*reinterpret_cast<const uint8_t*>(src) << (8 * i);
  }
  return word;
}

// N: times that a wave takes as many rows as fit it; all loads are on their way before
// the first is used.
template <typename T, int D, bool TO_PACKED, int N>
__global__ __launch_bounds__(256) void packed_move_kernel(PackedMoveParams p) {
  constexpr int LANES = D / 8;                        // lanes of a row
  constexpr int STEP = 64 / LANES;                    // rows of a wave at a time
  const int lane = threadIdx.x & 63, u = lane % LANES;
  const int nkv = p.packed.nkv;
  const int64_t chunks = (p.rows + N * STEP - 1) / (N * STEP), items = chunks * nkv * p.layers;
  for (int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); item < items;
       item += (int64_t)gridDim.x * 4) {
    const int h = (int)(item % nkv);
    const int64_t c = item / nkv % chunks;
    const int l = (int)(item / nkv / chunks);
    PackedLayer pl = p.packed;
    pl.base += l * p.packed_layer;
    const int64_t first = c * (N * STEP) + lane / LANES;
    // a row that does not count is one that does not exist: slot -1.  The four lanes of
    // a group share a row, so they agree.
    int64_t slot[N], from[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t row = first + i * STEP;
      slot[i] = row < p.rows ? p.packed_slots[row] : -1;
      from[i] = row < p.rows && p.plain_slots ? p.plain_slots[row] : row;
    }
    char *rec[N], *k[N], *v[N];
    int s[N];
    bool in[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      in[i] = slot[i] >= 0 && slot[i] < pl.slots && from[i] >= 0 && from[i] < p.plain_rows;
      rec[i] = packed_record(pl, in[i] ? slot[i] : 0, h, D);
      s[i] = (int)(slot[i] & (PK_TILE - 1));
      const int64_t in_row = ((int64_t)h * D + 8 * u) * sizeof(T);
      k[i] = p.k + l * p.plain_layer + from[i] * p.k_stride + in_row;
      v[i] = p.v + l * p.plain_layer + from[i] * p.v_stride + in_row;
    }
    if constexpr (TO_PACKED) {
      Raw8<T> kr[N], vr[N];
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (in[i]) {
          kr[i].load(k[i]);
          vr[i].load(v[i]);
        }
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (in[i]) {
          float x[8], y[8];
          kr[i].values(x);
          vr[i].values(y);
          uint32_t kb, vb;
          const uint32_t kw = encode8(x, kb), vw = encode8(y, vb);
          *reinterpret_cast<uint32_t*>(rec[i] + k_word<D>(s[i], u)) = kw;
          v_put<D>(rec[i], s[i], u, vw);
          if (u % 4 == 0) {
            rec[i][k_scale<D>(s[i], u / 4)] = (char)kb;
            rec[i][v_scale<D>(s[i], u / 4)] = (char)vb;
          }
        }
    } else {
      uint32_t kw[N], vw[N], kb[N], vb[N];
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (in[i]) {
          kw[i] = *reinterpret_cast<const uint32_t*>(rec[i] + k_word<D>(s[i], u));
          vw[i] = v_get<D>(rec[i], s[i], u);
          kb[i] = (uint8_t)rec[i][k_scale<D>(s[i], u / 4)];
          vb[i] = (uint8_t)rec[i][v_scale<D>(s[i], u / 4)];
        }
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (in[i]) {
          put8(k[i], kw[i], __uint_as_float(kb[i] << 23), T{});
          put8(v[i], vw[i], __uint_as_float(vb[i] << 23), T{});
        }
    }
  }
}

// 65K tokens of 4 layers (8 kv heads of 128, bf16) took 325 + 270 us to pack and to load
// with one time, 304 + 237 with two, 308 + 240 with four; 171 tokens of 28 layers (2 kv
// heads) 4.1 + 3.9 with one, 4.3 + 4.0 with two, 5.5 + 4.6 with four: once where that
// leaves the chip's 8192 waves unfilled.
template <typename T, int D>
void launch_move(bool to_packed, const PackedMoveParams& p, hipStream_t s) {
  constexpr int STEP = 64 / (D / 8);
  const int64_t once = (p.rows + STEP - 1) / STEP * p.packed.nkv * p.layers;
  const bool twice = once > 2 * 8192;
  const int64_t items = twice ? (p.rows + 2 * STEP - 1) / (2 * STEP) * p.packed.nkv * p.layers : once;
  const dim3 grid((unsigned)std::min<int64_t>((items + 3) / 4, 1 << 16));
  if (to_packed && twice)
    hipLaunchKernelGGL((packed_move_kernel<T, D, true, 2>), grid, dim3(256), 0, s, p);
  else if (to_packed)
    hipLaunchKernelGGL((packed_move_kernel<T, D, true, 1>), grid, dim3(256), 0, s, p);
  else if (twice)
    hipLaunchKernelGGL((packed_move_kernel<T, D, false, 2>), grid, dim3(256), 0, s, p);
  else
    hipLaunchKernelGGL((packed_move_kernel<T, D, false, 1>), grid, dim3(256), 0, s, p);
}

}  // namespace

void launch_packed_move(int dtype, int d, bool to_packed, const PackedMoveParams& p, hipStream_t s) {
  if (dtype == KV_BF16) launch_move<bf16_t, 128>(to_packed, p, s);
  else if (d == 128) launch_move<float, 128>(to_packed, p, s);
  else if (d == 64) launch_move<float, 64>(to_packed, p, s);
  else launch_move<float, 32>(to_packed, p, s);
}

}  // namespace kvr

using namespace kvr;

namespace {

std::mutex g_mu;
std::set<const void*> g_packed;

uint64_t packed_bytes(const kv_model_desc& d, int32_t block_size, int64_t num_blocks) {
  const unsigned __int128 n = (unsigned __int128)d.num_layers * (uint64_t)num_blocks * (uint64_t)d.num_kv_heads *
                              (uint64_t)(block_size / PK_TILE) * 17 * (uint64_t)d.head_dim;
  return n > (unsigned __int128)INT64_MAX ? 0 : (uint64_t)n;
}

kv_status check_packed(const kv_model_desc* desc, int32_t block_size, int64_t num_blocks) {
  const kv_status st = check_desc(desc);
  if (st != KV_OK) return st;
  if (desc->head_dim % PK_GROUP != 0)
    return kvr_err::set(KV_EINVAL, "packed arenas need head_dim in {32, 64, 128}");
  if (block_size <= 0 || block_size % PK_TILE != 0)
    return kvr_err::set(KV_EINVAL, "packed arenas need a block_size that is a positive multiple of 16");
  if (num_blocks <= 0 || packed_bytes(*desc, block_size, num_blocks) == 0)
    return kvr_err::set(KV_EINVAL, "num_blocks must be positive and the arena below 2^63 bytes");
  return KV_OK;
}

PackedMoveParams move_params(const kv_packed* a, int32_t layer, int layers) {
  PackedMoveParams p{};
  p.packed = packed_layer(a, layer);
  p.packed_layer = (int64_t)(packed_bytes(a->desc, a->block_size, a->num_blocks) / a->desc.num_layers);
  p.layers = layers;
  return p;
}

// one layer's rows, either way
kv_status move_rows(kv_packed* a, bool to_packed, int32_t layer, const void* k, int64_t k_stride,
                    const void* v, int64_t v_stride, const int64_t* slots, int64_t rows, void* stream) {
  if (!live_packed(a)) return kvr_err::set(KV_ESTATE, "unknown or released packed arena handle");
  const kv_model_desc& d = a->desc;
  const int64_t e = elem_bytes(d.dtype), row = (int64_t)d.num_kv_heads * d.head_dim;
  if (layer < 0 || layer >= d.num_layers)
    return kvr_err::set(KV_EINVAL, "layer %d outside [0, %d)", layer, d.num_layers);
  if (rows < 0 || rows > INT32_MAX) return kvr_err::set(KV_EINVAL, "rows must be 0 .. 2^31 - 1");
  if (rows == 0) return kvr_err::clear();
  if (!k || !v || !slots) return kvr_err::set(KV_EINVAL, "null k, v or slots");
  if (k_stride < row || v_stride < row)
    return kvr_err::set(KV_EINVAL, "a stride is below the row's %lld elements", (long long)row);
  if (((uintptr_t)k | (uintptr_t)v | (uintptr_t)(k_stride * e) | (uintptr_t)(v_stride * e)) % 4 != 0 ||
      (uintptr_t)slots % 8 != 0)
    return kvr_err::set(KV_EINVAL, "k, v and their strides need boundaries of 4 bytes, slots one of 8");
  DeviceGuard dg(a->device);
  const kv_status st = device_ready(dg, a->device);
  if (st != KV_OK) return st;
  PackedMoveParams p = move_params(a, layer, 1);
  p.k = static_cast<char*>(const_cast<void*>(k));
  p.v = static_cast<char*>(const_cast<void*>(v));
  p.k_stride = k_stride * e;
  p.v_stride = v_stride * e;
  p.plain_rows = rows;
  p.packed_slots = slots;
  p.rows = rows;
  launch_packed_move(d.dtype, d.head_dim, to_packed, p, reinterpret_cast<hipStream_t>(stream));
  return launched();
}

}  // namespace

void kvr::packed_store_rows(const kv_packed* a, int32_t layer, const void* k, const void* v, const int64_t* slots,
                            int64_t rows, hipStream_t s) {
  const kv_model_desc& d = a->desc;
  PackedMoveParams p = move_params(a, layer, 1);
  p.k = static_cast<char*>(const_cast<void*>(k));
  p.v = static_cast<char*>(const_cast<void*>(v));
  p.k_stride = p.v_stride = (int64_t)d.num_kv_heads * d.head_dim * elem_bytes(d.dtype);
  p.plain_rows = p.rows = rows;
  p.packed_slots = slots;
  launch_packed_move(d.dtype, d.head_dim, true, p, s);
}

namespace {

// every layer, between the two arenas
kv_status move_all(bool to_packed, kv_arena* arena, const int64_t* arena_slots, kv_packed* packed,
                   const int64_t* packed_slots, int64_t rows, void* stream) {
  if (!live_arena(arena)) return kvr_err::set(KV_ESTATE, "unknown or released arena handle");
  if (!live_packed(packed)) return kvr_err::set(KV_ESTATE, "unknown or released packed arena handle");
  const kv_model_desc &d = arena->desc, &b = packed->desc;
  if (d.num_layers != b.num_layers || d.num_kv_heads != b.num_kv_heads || d.head_dim != b.head_dim ||
      d.dtype != b.dtype)
    return kvr_err::set(KV_ESTATE, "the arenas describe different models");
  if (arena->device != packed->device) return kvr_err::set(KV_ESTATE, "the arenas are on different devices");
  if (rows < 0 || rows > INT32_MAX) return kvr_err::set(KV_EINVAL, "rows must be 0 .. 2^31 - 1");
  if (rows == 0) return kvr_err::clear();
  if (!arena_slots || !packed_slots) return kvr_err::set(KV_EINVAL, "null slots");
  if (((uintptr_t)arena_slots | (uintptr_t)packed_slots) % 8 != 0)
    return kvr_err::set(KV_EINVAL, "slots need a boundary of 8 bytes");
  DeviceGuard dg(packed->device);
  const kv_status st = device_ready(dg, packed->device);
  if (st != KV_OK) return st;
  const int64_t row = (int64_t)d.num_kv_heads * d.head_dim * elem_bytes(d.dtype);
  const int64_t plane = arena->num_blocks * arena->block_size * row;
  PackedMoveParams p = move_params(packed, 0, d.num_layers);
  p.k = static_cast<char*>(arena->base);
  p.v = p.k + plane;
  p.k_stride = p.v_stride = row;
  p.plain_layer = 2 * plane;
  p.plain_slots = arena_slots;
  p.plain_rows = arena->num_blocks * arena->block_size;
  p.packed_slots = packed_slots;
  p.rows = rows;
  launch_packed_move(d.dtype, d.head_dim, to_packed, p, reinterpret_cast<hipStream_t>(stream));
  return launched();
}

}  // namespace

bool kvr::live_packed(const kv_packed* a) {
  std::lock_guard<std::mutex> g(g_mu);
  return a && g_packed.count(a);
}

PackedLayer kvr::packed_layer(const kv_packed* a, int32_t layer) {
  const int64_t bytes = (int64_t)(packed_bytes(a->desc, a->block_size, a->num_blocks) / a->desc.num_layers);
  return PackedLayer{static_cast<char*>(a->base) + layer * bytes, a->num_blocks * a->block_size, a->block_size,
                     a->desc.num_kv_heads};
}

extern "C" {

uint64_t kv_packed_bytes(const kv_model_desc* desc, int32_t block_size, int64_t num_blocks) {
  return check_packed(desc, block_size, num_blocks) == KV_OK ? packed_bytes(*desc, block_size, num_blocks) : 0;
}

kv_status kv_packed_bind(void* base, uint64_t bytes, const kv_model_desc* desc, int32_t block_size,
                         int64_t num_blocks, int32_t device, kv_packed_t* out) {
  if (!out) return kvr_err::set(KV_EINVAL, "null output handle");
  *out = nullptr;
  if (!base) return kvr_err::set(KV_EINVAL, "null packed arena base");
  kv_status st = check_packed(desc, block_size, num_blocks);
  if (st != KV_OK) return st;
  if ((uintptr_t)base % 16 != 0) return kvr_err::set(KV_EINVAL, "packed arenas need a boundary of 16 bytes");
  if (packed_bytes(*desc, block_size, num_blocks) > bytes)
    return kvr_err::set(KV_EINVAL, "packed arena of %llu bytes is smaller than its geometry needs",
                        (unsigned long long)bytes);
  int* flag = nullptr;
  st = probe_memory(base, device, &flag);
  if (st != KV_OK) return st;
  {
    DeviceGuard dg(device);
    (void)hipFree(flag);
  }
  try {
    std::unique_ptr<kv_packed> a(new kv_packed{base, bytes, *desc, block_size, num_blocks, device});
    DeviceGuard dg(device);
    if (hipEventCreateWithFlags(&a->staged, hipEventDisableTiming) != hipSuccess) {
      (void)hipGetLastError();
      return kvr_err::set(KV_EDEVICE, "event creation failed");
    }
    std::lock_guard<std::mutex> g(g_mu);
    g_packed.insert(a.get());
    *out = a.release();
  } catch (const std::bad_alloc&) {
    return kvr_err::set(KV_ENOMEM, "host allocation failed");
  }
  return kvr_err::clear();
}

kv_status kv_packed_release(kv_packed_t packed) {
  {
    std::lock_guard<std::mutex> g(g_mu);
    if (!packed || !g_packed.count(packed))
      return kvr_err::set(KV_ESTATE, "unknown or released packed arena handle");
    g_packed.erase(packed);
  }
  DeviceGuard dg(packed->device);
  if (packed->staged_pending) (void)hipEventSynchronize(packed->staged);
  if (packed->pinned) (void)hipHostFree(packed->pinned);
  (void)hipEventDestroy(packed->staged);
  delete packed;
  return kvr_err::clear();
}

kv_status kv_packed_store(kv_packed_t packed, int32_t layer, const void* k, int64_t k_stride, const void* v,
                          int64_t v_stride, const int64_t* slots, int64_t rows, void* stream) {
  return move_rows(packed, true, layer, k, k_stride, v, v_stride, slots, rows, stream);
}

kv_status kv_packed_load(kv_packed_t packed, int32_t layer, void* k, int64_t k_stride, void* v, int64_t v_stride,
                         const int64_t* slots, int64_t rows, void* stream) {
  return move_rows(packed, false, layer, k, k_stride, v, v_stride, slots, rows, stream);
}

kv_status kv_packed_park(kv_arena_t arena, const int64_t* arena_slots, kv_packed_t packed,
                         const int64_t* packed_slots, int64_t rows, void* stream) {
  return move_all(true, arena, arena_slots, packed, packed_slots, rows, stream);
}

kv_status kv_packed_restore(kv_packed_t packed, const int64_t* packed_slots, kv_arena_t arena,
                            const int64_t* arena_slots, int64_t rows, void* stream) {
  return move_all(false, arena, arena_slots, packed, packed_slots, rows, stream);
}

}  // extern "C"
