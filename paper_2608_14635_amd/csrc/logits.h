// Logits of a row, read in pieces of 16 bytes, and sums of their exponentials (log
// probabilities, the policy loss).
//
// In log2 units, with c = scale log2 e and m the largest logit of a chunk, t_v = fma(c, z_v,
// -C) with C = c m rounded: one operation, whose common shift, the rounding of C, is taken
// out where chunks meet.  Where C is so large that its rounding would count, t_v = (z_v - m) c.
#pragma once
#include <type_traits>

#include "common.h"

namespace kvr {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));

// 16 bytes of logits, on any boundary of their elements, and their values.
template <typename T> struct Piece;
template <> struct Piece<float> {
  static constexpr int N = 4;
  f32x4 w;
  __device__ __forceinline__ void load(const float* p) { w = *reinterpret_cast<const f32x4_a4*>(p); }
  __device__ __forceinline__ void set(int j, float v) { w[j] = v; }
  __device__ __forceinline__ float value(int j) const { return w[j]; }
  __device__ __forceinline__ void put(const float* v) { w = f32x4{v[0], v[1], v[2], v[3]}; }
  __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<f32x4_a4*>(p) = w; }
  // past the caches: nothing reads it soon
  __device__ __forceinline__ void store_past(float* p) const {
    __builtin_nontemporal_store(w, reinterpret_cast<f32x4_a4*>(p));
  }
};
template <> struct Piece<bf16_t> {
  static constexpr int N = 8;
  u32x4 w;
  __device__ __forceinline__ void load(const bf16_t* p) { w = *reinterpret_cast<const u32x4_a2*>(p); }
  __device__ __forceinline__ void set(int j, float v) {  // of a bf16 number
    const uint32_t b = __float_as_uint(v) >> 16;
    w[j / 2] = j % 2 ? (w[j / 2] & 0xffffu) | b << 16 : (w[j / 2] & 0xffff0000u) | b;
  }
  __device__ __forceinline__ float value(int j) const {
    return __uint_as_float(j % 2 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
  }
  __device__ __forceinline__ void put(const float* v) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      w[j] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)v[2 * j], (__bf16)v[2 * j + 1]});
  }
  __device__ __forceinline__ void store(bf16_t* p) const { *reinterpret_cast<u32x4_a2*>(p) = w; }
  __device__ __forceinline__ void store_past(bf16_t* p) const {
    __builtin_nontemporal_store(w, reinterpret_cast<u32x4_a2*>(p));
  }
};

// f over the wave's lanes, in every lane: neighbours, pairs, fours and eights of a row of
// 16 by lane moves within it, then the rows.
template <typename F>
__device__ __forceinline__ float over_wave(float v, F f) {
  const auto moved = [&](auto ctrl) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  v = f(v, moved(std::integral_constant<int, 0xb1>{}));   // quad_perm 1 0 3 2
  v = f(v, moved(std::integral_constant<int, 0x4e>{}));   // quad_perm 2 3 0 1
  v = f(v, moved(std::integral_constant<int, 0x141>{}));  // row_half_mirror
  v = f(v, moved(std::integral_constant<int, 0x140>{}));  // row_mirror
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float max_over_wave(float v) {
  return over_wave(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float sum_over_wave(float v) {
  return over_wave(v, [](float a, float b) { return a + b; });
}

// What logits are taken relative to: -infinity stands for no logit above it, and
// differences with it would be NaN.
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.0f : m; }
// C of a maximum: rounded, not contracted into what it enters.
__device__ __forceinline__ float c_of(float m, float scale2) {
#pragma clang fp contract(off)
  return m * scale2;
}
// Whether C stands for c m up to 2^-5.
__device__ __forceinline__ bool by_c(float c) { return fabsf(c) < 0x1p20f; }

// scale (a - b) - off.  A difference that passes the largest number is taken of the halves.
__device__ __forceinline__ float scaled_difference(float a, float b, float scale, float off) {
  const float d = a - b;
  return fabsf(d) < INFINITY ? fmaf(d, scale, -off) : fmaf(2.0f, (0.5f * a - 0.5f * b) * scale, -off);
}

// A chunk's largest logit and sums, added to those of its row, whose t is relative to
// `base`: by the two logits, and without the rounding of the chunk's C.
__device__ __forceinline__ void add_chunk(float m, float chunk_l, float chunk_s, float base, float scale2, float& l,
                                          float& s) {
  const float cm = c_of(base_of(m), scale2), off = by_c(cm) ? fmaf(base_of(m), scale2, -cm) : 0.0f;
  const float x = fmaxf(scaled_difference(m, base, scale2, off), -1e30f);
  const float e = __builtin_amdgcn_exp2f(x);
  l = fmaf(chunk_l, e, l);
  s += e * fmaf(x, chunk_l, chunk_s);
}

}  // namespace kvr
