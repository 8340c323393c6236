// Device helpers shared by the kernel files: vector types, 16-bit conversions, code rows widened for the matrix cores, lane swaps.
#pragma once
#include "tkv_internal.h"

namespace tkv {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(2))) unsigned int u32x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// type of K, V and q as a template argument: binary32, bfloat16, binary16
constexpr int KT_F32 = 0, KT_BF16 = 1, KT_F16 = 2;

struct __attribute__((packed, aligned(2))) PackedU32x4 { u32x4 v; };   // 16 bytes at any 16-bit element

__device__ __forceinline__ float add_swap32(float a, float b) {      // lanes 0..31: a's halves added; 32..63: b's
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), false, false);
  return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}
__device__ __forceinline__ uint16_t f32_to_bf16(float f) {
  uint32_t u = __builtin_bit_cast(uint32_t, f);
  u += 0x7fffu + ((u >> 16) & 1u);
  return (uint16_t)(u >> 16);
}
__device__ __forceinline__ float half_of(uint32_t w, int hi) {
  return (float)__builtin_bit_cast(_Float16, (uint16_t)(hi ? (w >> 16) : (w & 0xffffu)));
}

// Code values (one byte each, or two per byte) as 16-bit floating point, sign-extended: at most 7 significant bits, so the
// matrix cores multiply them exactly.  Two values per 32-bit word, low element first.
template <int KT>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
  if constexpr (KT == KT_BF16) return __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, hi), __builtin_bit_cast(uint32_t, lo), 0x07060302u);
  else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(lo, hi));
}
__device__ __forceinline__ float sbyte_f(uint32_t w, int n) { return (float)(int8_t)(w >> (8 * n)); }              // byte n of w
__device__ __forceinline__ float snib_f(uint32_t w, int n) { return (float)((int32_t)(w << (28 - 4 * n)) >> 28); }   // nibble n of w
// one word of int8 codes (4) -> two words; one word of int4 codes (8) -> four words
template <int KT>
__device__ __forceinline__ void widen_int8(uint32_t w, uint32_t& o0, uint32_t& o1) {
  o0 = pack16<KT>(sbyte_f(w, 0), sbyte_f(w, 1));
  o1 = pack16<KT>(sbyte_f(w, 2), sbyte_f(w, 3));
}
template <int KT>
__device__ __forceinline__ u32x4 widen_int4(uint32_t w) {
  return u32x4{pack16<KT>(snib_f(w, 0), snib_f(w, 1)), pack16<KT>(snib_f(w, 2), snib_f(w, 3)),
               pack16<KT>(snib_f(w, 4), snib_f(w, 5)), pack16<KT>(snib_f(w, 6), snib_f(w, 7))};
}

}  // namespace tkv
