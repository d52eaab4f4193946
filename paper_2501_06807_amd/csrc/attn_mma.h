// Matrix-core pieces that the attentions share: operand types, weights to 16 bits, transposes of value rows in registers.
#pragma once
#include "paged_dev.h"

namespace mpc {
namespace dev {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// c + a b over 32 channels (keys): lane (g = lane / 16, c = lane % 16) holds row (column) c of a (b) at the eight places
// 8 g .. 8 g + 7; of the result it holds column c, rows 4 g .. 4 g + 3. Which channel (key) a place stands for is the
// caller's choice, the same for both operands.
template <class DT>
__device__ __forceinline__ f32x4 mma(const uint4& a, const uint4& b, f32x4 c) {
  if constexpr (DT::kCode == MPC_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
// The same in fp32 over four channels (keys), a place to each g.
__device__ __forceinline__ f32x4 mma(float a, float b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// Two fp32 values as a pair of the 16-bit type, to nearest even.
template <class DT>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const f32x2 x = {lo, hi};
  if constexpr (DT::kCode == MPC_BF16)
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2_t));
  else
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, f16x2_t));
}

// Codes HI, HI + 1 of a word as a pair of the 16-bit type (exact: both hold every e4m3 value).
template <class DT, bool HI>
__device__ __forceinline__ uint32_t widen2(uint32_t w) {
  if constexpr (DT::kCode == MPC_BF16)
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, HI));
  else
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)w, 1.0f, HI));
}

// max over the four lanes that hold a column (c, c + 16, c + 32, c + 48)
__device__ __forceinline__ float column_max(float x) {
  x = xor_combine<16>(x, [](float a, float b) { return fmaxf(a, b); });
  return xor_combine<32>(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float column_sum(float x) {
  x = xor_combine<16>(x, [](float a, float b) { return a + b; });
  return xor_combine<32>(x, [](float a, float b) { return a + b; });
}

// Values that are not finite, as numbers that add up without mixing over the 32 keys of a tile: +infinity 1, -infinity 64,
// NaN 4096.
constexpr float kPlusInf = 1.f, kMinusInf = 64.f, kNan = 4096.f;

// Whether a word of the 16-bit type, or of fp32, holds a value that is not finite.
template <class DT>
__device__ __forceinline__ bool not_finite(uint32_t w) {
  if constexpr (DT::kElt == 4) return (w & 0x7F800000u) == 0x7F800000u;
  constexpr uint32_t lo = DT::kCode == MPC_BF16 ? 0x7F80u : 0x7C00u, hi = lo << 16;
  return (w & lo) == lo || (w & hi) == hi;
}
// Largest magnitude bits of the 16-bit values so far, by half, and whether they say that one was not finite.
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t max_magnitude(uint32_t top, uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top), __builtin_bit_cast(u16x2, w & 0x7FFF7FFFu)));
}
// Takes the values that are not finite out of a word (zero in their place) and returns what they were.
template <class DT>
__device__ __forceinline__ uint32_t take_not_finite(uint32_t& w) {
  constexpr bool B = DT::kCode == MPC_BF16;
  constexpr uint32_t E = DT::kElt == 4 ? 0x7F800000u : B ? 0x7F80u : 0x7C00u;
  constexpr uint32_t plus = DT::kElt == 4 ? 0x3F800000u : B ? 0x3F80u : 0x3C00u, minus = DT::kElt == 4 ? 0x42800000u : B ? 0x4280u : 0x5400u,
                     nan = DT::kElt == 4 ? 0x45800000u : B ? 0x4580u : 0x6C00u;
  constexpr uint32_t mask = DT::kElt == 4 ? 0xFFFFFFFFu : 0xFFFFu;
  uint32_t what = 0;
#pragma unroll
  for (int i = 0; i < (DT::kElt == 4 ? 1 : 2); ++i) {
    const uint32_t x = w >> 16 * i & mask;
    if ((x & E) != E) continue;
    what |= ((x & (mask >> 1)) != E ? nan : x == E ? plus : minus) << 16 * i;
    w &= ~(mask << 16 * i);
  }
  return what;
}
// A sum of such numbers as what adding the values gives.
__device__ __forceinline__ float not_finite_sum(float n) {
  const int i = (int)n, plus = i & 63, minus = i >> 6 & 63, nan = i >> 12;
  if (nan || (plus && minus)) return __uint_as_float(0x7FC00000u);
  return plus ? INFINITY : minus ? -INFINITY : 0.f;
}

}  // namespace dev
}  // namespace mpc
