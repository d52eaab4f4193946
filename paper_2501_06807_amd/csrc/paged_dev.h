// Device helpers of the paged cache: 8-bit codes, page scales, row addresses.
#pragma once
#include "paged.h"

namespace mpc {
namespace dev {

// Pairs of e4m3 codes and fp32 values (v_cvt_pk_*_fp8: to nearest even, subnormals kept).
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
__device__ __forceinline__ void decode4(uint32_t w, float* out) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  out[0] = lo[0];
  out[1] = lo[1];
  out[2] = hi[0];
  out[3] = hi[1];
}

// Codes of 4 bits (e2m1), eight channels to a word, the even one of a byte low; scale: 2^e, of which the conversions take the
// exponent (all ones: NaN, as the scale byte 255 says).
__device__ __forceinline__ float mx4_scale(uint32_t byte) { return __uint_as_float((byte & 255u) << 23); }
__device__ __forceinline__ void decode8(uint32_t w, float scale, float* out) {
  const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
  const auto c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
  out[0] = a[0];
  out[1] = a[1];
  out[2] = b[0];
  out[3] = b[1];
  out[4] = c[0];
  out[5] = c[1];
  out[6] = d[0];
  out[7] = d[1];
}
// The same as bf16 pairs (exact: bf16 holds every code at every scale).
__device__ __forceinline__ uint4 widen8(uint32_t w, float scale) {
  return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2)),
                    __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3)));
}

// Codes of eight values in units of their scale: to nearest, halves to even codes, what is beyond 6 to 6.
__device__ __forceinline__ uint32_t encode8(const float* x) {
  uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, x[0], x[1], 1.f, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], 1.f, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], 1.f, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], 1.f, 3);
}
// Exponent s of a block's scale 2^s: the least with amax <= 6 * 2^s = 1.5 * 2^(s + 2), off the bits of amax, up to 125 (6 * 2^126
// is no fp32 value).
__device__ __forceinline__ int mx4_exponent(uint32_t amax_bits) {
  if (amax_bits == 0) return 0;
  const int s = (int)(amax_bits >> 23) - 127 - 2 + ((amax_bits & 0x7FFFFFu) > 0x400000u ? 1 : 0);
  return min(max(s, -126), 125);
}

// Exponent s of a page's scale 2^s: the least with amax <= 448 * 2^s = 1.75 * 2^(s + 8), read off the bits of amax.
__device__ __forceinline__ int scale_exponent(uint32_t amax_bits) {
  if (amax_bits == 0) return 0;
  const int s = (int)(amax_bits >> 23) - 127 - 8 + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return max(s, -126);
}
__device__ __forceinline__ float pow2(int s) { return __uint_as_float((uint32_t)(s + 127) << 23); }

// Magnitude bits of a finite value, 0 for the others: page maxima are taken over the finite values.
__device__ __forceinline__ uint32_t finite_bits(float x) {
  const uint32_t u = __float_as_uint(x) & 0x7FFFFFFFu;
  return u < 0x7F800000u ? u : 0u;
}
// A value in units of its page's scale, as the code conversion takes it: infinities to the largest code.
__device__ __forceinline__ float to_code_range(float x, float inv) {
  const float y = x * inv;
  return y != y ? y : fminf(fmaxf(y, -448.f), 448.f);
}

// Workgroup ids are dealt round-robin over the dies; each die gets one contiguous range of the n items, so that neighbours,
// which read the same rows, share its L2.
constexpr unsigned kDies = 8;
__device__ __forceinline__ unsigned by_die(unsigned id, unsigned n) {
  const unsigned q = n / kDies, r = n % kDies, x = id % kDies, slot = id / kDies;
  return x < r ? x * (q + 1) + slot : r * (q + 1) + (x - r) * q + slot;
}

// A value that the launch does not write, at an address that is the same over the wave: through the scalar cache, so that
// it has a counter of its own and waiting for it does not wait for the rows in flight.
template <class T>
__device__ __forceinline__ T load_uniform(const T* p) {
  return *(const __attribute__((address_space(4))) T*)(uintptr_t)p;
}

// Page id of logical page pg (not negative) of sequence b, or -1 where the table or the pool has none, in two steps: the
// table's entry, asked for early (b and pg the same over the wave, or with a lane to each), and what it says.
__device__ __forceinline__ int page_entry(const PagedCache& c, int b, int pg) {
  return load_uniform(c.table + (size_t)b * c.max_pages + min(pg, c.max_pages - 1));
}
__device__ __forceinline__ int page_of_entry(const PagedCache& c, int entry, int pg) {
  return pg < c.max_pages && (unsigned)entry < (unsigned)c.n_pages ? entry : -1;
}
__device__ __forceinline__ int page_id_lane(const PagedCache& c, int b, int pg) {
  return page_of_entry(c, c.table[(size_t)b * c.max_pages + min(pg, c.max_pages - 1)], pg);
}
// Index of (layer, page, head) in the pool.
__device__ __forceinline__ size_t page_unit(const PagedCache& c, int l, int id, int h) {
  return ((size_t)l * c.n_pages + id) * c.Hkv + h;
}

}  // namespace dev
}  // namespace mpc
