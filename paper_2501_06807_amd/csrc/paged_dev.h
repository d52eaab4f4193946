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
