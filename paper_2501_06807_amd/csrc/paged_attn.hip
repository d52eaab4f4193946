// Attention of new tokens over a paged cache.
#include "attn_rows.h"

namespace mpc {
namespace {

using namespace dev;

template <class DT, int D, bool CODES>
struct PagedKeys {
  const PagedCache& c;
  int l, b, h, rows, full;  // rows in the cache; rows of complete pages
  __device__ PagedKeys(const PagedCache& c_, int l_, int b_, int h_) : c(c_), l(l_), b(b_), h(h_) {
    rows = min(c.len(b), c.cap());
    full = CODES ? rows & ~(c.page - 1) : rows;
  }
  __device__ int limit() const { return rows; }
  __device__ bool has(int j) const { return j >= full || page_id(c, b, j >> c.log_page) >= 0; }
  __device__ void load8(int j, bool is_v, int e, float* out) const {
    if (CODES && j >= full) {
      const size_t row = (((size_t)l * c.B + b) * c.Hkv + h) * (2 * c.page) + (j & (2 * c.page - 1));
      dev::load8<DT>((is_v ? c.v_tail : c.k_tail) + (row * D + e) * DT::kElt, out);
      return;
    }
    const size_t unit = page_unit(c, l, page_id(c, b, j >> c.log_page), h);
    const size_t at = (unit * c.page + (j & (c.page - 1))) * D + e;
    if constexpr (CODES) {
      const uint2 w = *(const uint2*)((is_v ? c.v : c.k) + at);
      const float s = (is_v ? c.vs : c.ks)[unit];
      decode4(w.x, out);
      decode4(w.y, out + 4);
#pragma unroll
      for (int i = 0; i < 8; ++i) out[i] *= s;
    } else {
      dev::load8<DT>((is_v ? c.v : c.k) + at * DT::kElt, out);
    }
  }
};

template <class DT, int D, bool CODES>
__global__ __launch_bounds__(kRowWaves* kWave) void k_paged_rows(PagedAttnArgs a) {
  __shared__ float s_q[kRowWaves][D];
  const int w = threadIdx.x / kWave;
  const int64_t r = (int64_t)blockIdx.x * kRowWaves + w;
  if (r >= (int64_t)a.L * a.B * a.Hq * a.n) return;
  const int t = (int)(r % a.n), u = (int)(r / a.n);
  const int hq = u % a.Hq, b = u / a.Hq % a.B, l = u / a.Hq / a.B;
  const int valid = a.c.valid(b);
  if (t >= valid) return;
  const PagedKeys<DT, D, CODES> keys(a.c, l, b, hq / (a.Hq / a.Hkv));
  attend_row<DT, D>(a, keys, l, b, hq, t, a.c.len(b) - valid + t, s_q[w]);
}

template <class DT, int D>
hipError_t launch(const PagedAttnArgs& a, hipStream_t st) {
  const int64_t blocks = ((int64_t)a.L * a.B * a.Hq * a.n + kRowWaves - 1) / kRowWaves;
  if (blocks >= ((int64_t)1 << 31)) return hipErrorInvalidValue;
  if (a.c.ks)
    hipLaunchKernelGGL((k_paged_rows<DT, D, true>), dim3((unsigned)blocks), dim3(kRowWaves * kWave), 0, st, a);
  else
    hipLaunchKernelGGL((k_paged_rows<DT, D, false>), dim3((unsigned)blocks), dim3(kRowWaves * kWave), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attn(const PagedAttnArgs& a, int dtype, int D, hipStream_t st) {
  if (dtype == MPC_FP32) return D == 64 ? launch<F32, 64>(a, st) : launch<F32, 128>(a, st);
  if (dtype == MPC_FP16) return D == 64 ? launch<F16, 64>(a, st) : launch<F16, 128>(a, st);
  return D == 64 ? launch<BF16, 64>(a, st) : launch<BF16, 128>(a, st);
}

}  // namespace mpc
