// Attention of a prompt's rows over its keys in fp32: a wave to a row for now.
#include "attn_rows.h"

namespace mpc {
namespace {

using namespace dev;

template <class DT, int D>
struct PlainKeys {
  const PromptAttnArgs& a;
  int l, b, h, rows;
  __device__ int limit() const { return rows; }
  __device__ bool has(int) const { return true; }
  __device__ void load8(int j, bool is_v, int e, float* out) const {
    dev::load8<DT>((is_v ? a.v : a.k).at(l, b, h, j) + e * DT::kElt, out);
  }
};

template <class DT, int D>
__global__ __launch_bounds__(kRowWaves* kWave) void k_prompt_rows(PromptAttnArgs a) {
  __shared__ float s_q[kRowWaves][D];
  const int w = threadIdx.x / kWave;
  const int64_t r = (int64_t)blockIdx.x * kRowWaves + w;
  if (r >= (int64_t)a.L * a.B * a.Hq * a.n) return;
  const int t = (int)(r % a.n), u = (int)(r / a.n);
  const int hq = u % a.Hq, b = u / a.Hq % a.B, l = u / a.Hq / a.B;
  const int q_len = a.q_lens ? min(max(a.q_lens[b], 0), a.n) : a.n;
  const int k_len = a.k_lens ? min(max(a.k_lens[b], 0), a.T) : a.T;
  if (t >= q_len) return;
  const PlainKeys<DT, D> keys{a, l, b, hq / (a.Hq / a.Hkv), k_len};
  attend_row<DT, D>(a, keys, l, b, hq, t, k_len - q_len + t, s_q[w]);
}

template <int D>
hipError_t launch(const PromptAttnArgs& a, hipStream_t st) {
  const int64_t blocks = ((int64_t)a.L * a.B * a.Hq * a.n + kRowWaves - 1) / kRowWaves;
  if (blocks >= ((int64_t)1 << 31)) return hipErrorInvalidValue;
  hipLaunchKernelGGL((k_prompt_rows<F32, D>), dim3((unsigned)blocks), dim3(kRowWaves * kWave), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_prompt_attn_fp32(const PromptAttnArgs& a, int D, hipStream_t st) {
  return D == 64 ? launch<64>(a, st) : launch<128>(a, st);
}

}  // namespace mpc
