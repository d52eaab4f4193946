// Attention of query rows over keys, a wave to a row: the keys in blocks of 64, a lane to a key for the scores, then
// lanes over the channels for the values; running maximum and sum, everything in fp32.
#pragma once
#include "paged_dev.h"

namespace mpc {
namespace dev {

constexpr int kRowWaves = 4;

// KEYS: limit() rows, has(j), load8(j, is_v, e, out) of row j's channels e .. e + 7.
template <class DT, int D, class KEYS>
__device__ __forceinline__ void attend_row(const AttnArgs& a, const KEYS& keys, int l, int b, int hq, int t, int p,
                                           float* s_q) {
  constexpr int CL = D / 8, KG = kWave / CL;  // lanes to a value row, value rows at once
  const int lane = threadIdx.x % kWave;
  for (int e = lane; e < D; e += kWave) s_q[e] = load_elt<DT>(a.q.at(l, b, hq, t), e);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  float m = -INFINITY, sum = 0.f, acc[8] = {};
  const int end = min(p + 1, keys.limit());
  for (int j0 = 0; j0 < end; j0 += kWave) {
    if (a.window && j0 >= a.sinks && j0 + kWave - 1 <= p - a.window) continue;
    const int j = j0 + lane;
    const bool see = j < end && (!a.window || j > p - a.window || j < a.sinks) && keys.has(j);
    float s = -INFINITY;
    if (see) {
      float x = 0.f;
      for (int e = 0; e < D; e += 8) {
        float k[8];
        keys.load8(j, false, e, k);
#pragma unroll
        for (int i = 0; i < 8; ++i) x = fmaf(k[i], s_q[e + i], x);
      }
      s = x * a.qscale;
    }
    float top = s;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
    const float m_new = fmaxf(m, top), base = m_new == -INFINITY ? 0.f : m_new;
    const float w = see ? fast_exp2(s - base) : 0.f, r = fast_exp2(m - base);
    sum = sum * r + wave_sum(w);
    m = m_new;
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] *= r;
    const unsigned long long seen = __ballot(see);
    for (int k = 0; k < kWave; k += KG) {
      const int jj = k + lane / CL;
      const float wj = __shfl(w, jj);
      if (!(seen >> jj & 1)) continue;
      float v[8];
      keys.load8(j0 + jj, true, lane % CL * 8, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[i] = fmaf(wj, v[i], acc[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int o = CL; o < kWave; o <<= 1) acc[i] += __shfl_xor(acc[i], o);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  char* out = a.out.at(l, b, hq, t);
  if (lane < CL)
#pragma unroll
    for (int i = 0; i < 8; ++i) store_elt<DT>(out, lane * 8 + i, sum == 0.f ? 0.f : acc[i] * inv);
  if (a.lse && lane == 0)
    a.lse[(((size_t)l * a.B + b) * a.Hq + hq) * a.n + t] =
        sum == 0.f ? -INFINITY : (m + __log2f(sum)) * 0.69314718055994531f;
}

}  // namespace dev
}  // namespace mpc
