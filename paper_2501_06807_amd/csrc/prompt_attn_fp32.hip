// Attention of a prompt's rows over its keys in fp32.
//
// A workgroup takes 16 RT query rows of one kv head (the G heads of the group times the tokens), and its waves divide the
// tiles of 16 keys, which come straight from memory into registers: fp32 products (16x16x4, a sixteenth of the 16-bit
// rate) leave the caches time to bring the rows, and short prompts have many workgroups this way. The waves' parts meet in
// LDS. The scores, weights and products of a tile are those of the paged attention. 512 rows and keys of 12 heads of 64: 16 us
// (the products alone 2.6 at the rate of a large fp32 product, 153 TFLOP/s): up to eight tiles one after the other, each with
// four chains of four dependent products for its scores and a memory round trip (one chain of 16: 16 us too).
#include "paged_attn_dev.h"

namespace mpc {
namespace {

using namespace dev;
constexpr int kFp32Waves = 4;

template <int D, int RT>
__global__ __launch_bounds__(kFp32Waves* kWave, RT == 1 ? 2 : 1) void k_prompt_fp32(PromptAttnArgs a) {
  using TL = PagedTile<F32, D, false, RT>;
  constexpr int NT = TL::NT, RW = 16 * RT, NW = kFp32Waves, KT = TL::TK;
  const int lane = threadIdx.x % kWave, g = lane / 16, col = lane % 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int G = a.Hq / a.Hkv, log_g = __builtin_ctz(G);
  __shared__ __align__(16) f32x4 s_o[NW / 2][NT][kWave];
  __shared__ float s_ml[NW][RT][2][kWave];

  // units of the last rows first: under the causal rule they see the most keys
  const unsigned groups = (unsigned)(((unsigned long long)a.n * G + RW - 1) / RW);
  const unsigned rg = groups - 1 - blockIdx.x % groups, u = blockIdx.x / groups;
  const int h = u % a.Hkv, b = u / a.Hkv % a.B, l = u / a.Hkv / a.B;
  const int q_len = a.q_lens ? min(max(load_uniform(a.q_lens + b), 0), a.n) : a.n;
  const int rows = a.k_lens ? min(max(load_uniform(a.k_lens + b), 0), a.T) : a.T;
  const long long r0 = (long long)rg * RW, r_end = min((long long)q_len << log_g, r0 + RW);
  if (r0 >= r_end) return;
  const int start = rows - q_len;
  const int lo = start + (int)(r0 >> log_g), hi = start + (int)((r_end - 1) >> log_g);
  // tiles [0, skip) and [at, all)
  const int all = max(0, (min(hi + 1, rows) + KT - 1) / KT);
  int skip = 0, at = 0;
  if (a.window) {
    skip = min((a.sinks + KT - 1) / KT, all);
    at = max(skip, min(max(lo - a.window + 1, 0) / KT, all));
  }
  const int n_tiles = skip + all - at;
  auto first_key = [&](int i) { return (i < skip ? i : i - skip + at) * KT; };

  PagedWave<F32, D, false, RT> w;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const long long r = r0 + 16 * rt + col;
    const bool ok = r < r_end;
    const int t = ok ? (int)(r >> log_g) : 0, hq = h * G + (ok ? (int)(r & (G - 1)) : 0);
    w.pos[rt] = ok ? start + t : -kMaxRows;
    const char* row = a.q.at(l, b, hq, t);
#pragma unroll
    for (int i = 0; i < TL::QF; i += 4) {
      const uint4 y = ldg16(row + TL::q_channel(i, g) * 4);
      w.q[rt][i] = ok ? __uint_as_float(y.x) : 0.f;
      w.q[rt][i + 1] = ok ? __uint_as_float(y.y) : 0.f;
      w.q[rt][i + 2] = ok ? __uint_as_float(y.z) : 0.f;
      w.q[rt][i + 3] = ok ? __uint_as_float(y.w) : 0.f;
    }
  }
  w.clear();
  const char *kb = a.k.at(l, b, h, 0) + g * 16, *vb = a.v.at(l, b, h, 0) + col * (TL::VW * 4);
  auto load_k = [&](int i, uint4 (*k)[TL::KL]) {
    const char* p = kb + min(first_key(i) + col, rows - 1) * a.k.token;
#pragma unroll
    for (int n = 0; n < TL::KL; ++n) k[0][n] = ldg16(p + n * 64);
  };
  auto load_v = [&](int i, uint32_t (*v)[TL::VW]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) load_words<TL::VW>(vb + min(first_key(i) + 4 * g + j, rows - 1) * a.v.token, v[j]);
  };
  int i = wave;
  if (i < n_tiles) {
    uint4 k[1][TL::KL];
    uint32_t v[TL::VK][TL::VW];
    load_k(i, k);
    load_v(i, v);
    const bool have[1] = {true};
    const float sc[1] = {a.qscale};
    for (;;) {
      const int i1 = i + NW < n_tiles ? i + NW : i;
      const int k0 = first_key(i), k1 = k0 + KT - 1;
      const bool edge = !(k1 < rows && k1 <= lo && (!a.window || k0 > hi - a.window || k1 < a.sinks));
      f32x4 s[RT][1];
      w.template scores<false>(k, s);
      load_k(i1, k);
      float p[RT][TL::VK];
      w.weights(s, sc, nullptr, a, edge, k0, rows, have, p);
      float x[TL::VK][NT];
      w.template operands<false>(v, x);
      w.add_values(x, p, a, edge, k0, rows, have, lo, hi, nullptr);
      load_v(i1, v);
      if (i1 == i) break;
      i = i1;
    }
  }

#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    s_ml[wave][rt][0][lane] = w.m[rt];
    s_ml[wave][rt][1][lane] = column_sum(w.l[rt]);
  }
  __syncthreads();
  float M[RT], L[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    M[rt] = -INFINITY;
    L[rt] = 0.f;
#pragma unroll
    for (int n = 0; n < NW; ++n) M[rt] = fmaxf(M[rt], s_ml[n][rt][0][lane]);
    const float b0 = M[rt] == -INFINITY ? 0.f : M[rt];
#pragma unroll
    for (int n = 0; n < NW; ++n) L[rt] += s_ml[n][rt][1][lane] * fast_exp2(s_ml[n][rt][0][lane] - b0);
    const float move = fast_exp2(w.m[rt] - b0);
#pragma unroll
    for (int t = 0; t < NT; ++t) w.o[rt][t] *= move;
  }
#pragma unroll
  for (int n = NW / 2; n > 0; n /= 2) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      if (wave >= n && wave < 2 * n)
#pragma unroll
        for (int t = 0; t < NT; ++t) s_o[wave - n][t][lane] = w.o[rt][t];
      __syncthreads();
      if (wave < n)
#pragma unroll
        for (int t = 0; t < NT; ++t) w.o[rt][t] += s_o[wave][t][lane];
      if (rt + 1 < RT || n > 1) __syncthreads();
    }
  }
  if (wave > 0) return;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const long long r = r0 + 16 * rt + col;
    if (r >= r_end) continue;
    const int t = (int)(r >> log_g), hq = h * G + (int)(r & (G - 1));
    const float inv = L[rt] == 0.f ? 0.f : 1.f / L[rt];
    char* out = a.out.at(l, b, hq, t);
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int n = 0; n < NT; n += 4) {
        float4 y = make_float4(w.o[rt][n][e], w.o[rt][n + 1][e], w.o[rt][n + 2][e], w.o[rt][n + 3][e]);
        y = L[rt] == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(y.x * inv, y.y * inv, y.z * inv, y.w * inv);
        *(float4*)(out + ((4 * g + e) * NT + n) * 4) = y;
      }
    if (a.lse && g == 0)
      a.lse[(((size_t)l * a.B + b) * a.Hq + hq) * a.n + t] =
          L[rt] == 0.f ? -INFINITY : (M[rt] + __log2f(L[rt])) * 0.69314718055994531f;
  }
}

template <int D, int RT>
hipError_t launch(const PromptAttnArgs& a, hipStream_t st) {
  const long long groups = ((long long)a.n * (a.Hq / a.Hkv) + 16 * RT - 1) / (16 * RT), units = (long long)a.L * a.B * a.Hkv * groups;
  if (units >= (1ll << 31)) return hipErrorInvalidValue;
  hipLaunchKernelGGL((k_prompt_fp32<D, RT>), dim3((unsigned)units), dim3(kFp32Waves * kWave), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_prompt_attn_fp32(const PromptAttnArgs& a, int D, hipStream_t st) {
  // two 16-row tiles read K and V half as often; one where that would leave compute units without a workgroup
  const bool two = (long long)a.L * a.B * a.Hq * a.n >= 32ll * 2 * kNumCU;
  if (D == 64) return two ? launch<64, 2>(a, st) : launch<64, 1>(a, st);
  return two ? launch<128, 2>(a, st) : launch<128, 1>(a, st);
}

}  // namespace mpc
