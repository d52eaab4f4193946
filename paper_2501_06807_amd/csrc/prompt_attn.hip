// Attention of a prompt's rows over its keys, with an optional sliding window and sinks.
//
// 16-bit types (k_prompt): a workgroup of four waves (or two groups of four, which halve the keys) takes 128 rows of one
// query head, a wave 32 of them. Tiles of keys go through LDS, double-buffered, the next one in registers meanwhile.
// A wave computes S^T = K Q^T in 32x32x16 products: a lane then holds 16 scores of one row for each 32 keys, the other
// half of the row's lying 32 lanes on, and its weights, packed to 16 bits, are the operand of O^T += V^T P^T as they
// stand; V comes from LDS through the transposing reads of gfx950 (four keys of one channel to a lane).
// The row's reference (what its exponents are taken against) moves only when a score passes it by 2^8, so that the
// accumulators are seldom rescaled; weights are at most 2^8 (fp16: 2^15, lifted so that only those below 2^-21 of the
// reference lose bits), their sum and the accumulators fp32. Weights are rounded once to the type: a second product with what
// the rounding leaves takes 818 us instead of 640 in the first case below, and 1306 instead of 1050 behind the window, for
// outputs that are off by 0.0017 of their size instead of 0.0022 (their own rounding: 0.0017).
//
// 8K rows and keys of 32 heads of 128 in bf16: 631 to 640 us, 862 TFLOP/s of the products that the rows need (a large bf16
// product of the library: 1229). The matrix unit is busy 40% of the cycles, the vector unit as much (a quarter of it
// exponentials), at 2.07 GHz. Both units side by side, in a written-out pipeline that takes the next tile's scores beside this one's
// weights, gave 2% there and cost 4% behind a window: the clock falls as the units fill. 32-key tiles instead of 64 (which
// spill): 1072 -> 730 us; whole tiles apart from edge tiles, and the values asked for before the scores: 640. A window of
// 1024 over four prompts of up to 16K: 1045 us; a block of 128 rows visits 37 tiles for 32 full ones' worth of keys, 11 of
// them with masks (one check of the staged values instead of one of every fragment, 2130 -> 1383; the dies dividing the heads
// instead of the sequences, 1376 -> 1078).
#include "attn_mma.h"

namespace mpc {
namespace {

using namespace dev;

constexpr int kRowsWave = 32, kRowsGroup = 4 * kRowsWave;
constexpr float kSlack = 8.f;  // log2 of how far a weight may pass 1 before its row's reference moves

// The tiles of KT keys that rows at positions lo .. hi may see, as a list: first the `edge` ones, which some row may not see
// whole (those of the sinks, at the window's start and at the diagonal), then those that every row sees. Keys may be taken in
// any order.
struct Tiles {
  int n, edge;
  int skip, at, f0, f1;  // sinks [0, skip), window [at, ...) with [f0, f1) seen whole
  __device__ int id(int i) const {
    if (i >= edge) return f0 + i - edge;
    if (i < skip) return i;
    i += at - skip;
    return i < f0 ? i : i - f0 + f1;
  }
};
__device__ __forceinline__ Tiles tiles_of(const AttnArgs& a, int lo, int hi, int rows, int KT) {
  Tiles t;
  const int all = max(0, (min(hi + 1, rows) + KT - 1) / KT);
  t.skip = t.at = t.f0 = 0;
  if (a.window) {
    t.skip = min((a.sinks + KT - 1) / KT, all);
    t.at = max(t.skip, min(max(lo - a.window + 1, 0) / KT, all));
    t.f0 = max(t.at, min((max(hi - a.window + 1, 0) + KT - 1) / KT, all));
  }
  t.f1 = max(t.f0, (max(min(lo, rows - 1), -1) + 1) / KT);
  t.edge = t.skip + (t.f0 - t.at) + (all - t.f1);
  t.n = t.edge + (t.f1 - t.f0);
  return t;
}

// Whether any row at positions lo .. hi sees any of the keys [k0, k1].
__device__ __forceinline__ bool seen_by(const AttnArgs& a, int k0, int k1, int lo, int hi, int rows) {
  return k0 <= hi && k0 < rows && (!a.window || k1 > lo - a.window || k0 < a.sinks);
}

template <class DT, int D, int NS>
__global__ __launch_bounds__(256 * NS, 2) void k_prompt(PromptAttnArgs a) {
  constexpr int KT = 32, KB = KT / 32;  // keys of a tile, and its 32-key blocks
  constexpr int CH = D / 8, KSTEPS = D / 16, DB = D / 32, THREADS = 256;
  constexpr float LIFT = DT::kCode == MPC_FP16 ? 7.f : 0.f;  // of the weights' exponents, also in their sum
  constexpr int PER = KT * CH / THREADS;  // chunks of K (and of V) that a thread stages
  __shared__ uint4 s_k[NS][2][KT * CH], s_v[NS][2][KT * CH];
  __shared__ int s_bad[NS][2];  // the last round whose values, staged for an edge, were not all finite
  const int tid = threadIdx.x % THREADS, lane = tid % kWave, q32 = lane & 31, hl = lane >> 5;
  const int grp = __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int G = a.Hq / a.Hkv;

  // item: (kv head, layer, sequence), then the blocks of rows from the last one on, then the heads of the group; so the dies
  // divide the heads, and sequences of different lengths fall to all of them
  const unsigned id = by_die(blockIdx.x, gridDim.x);
  const unsigned nqb = (a.n + kRowsGroup - 1) / kRowsGroup;
  const int gq = id % G, qb = nqb - 1 - id / G % nqb;
  const unsigned u = id / G / nqb;
  const int b = u % a.B, l = u / a.B % a.L, h = u / a.B / a.L, hq = h * G + gq;
  const int q_len = a.q_lens ? min(max(load_uniform(a.q_lens + b), 0), a.n) : a.n;
  const int rows = a.k_lens ? min(max(load_uniform(a.k_lens + b), 0), a.T) : a.T;
  if (qb * kRowsGroup >= q_len) return;
  const int start = rows - q_len;
  const int g_lo = start + qb * kRowsGroup, g_hi = start + min(q_len, (qb + 1) * kRowsGroup) - 1;
  const Tiles tl = tiles_of(a, g_lo, g_hi, rows, KT);
  const int r0 = qb * kRowsGroup + wave * kRowsWave, t = r0 + q32;
  const int lo = start + r0, hi = min(lo + kRowsWave - 1, g_hi);  // the wave's rows; none where hi < lo
  const int pos = start + t;

  // a negative scale is taken into the queries
  // zero times a masked score would be NaN: the smallest number that is not zero instead, 5e-7 times the largest score
  const float c = fmaxf(fabsf(a.qscale), 0x1p-149f);
  const uint32_t flip = a.qscale < 0.f ? 0x80008000u : 0u;
  uint4 q[KSTEPS];
  {
    const char* row = a.q.at(l, b, hq, min(t, q_len - 1)) + hl * 16;
#pragma unroll
    for (int i = 0; i < KSTEPS; ++i) {
      uint4 x = ldg16(row + i * 32);
      q[i] = make_uint4(x.x ^ flip, x.y ^ flip, x.z ^ flip, x.w ^ flip);
    }
  }
  f32x16 o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  float ref = -INFINITY, sum = 0.f;  // reference (in units of the exponent) and sum over this lane's keys

  uint4 kr[PER], vr[PER];
  const char *kbase = a.k.at(l, b, h, 0), *vbase = a.v.at(l, b, h, 0);
  // this thread's chunks of a tile, from the tile's first row
  int64_t k_off[PER], v_off[PER];
#pragma unroll
  for (int n = 0; n < PER; ++n) {
    const int x = tid + n * THREADS;
    k_off[n] = x / CH * a.k.token + x % CH * 16;
    v_off[n] = x / CH * a.v.token + x % CH * 16;
  }
  auto fetch = [&](int i) {
    const int k0 = tl.id(i) * KT;
    if (k0 + KT <= rows) {
      const char *kp = kbase + k0 * a.k.token, *vp = vbase + k0 * a.v.token;
#pragma unroll
      for (int n = 0; n < PER; ++n) {
        kr[n] = ldg16(kp + k_off[n]);
        vr[n] = ldg16(vp + v_off[n]);
      }
    } else {
#pragma unroll
      for (int n = 0; n < PER; ++n) {
        const int x = tid + n * THREADS, row = min(k0 + x / CH, rows - 1);
        kr[n] = ldg16(kbase + row * a.k.token + x % CH * 16);
        vr[n] = ldg16(vbase + row * a.v.token + x % CH * 16);
      }
    }
  };
  auto stash = [&](int buf) {
#pragma unroll
    for (int n = 0; n < PER; ++n) {
      const int x = tid + n * THREADS;
      s_k[grp][buf][tile_chunk_k<D>(x / CH, x % CH)] = kr[n];
      s_v[grp][buf][tile_chunk_v<D>(x / CH, x % CH)] = vr[n];
    }
  };
  auto staged_not_finite = [&]() {
    uint32_t top = 0;
#pragma unroll
    for (int n = 0; n < PER; ++n) top = max_magnitude(max_magnitude(max_magnitude(max_magnitude(top, vr[n].x), vr[n].y), vr[n].z), vr[n].w);
    return not_finite<DT>(top);
  };
  // The tile of round n; EDGE: some row of the wave may not see some key of it.
  auto tile = [&](auto edge, int k0, int buf, int n) {
    constexpr bool EDGE = decltype(edge)::value;
    const uint4* sk = s_k[grp][buf];
    const char* sv = (const char*)s_v[grp][buf];
    // places 0..3 and 4..7 of half hl in a product over 16 keys are keys 4 hl .. and 8 + 4 hl ..
    const int vrow = 4 * hl + ((lane & 15) >> 2);  // row whose piece this lane asks for, and the piece's 16-byte chunk
    const int vcol = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), vbyte = (lane & 1) * 8;
    auto values = [&](int kb, int st, uint32_t (*v)[4]) {
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int row = 32 * kb + 16 * st + 8 * e + vrow;
          const char* at = sv + tile_chunk_v<D>(row, 4 * d + vcol) * 16 + vbyte;
          const auto x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)at);
          const uint2 y = __builtin_bit_cast(uint2, x);
          v[d][2 * e] = y.x;
          v[d][2 * e + 1] = y.y;
        }
    };
    const int bad = EDGE ? s_bad[grp][buf] : 0;
    uint4 kf[KB][KSTEPS];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) kf[kb][ks] = sk[tile_chunk_k<D>(kb * 32 + q32, 2 * ks + hl)];
    // the values are asked for before the scores are taken, so that they are there when the weights are
    uint32_t vf[KB][2][DB][4];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int st = 0; st < 2; ++st) values(kb, st, vf[kb][st]);
    __builtin_amdgcn_sched_barrier(0);
    f32x16 s[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KSTEPS; ++ks) s[kb] = mma32<DT>(kf[kb][ks], q[ks], s[kb]);
    }
    if constexpr (EDGE) {
      // the lane's keys lie (8 (r / 4) + r % 4) behind this one
      const int j0 = k0 + 4 * hl;
      if (k0 + KT - 1 > min(lo, rows - 1)) {
        const int last = min(pos, rows - 1) - j0;
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (32 * kb + 8 * (r >> 2) + (r & 3) > last) s[kb][r] = -INFINITY;
      }
      if (a.window && k0 <= hi - a.window && k0 + KT > a.sinks) {
        const int gone = pos - a.window - j0, sinks = a.sinks - j0;
        if (k0 < a.sinks) {
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int j = 32 * kb + 8 * (r >> 2) + (r & 3);
              if (j <= gone && j >= sinks) s[kb][r] = -INFINITY;
            }
        } else {
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              if (32 * kb + 8 * (r >> 2) + (r & 3) <= gone) s[kb][r] = -INFINITY;
        }
      }
    }
    float top = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) top = fmaxf(top, s[kb][r]);
    if (__any(top * c > ref + kSlack || (ref == -INFINITY && top > -INFINITY))) {
      top = xor_combine<32>(top, [](float x, float y) { return fmaxf(x, y); });
      const float was = ref;
      ref = top == -INFINITY ? ref : fmaxf(ref, top * c);
      // exp2(-inf - 0) = 0: nothing was there to move
      const float move = fast_exp2(was - (ref == -INFINITY ? 0.f : ref));
      sum *= move;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= move;
    }
    const float base = (ref == -INFINITY ? 0.f : ref) - LIFT;
    uint32_t p[KB][8];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        const float w0 = fast_exp2(fmaf(s[kb][r], c, -base)), w1 = fast_exp2(fmaf(s[kb][r + 1], c, -base));
        sum += w0 + w1;
        p[kb][r / 2] = pack2<DT>(w0, w1);
      }
    // O^T += V^T P^T, 16 keys at a time
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const uint4 w = make_uint4(p[kb][4 * st], p[kb][4 * st + 1], p[kb][4 * st + 2], p[kb][4 * st + 3]);
        uint32_t(*v)[4] = vf[kb][st];
        if constexpr (EDGE) {
          // Values that are not finite, in keys that some row does not see, must not meet that row's weight of zero: they
          // are added apart, to the rows that see them
          if (__builtin_amdgcn_readfirstlane(bad) == n) {
            const int j0 = k0 + 32 * kb + 16 * st + 4 * hl;
            float one[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int j = j0 + (e >= 4 ? 8 : 0) + (e & 3);
              one[e] = j <= pos && j < rows && (!a.window || j > pos - a.window || j < a.sinks) ? 1.f : 0.f;
            }
            const uint4 w1 = make_uint4(pack2<DT>(one[0], one[1]), pack2<DT>(one[2], one[3]), pack2<DT>(one[4], one[5]), pack2<DT>(one[6], one[7]));
#pragma unroll
            for (int d = 0; d < DB; ++d) {
              uint32_t what[4];
#pragma unroll
              for (int n = 0; n < 4; ++n) what[n] = take_not_finite<DT>(v[d][n]);
              f32x16 y;
#pragma unroll
              for (int r = 0; r < 16; ++r) y[r] = 0.f;
              y = mma32<DT>(make_uint4(what[0], what[1], what[2], what[3]), w1, y);
#pragma unroll
              for (int r = 0; r < 16; ++r) o[d][r] += not_finite_sum(y[r]);
            }
          }
        }
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] = mma32<DT>(make_uint4(v[d][0], v[d][1], v[d][2], v[d][3]), w, o[d]);
      }
  };
  // the groups take every NS-th tile of the list; all of them run the same number of rounds, and change from edge tiles to
  // whole ones in the same round (the edge form takes any tile)
  const int rounds = (tl.n + NS - 1) / NS, edges = (tl.edge + NS - 1) / NS;
  if (grp < tl.n) fetch(grp);
  if (threadIdx.x < 2 * NS) (&s_bad[0][0])[threadIdx.x] = -1;
  __syncthreads();
  auto round = [&](auto edge, int n) {
    constexpr bool EDGE = decltype(edge)::value;
    const int i = n * NS + grp, buf = n & 1;
    if (i < tl.n) {
      if (EDGE && staged_not_finite()) s_bad[grp][buf] = n;
      stash(buf);
    }
    __syncthreads();
    if (i + NS < tl.n) fetch(i + NS);
    if (i >= tl.n || hi < lo) return;
    const int k0 = tl.id(i) * KT;
    if (EDGE && !seen_by(a, k0, k0 + KT - 1, lo, hi, rows)) return;
    tile(edge, k0, buf, n);
  };
  for (int n = 0; n < edges; ++n) round(std::true_type{}, n);
  for (int n = edges; n < rounds; ++n) round(std::false_type{}, n);

  sum = xor_combine<32>(sum, [](float x, float y) { return x + y; });
  if constexpr (NS == 2) {
    // the second group's part to the first, through the tiles' LDS
    constexpr int HALF = DB / 2;
    float* s_o = (float*)&s_k[0][0][0];  // [4 waves][HALF * 16][64 lanes] each for a half of the channels
    float* s_st = (float*)&s_v[0][0][0];
    const float mine = ref;
    __syncthreads();
    if (grp == 1) {
      s_st[(wave * 2) * kWave + lane] = ref;
      s_st[(wave * 2 + 1) * kWave + lane] = sum;
    }
    __syncthreads();
    float f0 = 1.f, f1 = 0.f;
    if (grp == 0) {
      const float r1 = s_st[(wave * 2) * kWave + lane], sum1 = s_st[(wave * 2 + 1) * kWave + lane];
      ref = fmaxf(mine, r1);
      const float base = ref == -INFINITY ? 0.f : ref;
      f0 = fast_exp2(mine - base);
      f1 = fast_exp2(r1 - base);
      sum = sum * f0 + sum1 * f1;
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      __syncthreads();
      if (grp == 1)
#pragma unroll
        for (int d = 0; d < HALF; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) s_o[((wave * HALF + d) * 16 + r) * kWave + lane] = o[e * HALF + d][r];
      __syncthreads();
      if (grp == 0)
#pragma unroll
        for (int d = 0; d < HALF; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            o[e * HALF + d][r] = o[e * HALF + d][r] * f0 + s_o[((wave * HALF + d) * 16 + r) * kWave + lane] * f1;
    }
    if (grp == 1) return;
  }
  if (t >= q_len) return;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  char* out = a.out.at(l, b, hq, t);
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = sum == 0.f ? 0.f : o[d][r + e] * inv;
      *(uint2*)(out + (32 * d + 2 * r + 4 * hl) * 2) = make_uint2(pack2<DT>(y[0], y[1]), pack2<DT>(y[2], y[3]));
    }
  if (a.lse && hl == 0)
    a.lse[(((size_t)l * a.B + b) * a.Hq + hq) * a.n + t] =
        sum == 0.f ? -INFINITY : (ref - LIFT + __log2f(sum)) * 0.69314718055994531f;
}

template <class DT, int D>
hipError_t launch16(const PromptAttnArgs& a, hipStream_t st) {
  const long long items = (long long)a.L * a.B * a.Hq * ((a.n + kRowsGroup - 1) / kRowsGroup);
  if (items >= (1ll << 31)) return hipErrorInvalidValue;
  // where one workgroup to a compute unit is all there is, two groups halve each one's keys
  if (items <= kNumCU)
    hipLaunchKernelGGL((k_prompt<DT, D, 2>), dim3((unsigned)items), dim3(512), 0, st, a);
  else
    hipLaunchKernelGGL((k_prompt<DT, D, 1>), dim3((unsigned)items), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_prompt_attn_fp32(const PromptAttnArgs& a, int D, hipStream_t st);

hipError_t launch_prompt_attn(const PromptAttnArgs& a, int dtype, int D, hipStream_t st) {
  if (dtype == MPC_FP32) return launch_prompt_attn_fp32(a, D, st);
  if (dtype == MPC_FP16) return D == 64 ? launch16<F16, 64>(a, st) : launch16<F16, 128>(a, st);
  return D == 64 ? launch16<BF16, 64>(a, st) : launch16<BF16, 128>(a, st);
}

}  // namespace mpc
