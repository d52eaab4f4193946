// Attention behind shared rows, 16-bit types: the kernel of the shared rows for units of 128 query rows, and own rows after them.
//
// A workgroup has four waves, a wave 32 of the unit's rows; a tile of 32 keys goes through LDS once for them: rows of the element type
// straight from memory, two tiles ahead of the one that is worked on, codes a tile ahead in registers, which become 16-bit
// values on the way. S^T = K Q^T and O^T += V^T P^T are 32x32x16 products, as in the prompt attention: a lane has 16 scores of
// one row for each 32 keys, and its weights, packed, are the next product's operand; V comes from LDS through the transposing
// reads. Two workgroups to a compute unit, which wait for each other nowhere: one of eight waves, in two groups that divide the
// keys and join in LDS, took 114 us against 109 in the last case below in turn on one card, and as long in the other two.
// A row's reference moves only when a score passes it by 2^8. A weight is multiplied in two parts of the type, as in the paged
// attention (over codes in bf16 ones for both types, since values times page or block scales have no place in fp16's range).
// In turn on one card, weights rounded once and in two parts: 611 and 763 us, 62 and 67, 110 and 129 in the cases below; rounded
// once, outputs are off by 0.0020 of their size instead of 0.0017 in bf16 and by 0.00027 instead of 0.00021 in fp16. Figures
// of what else was tried are of the kernel with weights rounded once.
//
// Eight prompts of up to 256 tokens behind 16K rows of fp16 pages (8 kv heads of 128, 6736 query rows to each), 454 GFLOP: 746 to
// 775 us on different cards, up to 608 TFLOP/s, 912 with the second parts' products (a large product of the library: 1078). The matrix unit
// is busy 43% of the cycles, the vector unit as much; 94% of the reads hit the L2. On the way there: masks and values that are not
// finite in a loop of their own (spills: 1341 to 871 us), page ids and offsets in registers of a window of 64 halves instead
// of scalar loads and 64-bit products (871 to 729, 646 to 614), rows of shorter prompts not padded (726 to 678), runs from
// their end on (677 to 646; before it 93% of the reads missed the L2). Not kept: units of 256 rows (691 of 678), tiles
// straight to LDS in rounds of two (765), priority to the matrix operations (616 of 614), all in workgroups of eight waves; the
// next tile's scores beside this one's weights (681 of 664 under the profiler). Tiles straight to LDS instead of through
// registers: no time here, 52 to 50 us of the next case's first launch.
// 32 sequences behind 32K rows of bf16 pages, 128 query rows to each of 8 kv heads: 65 to 71 us, 182 MB (28 us at the rate of a
// large read), 10 of them for the join of 66 parts to a row, the rest for the shared rows, the own ones and what lies between.
// 48 sequences of four drafts behind 20K rows of 4-bit pages, 768 query rows to each of 8 kv heads (63 GFLOP): 128 to 130 us, most of
// it for the shared rows, whose codes are widened once for 128 query rows.
#pragma once
#include "shared_attn_dev.h"

namespace mpc {
namespace dev {

// 16 bytes from p + off to the lane's place behind `at` (p and `at` the same over the wave), without a register between.
__device__ __forceinline__ void load_to_lds(const char* p, int off, uint4* at) {
  const uint32_t lds = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint4*)at);
  uint32_t was;
  asm volatile(
      "s_mov_b32 %0, m0\n\t"
      "s_mov_b32 m0, %1\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %2, %3\n\t"
      "s_mov_b32 m0, %0"
      : "=&s"(was)
      : "s"(lds), "v"(off), "s"(p)
      : "memory");
}
// Waits for a wave's loads but the last N (`some`) or for all of them, and for its LDS operations, then for the workgroup.
template <int N>
__device__ __forceinline__ void wait_loads(bool some) {
  if (some)
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
  else
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

template <class DT, int D, int FMT>
__device__ __forceinline__ void shared_wide(const SharedArgs& a, const Plan& plan) {
  constexpr bool C8 = FMT == MPC_PAGE_E4M3, C4 = FMT == MPC_PAGE_MX4, CODES = C8 || C4;
  constexpr bool H = DT::kCode == MPC_FP16, SPLIT = C4 && H;
  using QT = std::conditional_t<C4, BF16, DT>;    // type of the scores' product
  using PV = std::conditional_t<CODES, BF16, DT>;  // and of the values'
  constexpr int KT = 32, CH = D / 8, KSTEPS = D / 16, DB = D / 32, THREADS = 256, PS = D + kPartTail;
  constexpr float LIFT = PV::kCode == MPC_FP16 ? 7.f : 0.f;  // of the weights' exponents, also in their sum
  constexpr float SLACK = 8.f;                               // log2 of how far a weight may pass 1 before its reference moves
  constexpr int PER = CODES ? 1 : KT * CH / THREADS;         // pieces of K (and of V) that a thread stages
  constexpr int PCH = CODES ? D / 8 : 8;                     // channels of a piece
  constexpr int RB = C4 ? D / 2 : C8 ? D : 2 * D;            // bytes of a page's row
  // Codes: a tile in registers and two in LDS; others go straight to LDS, two tiles ahead of the one that is worked on.
  constexpr int NB = CODES ? 2 : 3;
  __shared__ uint4 s_k[NB][KT * CH], s_v[NB][KT * CH];
  __shared__ int s_bad[NB];        // codes: the last round whose values, staged for an edge, were not all finite; else [0]: the run is taken again
  __shared__ uint4 s_q2[SPLIT ? 4 : 1][KSTEPS][SPLIT ? kWave : 1];  // second parts of the queries (registers do not hold them)
  __shared__ int s_range[4][2];    // positions of the waves' rows
  const PagedCache& c = a.c;
  const int tid = threadIdx.x, lane = tid % kWave, q32 = lane & 31, hl = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);

  const unsigned total = plan.shared, id = by_die(blockIdx.x, gridDim.x);
  const unsigned per = (total + gridDim.x - 1) / gridDim.x;
  if ((unsigned long long)id * per >= total) return;
  const unsigned first = id * per, last = min(first + per, total);
  int gi = last_from(a.groups, last - 1, [&](int i) { return plan.group[i].block0; });
  // a negative scale is taken into the queries (8-bit codes: it stays with the pages' scales); zero times a masked score would be
  // NaN: the smallest number that is not zero instead
  const float qs = C8 ? a.qscale : fmaxf(fabsf(a.qscale), 0x1p-149f);
  const uint32_t flip = !C8 && a.qscale < 0.f ? 0x80008000u : 0u;

  // The run is taken from its end on, and a whole unit's blocks from the one on that the time says, so that workgroups with units
  // of the same keys are at the same keys at a time (their L2 has them once for all): what a run ends with begins at a
  // unit's first key, what it begins with ends at a unit's last one.
  unsigned x_end = last;
  while (x_end > first) {
    while (gi > 0 && x_end <= same(plan.group[gi].block0)) --gi;
    const SharedGroup* gp = plan.group + gi;
    const int f0 = same(gp->f0), nb = same(gp->nb), rts = same(gp->rt);
    const int base = same(gp->base), skip = same(gp->skip), at = same(gp->at);
    const unsigned block0 = same(gp->block0), in = x_end - 1 - block0;
    const int u = __builtin_amdgcn_readfirstlane(in / (unsigned)nb), blk_end = __builtin_amdgcn_readfirstlane(in - u * (unsigned)nb) + 1;
    const unsigned unit0 = block0 + u * (unsigned)nb;  // the unit's first block
    const int blk = first > unit0 ? (int)(first - unit0) : 0;
    const int lh = u / rts, h = lh % a.Hkv, l = lh / a.Hkv, r0 = u % rts * 128;
    const int i0 = blk * a.shared_block, i1 = min(blk_end * a.shared_block, same(gp->tiles));

    const SharedRow row = shared_row(a, plan.seq, gp, r0 + 32 * wave + q32);
    // a row that is not there sees every key, so that it makes no tile an edge; nobody reads it
    const int pos = row.live ? row.pos : kMaxRows;
    int lo = row.live ? pos : kMaxRows, hi = row.live ? pos : -kMaxRows;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      lo = min(lo, __shfl_xor(lo, o));
      hi = max(hi, __shfl_xor(hi, o));
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
    if (lane == 0) {
      s_range[wave][0] = lo;
      s_range[wave][1] = hi;
    }
    if (tid < NB) s_bad[tid] = -1;
    uint4 q[KSTEPS];
    {
      const int t = row.in_seq >> a.log_g, hq = (h << a.log_g) + row.in_seq - (t << a.log_g);
      const char* p = a.q.at(l, row.b, hq, t) + hl * 16;
#pragma unroll
      for (int i = 0; i < KSTEPS; ++i) {
        const uint4 y = ldg16(p + i * 32);
        q[i] = make_uint4(y.x ^ flip, y.y ^ flip, y.z ^ flip, y.w ^ flip);
        if constexpr (SPLIT) {
          uint4 rest;
          split_bf16(q[i], rest);
          s_q2[wave][i][lane] = rest;
        }
      }
    }
    f32x16 o[DB];
    float ref, sum;  // reference (in units of the exponent) and sum over this lane's keys
    __syncthreads();
    int g_lo = kMaxRows, g_hi = -kMaxRows;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      g_lo = min(g_lo, s_range[i][0]);
      g_hi = max(g_hi, s_range[i][1]);
    }
    g_lo = __builtin_amdgcn_readfirstlane(g_lo);
    g_hi = __builtin_amdgcn_readfirstlane(g_hi);

    // The run's tiles: first those that some row may not see whole (ahead of [w0, w1) and behind it), then those that every row
    // sees as far as their pages have rows.
    int w0 = i0, w1 = min(i1, (max(g_lo, -1) + 1) / KT - (a.window ? at - skip : 0));
    if (a.window) w0 = skip + max(0, (max(g_hi - a.window + 1, 0) + KT - 1) / KT - at);
    w0 = min(max(w0, i0), i1);
    w1 = max(w1, w0);
    const int edges = w0 - i0 + i1 - w1;
    auto key_of = [&](int i) { return (i < skip ? i : i - skip + at) * KT; };
    // whole tiles lie side by side; they are taken from number `turn` on
    const int whole0 = key_of(w0), n_whole = w1 - w0, whole_end = whole0 + n_whole * KT;
    const int turn = blk == 0 && blk_end == nb ? min((int)((last - x_end) % (unsigned)nb) * a.shared_block, max(n_whole - 1, 0)) : 0;
    auto whole_key = [&](int j) {
      const int i = j - edges + turn;
      return whole0 + (i >= n_whole ? i - n_whole : i) * KT;
    };
    auto key0 = [&](int j) { return j >= edges ? whole_key(j) : key_of(j < w0 - i0 ? i0 + j : w1 + j - (w0 - i0)); };
    // This (layer, kv head)'s rows of page 0, and bytes from a page to the next.
    const size_t page0 = page_unit(c, l, 0, h), page_bytes = (size_t)c.Hkv * c.page * RB;
    const char *k_page = c.k + page0 * c.page * RB, *v_page = c.v + page0 * c.page * RB;
    // A window of 64 halves (16 keys) from number `win` on, a lane to each: where its first row lies behind page 0's (that one where
    // there is no page: its rows are not used), whether there is one, and (8-bit codes) its page's scales.
    int win = -kWave;
    uint32_t w_lo = 0, w_hi = 0;
    unsigned long long w_has = 0;
    float w_ks = 0.f, w_vs = 0.f;
    auto load_window = [&](int half) {
      win = half;
      const int i = half + lane, pg = (16 * i) >> c.log_page;
      const int entry = c.table[(size_t)f0 * c.max_pages + min(pg, c.max_pages - 1)], id = page_of_entry(c, entry, pg);
      const size_t at = max(id, 0) * page_bytes + (size_t)((16 * i) & (c.page - 1)) * RB;
      w_lo = (uint32_t)at;
      w_hi = (uint32_t)(at >> 32);
      w_has = __ballot(id >= 0 && 16 * i < base);
      if constexpr (C8) {
        w_ks = c.ks[page0 + (size_t)max(id, 0) * c.Hkv];
        w_vs = c.vs[page0 + (size_t)max(id, 0) * c.Hkv];
      }
    };
    uint4 kr[CODES ? PER : 1], vr[CODES ? PER : 1];
    uint32_t kx = 0, vx = 0;                       // 4-bit codes: the piece's scale bytes
    float ks[2] = {1.f, 1.f}, vs[2] = {1.f, 1.f};  // 8-bit codes: the halves' page scales
    const int lane_row = (tid / 8 & 15) * RB + tid % 8 * (RB / 8);
    // a lane's place in LDS is fixed: which chunk of the row it asks for puts it where the exchange within the row wants it
    const int k_lane = (tid / CH & 15) * RB + tile_chunk_k<D>(tid / CH, tid % CH) % CH * 16;
    const int v_lane = (tid / CH & 15) * RB + tile_chunk_v<D>(tid / CH, tid % CH) % CH * 16;
    int k_at = 0;         // the fetched tile's first key
    unsigned has_at = 0;  // and whether its halves have a page
    auto fetch = [&](int k0, int buf) {
      int i = (k0 >> 4) - win;
      if ((unsigned)i >= kWave - 1) {
        load_window(k0 >> 4);
        i = 0;
      }
      k_at = k0;
      has_at = (unsigned)(w_has >> i) & 3u;
      size_t at[2];
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        at[hf] = (uint32_t)__builtin_amdgcn_readlane(w_lo, i + hf) | (size_t)(uint32_t)__builtin_amdgcn_readlane(w_hi, i + hf) << 32;
        if constexpr (C8) {
          ks[hf] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w_ks), i + hf));
          vs[hf] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w_vs), i + hf));
        }
      }
      if constexpr (CODES) {  // (a wave's rows lie in one half)
        const size_t from = wave >= 2 ? at[1] : at[0];
        const char *kp = k_page + from + lane_row, *vp = v_page + from + lane_row;
        if constexpr (RB / 8 == 16) {
          kr[0] = ldg16(kp);
          vr[0] = ldg16(vp);
        } else if constexpr (RB / 8 == 8) {
          const uint2 y = *(const uint2*)kp, z = *(const uint2*)vp;
          kr[0] = make_uint4(y.x, y.y, 0, 0);
          vr[0] = make_uint4(z.x, z.y, 0, 0);
        } else {
          kr[0] = make_uint4(*(const uint32_t*)kp, 0, 0, 0);
          vr[0] = make_uint4(*(const uint32_t*)vp, 0, 0, 0);
        }
        if constexpr (C4) {
          constexpr int SB = D / kMx4Block;
          const int slot = (k0 + (wave >= 2 ? 16 : 0)) & (c.page - 1);
          const size_t s_at = page0 * SB * c.page + from / RB * SB - slot * (SB - 1);
          const int lane_scale = tid % 8 * PCH / kMx4Block * c.page + (tid / 8 & 15);
          kx = (c.kx + s_at)[lane_scale];
          vx = (c.vx + s_at)[lane_scale];
        }
      } else {
#pragma unroll
        for (int n = 0; n < PER; ++n) {  // (a half to each n, or to each pair of waves)
          const bool second = PER == 2 ? n == 1 : wave >= 2;
          const size_t from = second ? at[1] : at[0];
          const int y = wave * kWave + n * THREADS;
          load_to_lds(k_page + from, k_lane, s_k[buf] + y);
          if (has_at >> (second ? 1 : 0) & 1)
            load_to_lds(v_page + from, v_lane, s_v[buf] + y);
          else  // values that have no page must not be anything
            s_v[buf][y + lane] = make_uint4(0, 0, 0, 0);
        }
      }
    };
    // Eight channels of a piece as 16-bit values.
    auto widened = [&](auto type, const uint4& y, int part, uint32_t xb) {
      using T = decltype(type);
      if constexpr (C4) {
        return widen8(part == 0 ? y.x : y.y, mx4_scale(xb));
      } else {
        const uint32_t w0 = part == 0 ? y.x : y.z, w1 = part == 0 ? y.y : y.w;
        return make_uint4(widen2<T, false>(w0), widen2<T, true>(w0), widen2<T, false>(w1), widen2<T, true>(w1));
      }
    };
    // Codes: stages the fetched tile, with zeros for values that have no page; whether it held values that are not finite (edge).
    auto stash = [&](auto edge_, int buf, const bool* have) {
      constexpr bool edge = decltype(edge_)::value;
      uint32_t top = 0;
      auto seen = [&](const uint4& y) { top = max_magnitude(max_magnitude(max_magnitude(max_magnitude(top, y.x), y.y), y.z), y.w); };
      if constexpr (CODES) {
        const int r = tid / 8, piece = tid % 8;
#pragma unroll
        for (int n = 0; n < PCH / 8; ++n) {
          const int chunk = piece * (PCH / 8) + n;
          uint4 y = widened(PV{}, vr[0], n, vx);
          if (!(wave >= 2 ? have[1] : have[0])) y = make_uint4(0, 0, 0, 0);
          if (edge) seen(y);
          s_k[buf][tile_chunk_k<D>(r, chunk)] = widened(QT{}, kr[0], n, kx);
          s_v[buf][tile_chunk_v<D>(r, chunk)] = y;
        }
      }
      return not_finite<PV>(top);
    };
    // The tile of round n at key k0; EDGE: some row of the wave may not see some key of it.
    auto tile = [&](auto edge, int k0, int buf, int n, const bool* have, const float* kss, const float* vss) {
      constexpr bool EDGE = decltype(edge)::value;
      const uint4* sk = s_k[buf];
      const char* sv = (const char*)s_v[buf];
      // places 0..3 and 4..7 of half hl in a product over 16 keys are keys 4 hl .. and 8 + 4 hl ..
      const int vrow = 4 * hl + ((lane & 15) >> 2);  // row whose piece this lane asks for, and the piece's 16-byte chunk
      const int vcol = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1), vbyte = (lane & 1) * 8;
      bool bad = EDGE && CODES && __builtin_amdgcn_readfirstlane(s_bad[buf]) == n;
      uint4 kf[KSTEPS];
#pragma unroll
      for (int i = 0; i < KSTEPS; ++i) kf[i] = sk[tile_chunk_k<D>(q32, 2 * i + hl)];
      // the values are asked for before the scores are taken, so that they are there when the weights are
      uint32_t vf[2][DB][4];
#pragma unroll
      for (int st = 0; st < 2; ++st)
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const char* p = sv + tile_chunk_v<D>(16 * st + 8 * e + vrow, 4 * d + vcol) * 16 + vbyte;
            const uint2 y = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p));
            vf[st][d][2 * e] = y.x;
            vf[st][d][2 * e + 1] = y.y;
          }
      __builtin_amdgcn_sched_barrier(0);
      f32x16 s;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
      for (int i = 0; i < KSTEPS; ++i) {
        if constexpr (SPLIT) s = mma32<QT>(kf[i], s_q2[wave][i][lane], s);
        s = mma32<QT>(kf[i], q[i], s);
      }
      // the lane's keys lie 8 (r / 4) + r % 4 behind this one
      const int j0 = k0 + 4 * hl;
      auto sees = [&](int j) { return j <= pos && (!a.window || j > pos - a.window || j < a.sinks); };  // (of those that exist)
      const float cc[2] = {C8 ? (have[0] ? qs * kss[0] : 1.f) : qs, C8 ? (have[1] ? qs * kss[1] : 1.f) : qs};
      auto key = [&](int r) { return j0 + 8 * (r >> 2) + (r & 3); };
      if (!(have[0] && have[1])) {
        asm volatile("");  // (a branch, not a selection for each score)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = have[r >> 3] ? s[r] : -INFINITY;
      }
      float top = -INFINITY;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if constexpr (C8) {
          const float y = s[r] * cc[r >> 3];
          top = fmaxf(top, !EDGE || sees(key(r)) ? y : -INFINITY);
        } else {
          if constexpr (EDGE) s[r] = sees(key(r)) ? s[r] : -INFINITY;
          top = fmaxf(top, s[r]);
        }
      }
      if constexpr (!C8) top *= qs;
      if (__any(top > ref + SLACK || (ref == -INFINITY && top > -INFINITY))) {
        top = xor_combine<32>(top, [](float p, float q) { return fmaxf(p, q); });
        const float was = ref;
        ref = top == -INFINITY ? ref : fmaxf(ref, top);
        // exp2(-inf - 0) = 0: nothing was there to move
        const float move = fast_exp2(was - (ref == -INFINITY ? 0.f : ref));
        sum *= move;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[d][r] *= move;
      }
      const float zero = (ref == -INFINITY ? 0.f : ref) - LIFT;
      uint32_t p[8], p2[8];  // weights in two parts of the type: rounded, and what that leaves, rounded
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        float w0 = fast_exp2(fmaf(s[r], cc[r >> 3], -zero)), w1 = fast_exp2(fmaf(s[r + 1], cc[r >> 3], -zero));
        if constexpr (C8 && EDGE) {
          w0 = sees(key(r)) ? w0 : 0.f;
          w1 = sees(key(r + 1)) ? w1 : 0.f;
        }
        sum += w0 + w1;
        if constexpr (C8) {  // a page that the row sees nothing of does not reach it, whatever its scale is
          const float f = have[r >> 3] ? vss[r >> 3] : 0.f;
          w0 = EDGE && w0 == 0.f ? 0.f : w0 * f;
          w1 = EDGE && w1 == 0.f ? 0.f : w1 * f;
        }
        p[r / 2] = pack2<PV>(w0, w1);
        const float2 x = unpack2<PV>(p[r / 2]);
        p2[r / 2] = pack2<PV>(w0 - x.x, w1 - x.y);
      }
      if constexpr (EDGE && !CODES) {
        uint32_t most = 0;
#pragma unroll
        for (int i = 0; i < 8 * DB; ++i) most = max_magnitude(most, vf[i / (4 * DB)][i / 4 % DB][i % 4]);
        bad = __any(not_finite<PV>(most));
      }
      // O^T += V^T P^T, 16 keys at a time
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const uint4 w = make_uint4(p[4 * st], p[4 * st + 1], p[4 * st + 2], p[4 * st + 3]);
        uint32_t(*v)[4] = vf[st];
        if constexpr (EDGE) {
          // Values that are not finite, in keys that some row does not see, must not meet that row's weight of zero: they are
          // added apart, to the rows that see them
          if (bad) {
            float one[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) one[e] = sees(j0 + 16 * st + (e >= 4 ? 8 : 0) + (e & 3)) ? 1.f : 0.f;
            const uint4 w1 = make_uint4(pack2<PV>(one[0], one[1]), pack2<PV>(one[2], one[3]), pack2<PV>(one[4], one[5]), pack2<PV>(one[6], one[7]));
#pragma unroll
            for (int d = 0; d < DB; ++d) {
              uint32_t what[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) what[e] = take_not_finite<PV>(v[d][e]);
              f32x16 y;
#pragma unroll
              for (int r = 0; r < 16; ++r) y[r] = 0.f;
              y = mma32<PV>(make_uint4(what[0], what[1], what[2], what[3]), w1, y);
#pragma unroll
              for (int r = 0; r < 16; ++r) o[d][r] += not_finite_sum(y[r]);
            }
          }
        }
#pragma unroll
        for (int d = 0; d < DB; ++d) {
          const uint4 y = make_uint4(v[d][0], v[d][1], v[d][2], v[d][3]);
          o[d] = mma32<PV>(y, make_uint4(p2[4 * st], p2[4 * st + 1], p2[4 * st + 2], p2[4 * st + 3]), o[d]);
          o[d] = mma32<PV>(y, w, o[d]);
        }
      }
    };

    const int tiles = i1 - i0;
    int place, k_next = 0, k_now;  // straight to LDS: the tile's place there, and the tile that is on its way behind it
    unsigned has_next = 0, has_now;
    auto round = [&](auto edge, int n) {
      constexpr bool EDGE = decltype(edge)::value;
      const int ahead = n + NB - 1, k0 = k_now, buf = CODES ? n & 1 : place;
      const bool have[2] = {(has_now & 1) != 0, (has_now & 2) != 0};
      const float kss[2] = {ks[0], ks[1]}, vss[2] = {vs[0], vs[1]};
      if constexpr (CODES) {
        if (stash(edge, buf, have) && EDGE) s_bad[buf] = n;
        __syncthreads();
      } else {
        // this tile's loads have arrived when no more than the next one's are on their way (fewer than 2 PER where it has zeros)
        wait_loads<2 * PER>(n + 1 < tiles && has_next == 3);
        k_now = k_next;
        has_now = has_next;
      }
      if (ahead < tiles) {
        int next = (CODES ? k0 : k_next) + KT;
        if (EDGE)
          next = key0(ahead);
        else if (next >= whole_end)
          next -= n_whole * KT;
        fetch(next, buf == 0 ? NB - 1 : buf - 1);  // (where the tile before this one was)
        (CODES ? k_now : k_next) = k_at;
        (CODES ? has_now : has_next) = has_at;
      }
      if (lo <= hi) tile(edge, k0, buf, n, have, kss, vss);
      if (!CODES) place = buf == NB - 1 ? 0 : buf + 1;
    };
    // Whole tiles multiply every value with every weight. An infinity times a weight that is zero in its type would be NaN: where an
    // accumulator ends up not finite beside a finite sum, the run is taken once more with every tile as an edge (a check of
    // every tile's values would cost all of them). Codes hold no infinities, and a NaN needs no sign.
    int n_edge = edges;
    for (;;) {
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
      ref = -INFINITY;
      sum = 0.f;
      place = 0;
      fetch(key0(0), 0);
      k_now = k_at;
      has_now = has_at;
      if (!CODES && tiles > 1) {
        fetch(key0(1), 1);
        k_next = k_at;
        has_next = has_at;
      }
      for (int n = 0; n < n_edge; ++n) round(std::true_type{}, n);
      for (int n = n_edge; n < tiles; ++n) round(std::false_type{}, n);
      sum = xor_combine<32>(sum, [](float p, float q) { return p + q; });
      if (CODES || n_edge == tiles) break;
      float zero = 0.f;  // NaN where an accumulator is not finite
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) zero = fmaf(o[d][r], 0.f, zero);
      if (row.live && zero != 0.f && sum * 0.f == 0.f) s_bad[0] = 0;
      __syncthreads();
      if (__builtin_amdgcn_readfirstlane(s_bad[0]) != 0) break;
      n_edge = tiles;
    }

    if (row.live) {
      float* part = blk == 0 ? a.shared.head + part_row(a, lh, row.b, row.in_seq) * PS : a.shared.more + ((size_t)id * 128 + 32 * wave + q32) * PS;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4) *(float4*)(part + 32 * d + 2 * r + 4 * hl) = make_float4(o[d][r], o[d][r + 1], o[d][r + 2], o[d][r + 3]);
      if (hl == 0) *(float2*)(part + D) = make_float2(ref - LIFT, sum);
    }
    __syncthreads();  // the LDS buffers are free again
    x_end = unit0 + blk;
  }
}

// Shared rows, then own ones, in units of 16 query rows (units of 32, in a launch of their own for want of registers, took as long:
// 616 us of what then was 614 for the eight prompts).
template <class DT, int D, int FMT>
__global__ __launch_bounds__(kWideWaves * kWave, 2) void k_shared_wide(SharedArgs a) {
  __shared__ PlanSpace space;
  const Plan plan = plan_of<FMT == MPC_PAGE_E4M3>(a, space);
  shared_wide<DT, D, FMT>(a, plan);
  own_rows_of<DT, D, FMT, 1, kWideWaves>(a, plan);
}

}  // namespace dev
}  // namespace mpc
