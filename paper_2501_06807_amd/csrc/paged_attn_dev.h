// Attention of new tokens over a paged cache on the matrix cores.
//
// A work unit is one (sequence, layer, kv head) and a group of 16 RT of its query rows (the G heads of the group times the
// new tokens), which K and V are read once for. Its keys come in tiles (32 keys, 16 in fp32), a tile for each wave of the
// workgroup to a block. The grid divides the blocks of all units evenly, whatever the lengths: a workgroup takes a run of blocks, and a
// unit that several of them share is joined by the last one to arrive. Lengths are read on the device, so a captured
// graph follows them.
//
// Of a tile a wave computes the scores transposed, S^T = K Q^T, so that a lane's four to eight scores belong to one
// query row and its weights are already the other operand of O^T += V^T P^T: no lane exchange but the row maximum's.
// The contraction's places are bound to channels and keys so that every load is 8 or 16 bytes of a row; V's rows meet in
// registers (byte permutes), and nothing passes through LDS until the waves' parts are joined.
// Running maximum m, sum l and the accumulators are fp32. 16-bit types multiply a weight in two parts of the type, its rounding
// and that of the rest, which holds it to half a step of half a step; fp32 multiplies in fp32. The second product of each value
// costs single and drafted tokens no time (one part and two: 371 us and 371 in the first case below, 61.6 and 61.0 in the
// second, 37.7 and 31.4 for the drafts, whose kernel no longer spills); chunks of more than 16 query rows to a unit over codes
// take 1.05 to 1.2 times as long (1000 rows of 32 heads over 20K rows of 8: 1076 us and 1272; over 16-bit pages 1460 and 1446).
// The outputs' error falls from 0.0018 to 0.0017 of their size, what rounding them to bf16 costs. Codes
// widen exactly to either 16-bit type. A page's value scale goes into a bf16 weight, whose range takes it; fp16 weights have no
// such range: they are lifted by 2^14, so that only weights below 2^-28 of the largest lose bits of their first part, and the
// scale is applied to a tile's product in fp32.
//
// 4-bit codes have a scale for each 32 channels of a row, so they become bf16 values with their scale (v_cvt_scalef32, exact) before they
// are transposed; fp16, whose range does not hold code times scale, is multiplied in bf16 too, with the queries in two parts
// (8 + 3 places, exact).
//
// Reading K and V bounds it: 4 x 32K rows, 2 layers of 32 heads of 128 over 8-bit pages, 2.1 GB in 371 us (5.8 TB/s); one
// sequence of 128K rows and 8 kv heads, 268 MB in 61 us, of which about 12 are not reading: the launch, the chain of
// lengths, table entry and first rows (4), and the joins (4 to 8). The same rows of 4-bit codes: 1.14 GB in 201 us (5.7 TB/s; a
// tile's 230 vector operations keep that unit busy half of the time, and tiles two ahead instead of one gain nothing, 206), three drafts
// over 128K rows 143 MB in 46 us. In between the dies differ: their workgroups read at rates
// 35% apart, so that the even division ends with the slowest (41 us on average, 48 on the last). Keys two tiles ahead instead
// of one changed nothing (373 and 63 us), nor did runs of at least four blocks where there is enough work. 32 sequences of
// four drafted tokens behind a window of 1024 (16-bit pages of 16 rows) take 32 us, 136 MB (147 fetched): each workgroup has
// one unit of 34 tiles, five rounds of its waves, and nothing beside the start, the last round and the end. A table entry or a
// scale read through the vector cache waits for every row in flight: the scalar cache took the first case from 426 to 365.
#pragma once
#include "attn_mma.h"

namespace mpc {
namespace dev {


template <class DT, int D, int FMT, int RT>
struct PagedTile {
  static constexpr bool F = DT::kElt == 4;
  static constexpr bool C8 = FMT == MPC_PAGE_E4M3, C4 = FMT == MPC_PAGE_MX4;  // codes of 8 bits, or of 4
  static constexpr int TK = F ? 16 : 32;       // keys of a tile
  static constexpr int HALVES = TK / 16;       // 16-key halves, each inside one page
  static constexpr int NT = D / 16;            // 16-channel tiles of the output; channel (4 g + r) * NT + t in tile t
  static constexpr int KB = F ? 4 : 2;         // element bytes
  static constexpr int RB = C4 ? D / 2 : D * (C8 ? 1 : KB);  // bytes of a page's row
  static constexpr int KL = RB < 64 ? 1 : RB / 64;  // 16-byte loads of a lane's key row (four lanes to a row; 8 bytes where a row has 32)
  static constexpr int KLT = D * KB / 64;      // the same of a tail row
  static constexpr int VK = F ? 4 : 8;         // keys of a lane's value rows
  static constexpr int VWT = NT * KB / 4;      // words of a lane's piece of a tail row
  static constexpr int VW = C4 ? 1 : NT * (C8 ? 1 : KB) / 4;  // and of a page's row (4 bits, d 64: half a word)
  static constexpr int SB = D / kMx4Block;     // 4 bits: scales of a row
  // Type of the values' product, and of the scores' with 4-bit codes: what holds every code times its scale. fp16 does not,
  // so its queries are multiplied in two bf16 parts (exact: 8 + 3 places), the second part's frags behind the first's.
  using PV = std::conditional_t<C4 && !F, BF16, DT>;
  static constexpr bool SPLIT = C4 && DT::kCode == MPC_FP16;
  // queries: 16-bit frags of 32 channels, or fp32 words of 4
  static constexpr int QF = F ? D / 4 : D / 32, QN = SPLIT ? 2 * QF : QF;
  using QFrag = std::conditional_t<F, float, uint4>;
  // fp16: exponents of the weights are lifted by this (also in the sum), and page scales applied to products
  static constexpr bool H = PV::kCode == MPC_FP16;
  static constexpr float LIFT = H ? 14.f : 0.f;

  // First channel of query fragment i of lane group g (fp32: of word i).
  __device__ static int q_channel(int i, int g) {
    if constexpr (C4) return g * (D / 4) + i * (F ? 1 : 8);
    if constexpr (F) return C8 ? i / 16 * 64 + g * 16 + i % 16 : i / 4 * 16 + g * 4 + i % 4;
    return C8 ? i / 2 * 64 + g * 16 + i % 2 * 8 : i * 32 + g * 8;
  }
  // Key (of the tile) of value place j of lane group g.
  __device__ static int v_key(int j, int g) { return j < 4 ? 4 * g + j : 16 + 4 * g + j - 4; }
};

template <int W>
__device__ __forceinline__ void load_words(const char* p, uint32_t* w) {
  if constexpr (W == 1) {
    w[0] = *(const uint32_t*)p;
  } else if constexpr (W == 2) {
    const uint2 x = *(const uint2*)p;
    w[0] = x.x;
    w[1] = x.y;
  } else {
#pragma unroll
    for (int i = 0; i < W / 4; ++i) {
      const uint4 x = ldg16(p + i * 16);
      w[4 * i] = x.x;
      w[4 * i + 1] = x.y;
      w[4 * i + 2] = x.z;
      w[4 * i + 3] = x.w;
    }
  }
}

// The state of a wave's rows: column c of each 16-row tile is a query row.
template <class DT, int D, int FMT, int RT>
struct PagedWave {
  using TL = PagedTile<DT, D, FMT, RT>;
  static constexpr bool F = TL::F, C8 = TL::C8, C4 = TL::C4, CODES = C8 || C4;
  typename TL::QFrag q[RT][TL::QN];
  f32x4 o[RT][TL::NT];
  float m[RT], l[RT];  // running maximum of the column; sum over this lane's keys
  int pos[RT];         // position of the column's row, or one that sees nothing

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
      for (int t = 0; t < TL::NT; ++t) o[rt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
      m[rt] = -INFINITY;
      l[rt] = 0.f;
    }
  }

  // s += K Q^T of one tile: keys in the rows, query rows in the columns. kx: scale bytes of this lane's codes (4 bits).
  template <bool TAIL>
  __device__ __forceinline__ void scores(const uint4 (*k)[TAIL ? TL::KLT : TL::KL], f32x4 (*s)[TL::HALVES], const uint32_t* kx = nullptr) const {
#pragma unroll
    for (int h = 0; h < TL::HALVES; ++h) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) s[rt][h] = f32x4{0.f, 0.f, 0.f, 0.f};
      if constexpr (F) {
        // four chains of products, one for each word of a row's piece: a chain's sum is rounded at every step of it
        f32x4 y[RT][4];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int e = 0; e < 4; ++e) y[rt][e] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < (TAIL ? TL::KLT : TL::KL); ++i) {
          const uint32_t w[4] = {k[h][i].x, k[h][i].y, k[h][i].z, k[h][i].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if constexpr (C4) {
              if (e >= D / 32) continue;  // (d 64: two words)
              float x[8];
              decode8(w[e], mx4_scale(kx[h]), x);
#pragma unroll
              for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) y[rt][(8 * e + n) / (D / 16)] = mma(x[n], q[rt][8 * e + n], y[rt][(8 * e + n) / (D / 16)]);
            } else if constexpr (C8 && !TAIL) {
              float x[4];
              decode4(w[e], x);
#pragma unroll
              for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) y[rt][e] = mma(x[n], q[rt][16 * i + 4 * e + n], y[rt][e]);
            } else {
#pragma unroll
              for (int rt = 0; rt < RT; ++rt) y[rt][e] = mma(__uint_as_float(w[e]), q[rt][4 * i + e], y[rt][e]);
            }
          }
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) s[rt][h] = (y[rt][0] + y[rt][1]) + (y[rt][2] + y[rt][3]);
      } else if constexpr (C4) {
        const uint32_t w[4] = {k[h][0].x, k[h][0].y, k[h][0].z, k[h][0].w};
        const float scale = mx4_scale(kx[h]);
#pragma unroll
        for (int i = 0; i < TL::QF; ++i) {
          const uint4 x = widen8(w[i], scale);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            if constexpr (TL::SPLIT) s[rt][h] = mma<BF16>(x, q[rt][TL::QF + i], s[rt][h]);
            s[rt][h] = mma<BF16>(x, q[rt][i], s[rt][h]);
          }
        }
      } else if constexpr (C8 && !TAIL) {
#pragma unroll
        for (int i = 0; i < TL::KL; ++i) {
          const uint4& x = k[h][i];
          const uint4 lo8 = make_uint4(widen2<DT, false>(x.x), widen2<DT, true>(x.x), widen2<DT, false>(x.y), widen2<DT, true>(x.y));
          const uint4 hi8 = make_uint4(widen2<DT, false>(x.z), widen2<DT, true>(x.z), widen2<DT, false>(x.w), widen2<DT, true>(x.w));
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            s[rt][h] = mma<DT>(lo8, q[rt][2 * i], s[rt][h]);
            s[rt][h] = mma<DT>(hi8, q[rt][2 * i + 1], s[rt][h]);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < TL::QF; ++i)
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) s[rt][h] = mma<DT>(k[h][i], q[rt][i], s[rt][h]);
      }
    }
  }

  // Whether the row at position p sees key j (of those that exist).
  __device__ static __forceinline__ bool sees(const AttnArgs& a, int p, int j) {
    return j <= p && (!a.window || j > p - a.window || j < a.sinks);
  }

  // Whether the row at position p sees any of the 16 keys from j0 on (of those that exist).
  __device__ static __forceinline__ bool sees_half(const AttnArgs& a, int p, int j0) {
    return j0 <= p && (!a.window || j0 + 15 > p - a.window || j0 < a.sinks);
  }

  // Scores to weights (by value place): scale c and weight factor f of each half; maximum and sum follow. With `edge`
  // some row may not see some key; have: halves that exist, rows: rows that do.
  __device__ __forceinline__ void weights(const f32x4 (*s)[TL::HALVES], const float* c, const float* f, const AttnArgs& a,
                                          bool edge, int k0, int rows, const bool* have, float (*p)[TL::VK]) {
    const int g = (threadIdx.x % kWave) / 16;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
      for (int h = 0; h < TL::HALVES; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) p[rt][4 * h + r] = s[rt][h][r] * c[h];
      if (edge) {
#pragma unroll
        for (int h = 0; h < TL::HALVES; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int j = k0 + 16 * h + 4 * g + r;
            if (!(have[h] && j < rows && sees(a, pos[rt], j))) p[rt][4 * h + r] = -INFINITY;
          }
      }
      float top = p[rt][0];
#pragma unroll
      for (int j = 1; j < TL::VK; ++j) top = fmaxf(top, p[rt][j]);
      top = column_max(top);
      if (__any(top > m[rt])) {
        const float m_new = fmaxf(m[rt], top);
        // exp2(-inf - 0) = 0: nothing was there to move
        const float move = fast_exp2(m[rt] - (m_new == -INFINITY ? 0.f : m_new));
        m[rt] = m_new;
        l[rt] *= move;
#pragma unroll
        for (int t = 0; t < TL::NT; ++t) o[rt][t] *= move;
      }
      const float base = (m[rt] == -INFINITY ? 0.f : m[rt]) - TL::LIFT;
      // The exponent s c - base in one rounding: what the product alone would lose, half a step of the score's size, is as
      // large as that step in the weight (scores of 4000 in fp32: outputs off by 6e-6).
      float e[TL::VK];
#pragma unroll
      for (int j = 0; j < TL::VK; ++j) e[j] = fmaf(s[rt][j / 4][j % 4], c[j / 4], -base);
      if (edge) {
#pragma unroll
        for (int j = 0; j < TL::VK; ++j) e[j] = p[rt][j] == -INFINITY ? -INFINITY : e[j];
      }
#pragma unroll
      for (int j = 0; j < TL::VK; ++j) {
        p[rt][j] = fast_exp2(e[j]);
        l[rt] += p[rt][j];
      }
      if (f) {
#pragma unroll
        for (int h = 0; h < TL::HALVES; ++h) {
          // a page that the row sees nothing of does not reach it, whatever its scale is
          const float fh = !edge || sees_half(a, pos[rt], k0 + 16 * h) ? f[h] : 0.f;
#pragma unroll
          for (int r = 0; r < 4; ++r) p[rt][4 * h + r] *= fh;
        }
      }
    }
  }

  // Value rows as 16-bit operands, one for each channel tile: the places of a channel side by side. vx: the scale bytes of
  // four keys of each half (4 bits).
  template <bool TAIL>
  __device__ static __forceinline__ void operands(const uint32_t (*v)[TAIL ? TL::VWT : TL::VW], uint32_t (*w)[4], const uint32_t* vx = nullptr) {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      if constexpr (C4) {
        const float sa = mx4_scale(vx[p / 2] >> 16 * (p % 2)), sb = mx4_scale(vx[p / 2] >> (16 * (p % 2) + 8));
        const uint4 a = widen8(v[2 * p][0], sa), b = widen8(v[2 * p + 1][0], sb);
        const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int n = 0; n < TL::NT / 2; ++n) {
          w[2 * n][p] = __builtin_amdgcn_perm(y[n], x[n], 0x05040100u);
          w[2 * n + 1][p] = __builtin_amdgcn_perm(y[n], x[n], 0x07060302u);
        }
      } else if constexpr (C8 && !TAIL) {
#pragma unroll
        for (int i = 0; i < TL::VW; ++i) {
          const uint32_t a = v[2 * p][i], b = v[2 * p + 1][i];
          const uint32_t x = __builtin_amdgcn_perm(b, a, 0x05010400u), y = __builtin_amdgcn_perm(b, a, 0x07030602u);
          w[4 * i][p] = widen2<DT, false>(x);
          w[4 * i + 1][p] = widen2<DT, true>(x);
          w[4 * i + 2][p] = widen2<DT, false>(y);
          w[4 * i + 3][p] = widen2<DT, true>(y);
        }
      } else {
#pragma unroll
        for (int i = 0; i < TL::VWT; ++i) {
          const uint32_t a = v[2 * p][i], b = v[2 * p + 1][i];
          w[2 * i][p] = __builtin_amdgcn_perm(b, a, 0x05040100u);
          w[2 * i + 1][p] = __builtin_amdgcn_perm(b, a, 0x07060302u);
        }
      }
    }
  }
  // Value rows as fp32 operands.
  template <bool TAIL>
  __device__ static __forceinline__ void operands(const uint32_t (*v)[TAIL ? TL::VWT : TL::VW], float (*x)[TL::NT], const uint32_t* vx = nullptr) {
#pragma unroll
    for (int j = 0; j < TL::VK; ++j) {
      if constexpr (C4) {
        float y[8];
        decode8(v[j][0], mx4_scale(vx[j / 4] >> 8 * (j % 4)), y);
#pragma unroll
        for (int i = 0; i < TL::NT; ++i) x[j][i] = y[i];
      } else if constexpr (C8 && !TAIL) {
#pragma unroll
        for (int i = 0; i < TL::VW; ++i) decode4(v[j][i], x[j] + 4 * i);
      } else {
#pragma unroll
        for (int i = 0; i < TL::NT; ++i) x[j][i] = __uint_as_float(v[j][i]);
      }
    }
  }

  // o += V^T P^T. With `edge`: value rows that no row of the group sees do not enter (zero times what they hold might not
  // be zero). Values that are not finite are added apart, to the rows that see them: a weight's second part may be zero, or
  // below zero, and with `edge` some rows do not see them at all. (Codes hold no infinities, and a NaN needs no sign: those of
  // tiles that every row sees stay where they are.) lo, hi: the smallest and largest position of the group's rows.
  // scale: factors of the halves' products, or null.
  __device__ __forceinline__ void add_values(uint32_t (*w)[4], const float (*p)[TL::VK], const AttnArgs& a, bool edge, int k0,
                                             int rows, const bool* have, int lo, int hi, const float* scale) {
    using PV = typename TL::PV;
    const int g = (threadIdx.x % kWave) / 16;
    if (edge) {
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        uint32_t keep = 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int j = 2 * n + i, key = k0 + TL::v_key(j, g);
          const bool any = have[j / 4] && key < rows && key <= hi && (!a.window || key > lo - a.window || key < a.sinks);
          keep |= any ? 0xFFFFu << 16 * i : 0u;
        }
#pragma unroll
        for (int t = 0; t < TL::NT; ++t) w[t][n] &= keep;
      }
    }
    if (edge || !CODES) {
      uint32_t top = 0;
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int t = 0; t < TL::NT; ++t) top = max_magnitude(top, w[t][n]);
      if (__any(not_finite<PV>(top))) {
        float one[RT][TL::VK];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int j = 0; j < TL::VK; ++j) one[rt][j] = sees(a, pos[rt], k0 + TL::v_key(j, g)) ? 1.f : 0.f;
#pragma unroll
        for (int t = 0; t < TL::NT; ++t) {
          uint32_t what[4];
#pragma unroll
          for (int n = 0; n < 4; ++n) what[n] = take_not_finite<PV>(w[t][n]);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            const f32x4 y = mma<PV>(words(what), packed<PV>(one[rt]), f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int r = 0; r < 4; ++r) o[rt][t][r] += not_finite_sum(y[r]);
          }
        }
      }
    }
    // A weight is multiplied in two parts of the type, itself rounded and the rest of that, rounded: it loses half a step of
    // half a step (2^-16 in bf16), not the half step that the output's own rounding would have beside it.
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const uint4 x = packed<PV>(p[rt]);
      float rest[TL::VK];
      unpack<PV>(x, rest);
#pragma unroll
      for (int j = 0; j < TL::VK; ++j) rest[j] = p[rt][j] - rest[j];
      const uint4 y = packed<PV>(rest);
      if (!scale) {
#pragma unroll
        for (int t = 0; t < TL::NT; ++t) o[rt][t] = mma<PV>(words(w[t]), x, mma<PV>(words(w[t]), y, o[rt][t]));
      } else if (!edge && scale[0] == scale[1]) {
#pragma unroll
        for (int t = 0; t < TL::NT; ++t) o[rt][t] += mma<PV>(words(w[t]), x, mma<PV>(words(w[t]), y, f32x4{0.f, 0.f, 0.f, 0.f})) * scale[0];
      } else {  // two pages of 16 rows, or rows that see nothing of one half (its scale does not reach them)
        const float s0 = !edge || sees_half(a, pos[rt], k0) ? scale[0] : 0.f, s1 = !edge || sees_half(a, pos[rt], k0 + 16) ? scale[1] : 0.f;
        const uint4 x0 = make_uint4(x.x, x.y, 0, 0), x1 = make_uint4(0, 0, x.z, x.w), y0 = make_uint4(y.x, y.y, 0, 0), y1 = make_uint4(0, 0, y.z, y.w);
#pragma unroll
        for (int t = 0; t < TL::NT; ++t)
          o[rt][t] += mma<PV>(words(w[t]), x0, mma<PV>(words(w[t]), y0, f32x4{0.f, 0.f, 0.f, 0.f})) * s0 +
                      mma<PV>(words(w[t]), x1, mma<PV>(words(w[t]), y1, f32x4{0.f, 0.f, 0.f, 0.f})) * s1;
      }
    }
  }
  __device__ static __forceinline__ uint4 words(const uint32_t* w) { return make_uint4(w[0], w[1], w[2], w[3]); }
  template <class PV>
  __device__ static __forceinline__ uint4 packed(const float* y) {
    return make_uint4(pack2<PV>(y[0], y[1]), pack2<PV>(y[2], y[3]), pack2<PV>(y[4], y[5]), pack2<PV>(y[6], y[7]));
  }
  // The same in fp32.
  __device__ __forceinline__ void add_values(float (*x)[TL::NT], const float (*p)[TL::VK], const AttnArgs& a, bool edge, int k0,
                                             int rows, const bool* have, int lo, int hi, const float*) {
    const int g = (threadIdx.x % kWave) / 16;
    if (edge) {
      bool bad = false;
#pragma unroll
      for (int j = 0; j < TL::VK; ++j) {
        const int key = k0 + TL::v_key(j, g);
        const bool any = have[j / 4] && key < rows && key <= hi && (!a.window || key > lo - a.window || key < a.sinks);
#pragma unroll
        for (int t = 0; t < TL::NT; ++t) {
          x[j][t] = any ? x[j][t] : 0.f;
          bad |= not_finite<F32>(__float_as_uint(x[j][t]));
        }
      }
      if (lo != hi && __any(bad)) {
        float one[RT][TL::VK];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int j = 0; j < TL::VK; ++j) one[rt][j] = sees(a, pos[rt], k0 + TL::v_key(j, g)) ? 1.f : 0.f;
#pragma unroll
        for (int t = 0; t < TL::NT; ++t) {
          float what[TL::VK];
#pragma unroll
          for (int j = 0; j < TL::VK; ++j) {
            uint32_t u = __float_as_uint(x[j][t]);
            what[j] = __uint_as_float(take_not_finite<F32>(u));
            x[j][t] = __uint_as_float(u);
          }
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            f32x4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < TL::VK; ++j) y = mma(what[j], one[rt][j], y);
#pragma unroll
            for (int r = 0; r < 4; ++r) o[rt][t][r] += not_finite_sum(y[r]);
          }
        }
      }
    }
#pragma unroll
    for (int j = 0; j < TL::VK; ++j)
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int t = 0; t < TL::NT; ++t) o[rt][t] = mma(x[j][t], p[rt][j], o[rt][t]);
  }
};

// This lane's pieces of a query row (zeros where there is none).
template <class DT, int D, int FMT, int RT>
__device__ __forceinline__ void load_query_row(PagedWave<DT, D, FMT, RT>& w, int rt, const char* row, bool ok) {
  using TL = PagedTile<DT, D, FMT, RT>;
  const int g = (threadIdx.x % kWave) / 16;
  if constexpr (TL::F) {
#pragma unroll
    for (int i = 0; i < TL::QF; i += 4) {
      const uint4 y = ldg16(row + TL::q_channel(i, g) * 4);
      w.q[rt][i] = ok ? __uint_as_float(y.x) : 0.f;
      w.q[rt][i + 1] = ok ? __uint_as_float(y.y) : 0.f;
      w.q[rt][i + 2] = ok ? __uint_as_float(y.z) : 0.f;
      w.q[rt][i + 3] = ok ? __uint_as_float(y.w) : 0.f;
    }
  } else {
#pragma unroll
    for (int i = 0; i < TL::QF; ++i) {
      const uint4 y = ldg16(row + TL::q_channel(i, g) * 2);
      w.q[rt][i] = ok ? y : make_uint4(0, 0, 0, 0);
      if constexpr (TL::SPLIT) split_bf16(w.q[rt][i], w.q[rt][TL::QF + i]);
    }
  }
}

// The pages' rows that a unit's rows look at, in tiles: [from, from + skip), then from `at` on; keys [base, full) of them.
struct PageRows {
  int skip, at, from, base, full;
};

// A wave's tiles i, i + STEP, .. (before i_end) of (sequence b's table, layer l, kv head h), for rows at positions lo .. hi; takes
// the queries in beside the first loads.
template <class DT, int D, int FMT, int RT, int STEP, class Queries>
__device__ __forceinline__ void walk_pages(PagedWave<DT, D, FMT, RT>& w, const AttnArgs& a, const PagedCache& c, int b, int l, int h,
                                           const PageRows& r, int i, int i_end, int lo, int hi, Queries load_queries) {
  using TL = PagedTile<DT, D, FMT, RT>;
  constexpr bool C8 = TL::C8, C4 = TL::C4;
  constexpr int NT = TL::NT;
  const int lane = threadIdx.x % kWave, g = lane / 16, col = lane % 16;
  auto page_tile = [&](int i) { return i < r.skip ? r.from + i : i - r.skip + r.at; };
  auto page_at = [&](int i, int hf) { return (page_tile(i) * TL::TK + 16 * hf) >> c.log_page; };
  // table entries of a tile's halves, and the page ids that they give (-1 where there is none)
  auto entries_of = [&](int i, int* e) {
#pragma unroll
    for (int hf = 0; hf < TL::HALVES; ++hf) e[hf] = page_entry(c, b, page_at(i, hf));
  };
  auto ids_of = [&](int i, const int* e, int* id) {
#pragma unroll
    for (int hf = 0; hf < TL::HALVES; ++hf) id[hf] = page_of_entry(c, e[hf], page_at(i, hf));
  };
  // This (layer, kv head)'s part of page 0 and the bytes (scales) from a page to the next; a lane's place in a half's rows.
  const size_t unit0 = page_unit(c, l, 0, h), page_bytes = (size_t)c.Hkv * c.page * TL::RB;
  const char *k_page = c.k + unit0 * c.page * TL::RB, *v_page = c.v + unit0 * c.page * TL::RB;
  const unsigned k_lane = col * TL::RB + g * (TL::RB < 64 ? 8 : 16), v_lane = 4 * g * TL::RB + col * (TL::RB / 16);
  const uint8_t *kx_page = C4 ? c.kx + unit0 * (TL::SB * c.page) : nullptr, *vx_page = C4 ? c.vx + unit0 * (TL::SB * c.page) : nullptr;
  const unsigned kx_lane = g * TL::SB / 4 * c.page + col, vx_lane = col * TL::SB / 16 * c.page + 4 * g;
  // a half's first row (page 0 where it has no page: its rows are not used)
  auto slot_of = [&](int i, int hf) { return (page_tile(i) * TL::TK + 16 * hf) & (c.page - 1); };
  auto load_k = [&](int i, const int* id, uint4 (*k)[TL::KL], float* ks, uint32_t* kx) {
#pragma unroll
    for (int hf = 0; hf < TL::HALVES; ++hf) {
      const int n = max(id[hf], 0), slot = slot_of(i, hf);
      const char* p = k_page + (n * page_bytes + (size_t)slot * TL::RB);
      if constexpr (TL::RB < 64) {
        const uint2 x = *(const uint2*)(p + k_lane);
        k[hf][0] = make_uint4(x.x, x.y, 0, 0);
      } else {
#pragma unroll
        for (int m = 0; m < TL::KL; ++m) k[hf][m] = ldg16(p + k_lane + m * 64);
      }
      if constexpr (C8) ks[hf] = load_uniform(c.ks + unit0 + (size_t)n * c.Hkv);
      if constexpr (C4) kx[hf] = (kx_page + ((size_t)n * c.Hkv * (TL::SB * c.page) + slot))[kx_lane];
    }
  };
  auto load_v = [&](int i, const int* id, uint32_t (*v)[TL::VW], float* vs, uint32_t* vx) {
#pragma unroll
    for (int hf = 0; hf < TL::HALVES; ++hf) {
      const int n = max(id[hf], 0), slot = slot_of(i, hf);
      const char* p = v_page + (n * page_bytes + (size_t)slot * TL::RB);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (TL::RB < 64)
          v[4 * hf + j][0] = *(const uint16_t*)(p + v_lane + j * TL::RB);
        else
          load_words<TL::VW>(p + v_lane + j * TL::RB, v[4 * hf + j]);
      }
      if constexpr (C8) vs[hf] = load_uniform(c.vs + unit0 + (size_t)n * c.Hkv);
      if constexpr (C4) vx[hf] = *(const uint32_t*)(vx_page + ((size_t)n * c.Hkv * (TL::SB * c.page) + slot) + vx_lane);
    }
  };
  using Operand = std::conditional_t<TL::F, float[TL::VK][NT], uint32_t[NT][4]>;
  if (i < i_end) {
    // A tile's keys are dead after the scores and its values after the transpose: the next tile's loads go out there,
    // into the same registers, and are waited for a tile's work later.
    uint4 k[TL::HALVES][TL::KL];
    uint32_t v[TL::VK][TL::VW];
    float ks[TL::HALVES], vs[TL::HALVES];
    uint32_t kx[TL::HALVES], vx[TL::HALVES];
    int id[TL::HALVES], next[TL::HALVES], entry[TL::HALVES];
    entries_of(i, entry);
    ids_of(i, entry, id);
    load_k(i, id, k, ks, kx);
    load_v(i, id, v, vs, vx);
    load_queries();
    auto after = [&](int n) { return n + STEP < i_end ? n + STEP : n; };
    entries_of(after(i), entry);
    for (;;) {
      // the last tile asks for itself again, so that every pass has the same loads in flight and waits for its own only
      const int i1 = after(i);
      const int k0 = page_tile(i) * TL::TK, k1 = k0 + TL::TK - 1;
      bool have[TL::HALVES], all = true;
      float sc[TL::HALVES], vf[TL::HALVES];
#pragma unroll
      for (int hf = 0; hf < TL::HALVES; ++hf) {
        have[hf] = id[hf] >= 0 && k0 + 16 * hf < r.full && k0 + 16 * hf >= r.base;
        all = all && have[hf];
      }
      const bool edge = !(all && k1 < r.full && k1 <= lo && (!a.window || k0 > hi - a.window || k1 < a.sinks));
      f32x4 sr[RT][TL::HALVES];
      w.template scores<false>(k, sr, kx);
#pragma unroll
      for (int hf = 0; hf < TL::HALVES; ++hf) {
        sc[hf] = C8 ? (have[hf] ? a.qscale * ks[hf] : 0.f) : a.qscale;
        vf[hf] = C8 ? (have[hf] ? vs[hf] : 0.f) : 1.f;
      }
      ids_of(i1, entry, next);
      load_k(i1, next, k, ks, kx);
      entries_of(after(i1), entry);
      float p[RT][TL::VK];
      w.weights(sr, sc, C8 && !TL::H ? vf : nullptr, a, edge, k0, r.full, have, p);
      Operand x;
      w.template operands<false>(v, x, vx);
      load_v(i1, next, v, vs, vx);
#pragma unroll
      for (int hf = 0; hf < TL::HALVES; ++hf) id[hf] = next[hf];
      w.add_values(x, p, a, edge, k0, r.full, have, lo, hi, C8 && TL::H ? vf : nullptr);
      if (i1 == i) break;
      i = i1;
    }
  }
  else {
    load_queries();
  }
}

// The same for tiles of a page that is not complete, rows [full, rows), from the ring (8-bit codes).
template <class DT, int D, int RT, int STEP>
__device__ __forceinline__ void walk_tail(PagedWave<DT, D, MPC_PAGE_E4M3, RT>& w, const AttnArgs& a, const PagedCache& c, int b, int l,
                                          int h, int full, int rows, int i, int i_end, int lo, int hi) {
  using TL = PagedTile<DT, D, MPC_PAGE_E4M3, RT>;
  constexpr int NT = TL::NT;
  const int lane = threadIdx.x % kWave, g = lane / 16, col = lane % 16;
  for (; i < i_end; i += STEP) {
    const int k0 = full + i * TL::TK;
    if (k0 >= rows) break;
    const size_t ring = (((size_t)l * c.B + b) * c.Hkv + h) * (2 * c.page);
    auto row = [&](const char* base_, int j) { return base_ + (ring + (j & (2 * c.page - 1))) * (size_t)(D * TL::KB); };
    uint4 kr[TL::HALVES][TL::KLT];
    uint32_t vr[TL::VK][TL::VWT];
#pragma unroll
    for (int hf = 0; hf < TL::HALVES; ++hf)
#pragma unroll
      for (int e = 0; e < TL::KLT; ++e)
        kr[hf][e] = ldg16(row(c.k_tail, k0 + 16 * hf + col) + TL::q_channel(TL::F ? 4 * e : e, g) * TL::KB);
#pragma unroll
    for (int j = 0; j < TL::VK; ++j)
      load_words<TL::VWT>(row(c.v_tail, k0 + TL::v_key(j, g)) + col * (TL::VWT * 4), vr[j]);
    const bool have[2] = {true, true};
    const float sc[2] = {a.qscale, a.qscale};
    f32x4 sr[RT][TL::HALVES];
    w.template scores<true>(kr, sr);
    float p[RT][TL::VK];
    w.weights(sr, sc, nullptr, a, true, k0, rows, have, p);
    std::conditional_t<TL::F, float[TL::VK][NT], uint32_t[NT][4]> x;
    w.template operands<true>(vr, x);
    w.add_values(x, p, a, true, k0, rows, have, lo, hi, nullptr);
  }
}

// Maxima, sums and accumulators of a workgroup's waves into those of wave 0 (M and Lsum: of every wave).
template <class DT, int D, int FMT, int RT>
__device__ __forceinline__ void join_waves(PagedWave<DT, D, FMT, RT>& w, int wave, float (*s_ml)[RT][2][kWave],
                                           f32x4 (*s_o)[PagedTile<DT, D, FMT, RT>::NT][kWave], float* M, float* Lsum) {
  constexpr int NT = PagedTile<DT, D, FMT, RT>::NT, NW = paged_waves(RT);
  const int lane = threadIdx.x % kWave;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    s_ml[wave][rt][0][lane] = w.m[rt];
    s_ml[wave][rt][1][lane] = column_sum(w.l[rt]);
  }
  __syncthreads();
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    M[rt] = -INFINITY;
    Lsum[rt] = 0.f;
#pragma unroll
    for (int n = 0; n < NW; ++n) M[rt] = fmaxf(M[rt], s_ml[n][rt][0][lane]);
    const float b0 = M[rt] == -INFINITY ? 0.f : M[rt];
#pragma unroll
    for (int n = 0; n < NW; ++n) Lsum[rt] += s_ml[n][rt][1][lane] * fast_exp2(s_ml[n][rt][0][lane] - b0);
    const float move = fast_exp2(w.m[rt] - b0);
#pragma unroll
    for (int t = 0; t < NT; ++t) w.o[rt][t] *= move;
  }
  // half of the waves to the other half, until one has everything
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
}

template <class DT, int D, int FMT, int RT>
__global__ __launch_bounds__(paged_waves(RT) * kWave) void k_paged_attn(PagedAttnArgs a) {
  using TL = PagedTile<DT, D, FMT, RT>;
  constexpr bool C8 = TL::C8;
  constexpr int NT = TL::NT, RW = 16 * RT, NW = paged_waves(RT), THREADS = NW * kWave;
  const PagedCache& c = a.c;
  const int lane = threadIdx.x % kWave, g = lane / 16, col = lane % 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int G = 1 << a.log_g;
  __shared__ __align__(16) f32x4 s_o[NW / 2][NT][kWave];
  __shared__ float s_ml[NW][RT][2][kWave];
  __shared__ float s_join[2][RW];
  __shared__ int s_last;

  // Work of sequence b: units (layer, kv head, row group) of nb blocks each.
  struct Seq {
    int valid, len, rows, start, groups, full, tiles, skip, at, nb;  // tiles of pages: [from, from + skip) and [at, ..)
  };
  auto seq_of = [&](int len, int valid) {
    Seq s;
    s.valid = min(max(valid, 0), c.n_new);
    s.len = min(max(len, 0), kMaxRows);
    s.rows = min(s.len, c.cap());
    s.start = s.len - s.valid;
    s.groups = ((s.valid << a.log_g) + RW - 1) / RW;
    s.full = C8 ? s.rows & ~(c.page - 1) : s.rows;
    const int all = (s.full + TL::TK - 1) / TL::TK;
    s.skip = all;
    s.at = all;
    if (a.window) {
      s.skip = min((a.sinks + TL::TK - 1) / TL::TK, all);
      s.at = max(s.skip, min(max(s.start - a.window + 1, 0) / TL::TK, all));
    }
    s.tiles = s.skip + all - s.at;
    const int tail = (s.rows - s.full + TL::TK - 1) / TL::TK;
    s.nb = max(1, (s.tiles + tail + NW - 1) / NW);
    return s;
  };
  auto seq = [&](int b) { return seq_of(load_uniform(c.lens + b), c.n_valid ? load_uniform(c.n_valid + b) : c.n_new); };
  const int per_group = a.L * a.Hkv;
  auto blocks_of = [&](const Seq& s) { return (unsigned)(s.groups * per_group) * (unsigned)s.nb; };
  // all blocks (below 2^31, as the host has checked for the longest sequences), sequences to lanes
  unsigned total = 0, mine = 0;
  int my_len = 0, my_valid = 0;
  for (int b0 = 0; b0 < a.B; b0 += kWave) {
    const bool in = b0 + lane < a.B;
    my_len = in ? c.lens[b0 + lane] : 0;
    my_valid = in ? c.n_valid ? c.n_valid[b0 + lane] : c.n_new : 0;
    mine = blocks_of(seq_of(my_len, my_valid));
    total += wave_sum(mine);
  }
  total = __builtin_amdgcn_readfirstlane(total);
  if (total == 0) return;
  const unsigned per = (total + gridDim.x - 1) / gridDim.x;
  if ((unsigned long long)blockIdx.x * per >= total) return;
  const unsigned first = blockIdx.x * per, last = min(first + per, total);
  // the sequence of the first block
  int b = 0;
  unsigned base = 0;  // blocks of the sequences before b
  Seq s;
  for (int b0 = 0;; b0 += kWave) {
    if (a.B > kWave) {
      const bool in = b0 + lane < a.B;
      my_len = in ? c.lens[b0 + lane] : 0;
      my_valid = in ? c.n_valid ? c.n_valid[b0 + lane] : c.n_new : 0;
      mine = blocks_of(seq_of(my_len, my_valid));
    }
    unsigned sum = mine;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const unsigned x = __shfl_up(sum, o);
      if (lane >= o) sum += x;
    }
    const unsigned long long past = __ballot(base + sum > first);
    if (past) {
      const int at = __builtin_amdgcn_readfirstlane(__ffsll((long long)past) - 1);
      b = b0 + at;
      base += __builtin_amdgcn_readlane(sum - mine, at);
      s = seq_of(__builtin_amdgcn_readlane(my_len, at), __builtin_amdgcn_readlane(my_valid, at));
      break;
    }
    base += __builtin_amdgcn_readlane(sum, kWave - 1);
  }

  PagedWave<DT, D, FMT, RT> w;
  unsigned x = first;
  while (x < last) {
    while (x >= base + blocks_of(s)) {
      base += blocks_of(s);
      s = seq(++b);
    }
    const unsigned in = x - base;
    const int u = __builtin_amdgcn_readfirstlane(in / (unsigned)s.nb), blk = __builtin_amdgcn_readfirstlane(in - u * (unsigned)s.nb);
    const int blk_end = min(s.nb, blk + (int)(last - x));
    const int rg = u % s.groups, lh = u / s.groups, h = lh % a.Hkv, l = lh / a.Hkv;
    const unsigned unit0 = x - blk;  // the unit's first block

    // rows: token t, head hq of the group, in the order t * G + hq
    const int r0 = rg * RW, r_end = min(s.valid << a.log_g, r0 + RW);
    const int lo = s.start + (r0 >> a.log_g), hi = s.start + ((r_end - 1) >> a.log_g);
    w.clear();

    auto load_queries = [&]() {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const int r = r0 + 16 * rt + col;
        const bool ok = r < r_end;
        const int t = ok ? r >> a.log_g : 0, hq = h * G + (ok ? r - t * G : 0);
        w.pos[rt] = ok ? s.start + t : -kMaxRows;
        load_query_row<DT, D, FMT, RT>(w, rt, a.q.at(l, b, hq, t), ok);
      }
    };
    walk_pages<DT, D, FMT, RT, NW>(w, a, c, b, l, h, PageRows{s.skip, s.at, 0, 0, s.full}, blk * NW + wave, min(blk_end * NW, s.tiles), lo, hi, load_queries);
    if constexpr (C8) {
      int n = blk * NW + wave;
      if (n < s.tiles) n += (s.tiles - n + NW - 1) / NW * NW;
      walk_tail<DT, D, RT, NW>(w, a, c, b, l, h, s.full, s.rows, n - s.tiles, blk_end * NW - s.tiles, lo, hi);
    }

    float M[RT], Lsum[RT];
    join_waves<DT, D, FMT, RT>(w, wave, s_ml, s_o, M, Lsum);

    const unsigned w0 = unit0 / per, w1 = (unit0 + s.nb - 1) / per;  // workgroups that share the unit
    const bool alone = w0 == w1;
    const int n_rows = r_end - r0;
    // parts: a workgroup's run starts inside at most one unit and ends inside at most one other
    float* part = a.part + ((size_t)blockIdx.x * 2 + (x > first ? 1 : 0)) * a.part_rows * (D + 2);
    if (wave == 0) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const int r = 16 * rt + col;
        if (r >= n_rows) continue;
        const int t = (r0 + r) >> a.log_g, hq = h * G + (r0 + r) - t * G;
        const float inv = Lsum[rt] == 0.f ? 0.f : 1.f / Lsum[rt];
        char* out = a.out.at(l, b, hq, t);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float y[NT];
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            y[n] = w.o[rt][n][e];
            if (alone) y[n] = Lsum[rt] == 0.f ? 0.f : y[n] * inv;
          }
          const int ch = (4 * g + e) * NT;
          if (alone) {
#pragma unroll
            for (int n = 0; n < NT; n += 2) {
              if constexpr (TL::F)
                *(float2*)(out + (ch + n) * 4) = make_float2(y[n], y[n + 1]);
              else
                *(uint32_t*)(out + (ch + n) * 2) = pack2<DT>(y[n], y[n + 1]);
            }
          } else {
#pragma unroll
            for (int n = 0; n < NT; n += 2) st_coherent2(part + r * (D + 2) + ch + n, y[n], y[n + 1]);
          }
        }
        if (g == 0) {
          if (alone) {
            if (a.lse)
              a.lse[(((size_t)l * a.B + b) * a.Hq + hq) * a.n + t] =
                  Lsum[rt] == 0.f ? -INFINITY : (M[rt] - TL::LIFT + __log2f(Lsum[rt])) * 0.69314718055994531f;
          } else {
            st_coherent2(part + r * (D + 2) + D, M[rt], Lsum[rt]);
          }
        }
      }
    }
    if (!alone) {
      // The last workgroup to arrive joins the parts. Every part is complete before its arrival is counted, and it is
      // read with device-coherent loads.
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
      const int share = __builtin_amdgcn_readfirstlane((int)(w1 - w0) + 1);
      int* cnt = a.cnt + w0;  // (no other shared unit starts in that workgroup's run)
      if (threadIdx.x == 0) {
        const int n = __hip_atomic_fetch_add(cnt, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        s_last = n == share - 1;
        if (s_last) __hip_atomic_store(cnt, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      __syncthreads();
      if (s_last) {
        // the first sharer's part is its second one unless its run starts with the unit
        const float* part0 = a.part + ((size_t)w0 * 2 + (w0 * per < unit0 ? 1 : 0)) * a.part_rows * (D + 2);
        const float* part1 = a.part + (size_t)w0 * 2 * a.part_rows * (D + 2);
        const unsigned step = 2 * a.part_rows * (D + 2);
        auto part_of = [&](int n) { return n == 0 ? part0 : part1 + (size_t)(n * step); };
        float* s_m = (float*)&s_o[0][0][0];  // maxima of `fit` parts, all rows
        const int fit = (int)(sizeof(s_o) / sizeof(float)) / n_rows;
        // a wave to a row, a lane to a part: the row's maximum and sum
        for (int r = wave; r < n_rows; r += NW) {
          float mx = -INFINITY, sum = 0.f;
          for (int n = lane; n < share; n += kWave) {
            const float2 ml = ld_coherent2(part_of(n) + r * (D + 2) + D);
            if (n < fit) s_m[n * n_rows + r] = ml.x;
            const float top = fmaxf(mx, ml.x), b0 = top == -INFINITY ? 0.f : top;
            sum = sum * fast_exp2(mx - b0) + ml.y * fast_exp2(ml.x - b0);
            mx = top;
          }
          float top = mx;
#pragma unroll
          for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
          const float b0 = top == -INFINITY ? 0.f : top;
          sum = wave_sum(sum * fast_exp2(mx - b0));
          if (lane == 0) {
            s_join[0][r] = b0;
            s_join[1][r] = sum;
          }
        }
        // a thread to two channels of a row, the parts divided over `ways` threads where there are enough
        const int items = n_rows * (D / 2);
        constexpr int AHEAD = 8;  // parts in flight
        for (int i0 = 0; i0 < items; i0 += THREADS) {
          const int ways = i0 == 0 && 2 * items <= THREADS ? THREADS / items : 1;
          const int item = i0 + (ways > 1 ? threadIdx.x % items : threadIdx.x), way = ways > 1 ? threadIdx.x / items : 0;
          const bool mine = item < items && way < ways;
          const int r = mine ? item / (D / 2) : 0, e = item % (D / 2) * 2;
          float x0 = 0.f, x1 = 0.f;
          for (int c0 = 0; c0 < share; c0 += fit) {
            __syncthreads();
            if (c0 > 0 || i0 > 0) {
              for (int n = threadIdx.x; n < min(fit, share - c0) * n_rows; n += THREADS)
                s_m[n] = ld_coherent(part_of(c0 + n / n_rows) + n % n_rows * (D + 2) + D);
              __syncthreads();
            }
            const float b0 = s_join[0][r];
            const int c1 = mine ? min(share, c0 + fit) : 0;
            for (int n0 = c0 + way; n0 < c1; n0 += AHEAD * ways) {
              float2 y[AHEAD];
#pragma unroll
              for (int n = 0; n < AHEAD; ++n) y[n] = ld_coherent2(part_of(min(n0 + n * ways, c1 - 1)) + r * (D + 2) + e);
#pragma unroll
              for (int n = 0; n < AHEAD; ++n) {
                const int k = n0 + n * ways;
                const float f = k < c1 ? fast_exp2(s_m[(min(k, c1 - 1) - c0) * n_rows + r] - b0) : 0.f;
                x0 = k < c1 ? fmaf(y[n].x, f, x0) : x0;
                x1 = k < c1 ? fmaf(y[n].y, f, x1) : x1;
              }
            }
          }
          if (ways > 1) {
            __syncthreads();
            float2* s_x = (float2*)&s_o[0][0][0];
            s_x[threadIdx.x] = make_float2(x0, x1);
            __syncthreads();
            if (way > 0) continue;
            for (int n = 1; n < ways; ++n) {
              x0 += s_x[item + n * items].x;
              x1 += s_x[item + n * items].y;
            }
          }
          if (!mine) continue;
          const float b0 = s_join[0][r], sum = s_join[1][r];
          const int t = (r0 + r) >> a.log_g, hq = h * G + (r0 + r) - t * G;
          const float inv = sum == 0.f ? 0.f : 1.f / sum;
          char* out = a.out.at(l, b, hq, t) + e * TL::KB;
          x0 = sum == 0.f ? 0.f : x0 * inv;
          x1 = sum == 0.f ? 0.f : x1 * inv;
          if constexpr (TL::F)
            *(float2*)out = make_float2(x0, x1);
          else
            *(uint32_t*)out = pack2<DT>(x0, x1);
          if (e == 0 && a.lse)
            a.lse[(((size_t)l * a.B + b) * a.Hq + hq) * a.n + t] =
                sum == 0.f ? -INFINITY : (b0 - TL::LIFT + __log2f(sum)) * 0.69314718055994531f;
        }
      }
    }
    __syncthreads();  // the LDS buffers are free again
    x += blk_end - blk;
  }
}

template <class DT, int D, int FMT, int RT>
hipError_t launch_paged(const PagedAttnArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((k_paged_attn<DT, D, FMT, RT>), dim3((unsigned)a.grid), dim3(paged_waves(RT) * kWave), 0, st, a);
  return hipGetLastError();
}

template <class DT, int FMT>
hipError_t launch_paged_format(const PagedAttnArgs& a, int D, hipStream_t st) {
  if (a.row_tiles == 1) return D == 64 ? launch_paged<DT, 64, FMT, 1>(a, st) : launch_paged<DT, 128, FMT, 1>(a, st);
  return D == 64 ? launch_paged<DT, 64, FMT, 2>(a, st) : launch_paged<DT, 128, FMT, 2>(a, st);
}

}  // namespace dev
}  // namespace mpc
