// Append of new tokens to a paged cache with the rotation of their positions.
//
// y0 = x0 c - x1 s, y1 = x0 s + x1 c for each channel pair; then rows to rows (queries, pages of the element type) or a page's
// rows to its scale 2^e (the least with amax <= 448 2^e) and codes. A row's channels are handled in pairs of 16-byte
// vectors, so that a thread holds both partners of every channel pair it rotates (vectors i and i + half the rotated ones),
// reads and writes each once, and may write in place. Every product and sum of the rotation is rounded on its own (no
// fused multiply-add), so that the rows, and with them the codes of a page, do not depend on how the compiler groups them.
//
// Memory bounds it: 32K tokens of 2 layers (32 query heads, 8 kv heads, d 128, fp16) into 8-bit pages 310 us, 4.8 TB/s of the
// bytes it has to move; four prompts of up to 8K tokens (32 heads, bf16) into 16-bit pages 218 us, 5.2 TB/s (a plain copy of
// the queries alone: 5.4). The angles are the second stream: a row of the rotary table is as large as a row of both
// types, so a thread reads it once for four heads, and the heads of a token run side by side (each head by itself: 719 us
// of the first case). One token of one layer takes 5.6 us, a chain of memory round trips (lengths, angles, rows).
// Work items in contiguous ranges per die cost 15% of the second case, and were not kept. Pages of 4-bit codes (move_rows4):
// four prompts of up to 8K tokens (32 heads of 128, fp16), 860 MB in 197 us, 4.4 TB/s; K and V alone 103 us (4.7 TB/s), 124 with
// the rotation, whose angles come from the L2 for every fourth head. One token of one layer takes 3 us.
#include "attn_mma.h"

namespace mpc {
namespace {

using namespace dev;
constexpr int kThreads = 256, kMaxPageThreads = 1024;  // (a page of 256 rows of 128 in fp32, four items to a thread)

template <class DT>
struct Pair {
  float a[DT::kVec], b[DT::kVec];
};

// Vectors of item i of a row: rotated ones first, then those that pass.
struct Item {
  int va, vb;
  bool turn;
};
template <class DT>
__device__ __forceinline__ Item item_of(int i, int rot) {
  const int h = rot / DT::kVec / 2;
  if (i < h) return {i, i + h, true};
  return {2 * i, 2 * i + 1, false};
}

// The (cos, sin) pairs of an item at a position, as they lie in the table: of vector va's channels (HALF), or of the pairs
// within both vectors.
template <class DT>
struct Angles {
  float4 t[DT::kVec / 2];
};
template <class DT>
__device__ __forceinline__ Angles<DT> angles_of(const RopeArgs& r, const Item& it, int pos) {
  constexpr int V = DT::kVec;
  const bool ok = pos >= 0 && pos < r.n_pos;
  const float2* cs = r.table + (size_t)(ok ? pos : 0) * (r.rot / 2);
  const float2 *lo = cs + it.va * (r.half ? V : V / 2), *hi = r.half ? lo + V / 2 : cs + it.vb * (V / 2);
  Angles<DT> x;
#pragma unroll
  for (int i = 0; i < V / 4; ++i) {
    x.t[i] = *(const float4*)(lo + 2 * i);
    x.t[V / 4 + i] = *(const float4*)(hi + 2 * i);
  }
  if (!ok)
#pragma unroll
    for (int i = 0; i < V / 2; ++i) x.t[i].x = x.t[i].y = x.t[i].z = x.t[i].w = __uint_as_float(0x7FC00000u);
  return x;
}

template <class DT>
__device__ __forceinline__ void turn_pair(Pair<DT>& x, bool half, const Angles<DT>& g) {
#pragma clang fp contract(off)
  constexpr int V = DT::kVec;
  float c[V], s[V], u[V], v[V];  // pair i is (u[i], v[i])
#pragma unroll
  for (int i = 0; i < V / 2; ++i) {
    c[2 * i] = g.t[i].x;
    s[2 * i] = g.t[i].y;
    c[2 * i + 1] = g.t[i].z;
    s[2 * i + 1] = g.t[i].w;
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float a = 2 * i < V ? x.a[2 * i < V ? 2 * i : 0] : x.b[2 * i < V ? 0 : 2 * i - V];
    const float b = 2 * i < V ? x.a[2 * i < V ? 2 * i + 1 : 0] : x.b[2 * i < V ? 0 : 2 * i + 1 - V];
    u[i] = half ? x.a[i] : a;
    v[i] = half ? x.b[i] : b;
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const float a = u[i], b = v[i];
    u[i] = a * c[i] - b * s[i];
    v[i] = a * s[i] + b * c[i];
  }
#pragma unroll
  for (int i = 0; i < V; ++i) {
    x.a[i] = half ? u[i] : i % 2 ? v[i / 2] : u[i / 2];
    x.b[i] = half ? v[i] : i % 2 ? v[V / 2 + i / 2] : u[V / 2 + i / 2];
  }
}

template <class DT>
__device__ __forceinline__ uint4 pack(const float* x) {
  if constexpr (DT::kVec == 4)
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  else
    return make_uint4(pack2<DT>(x[0], x[1]), pack2<DT>(x[2], x[3]), pack2<DT>(x[4], x[5]), pack2<DT>(x[6], x[7]));
}

// Both vectors of an item, turned, as the element type holds them.
template <class DT>
__device__ __forceinline__ void turn_item(uint4& a, uint4& b, bool half, const Angles<DT>& g) {
  Pair<DT> x;
  unpack<DT>(a, x.a);
  unpack<DT>(b, x.b);
  turn_pair<DT>(x, half, g);
  a = pack<DT>(x.a);
  b = pack<DT>(x.b);
}

// Rows to rows: the queries, and (KV) K and V into pages of the element type. A workgroup takes a run of tokens of one
// sequence and a few heads (q, k, then v): a thread has one item of one token, whose angles it reads once, in up to HPT
// heads.
struct Moves {
  int tokens, lanes;  // tokens of a workgroup (a power of two), and heads side by side
  int chunks, runs;   // head chunks and token runs of a (layer, sequence)
};
template <class DT, int D, bool KV, int HPT>
__device__ __forceinline__ void move_rows(const PagedAppendArgs& a, const Moves& m, unsigned block) {
  constexpr int NI = D / DT::kVec / 2;
  const PagedCache& c = a.c;
  const int heads = a.Hq + (KV ? 2 * c.Hkv : 0);
  const int chunk = block % (unsigned)m.chunks, run = block / (unsigned)m.chunks % (unsigned)m.runs;
  const int lb = block / (unsigned)m.chunks / (unsigned)m.runs, b = lb % c.B, l = lb / c.B;
  const int tr = threadIdx.x / NI, t = run * m.tokens + (tr & (m.tokens - 1)), lane = tr / m.tokens;
  const int valid = c.n_valid ? min(max(load_uniform(c.n_valid + b), 0), c.n_new) : c.n_new;
  if (t >= valid) return;
  const int j = min(max(load_uniform(c.lens + b), 0), kMaxRows) - valid + t;
  const int pos = a.pos0 ? load_uniform(a.pos0 + b) + t : j;
  const Item it = item_of<DT>(threadIdx.x % NI, a.rope.rot);
  const bool turned = a.rope.table && it.turn;
  const int h0 = chunk * HPT * m.lanes + lane;
  uint4 x[HPT], y[HPT];
#pragma unroll
  for (int k = 0; k < HPT; ++k) {
    const int hh = h0 + k * m.lanes;
    if (hh >= heads) continue;
    const char* src = hh < a.Hq ? a.q.at(l, b, hh, t) : hh < a.Hq + c.Hkv ? a.k.at(l, b, hh - a.Hq, t) : a.v.at(l, b, hh - a.Hq - c.Hkv, t);
    x[k] = ldg16(src + it.va * 16);
    y[k] = ldg16(src + it.vb * 16);
  }
  Angles<DT> g;
  if (turned) g = angles_of<DT>(a.rope, it, pos);
  const int id = KV && j >= 0 ? page_id_lane(c, b, j >> c.log_page) : -1;
#pragma unroll
  for (int k = 0; k < HPT; ++k) {
    const int hh = h0 + k * m.lanes;
    if (hh >= heads) continue;
    if (turned && hh < a.Hq + c.Hkv) turn_item<DT>(x[k], y[k], a.rope.half, g);
    char* dst;
    if (hh < a.Hq) {
      dst = a.q_out.at(l, b, hh, t);
    } else {
      const bool is_v = hh >= a.Hq + c.Hkv;
      const int h = hh - a.Hq - (is_v ? c.Hkv : 0);
      if (a.k_out.p && !is_v && j >= 0 && j < c.cap()) {
        char* row = a.k_out.at(l, b, h, t);
        *(uint4*)(row + it.va * 16) = x[k];
        *(uint4*)(row + it.vb * 16) = y[k];
      }
      if (id < 0) continue;
      dst = (is_v ? c.v : c.k) + (page_unit(c, l, id, h) * c.page + (j & (c.page - 1))) * (size_t)(D * DT::kElt);
    }
    *(uint4*)(dst + it.va * 16) = x[k];
    *(uint4*)(dst + it.vb * 16) = y[k];
  }
}

// Largest magnitude of one item's values so far, as float bits, and whether one was not finite.
template <class DT>
__device__ __forceinline__ uint32_t item_max(uint32_t top, const uint4& x) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (DT::kElt == 4)
      top = max(top, w[i] & 0x7FFFFFFFu);
    else
      top = max_magnitude(top, w[i]);  // both halves, still in the 16-bit type
  }
  return top;
}
template <class DT>
__device__ __forceinline__ uint32_t finite_max(uint32_t top, const uint4& x) {
  float f[DT::kVec];
  unpack<DT>(x, f);
#pragma unroll
  for (int e = 0; e < DT::kVec; ++e) top = max(top, finite_bits(f[e]));
  return top;
}
// The codes of a vector in units of the page's scale; clamped where some of the thread's values were not finite.
template <class DT>
__device__ __forceinline__ void store_codes(char* p, const uint4& x, float inv, bool odd) {
  float f[DT::kVec];
  unpack<DT>(x, f);
#pragma unroll
  for (int e = 0; e < DT::kVec; ++e) f[e] = odd ? to_code_range(f[e], inv) : f[e] * inv;
  if constexpr (DT::kVec == 4)
    *(uint32_t*)p = encode4(f[0], f[1], f[2], f[3]);
  else
    *(uint2*)p = make_uint2(encode4(f[0], f[1], f[2], f[3]), encode4(f[4], f[5], f[6], f[7]));
}

// One page of K or V of one (layer, sequence, head), a thread to IPT of its items: read (and rotated) once, kept in registers
// for the page's maximum and its codes, which are written when the page is complete, and for the ring rows of the new
// tokens in the last two pages. The ring rows of later pages lie where the first page's earlier rows lay; the workgroup that
// reads these writes those, after it.
template <class DT, int D, int IPT>
__device__ __forceinline__ void append_page(const PagedAppendArgs& a, unsigned block) {
  constexpr int NI = D / DT::kVec / 2, V = DT::kVec, RB = D * DT::kElt;
  __shared__ uint32_t s_max[kMaxPageThreads / kWave];
  const PagedCache& c = a.c;
  // K and V and the heads of one page side by side: they read the same angles
  const bool is_v = block & 1;
  const unsigned ph = (block >> 1) / (unsigned)c.Hkv;
  const int h = (block >> 1) - ph * c.Hkv, i = ph % (unsigned)a.np, lb = ph / (unsigned)a.np, b = lb % c.B, l = lb / c.B;
  const int u = lb * c.Hkv + h;
  const int len = min(max(load_uniform(c.lens + b), 0), kMaxRows);
  const int valid = c.n_valid ? min(max(load_uniform(c.n_valid + b), 0), c.n_new) : c.n_new;
  const int start = len - valid;
  if (valid == 0 || len == 0) return;
  const int p0 = max(start, 0) >> c.log_page, last = (len - 1) >> c.log_page, pg = p0 + i;
  if (pg > last || pg >= c.max_pages) return;
  const int entry = page_entry(c, b, pg);
  const int pos0 = a.pos0 ? load_uniform(a.pos0 + b) : start;
  const char* in = (is_v ? a.v : a.k).at(l, b, h, 0);
  const int64_t step = (is_v ? a.v : a.k).token;
  char* ring = (is_v ? c.v_tail : c.k_tail) + (size_t)u * (2 * c.page) * RB;
  const bool turned = a.rope.table && !is_v;
  uint4 x[IPT], y[IPT];
  Item it[IPT];
  // the items of `page` that are wanted: its new rows, and the earlier ones from the ring
  auto load = [&](int page, bool earlier) {
#pragma unroll
    for (int k = 0; k < IPT; ++k) {
      const int n = threadIdx.x + k * blockDim.x, j = (page << c.log_page) + n / NI;
      it[k] = item_of<DT>(n % NI, a.rope.rot);
      x[k] = y[k] = make_uint4(0, 0, 0, 0);
      const bool fresh = j >= start;
      if (fresh ? j < len : earlier) {
        const char* row = fresh ? in + (j - start) * step : ring + (size_t)(j & (2 * c.page - 1)) * RB;
        x[k] = ldg16(row + it[k].va * 16);
        y[k] = ldg16(row + it[k].vb * 16);
      }
    }
    if (turned)
#pragma unroll
      for (int k = 0; k < IPT; ++k) {
        const int j = (page << c.log_page) + (threadIdx.x + k * blockDim.x) / NI;
        if (it[k].turn && j >= start && j < len)
          turn_item<DT>(x[k], y[k], a.rope.half, angles_of<DT>(a.rope, it[k], pos0 + (j - start)));
      }
  };
  auto keep = [&](int page) {
#pragma unroll
    for (int k = 0; k < IPT; ++k) {
      const int j = (page << c.log_page) + (threadIdx.x + k * blockDim.x) / NI;
      if (j < start || j >= len) continue;
      char* row = ring + (size_t)(j & (2 * c.page - 1)) * RB;
      *(uint4*)(row + it[k].va * 16) = x[k];
      *(uint4*)(row + it[k].vb * 16) = y[k];
    }
  };
  const int id = page_of_entry(c, entry, pg);
  const bool whole = ((pg + 1) << c.log_page) <= len && id >= 0;
  const bool kept = i <= 1 && pg >= last - 1, plain = a.k_out.p && !is_v;
  if (!whole && !kept && !plain && !(i == 0 && last >= p0 + 2)) return;
  load(pg, whole);
  if (kept) keep(pg);
  if (plain) {
#pragma unroll
    for (int k = 0; k < IPT; ++k) {
      const int j = (pg << c.log_page) + (threadIdx.x + k * blockDim.x) / NI;
      if (j < start || j >= len) continue;
      char* row = a.k_out.at(l, b, h, j - start);
      *(uint4*)(row + it[k].va * 16) = x[k];
      *(uint4*)(row + it[k].vb * 16) = y[k];
    }
  }
  if (whole) {
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < IPT; ++k) top = item_max<DT>(item_max<DT>(top, x[k]), y[k]);
    const bool odd = not_finite<DT>(top);
    if (odd) {
      top = 0;
#pragma unroll
      for (int k = 0; k < IPT; ++k) top = finite_max<DT>(finite_max<DT>(top, x[k]), y[k]);
    } else if constexpr (DT::kElt == 2) {
      const uint32_t m = max(top & 0xFFFFu, top >> 16);
      top = __float_as_uint(DT::kCode == MPC_BF16 ? bf16_to_f32(m) : f16_to_f32(m));
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    if (blockDim.x > kWave) {
      if (threadIdx.x % kWave == 0) s_max[threadIdx.x / kWave] = top;
      __syncthreads();
      for (int w = 0; w < (int)blockDim.x / kWave; ++w) top = max(top, s_max[w]);
    }
    const int e2 = scale_exponent(top);
    const float inv = pow2(-e2);
    const size_t unit = page_unit(c, l, id, h);
    char* dst = (is_v ? c.v : c.k) + unit * c.page * (size_t)D;
    if (threadIdx.x == 0) (is_v ? c.vs : c.ks)[unit] = pow2(e2);
#pragma unroll
    for (int k = 0; k < IPT; ++k) {
      char* row = dst + (size_t)((threadIdx.x + k * blockDim.x) / NI) * D;
      store_codes<DT>(row + it[k].va * V, x[k], inv, odd);
      store_codes<DT>(row + it[k].vb * V, y[k], inv, odd);
    }
  }
  if (i == 0 && last >= p0 + 2) {
    __syncthreads();  // the earlier rows have been read
    for (int page = max(p0 + 2, last - 1); page <= last && page < c.max_pages; ++page) {
      load(page, false);
      keep(page);
    }
  }
}

// Largest finite magnitude of a vector's values as float bits, or kNanMark where one is a NaN.
constexpr uint32_t kNanMark = 0x7FFFFFFFu;
template <class DT>
__device__ __forceinline__ uint32_t block_max(const uint4& x) {
  const uint32_t top = item_max<DT>(0u, x);
  if (not_finite<DT>(top)) {
    float f[DT::kVec];
    unpack<DT>(x, f);
    bool nan = false;
#pragma unroll
    for (int e = 0; e < DT::kVec; ++e) nan |= f[e] != f[e];
    return nan ? kNanMark : finite_max<DT>(0u, x);
  }
  if constexpr (DT::kElt == 4) return top;
  const uint32_t m = max(top & 0xFFFFu, top >> 16);
  return __float_as_uint(DT::kCode == MPC_BF16 ? bf16_to_f32(m) : f16_to_f32(m));
}

// Rows of K or V into pages of 4-bit codes: a row's blocks of 32 channels have a scale each, so a row is final as it is
// written. Work is laid out as in move_rows, K and V apart; a row's lanes (of one wave) exchange the maxima of their vectors
// through LDS, since the partners of a rotated pair may lie in different blocks.
template <class DT, int D, int HPT>
__device__ __forceinline__ void move_rows4(const PagedAppendArgs& a, const Moves& m, unsigned block) {
  constexpr int NI = D / DT::kVec / 2, V = DT::kVec, NB = kMx4Block / V;  // vectors of a block
  __shared__ __align__(16) uint32_t s_max[kThreads / NI][2 * NI];
  const PagedCache& c = a.c;
  const int chunk = block % (unsigned)m.chunks, rest = block / (unsigned)m.chunks;
  const bool is_v = rest & 1;
  const int run = (unsigned)rest / 2 % (unsigned)m.runs, lb = (unsigned)rest / 2 / (unsigned)m.runs, b = lb % c.B, l = lb / c.B;
  const int tr = threadIdx.x / NI, t = run * m.tokens + (tr & (m.tokens - 1)), lane = tr / m.tokens;
  const int valid = c.n_valid ? min(max(load_uniform(c.n_valid + b), 0), c.n_new) : c.n_new;
  const int h0 = chunk * HPT * m.lanes + lane;
  if (t >= valid || h0 >= c.Hkv) return;
  const int j = min(max(load_uniform(c.lens + b), 0), kMaxRows) - valid + t;
  const int pos = a.pos0 ? load_uniform(a.pos0 + b) + t : j;
  const Item it = item_of<DT>(threadIdx.x % NI, a.rope.rot);
  const bool turned = a.rope.table && it.turn && !is_v;
  const Rows& in = is_v ? a.v : a.k;
  const char* src = in.at(l, b, h0, t);
  const int64_t src_step = m.lanes * in.head;
  uint4 x[HPT], y[HPT];
#pragma unroll
  for (int k = 0; k < HPT; ++k) {
    if (h0 + k * m.lanes >= c.Hkv) continue;
    x[k] = ldg16(src + k * src_step + it.va * 16);
    y[k] = ldg16(src + k * src_step + it.vb * 16);
  }
  Angles<DT> g;
  if (turned) g = angles_of<DT>(a.rope, it, pos);
  const int id = j >= 0 ? page_id_lane(c, b, j >> c.log_page) : -1;
  const bool plain = a.k_out.p && !is_v && j >= 0 && j < c.cap();
  const size_t unit = page_unit(c, l, max(id, 0), h0);
  const int slot = j & (c.page - 1);
  char* row = (is_v ? c.v : c.k) + (unit * c.page + slot) * (size_t)(D / 2);
  uint8_t* scale = (is_v ? c.vx : c.kx) + unit * (size_t)(D / kMx4Block * c.page) + slot;
#pragma unroll
  for (int k = 0; k < HPT; ++k) {
    if (h0 + k * m.lanes >= c.Hkv) continue;
    if (turned) turn_item<DT>(x[k], y[k], a.rope.half, g);
    if (plain) {
      char* o = a.k_out.at(l, b, h0 + k * m.lanes, t);
      *(uint4*)(o + it.va * 16) = x[k];
      *(uint4*)(o + it.vb * 16) = y[k];
    }
    if (id < 0) continue;
    s_max[tr][it.va] = block_max<DT>(x[k]);
    s_max[tr][it.vb] = block_max<DT>(y[k]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    char* to = row + (size_t)(k * m.lanes) * c.page * (D / 2);
    uint8_t* to_scale = scale + (size_t)(k * m.lanes) * (D / kMx4Block * c.page);
    auto put = [&](const uint4& z, int v) {
      uint32_t top = 0;
#pragma unroll
      for (int n = 0; n < NB; n += 4) {
        const uint4 w = *(const uint4*)&s_max[tr][v / NB * NB + n];
        top = max(top, max(max(w.x, w.y), max(w.z, w.w)));
      }
      const bool nan = top == kNanMark;
      const int e = nan ? 0 : mx4_exponent(top);
      const float inv = pow2(-e);
      float f[8] = {};
      unpack<DT>(z, f);
#pragma unroll
      for (int n = 0; n < V; ++n) f[n] *= inv;
      const uint32_t w = encode8(f);
      if constexpr (V == 8)
        *(uint32_t*)(to + v * 4) = w;
      else
        *(uint16_t*)(to + v * 2) = (uint16_t)w;
      if (v % NB == 0) to_scale[v / NB * c.page] = nan ? 255 : (uint8_t)(e + 127);
    };
    put(x[k], it.va);
    put(y[k], it.vb);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");  // the maxima have been read
    __builtin_amdgcn_wave_barrier();
  }
}

template <class DT, int D, int HPT>
__global__ __launch_bounds__(kThreads) void k_append_mx4(PagedAppendArgs a, Moves m4, Moves m, unsigned rows) {
  if (blockIdx.x < rows)
    move_rows4<DT, D, HPT>(a, m4, blockIdx.x);
  else
    move_rows<DT, D, false, HPT>(a, m, blockIdx.x - rows);
}

template <class DT, int D, int HPT>
__global__ __launch_bounds__(kThreads) void k_append_rows_paged(PagedAppendArgs a, Moves m) {
  move_rows<DT, D, true, HPT>(a, m, blockIdx.x);
}

// Pages first (they take longest), then the queries.
template <class DT, int D, int IPT, int HPT>
__global__ __launch_bounds__(IPT == 1 ? 2 * kWave : kMaxPageThreads) void k_append_pages(PagedAppendArgs a, Moves m, unsigned pages) {
  if (blockIdx.x < pages)
    append_page<DT, D, IPT>(a, blockIdx.x);
  else
    move_rows<DT, D, false, HPT>(a, m, blockIdx.x - pages);
}

// How the rows of `heads` heads are divided over workgroups of `slots` rows, hpt heads to a thread.
Moves moves_of(const PagedCache& c, int heads, int slots, int hpt) {
  Moves m{};
  m.tokens = 1;
  while (m.tokens < slots && m.tokens < c.n_new) m.tokens *= 2;
  m.lanes = slots / m.tokens;
  m.runs = (int)(((int64_t)c.n_new + m.tokens - 1) / m.tokens);
  m.chunks = (heads + hpt * m.lanes - 1) / (hpt * m.lanes);
  return m;
}

// Pages of 4-bit codes: rows of K and V first, then the queries.
template <class DT, int D>
hipError_t launch_mx4(const PagedAppendArgs& a, hipStream_t st) {
  constexpr int slots = kThreads / (D / DT::kVec / 2);
  const int64_t lb = (int64_t)a.c.L * a.c.B;
  auto blocks = [&](const Moves& m) { return lb * m.runs * m.chunks; };
  // four heads to a thread, where that leaves a few workgroups to a compute unit
  const int hpt = 2 * blocks(moves_of(a.c, a.c.Hkv, slots, 4)) >= 4 * kNumCU ? 4 : 1;
  const Moves m4 = moves_of(a.c, a.c.Hkv, slots, hpt), m = moves_of(a.c, a.Hq, slots, hpt);
  const int64_t rows = 2 * blocks(m4), all = rows + (a.Hq ? blocks(m) : 0);
  if (all >= ((int64_t)1 << 31)) return hipErrorInvalidValue;
  if (hpt == 4)
    hipLaunchKernelGGL((k_append_mx4<DT, D, 4>), dim3((unsigned)all), dim3(kThreads), 0, st, a, m4, m, (unsigned)rows);
  else
    hipLaunchKernelGGL((k_append_mx4<DT, D, 1>), dim3((unsigned)all), dim3(kThreads), 0, st, a, m4, m, (unsigned)rows);
  return hipGetLastError();
}

template <class DT, int D>
hipError_t launch(const PagedAppendArgs& a, hipStream_t st) {
  if (a.c.format == MPC_PAGE_MX4) return launch_mx4<DT, D>(a, st);
  constexpr int NI = D / DT::kVec / 2;
  const PagedCache& c = a.c;
  const int64_t lb = (int64_t)c.L * c.B;
  const bool codes = c.ks != nullptr;
  // a page's items are divided over threads four each, or one each where that would leave less than a wave
  const int items = c.page * NI, ipt = items >= 4 * kWave ? 4 : 1;
  const int threads = codes ? items / ipt : kThreads, slots = threads / NI, heads = a.Hq + (codes ? 0 : 2 * c.Hkv);
  Moves m{};
  m.tokens = 1;
  while (m.tokens < slots && m.tokens < c.n_new) m.tokens *= 2;
  m.lanes = slots / m.tokens;
  m.runs = (int)(((int64_t)c.n_new + m.tokens - 1) / m.tokens);
  // four heads to a thread, where that leaves a few workgroups to a compute unit
  const int64_t some = lb * m.runs * ((heads + 4 * m.lanes - 1) / (4 * m.lanes));
  const int hpt = some >= 4 * kNumCU ? 4 : 1;
  m.chunks = (heads + hpt * m.lanes - 1) / (hpt * m.lanes);
  const int64_t moves = lb * m.runs * m.chunks, pages = codes ? lb * c.Hkv * a.np * 2 : 0;
  if (moves + pages >= ((int64_t)1 << 31)) return hipErrorInvalidValue;
  const dim3 grid((unsigned)(moves + pages));
  const unsigned p = (unsigned)pages;
  if (!codes && hpt == 4)
    hipLaunchKernelGGL((k_append_rows_paged<DT, D, 4>), grid, dim3(threads), 0, st, a, m);
  else if (!codes)
    hipLaunchKernelGGL((k_append_rows_paged<DT, D, 1>), grid, dim3(threads), 0, st, a, m);
  else if (ipt == 4 && hpt == 4)
    hipLaunchKernelGGL((k_append_pages<DT, D, 4, 4>), grid, dim3(threads), 0, st, a, m, p);
  else if (ipt == 4)
    hipLaunchKernelGGL((k_append_pages<DT, D, 4, 1>), grid, dim3(threads), 0, st, a, m, p);
  else if (hpt == 4)
    hipLaunchKernelGGL((k_append_pages<DT, D, 1, 4>), grid, dim3(threads), 0, st, a, m, p);
  else
    hipLaunchKernelGGL((k_append_pages<DT, D, 1, 1>), grid, dim3(threads), 0, st, a, m, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_append(const PagedAppendArgs& a, int dtype, int D, hipStream_t st) {
  if (dtype == MPC_FP32) return D == 64 ? launch<F32, 64>(a, st) : launch<F32, 128>(a, st);
  if (dtype == MPC_FP16) return D == 64 ? launch<F16, 64>(a, st) : launch<F16, 128>(a, st);
  return D == 64 ? launch<BF16, 64>(a, st) : launch<BF16, 128>(a, st);
}

}  // namespace mpc
