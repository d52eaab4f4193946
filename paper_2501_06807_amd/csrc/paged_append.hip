// Append of new tokens to a paged cache with the rotation of their positions.
//
// A row's channels are handled in pairs of 16-byte vectors, so that a thread holds both partners of every channel
// pair it rotates (vectors i and i + half the rotated ones), reads and writes each once, and may write in place.
// Every product and sum of the rotation is rounded on its own (no fused multiply-add), so that the rows, and with
// them the codes of a page, do not depend on how the compiler groups them.
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

template <class DT>
__device__ __forceinline__ void turn_pair(Pair<DT>& x, const Item& it, const RopeArgs& r, int pos) {
#pragma clang fp contract(off)
  constexpr int V = DT::kVec;
  const bool ok = pos >= 0 && pos < r.n_pos;
  const float2* cs = r.table + (size_t)(ok ? pos : 0) * (r.rot / 2);
  const float bad = __uint_as_float(0x7FC00000u);
  if (r.half) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float2 t = cs[it.va * V + i];
      const float c = ok ? t.x : bad, s = ok ? t.y : bad;
      const float a = x.a[i], b = x.b[i];
      x.a[i] = a * c - b * s;
      x.b[i] = a * s + b * c;
    }
  } else {
    auto within = [&](float* y, int v) {
#pragma unroll
      for (int i = 0; i < V / 2; ++i) {
        const float2 t = cs[v * (V / 2) + i];
        const float c = ok ? t.x : bad, s = ok ? t.y : bad;
        const float a = y[2 * i], b = y[2 * i + 1];
        y[2 * i] = a * c - b * s;
        y[2 * i + 1] = a * s + b * c;
      }
    };
    within(x.a, it.va);
    within(x.b, it.vb);
  }
}

template <class DT>
__device__ __forceinline__ uint4 pack(const float* x) {
  if constexpr (DT::kVec == 4) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = DT::kCode == MPC_BF16 ? f32_to_bf16(x[2 * i]) : f32_to_f16(x[2 * i]);
      const uint32_t hi = DT::kCode == MPC_BF16 ? f32_to_bf16(x[2 * i + 1]) : f32_to_f16(x[2 * i + 1]);
      w[i] = lo | hi << 16;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// One item of one row, rotated where `r` asks for it, as the element type holds it.
template <class DT>
__device__ __forceinline__ void load_item(const char* row, const Item& it, const RopeArgs& r, int pos, uint4& a, uint4& b) {
  a = ldg16(row + it.va * 16);
  b = ldg16(row + it.vb * 16);
  if (!r.table || !it.turn) return;
  Pair<DT> x;
  unpack<DT>(a, x.a);
  unpack<DT>(b, x.b);
  turn_pair<DT>(x, it, r, pos);
  a = pack<DT>(x.a);
  b = pack<DT>(x.b);
}

// Rows to rows: the queries, and K and V into pages of the element type. Heads run q, k, v.
template <class DT, int D, bool KV>
__device__ __forceinline__ void move_rows(const PagedAppendArgs& a, int64_t block) {
  constexpr int NI = D / DT::kVec / 2;
  const PagedCache& c = a.c;
  const int heads = a.Hq + (KV ? 2 * c.Hkv : 0);
  const int64_t r0 = block * (blockDim.x / NI);
  const int64_t u0 = r0 / c.n_new;
  const unsigned t0 = (unsigned)(r0 - u0 * c.n_new) + threadIdx.x / NI;
  const int64_t u = u0 + t0 / (unsigned)c.n_new;
  const int t = (int)(t0 % (unsigned)c.n_new);
  if (u >= (int64_t)c.L * c.B * heads) return;
  const int hh = (int)((unsigned)u % (unsigned)heads), lb = (int)((unsigned)u / (unsigned)heads);
  const int b = lb % c.B, l = lb / c.B;
  const int valid = c.valid(b);
  if (t >= valid) return;
  const int j = c.len(b) - valid + t, pos = a.pos0 ? a.pos0[b] + t : j;
  const bool is_q = hh < a.Hq, is_v = hh >= a.Hq + c.Hkv;
  const int h = is_q ? hh : is_v ? hh - a.Hq - c.Hkv : hh - a.Hq;
  const char* src = is_q ? a.q.at(l, b, h, t) : is_v ? a.v.at(l, b, h, t) : a.k.at(l, b, h, t);
  char* dst;
  if (is_q) {
    dst = a.q_out.at(l, b, h, t);
  } else {
    if (j < 0) return;
    const int id = page_id(c, b, j >> c.log_page);
    if (id < 0) return;
    dst = (is_v ? c.v : c.k) + (page_unit(c, l, id, h) * c.page + (j & (c.page - 1))) * (size_t)(D * DT::kElt);
  }
  RopeArgs r = a.rope;
  if (is_v) r.table = nullptr;
  const Item it = item_of<DT>(threadIdx.x % NI, r.rot);
  uint4 x, y;
  load_item<DT>(src, it, r, pos, x, y);
  *(uint4*)(dst + it.va * 16) = x;
  *(uint4*)(dst + it.vb * 16) = y;
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
  const bool is_v = block & 1;
  const unsigned pu = block >> 1;
  const int i = pu % (unsigned)a.np, u = pu / (unsigned)a.np;
  const int h = u % c.Hkv, b = u / c.Hkv % c.B, l = u / c.Hkv / c.B;
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
  RopeArgs r = a.rope;
  if (is_v) r.table = nullptr;
  uint4 x[IPT], y[IPT];
  Item it[IPT];
  // the items of `page` that are wanted: its new rows, and the earlier ones from the ring
  auto load = [&](int page, bool earlier) {
#pragma unroll
    for (int k = 0; k < IPT; ++k) {
      const int n = threadIdx.x + k * blockDim.x, j = (page << c.log_page) + n / NI;
      it[k] = item_of<DT>(n % NI, r.rot);
      x[k] = y[k] = make_uint4(0, 0, 0, 0);
      if (j >= start && j < len) {
        load_item<DT>(in + (j - start) * step, it[k], r, pos0 + (j - start), x[k], y[k]);
      } else if (j < start && earlier) {
        const char* row = ring + (size_t)(j & (2 * c.page - 1)) * RB;
        x[k] = ldg16(row + it[k].va * 16);
        y[k] = ldg16(row + it[k].vb * 16);
      }
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
  const bool kept = i <= 1 && pg >= last - 1;
  if (!whole && !kept && !(i == 0 && last >= p0 + 2)) return;
  load(pg, whole);
  if (kept) keep(pg);
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

template <class DT, int D>
__global__ __launch_bounds__(kThreads) void k_append_rows_paged(PagedAppendArgs a) {
  move_rows<DT, D, true>(a, blockIdx.x);
}

// Pages first (they take longest), then the queries.
template <class DT, int D, int IPT>
__global__ __launch_bounds__(IPT == 1 ? 2 * kWave : kMaxPageThreads) void k_append_pages(PagedAppendArgs a, unsigned pages) {
  if (blockIdx.x < pages)
    append_page<DT, D, IPT>(a, blockIdx.x);
  else
    move_rows<DT, D, false>(a, blockIdx.x - pages);
}

template <class DT, int D>
hipError_t launch(const PagedAppendArgs& a, hipStream_t st) {
  constexpr int NI = D / DT::kVec / 2;
  const PagedCache& c = a.c;
  const int64_t lb = (int64_t)c.L * c.B;
  const bool codes = c.ks != nullptr;
  // a page's items are divided over threads four each, or one each where that would leave less than a wave
  const int items = c.page * NI, ipt = items >= 4 * kWave ? 4 : 1;
  const int threads = codes ? items / ipt : kThreads, per_block = threads / NI;
  const int64_t rows = lb * (a.Hq + (codes ? 0 : 2 * c.Hkv)) * c.n_new;
  const int64_t moves = (rows + per_block - 1) / per_block, pages = codes ? lb * c.Hkv * a.np * 2 : 0;
  if (moves + pages >= ((int64_t)1 << 31)) return hipErrorInvalidValue;
  const dim3 grid((unsigned)(moves + pages));
  if (!codes)
    hipLaunchKernelGGL((k_append_rows_paged<DT, D>), grid, dim3(threads), 0, st, a);
  else if (ipt == 4)
    hipLaunchKernelGGL((k_append_pages<DT, D, 4>), grid, dim3(threads), 0, st, a, (unsigned)pages);
  else
    hipLaunchKernelGGL((k_append_pages<DT, D, 1>), grid, dim3(threads), 0, st, a, (unsigned)pages);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_append(const PagedAppendArgs& a, int dtype, int D, hipStream_t st) {
  if (dtype == MPC_FP32) return D == 64 ? launch<F32, 64>(a, st) : launch<F32, 128>(a, st);
  if (dtype == MPC_FP16) return D == 64 ? launch<F16, 64>(a, st) : launch<F16, 128>(a, st);
  return D == 64 ? launch<BF16, 64>(a, st) : launch<BF16, 128>(a, st);
}

}  // namespace mpc
