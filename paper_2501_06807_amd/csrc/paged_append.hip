// Append of new tokens to a paged cache with the rotation of their positions.
//
// A row's channels are handled in pairs of 16-byte vectors, so that a thread holds both partners of every channel
// pair it rotates (vectors i and i + half the rotated ones), reads and writes each once, and may write in place.
// Every product and sum of the rotation is rounded on its own (no fused multiply-add), so that the rows, and with
// them the codes of a page, do not depend on how the compiler groups them.
#include "paged_dev.h"

namespace mpc {
namespace {

using namespace dev;
constexpr int kThreads = 256;

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
  constexpr int NI = D / DT::kVec / 2, ROWS = kThreads / NI;
  const PagedCache& c = a.c;
  const int heads = a.Hq + (KV ? 2 * c.Hkv : 0);
  const int64_t r0 = block * ROWS;
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

// One page of K or V of one (layer, sequence, head): codes once it is complete, and the ring rows of the new tokens in
// the last two pages. The ring rows of later pages lie where the first page's earlier rows lay; the workgroup that reads
// these writes those, after it.
template <class DT, int D>
__device__ __forceinline__ void append_page(const PagedAppendArgs& a, int64_t block) {
  constexpr int NI = D / DT::kVec / 2, V = DT::kVec, RB = D * DT::kElt;
  __shared__ uint32_t s_max[kThreads / kWave];
  const PagedCache& c = a.c;
  const bool is_v = block & 1;
  const int i = (int)((block >> 1) % a.np);
  const int u = (int)((block >> 1) / a.np);
  const int h = u % c.Hkv, b = u / c.Hkv % c.B, l = u / c.Hkv / c.B;
  const int valid = c.valid(b), len = c.len(b), start = len - valid;
  if (valid == 0 || len == 0) return;
  const int p0 = max(start, 0) >> c.log_page, last = (len - 1) >> c.log_page, pg = p0 + i;
  if (pg > last || pg >= c.max_pages) return;
  const Rows& in = is_v ? a.v : a.k;
  char* ring = (is_v ? c.v_tail : c.k_tail) + (size_t)u * (2 * c.page) * RB;
  const int items = c.page * NI;
  RopeArgs r = a.rope;
  if (is_v) r.table = nullptr;
  auto load = [&](int n, int page, uint4& x, uint4& y) -> Item {
    const int j = (page << c.log_page) + n / NI;
    const Item it = item_of<DT>(n % NI, r.rot);
    if (j >= start) {
      const int t = j - start;
      load_item<DT>(in.at(l, b, h, t), it, r, a.pos0 ? a.pos0[b] + t : j, x, y);
    } else {
      const char* row = ring + (size_t)(j & (2 * c.page - 1)) * RB;
      x = ldg16(row + it.va * 16);
      y = ldg16(row + it.vb * 16);
    }
    return it;
  };
  const int id = page_id(c, b, pg);
  if (((pg + 1) << c.log_page) <= len && id >= 0) {
    uint32_t top = 0;
    for (int n = threadIdx.x; n < items; n += kThreads) {
      uint4 x, y;
      load(n, pg, x, y);
      float f[V], g[V];
      unpack<DT>(x, f);
      unpack<DT>(y, g);
#pragma unroll
      for (int e = 0; e < V; ++e) top = max(top, max(finite_bits(f[e]), finite_bits(g[e])));
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    if (threadIdx.x % kWave == 0) s_max[threadIdx.x / kWave] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kThreads / kWave; ++w) top = max(top, s_max[w]);
    const int e2 = scale_exponent(top);
    const float inv = pow2(-e2);
    const size_t unit = page_unit(c, l, id, h);
    char* dst = (is_v ? c.v : c.k) + unit * c.page * (size_t)D;
    if (threadIdx.x == 0) (is_v ? c.vs : c.ks)[unit] = pow2(e2);
    for (int n = threadIdx.x; n < items; n += kThreads) {
      uint4 x, y;
      const Item it = load(n, pg, x, y);
      float f[V], g[V];
      unpack<DT>(x, f);
      unpack<DT>(y, g);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        f[e] = to_code_range(f[e], inv);
        g[e] = to_code_range(g[e], inv);
      }
      char* row = dst + (size_t)(n / NI) * D;
#pragma unroll
      for (int e = 0; e < V; e += 4) {
        *(uint32_t*)(row + it.va * V + e) = encode4(f[e], f[e + 1], f[e + 2], f[e + 3]);
        *(uint32_t*)(row + it.vb * V + e) = encode4(g[e], g[e + 1], g[e + 2], g[e + 3]);
      }
    }
  }
  auto keep = [&](int page) {
    for (int n = threadIdx.x; n < items; n += kThreads) {
      const int j = (page << c.log_page) + n / NI;
      if (j < start || j >= len) continue;
      uint4 x, y;
      const Item it = load(n, page, x, y);
      char* row = ring + (size_t)(j & (2 * c.page - 1)) * RB;
      *(uint4*)(row + it.va * 16) = x;
      *(uint4*)(row + it.vb * 16) = y;
    }
  };
  if (i <= 1 && pg >= last - 1) keep(pg);
  if (i == 0 && last >= p0 + 2) {
    __syncthreads();
    for (int page = max(p0 + 2, last - 1); page <= last && page < c.max_pages; ++page) keep(page);
  }
}

template <class DT, int D>
__global__ __launch_bounds__(kThreads) void k_append_rows_paged(PagedAppendArgs a) {
  move_rows<DT, D, true>(a, blockIdx.x);
}

template <class DT, int D>
__global__ __launch_bounds__(kThreads) void k_append_pages(PagedAppendArgs a, unsigned pages) {
  if (blockIdx.x < pages)
    append_page<DT, D>(a, blockIdx.x);
  else
    move_rows<DT, D, false>(a, blockIdx.x - pages);
}

template <class DT, int D>
hipError_t launch(const PagedAppendArgs& a, hipStream_t st) {
  constexpr int ROWS = kThreads / (D / DT::kVec / 2);
  const PagedCache& c = a.c;
  const int64_t lb = (int64_t)c.L * c.B;
  const bool codes = c.ks != nullptr;
  const int64_t rows = lb * (a.Hq + (codes ? 0 : 2 * c.Hkv)) * c.n_new;
  const int64_t moves = (rows + ROWS - 1) / ROWS, pages = codes ? lb * c.Hkv * a.np * 2 : 0;
  if (moves + pages >= ((int64_t)1 << 31)) return hipErrorInvalidValue;
  if (codes)
    hipLaunchKernelGGL((k_append_pages<DT, D>), dim3((unsigned)(moves + pages)), dim3(kThreads), 0, st, a, (unsigned)pages);
  else
    hipLaunchKernelGGL((k_append_rows_paged<DT, D>), dim3((unsigned)moves), dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_append(const PagedAppendArgs& a, int dtype, int D, hipStream_t st) {
  if (dtype == MPC_FP32) return D == 64 ? launch<F32, 64>(a, st) : launch<F32, 128>(a, st);
  if (dtype == MPC_FP16) return D == 64 ? launch<F16, 64>(a, st) : launch<F16, 128>(a, st);
  return D == 64 ? launch<BF16, 64>(a, st) : launch<BF16, 128>(a, st);
}

}  // namespace mpc
