// Rows of a paged cache, of any page format, as rows of the element type.
//
// A row's value is its code times its scale, rounded once to the element type (bf16 and fp32 hold it exactly). A thread has one
// 16-byte vector of a row, in up to HPT heads of K or V, so that a token's page id is looked up once for them.
//
// Memory bounds it: 32K rows of 4-bit codes, two layers of 8 heads of 128 in bf16, 340 MB in 79 us (4.3 TB/s; a large copy: 5.4), four
// prompts' rows of 32 heads in fp16 480 MB in 100 us (4.8). Four tokens to a thread instead of one 92 to 87 us, pointers that step
// from head to head instead of 64-bit products for each 87 to 77. The newest 500 rows of four sequences of 8-bit pages: 7.4 us.
#include "attn_mma.h"

namespace mpc {
namespace {

using namespace dev;
constexpr int kThreads = 256;

struct Reads {
  int tokens, lanes;        // tokens of a workgroup (a power of two), and heads side by side
  int chunks, sides, runs;  // head chunks, K and V, and token runs of a (layer, sequence)
};

template <class DT>
__device__ __forceinline__ uint4 pack(const float* x) {
  if constexpr (DT::kVec == 4)
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  else
    return make_uint4(pack2<DT>(x[0], x[1]), pack2<DT>(x[2], x[3]), pack2<DT>(x[4], x[5]), pack2<DT>(x[6], x[7]));
}

// A vector as it lies in a page, with its scale.
template <class DT, int FMT>
struct Piece {
  static constexpr int V = DT::kVec;
  uint4 w;
  float scale;
  __device__ void load(const char* p) {
    if constexpr (FMT == MPC_PAGE_SAME)
      w = ldg16(p);
    else if constexpr (FMT == MPC_PAGE_E4M3 && V == 8) {
      const uint2 x = *(const uint2*)p;
      w.x = x.x;
      w.y = x.y;
    } else if constexpr (FMT == MPC_PAGE_MX4 && V == 4)
      w.x = *(const uint16_t*)p;
    else
      w.x = *(const uint32_t*)p;
  }
  __device__ uint4 rows() const {
    if constexpr (FMT == MPC_PAGE_SAME) return w;
    float f[8];
    if constexpr (FMT == MPC_PAGE_MX4) {
      if constexpr (DT::kCode == MPC_BF16) return widen8(w.x, scale);
      decode8(w.x, scale, f);
    } else {
      decode4(w.x, f);
      if constexpr (V == 8) decode4(w.y, f + 4);
#pragma unroll
      for (int i = 0; i < V; ++i) f[i] *= scale;
    }
    return pack<DT>(f);
  }
};

// TPT tokens (a run apart) and HPT heads to a thread, all of their loads on the way at once.
template <class DT, int D, int FMT, int HPT, int TPT>
__global__ __launch_bounds__(kThreads) void k_read(PagedReadArgs a, Reads m) {
  constexpr int V = DT::kVec, NV = D / V;
  constexpr int BITS = FMT == MPC_PAGE_MX4 ? 4 : FMT == MPC_PAGE_E4M3 ? 8 : 8 * DT::kElt, RB = D * BITS / 8;
  const PagedCache& c = a.c;
  // a workgroup has heads of K or of V, then a run of tokens
  const int chunk = blockIdx.x % (unsigned)m.chunks, side = blockIdx.x / (unsigned)m.chunks % (unsigned)m.sides;
  const unsigned rest = blockIdx.x / (unsigned)m.chunks / (unsigned)m.sides;
  const int run = rest % (unsigned)m.runs, lb = rest / (unsigned)m.runs, b = lb % c.B, l = lb / c.B;
  const bool is_v = side == 1 || !a.k.p;
  const Rows& out = is_v ? a.v : a.k;
  const int tr = threadIdx.x / NV, v = threadIdx.x % NV, lane = tr / m.tokens, h0 = chunk * HPT * m.lanes + lane;
  if (h0 >= c.Hkv) return;
  const int valid = c.n_valid ? min(max(load_uniform(c.n_valid + b), 0), c.n_new) : c.n_new;
  const int len = min(max(load_uniform(c.lens + b), 0), kMaxRows), rows = min(len, c.cap());
  const int full = FMT == MPC_PAGE_E4M3 ? rows & ~(c.page - 1) : rows;
  const long long from = a.first ? (long long)load_uniform(a.first + b) : (long long)(len - valid);
  const int t0 = run * TPT * m.tokens + (tr & (m.tokens - 1));
  int j[TPT], id[TPT];  // rows of the cache, and their pages (-1: no such row)
#pragma unroll
  for (int q = 0; q < TPT; ++q) {
    const int t = t0 + q * m.tokens;
    const long long at = from + t;
    const bool ok = t < valid && at >= 0 && at < rows;
    j[q] = ok ? (int)at : 0;
    id[q] = page_id_lane(c, b, j[q] >> c.log_page);
    if (j[q] >= full) id[q] = 0;  // (a row of the ring needs no page)
    if (!ok) id[q] = -1;
  }
  // from one of the thread's heads to the next: pieces and scales of a page, rows
  const size_t step = (size_t)m.lanes * c.page * RB, scale_step = (size_t)m.lanes * (FMT == MPC_PAGE_MX4 ? D / kMx4Block * c.page : 1);
  const int64_t out_step = m.lanes * out.head;
  Piece<DT, FMT> x[TPT][HPT];
#pragma unroll
  for (int q = 0; q < TPT; ++q) {
    if (id[q] < 0) continue;
    if (FMT == MPC_PAGE_E4M3 && j[q] >= full) {
      const char* p = (is_v ? c.v_tail : c.k_tail) + (((size_t)lb * c.Hkv + h0) * (2 * c.page) + (j[q] & (2 * c.page - 1))) * (size_t)(D * DT::kElt) + v * 16;
      char* o = out.at(l, b, h0, t0 + q * m.tokens) + v * 16;
      for (int k = 0; k < HPT && h0 + k * m.lanes < c.Hkv; ++k) {
        *(uint4*)o = ldg16(p);
        p += (size_t)m.lanes * (2 * c.page) * (D * DT::kElt);
        o += out_step;
      }
      continue;
    }
    const size_t unit = page_unit(c, l, id[q], h0);
    const int slot = j[q] & (c.page - 1);
    const char* p = (is_v ? c.v : c.k) + (unit * c.page + slot) * RB + v * (V * BITS / 8);
    const uint8_t* px = FMT == MPC_PAGE_MX4 ? (is_v ? c.vx : c.kx) + unit * (size_t)(D / kMx4Block * c.page) + v * V / kMx4Block * c.page + slot : nullptr;
    const float* ps = FMT == MPC_PAGE_E4M3 ? (is_v ? c.vs : c.ks) + unit : nullptr;
#pragma unroll
    for (int k = 0; k < HPT; ++k) {
      if (h0 + k * m.lanes >= c.Hkv) continue;
      x[q][k].load(p + k * step);
      if constexpr (FMT == MPC_PAGE_E4M3) x[q][k].scale = ps[k * scale_step];
      if constexpr (FMT == MPC_PAGE_MX4) x[q][k].scale = mx4_scale(px[k * scale_step]);
    }
  }
#pragma unroll
  for (int q = 0; q < TPT; ++q) {
    if (id[q] < 0 || (FMT == MPC_PAGE_E4M3 && j[q] >= full)) continue;
    char* o = out.at(l, b, h0, t0 + q * m.tokens) + v * 16;
#pragma unroll
    for (int k = 0; k < HPT; ++k)
      if (h0 + k * m.lanes < c.Hkv) *(uint4*)(o + k * out_step) = x[q][k].rows();
  }
}

template <class DT, int D, int FMT>
hipError_t launch(const PagedReadArgs& a, hipStream_t st) {
  constexpr int slots = kThreads / (D / DT::kVec);
  const PagedCache& c = a.c;
  Reads m{};
  m.sides = (a.k.p ? 1 : 0) + (a.v.p ? 1 : 0);
  m.tokens = 1;
  while (m.tokens < slots && m.tokens < c.n_new) m.tokens *= 2;
  m.lanes = slots / m.tokens;
  auto blocks = [&](int hpt, int tpt) {
    m.runs = (int)(((int64_t)c.n_new + m.tokens * tpt - 1) / (m.tokens * tpt));
    m.chunks = (c.Hkv + hpt * m.lanes - 1) / (hpt * m.lanes);
    return (int64_t)c.L * c.B * m.runs * m.sides * m.chunks;
  };
  // four heads and four tokens to a thread, where that leaves a few workgroups to a compute unit
  const bool many = blocks(4, 4) >= 4 * kNumCU;
  const int64_t n = many ? blocks(4, 4) : blocks(1, 1);
  if (n >= ((int64_t)1 << 31)) return hipErrorInvalidValue;
  if (many)
    hipLaunchKernelGGL((k_read<DT, D, FMT, 4, 4>), dim3((unsigned)n), dim3(kThreads), 0, st, a, m);
  else
    hipLaunchKernelGGL((k_read<DT, D, FMT, 1, 1>), dim3((unsigned)n), dim3(kThreads), 0, st, a, m);
  return hipGetLastError();
}

template <class DT>
hipError_t launch_type(const PagedReadArgs& a, int D, hipStream_t st) {
  if (a.c.format == MPC_PAGE_MX4) return D == 64 ? launch<DT, 64, MPC_PAGE_MX4>(a, st) : launch<DT, 128, MPC_PAGE_MX4>(a, st);
  if (a.c.format == MPC_PAGE_E4M3) return D == 64 ? launch<DT, 64, MPC_PAGE_E4M3>(a, st) : launch<DT, 128, MPC_PAGE_E4M3>(a, st);
  return D == 64 ? launch<DT, 64, MPC_PAGE_SAME>(a, st) : launch<DT, 128, MPC_PAGE_SAME>(a, st);
}

}  // namespace

hipError_t launch_paged_read(const PagedReadArgs& a, int dtype, int D, hipStream_t st) {
  if (dtype == MPC_FP32) return launch_type<F32>(a, D, st);
  return dtype == MPC_FP16 ? launch_type<F16>(a, D, st) : launch_type<BF16>(a, D, st);
}

}  // namespace mpc
