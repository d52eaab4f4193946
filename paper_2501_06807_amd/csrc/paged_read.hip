// Rows of a paged cache, of any page format, as rows of the element type.
//
// A row's value is its code times its scale, rounded once to the element type (bf16 and fp32 hold it exactly). A thread has one
// 16-byte vector of one token's row, in up to HPT heads of K and V, so that a token's page id is looked up once for them.
#include "attn_mma.h"

namespace mpc {
namespace {

using namespace dev;
constexpr int kThreads = 256;

struct Reads {
  int tokens, lanes;  // tokens of a workgroup (a power of two), and heads side by side
  int chunks, runs;   // head chunks and token runs of a (layer, sequence)
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

template <class DT, int D, int FMT, int HPT>
__global__ __launch_bounds__(kThreads) void k_read(PagedReadArgs a, Reads m) {
  constexpr int V = DT::kVec, NV = D / V;
  constexpr int BITS = FMT == MPC_PAGE_MX4 ? 4 : FMT == MPC_PAGE_E4M3 ? 8 : 8 * DT::kElt, RB = D * BITS / 8;
  const PagedCache& c = a.c;
  const int nk = a.k.p ? c.Hkv : 0, heads = nk + (a.v.p ? c.Hkv : 0);
  const int chunk = blockIdx.x % (unsigned)m.chunks, run = blockIdx.x / (unsigned)m.chunks % (unsigned)m.runs;
  const int lb = blockIdx.x / (unsigned)m.chunks / (unsigned)m.runs, b = lb % c.B, l = lb / c.B;
  const int tr = threadIdx.x / NV, v = threadIdx.x % NV, t = run * m.tokens + (tr & (m.tokens - 1)), lane = tr / m.tokens;
  const int valid = c.n_valid ? min(max(load_uniform(c.n_valid + b), 0), c.n_new) : c.n_new;
  if (t >= valid) return;
  const int len = min(max(load_uniform(c.lens + b), 0), kMaxRows), rows = min(len, c.cap());
  const long long at = (a.first ? (long long)load_uniform(a.first + b) : (long long)(len - valid)) + t;
  if (at < 0 || at >= rows) return;
  const int j = (int)at;
  const bool tail = FMT == MPC_PAGE_E4M3 && j >= (rows & ~(c.page - 1));
  const int id = tail ? 0 : page_id_lane(c, b, j >> c.log_page);
  if (id < 0) return;
  const int h0 = chunk * HPT * m.lanes + lane;
  if (tail) {
    for (int k = 0; k < HPT; ++k) {
      const int hh = h0 + k * m.lanes;
      if (hh >= heads) continue;
      const bool is_v = hh >= nk;
      const int h = hh - (is_v ? nk : 0);
      const size_t row = ((size_t)lb * c.Hkv + h) * (2 * c.page) + (j & (2 * c.page - 1));
      *(uint4*)((is_v ? a.v : a.k).at(l, b, h, t) + v * 16) = ldg16((is_v ? c.v_tail : c.k_tail) + row * (size_t)(D * DT::kElt) + v * 16);
    }
    return;
  }
  Piece<DT, FMT> x[HPT];
#pragma unroll
  for (int k = 0; k < HPT; ++k) {
    const int hh = h0 + k * m.lanes;
    if (hh >= heads) continue;
    const bool is_v = hh >= nk;
    const size_t unit = page_unit(c, l, id, hh - (is_v ? nk : 0));
    const int slot = j & (c.page - 1);
    x[k].load((is_v ? c.v : c.k) + (unit * c.page + slot) * RB + v * (V * BITS / 8));
    if constexpr (FMT == MPC_PAGE_E4M3) x[k].scale = (is_v ? c.vs : c.ks)[unit];
    if constexpr (FMT == MPC_PAGE_MX4)
      x[k].scale = mx4_scale((is_v ? c.vx : c.kx)[unit * (size_t)(D / kMx4Block * c.page) + v * V / kMx4Block * c.page + slot]);
  }
#pragma unroll
  for (int k = 0; k < HPT; ++k) {
    const int hh = h0 + k * m.lanes;
    if (hh >= heads) continue;
    const bool is_v = hh >= nk;
    *(uint4*)((is_v ? a.v : a.k).at(l, b, hh - (is_v ? nk : 0), t) + v * 16) = x[k].rows();
  }
}

template <class DT, int D, int FMT>
hipError_t launch(const PagedReadArgs& a, hipStream_t st) {
  constexpr int slots = kThreads / (D / DT::kVec);
  const PagedCache& c = a.c;
  const int heads = ((a.k.p ? 1 : 0) + (a.v.p ? 1 : 0)) * c.Hkv;
  Reads m{};
  m.tokens = 1;
  while (m.tokens < slots && m.tokens < c.n_new) m.tokens *= 2;
  m.lanes = slots / m.tokens;
  m.runs = (int)(((int64_t)c.n_new + m.tokens - 1) / m.tokens);
  auto blocks = [&](int hpt) {
    m.chunks = (heads + hpt * m.lanes - 1) / (hpt * m.lanes);
    return (int64_t)c.L * c.B * m.runs * m.chunks;
  };
  // four heads to a thread, where that leaves a few workgroups to a compute unit
  const int hpt = blocks(4) >= 4 * kNumCU ? 4 : 1;
  const int64_t n = blocks(hpt);
  if (n >= ((int64_t)1 << 31)) return hipErrorInvalidValue;
  if (hpt == 4)
    hipLaunchKernelGGL((k_read<DT, D, FMT, 4>), dim3((unsigned)n), dim3(kThreads), 0, st, a, m);
  else
    hipLaunchKernelGGL((k_read<DT, D, FMT, 1>), dim3((unsigned)n), dim3(kThreads), 0, st, a, m);
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
