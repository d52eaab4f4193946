// Attention behind shared rows: sizes, the plan of a call, made on the device from the groups and the lengths, and the join.
#include <algorithm>

#include "shared_attn_dev.h"

namespace mpc {
namespace {

using namespace dev;
constexpr int kJoinThreads = 256;

template <bool C8>
__global__ __launch_bounds__(kMaxGroups) void k_shared_plan(SharedArgs a) {
  __shared__ PlanScratch<kMaxGroups> tmp;
  make_plan<C8, kMaxGroups>(a, tmp, a.group, a.seq, a.total);
}

// The join: 10.6 us for 1024 rows of 66 parts each (33: 8.1), 24 for 54K rows of two or three (110 MB; a wave to a row, statistics before the
// accumulators: 14 and 59). A team of lanes, 16 bytes to each, has a query row, whose parts are those of its own rows and of the
// shared ones; where there are few rows, ALL teams of a workgroup have one row and every T-th part of it each.
template <class DT, int D, bool ALL>
__global__ __launch_bounds__(kJoinThreads) void k_shared_join(SharedArgs a) {
  constexpr int PS = D + kPartTail, LANES = D / 4, TEAMS = kJoinThreads / LANES, T = ALL ? TEAMS : 1, AHEAD = ALL ? 5 : 4;
  __shared__ float4 s_x[ALL ? TEAMS : 1][LANES];
  __shared__ float2 s_ml[ALL ? TEAMS : 1];
  const PagedCache& c = a.c;
  const int team = threadIdx.x / LANES, e = threadIdx.x % LANES * 4, way = ALL ? team : 0;
  const int per = c.n_new << a.log_g;
  const unsigned row = ALL ? blockIdx.x : blockIdx.x * TEAMS + team;  // (below 2^31, as the host has checked)
  if (row >= (unsigned)(a.L * a.Hkv) * (unsigned)a.B * (unsigned)per) return;
  const int in_seq = row % (unsigned)per, lhb = row / (unsigned)per, b = (unsigned)lhb % (unsigned)a.B, lh = (unsigned)lhb / (unsigned)a.B, t = in_seq >> a.log_g;
  const int valid = c.valid(b);
  if (t >= valid) return;
  const SharedSeq q = a.seq[b];
  // the parts of a unit: its first worker's, by row, then those of the workers that go on with it
  struct Side {
    const float *head, *more;
    int n;
  };
  auto side = [&](const Parts& p, unsigned total, unsigned x0, int nb, int in_unit) {
    Side s{p.head + (size_t)row * PS, nullptr, 0};
    if (nb > 0) {
      const unsigned share = (total + p.workers - 1) / p.workers, w0 = x0 / share, w1 = (x0 + nb - 1) / share;
      s.more = p.more + ((size_t)w0 * p.unit_rows + in_unit) * PS;
      s.n = (int)(w1 - w0) + 1;
    }
    return s;
  };
  const int units = ((valid << a.log_g) + a.own.unit_rows - 1) / a.own.unit_rows;
  const Side o = side(a.own, a.total->own, q.block0 + (unsigned)(lh * units + in_seq / a.own.unit_rows) * (unsigned)q.nb, q.nb,
                      in_seq % a.own.unit_rows);
  Side s{nullptr, nullptr, 0};
  if (q.group >= 0) {
    const SharedGroup g = a.group[q.group];
    const int in_group = q.row0 - g.row0 + in_seq;
    const unsigned u = (unsigned)(lh * g.rt + in_group / a.shared.unit_rows);
    s = side(a.shared, a.total->shared, g.block0 + u * (unsigned)g.nb, g.nb, in_group % a.shared.unit_rows);
  }
  const int all = o.n + s.n;
  const size_t own_step = (size_t)a.own.unit_rows * PS, shared_step = (size_t)a.shared.unit_rows * PS;
  auto at = [&](int n) {
    const bool own = n < o.n;
    const int k = own ? n : n - o.n;
    return k == 0 ? (own ? o.head : s.head) : own ? o.more + k * own_step : s.more + k * shared_step;
  };
  float m = -INFINITY, sum = 0.f;  // reference and sum so far
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int n0 = way; n0 < all; n0 += AHEAD * T) {
    float2 ml[AHEAD];
    float4 y[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (n0 + k * T >= all) continue;
      const float* p = at(n0 + k * T);
      ml[k] = *(const float2*)(p + D);
      y[k] = *(const float4*)(p + e);
    }
    float top = m;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) top = n0 + k * T < all ? fmaxf(top, ml[k].x) : top;
    const float ref = top == -INFINITY ? 0.f : top, move = fast_exp2(m - ref);
    m = top;
    sum *= move;
    x = make_float4(x.x * move, x.y * move, x.z * move, x.w * move);
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      if (n0 + k * T >= all) continue;
      const float f = fast_exp2(ml[k].x - ref);
      sum = fmaf(ml[k].y, f, sum);
      x = make_float4(fmaf(y[k].x, f, x.x), fmaf(y[k].y, f, x.y), fmaf(y[k].z, f, x.z), fmaf(y[k].w, f, x.w));
    }
  }
  if constexpr (ALL) {
    s_x[team][e / 4] = x;
    if (e == 0) s_ml[team] = make_float2(m, sum);
    __syncthreads();
    if (team > 0) return;
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < TEAMS; ++k) top = fmaxf(top, s_ml[k].x);
    const float ref = top == -INFINITY ? 0.f : top;
    m = top;
    sum = 0.f;
    x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < TEAMS; ++k) {
      const float f = fast_exp2(s_ml[k].x - ref);
      const float4 y = s_x[k][e / 4];
      sum = fmaf(s_ml[k].y, f, sum);
      x = make_float4(fmaf(y.x, f, x.x), fmaf(y.y, f, x.y), fmaf(y.z, f, x.z), fmaf(y.w, f, x.w));
    }
  }
  const int h = lh % a.Hkv, l = lh / a.Hkv, hq = (h << a.log_g) + in_seq - (t << a.log_g);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  char* out = a.out.at(l, b, hq, t) + e * DT::kElt;
  x = sum == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
  if constexpr (DT::kElt == 4)
    *(float4*)out = x;
  else
    *(uint2*)out = make_uint2(pack2<DT>(x.x, x.y), pack2<DT>(x.z, x.w));
  if (e == 0 && a.lse)
    a.lse[(((size_t)l * a.B + b) * a.Hq + hq) * a.n + t] =
        sum == 0.f ? -INFINITY : ((m == -INFINITY ? 0.f : m) + __log2f(sum)) * 0.69314718055994531f;
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

template <class DT, int D>
hipError_t launch_join_d(const SharedArgs& a, hipStream_t st) {
  constexpr int teams = kJoinThreads / (D / 4);
  const long long rows = (long long)a.L * a.Hkv * a.B * ((long long)a.c.n_new << a.log_g);
  if (rows < 16 * kNumCU)
    hipLaunchKernelGGL((k_shared_join<DT, D, true>), dim3((unsigned)rows), dim3(kJoinThreads), 0, st, a);
  else
    hipLaunchKernelGGL((k_shared_join<DT, D, false>), dim3((unsigned)((rows + teams - 1) / teams)), dim3(kJoinThreads), 0, st, a);
  return hipGetLastError();
}
template <class DT>
hipError_t launch_join(const SharedArgs& a, int D, hipStream_t st) {
  return D == 64 ? launch_join_d<DT, 64>(a, st) : launch_join_d<DT, 128>(a, st);
}

}  // namespace

// Shared rows in units of 128 query rows (16-bit types) where a group has more than 32 on average and units of 32 would have 2^18
// keys or more to read together, else of 32, or of 16 over codes where that is enough. Units of 32 and of 128, us, for 8 kv heads of
// 128 in bf16 (8-bit codes in fp16; 4-bit codes in bf16): 40 query rows to a kv head behind 1K shared rows 24 and 31 (25 and 29; 23
// and 27), behind 16K 37 and 37 (39 and 36; 37 and 34); 96 behind 4K 34 and 37 (34 and 36; 32 and 32), behind 16K 54 and 44 (52
// and 42; 49 and 41); 512 behind 1K 38 and 42 (40 and 41; 38 and 40), behind 8K 84 and 61 (93 and 63; 86 and 61); two groups of 1024
// behind 1K 78 and 59 (83 and 58; 79 and 55). 32 rows behind 16K: 32 and 31 (31 and 31; 30 and 30). The lengths are on the device:
// the table's room stands for the shared rows, so a short prompt in a large table is taken in units of 128.
// 16 rows in units of 16 and of 32: bf16 34 and 30, fp32 50 and 51 (1K shared rows: 38 and 30), 8-bit codes 28 and 30, 4-bit codes
// 25 and 28. Own rows in units of 16 where a sequence's rows fit, or beside the wide units, else of 32. Blocks are a tile to each
// wave of a workgroup (wide units: four tiles), and 64 keys of the own rows, which are taken by the waves
// of the kernel that takes the shared ones (more where the table has room for 2^31 such blocks).
SharedPlan shared_plan(int dtype, int format, int D, int L, int B, int Hq, int Hkv, int n, int cap, int groups) {
  SharedPlan p{};
  const long long each_seq = (long long)n * (Hq / Hkv), rows = B * each_seq, each = (rows + groups - 1) / groups, lh = (long long)L * Hkv;
  p.wide = dtype != MPC_FP32 && each > 32 && (double)lh * groups * ((each + 31) / 32) * cap >= 1 << 18;
  p.shared_rows = p.wide ? 128 : each <= 16 && format != MPC_PAGE_SAME ? 16 : 32;
  p.own_rows = each_seq <= 16 || p.wide ? 16 : 32;
  p.tile = dtype == MPC_FP32 ? 16 : 32;
  p.shared_block = p.wide ? 4 : paged_waves(p.shared_rows / 16);
  p.own_block = 64 / p.tile;
  p.shared_workers = p.wide ? 2 * kNumCU : kNumCU;
  p.own_workers = kNumCU * (p.wide ? 8 : paged_waves(p.shared_rows / 16));
  const PagedPlan unshared = paged_plan(dtype, D, L, B, Hq, Hkv, n, cap);
  // Fewer than 2^31 blocks: what the paged attention takes (fewer of them, of 256 keys) is taken here too, in blocks as much larger
  auto blocks = [&](long long units, int& block) {
    for (;; block *= 2) {
      const long long nb = cap / ((long long)p.tile * block) + 2;  // complete pages' tiles and the ring's may each be cut short
      if ((double)units * (double)nb < 2147483648.0) return units * nb;
      if (nb == 2 || unshared.blocks >= 1ll << 31) return 1ll << 31;
    }
  };
  p.blocks = std::max(blocks((rows / p.shared_rows + groups) * lh, p.shared_block),
                      blocks(B * ((each_seq + p.own_rows - 1) / p.own_rows) * lh, p.own_block));
  if (unshared.blocks >= 1ll << 31) p.blocks = unshared.blocks;
  const size_t row = (D + kPartTail) * sizeof(float), heads = align256((size_t)lh * rows * row);
  p.total = kPagedCntBytes;  // behind the counters of the paged attention, which a workspace of this serves too
  p.group = p.total + align256(sizeof(SharedTotals));
  p.seq = p.group + align256((size_t)groups * sizeof(SharedGroup));
  p.shared_head = p.seq + align256((size_t)B * sizeof(SharedSeq));
  // as many places for the workers' parts as any form has, so that a workspace made for the most tokens serves calls of fewer
  const size_t most_shared = (size_t)kNumCU * (dtype == MPC_FP32 ? 32 : 256), most_own = (size_t)kNumCU * 128;
  p.shared_more = p.shared_head + heads;
  p.own_head = p.shared_more + align256(most_shared * row);
  p.own_more = p.own_head + heads;
  p.ws_bytes = std::max(p.own_more + most_own * row, unshared.ws_bytes);
  return p;
}

hipError_t launch_shared_attn(const SharedArgs& a, int dtype, int D, hipStream_t st) {
  hipError_t e;
  if (a.B > kPlanLanes) {  // fewer: every workgroup makes the plan for itself
    if (a.c.format == MPC_PAGE_E4M3)
      hipLaunchKernelGGL(k_shared_plan<true>, dim3(1), dim3(kMaxGroups), 0, st, a);
    else
      hipLaunchKernelGGL(k_shared_plan<false>, dim3(1), dim3(kMaxGroups), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  e = a.c.format == MPC_PAGE_MX4 ? launch_shared_mx4(a, dtype, D, st)
      : dtype == MPC_FP32        ? launch_shared_fp32(a, D, st)
      : dtype == MPC_FP16        ? launch_shared_fp16(a, D, st)
                                 : launch_shared_bf16(a, D, st);
  if (e != hipSuccess) return e;
  if (dtype == MPC_FP32) return launch_join<F32>(a, D, st);
  return dtype == MPC_FP16 ? launch_join<F16>(a, D, st) : launch_join<BF16>(a, D, st);
}

}  // namespace mpc
