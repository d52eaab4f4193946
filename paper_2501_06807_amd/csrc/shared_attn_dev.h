// Attention behind shared rows: the kernel of the shared rows, for units of 16 or 32 query rows.
//
// A group's query rows (all its sequences' tokens and the G heads of a kv head) are one unit's rows as far as they fit, so K and
// V of the shared rows are read once for a unit instead of once for a sequence. The blocks of keys of all units are divided
// evenly over the grid; each workgroup writes what it has of a unit (accumulators, maxima and sums of the unit's rows), and the
// paged attention's kernel, which takes each sequence's own rows, joins these parts to its own.
#pragma once
#include "paged_attn_dev.h"

namespace mpc {
namespace dev {

// The group that block x falls to; groups to lanes.
__device__ __forceinline__ int group_of(const SharedArgs& sh, unsigned x) {
  const int lane = threadIdx.x % kWave;
  int g = 0;
  for (int g0 = 0; g0 < sh.groups; g0 += kWave) {
    const bool before = g0 + lane < sh.groups && sh.plan[g0 + lane].block0 <= x;
    const unsigned long long past = __ballot(before);
    if (past) g = g0 + 63 - __clzll((long long)past);
  }
  return __builtin_amdgcn_readfirstlane(g);
}

// A query row of a group: sequence, token, head of the kv head's group, position.
struct SharedRow {
  int b, in_seq, pos;
  bool live;
};
__device__ __forceinline__ SharedRow shared_row(const PagedAttnArgs& a, int f0, int f1, int row) {
  const PagedCache& c = a.c;
  const int per = c.n_new << a.log_g;
  SharedRow r;
  const int k = row / per;
  r.live = f0 + k < f1;
  r.b = r.live ? f0 + k : f0;
  r.in_seq = r.live ? row - k * per : 0;
  const int valid = c.valid(r.b), t = r.in_seq >> a.log_g;
  r.live = r.live && t < valid;
  r.pos = c.len(r.b) - valid + t;
  return r;
}

template <class DT, int D, int FMT, int RT>
__global__ __launch_bounds__(paged_waves(RT) * kWave) void k_shared_rows(PagedAttnArgs a) {
  using TL = PagedTile<DT, D, FMT, RT>;
  constexpr int NT = TL::NT, RW = 16 * RT, NW = paged_waves(RT);
  const PagedCache& c = a.c;
  const SharedArgs& sh = a.sh;
  const int lane = threadIdx.x % kWave, g = lane / 16, col = lane % 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  __shared__ __align__(16) f32x4 s_o[NW / 2][NT][kWave];
  __shared__ float s_ml[NW][RT][2][kWave];

  const unsigned total = load_uniform(sh.total), id = by_die(blockIdx.x, gridDim.x);
  const unsigned per = (total + gridDim.x - 1) / gridDim.x;
  if ((unsigned long long)id * per >= total) return;
  const unsigned first = id * per, last = min(first + per, total);
  int gi = group_of(sh, first);
  PagedWave<DT, D, FMT, RT> w;
  unsigned x = first;
  while (x < last) {
    while (gi + 1 < sh.groups && x >= load_uniform(&sh.plan[gi + 1].block0)) ++gi;
    const SharedGroup* gp = sh.plan + gi;
    const int f0 = load_uniform(&gp->f0), f1 = load_uniform(&gp->f1), nb = load_uniform(&gp->nb), rts = load_uniform(&gp->rt);
    const unsigned block0 = load_uniform(&gp->block0), in = x - block0;
    const int u = __builtin_amdgcn_readfirstlane(in / (unsigned)nb), blk = __builtin_amdgcn_readfirstlane(in - u * (unsigned)nb);
    const int blk_end = min(nb, blk + (int)(last - x));
    const int lh = u / rts, h = lh % a.Hkv, l = lh / a.Hkv, r0 = u % rts * RW;
    const unsigned start = x - blk;  // the unit's first block
    w.clear();
    SharedRow row[RT];
    int lo = kMaxRows, hi = -kMaxRows;  // positions of the unit's rows
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      row[rt] = shared_row(a, f0, f1, r0 + 16 * rt + col);
      // a row that is not there sees every key, so that it makes no tile an edge; nobody reads it
      w.pos[rt] = row[rt].live ? row[rt].pos : kMaxRows;
      lo = min(lo, row[rt].live ? row[rt].pos : kMaxRows);
      hi = max(hi, row[rt].live ? row[rt].pos : -kMaxRows);
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) {
      lo = min(lo, __shfl_xor(lo, o));
      hi = max(hi, __shfl_xor(hi, o));
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
    auto load_queries = [&]() {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const int t = row[rt].in_seq >> a.log_g, hq = (h << a.log_g) + row[rt].in_seq - (t << a.log_g);
        const char* p = a.q.at(l, row[rt].b, hq, t);
        load_query_row<DT, D, FMT, RT>(w, rt, p, row[rt].live);
      }
    };
    const int base = load_uniform(&gp->base);
    const PageRows rows{load_uniform(&gp->skip), load_uniform(&gp->at), 0, 0, base};
    walk_pages<DT, D, FMT, RT>(w, a, c, f0, l, h, rows, blk * NW + wave, min(blk_end * NW, load_uniform(&gp->tiles)), lo, hi, load_queries);
    float M[RT], Lsum[RT];
    join_waves<DT, D, FMT, RT>(w, wave, s_ml, s_o, M, Lsum);
    if (blk == 0 && threadIdx.x == 0) {
      const unsigned w0 = start / per, w1 = (start + nb - 1) / per;
      sh.unit[load_uniform(&gp->unit0) + u] = make_int2((int)w0, (int)(w1 - w0) + 1);
    }
    if (wave == 0) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        if (!row[rt].live) continue;
        float* part = blk == 0 ? sh.head + (((long long)lh * a.B + row[rt].b) * ((long long)c.n_new << a.log_g) + row[rt].in_seq) * (D + 2)
                               : sh.more + ((size_t)id * sh.unit_rows + 16 * rt + col) * (D + 2);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int n = 0; n < NT; n += 2) *(float2*)(part + (4 * g + e) * NT + n) = make_float2(w.o[rt][n][e], w.o[rt][n + 1][e]);
        if (g == 0) *(float2*)(part + D) = make_float2(M[rt], Lsum[rt]);
      }
    }
    __syncthreads();  // the LDS buffers are free again
    x += blk_end - blk;
  }
}

template <class DT, int D, int FMT, int RT>
hipError_t launch_shared_rt(const PagedAttnArgs& a, hipStream_t st) {
  hipError_t e;
  if (a.sh.unit_rows == 16)
    hipLaunchKernelGGL((k_shared_rows<DT, D, FMT, 1>), dim3((unsigned)a.sh.grid), dim3(paged_waves(1) * kWave), 0, st, a);
  else
    hipLaunchKernelGGL((k_shared_rows<DT, D, FMT, 2>), dim3((unsigned)a.sh.grid), dim3(paged_waves(2) * kWave), 0, st, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  hipLaunchKernelGGL((k_paged_attn<DT, D, FMT, RT, true>), dim3((unsigned)a.grid), dim3(paged_waves(RT) * kWave), 0, st, a);
  return hipGetLastError();
}

template <class DT, int FMT>
hipError_t launch_shared_format(const PagedAttnArgs& a, int D, hipStream_t st) {
  if (a.row_tiles == 1) return D == 64 ? launch_shared_rt<DT, 64, FMT, 1>(a, st) : launch_shared_rt<DT, 128, FMT, 1>(a, st);
  return D == 64 ? launch_shared_rt<DT, 64, FMT, 2>(a, st) : launch_shared_rt<DT, 128, FMT, 2>(a, st);
}

}  // namespace dev
}  // namespace mpc
