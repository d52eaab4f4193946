// Attention behind shared rows: the plan, the shared rows for units of 16 or 32 query rows, and the sequences' own rows.
//
// A group's query rows (all its sequences' tokens and the G heads of a kv head) are one unit's rows as far as they fit, so K and
// V of the shared rows are read once for a unit instead of once for a sequence; a softmax over both kinds of rows is the join of
// its parts over each, o = sum_p 2^(m_p - m) o_p / sum_p 2^(m_p - m) l_p with m = max_p m_p. The tiles' work is the paged
// attention's. Reading the keys bounds it: 64 sequences in four groups behind 8K rows of 8-bit pages, 32 heads of 128, 108 us,
// 350 MB (54 us at the rate of a large read): 66 for the shared rows, of which the two groups of 17 take two units of 16 rows and
// ask for theirs twice (units of 32: 74), 28 for the own ones (100 MB), 8 for the join. More than 64 sequences wait for
// the plan's launch: 64 behind 4K rows of bf16 pages, 8 kv heads, 42 us, 65 of them 54.
//
// Own rows are short and their units many, so a wave takes a run of them by itself: no LDS, no wait for another wave. Eight waves to
// a unit, joined in LDS and through memory as in the paged attention, took 103 us of what is 32 for the own rows above (with
// launches of their own), and 30 of 20 for 32 sequences of up to 700 rows. Blocks of 64 keys instead of 128: 20 and 16 us there.
// The workgroups of the shared rows go on with own rows when they are done (77 to 73 us for 32 sequences behind 32K rows).
#pragma once
#include "paged_attn_dev.h"

namespace mpc {
namespace dev {

// The last of n entries (in order) that is not beyond x; entries to lanes, 64 steps at a time.
template <class At>
__device__ __forceinline__ int last_from(int n, unsigned x, At at) {
  const int lane = threadIdx.x % kWave;
  int lo = 0;
  for (int step = 1 << 24; step > 0; step /= kWave) {
    if (step >= n) continue;
    const int i = lo + lane * step;
    const unsigned long long past = __ballot(i < n && at(i) <= x);
    lo += (63 - __clzll((long long)past)) * step;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// A sequence's own rows: the tiles of pages behind the shared ones (as PageRows has them), and of the ring.
struct OwnRows {
  int valid, len, rows, start, groups, full, tiles, all;  // tiles of pages, and with those of the ring
  PageRows pages;
};
template <bool C8>
__device__ __forceinline__ OwnRows own_rows(const SharedArgs& a, int len, int valid, int base, int unit_rows) {
  const PagedCache& c = a.c;
  const int tile = a.tile;
  OwnRows s;
  s.valid = min(max(valid, 0), c.n_new);
  s.len = min(max(len, 0), kMaxRows);
  s.rows = min(s.len, c.cap());
  s.start = s.len - s.valid;
  s.groups = ((s.valid << a.log_g) + unit_rows - 1) / unit_rows;
  s.full = C8 ? s.rows & ~(c.page - 1) : s.rows;
  const int all = (s.full + tile - 1) / tile;
  PageRows& p = s.pages;
  p.base = base;
  p.full = s.full;
  p.from = base / tile;
  p.skip = max(all - p.from, 0);
  p.at = max(all, p.from);
  if (a.window) {
    p.skip = max(min((a.sinks + tile - 1) / tile, all) - p.from, 0);
    p.at = max(p.from + p.skip, min(max(s.start - a.window + 1, 0) / tile, all));
  }
  s.tiles = p.skip + max(all - p.at, 0);
  s.all = s.tiles + (s.full < base ? 0 : (s.rows - s.full + tile - 1) / tile);
  return s;
}

// The plan is made by a wave of each workgroup where that has a lane to each sequence, else by a launch of its own.
constexpr int kPlanLanes = kWave;
template <int THREADS>
struct PlanScratch {
  int f[THREADS + 1], base[THREADS], lo[THREADS], hi[THREADS];
  unsigned wave[THREADS / kWave];
};
template <int THREADS>
__device__ __forceinline__ void plan_sync() {
  if constexpr (THREADS == kWave) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  } else {
    __syncthreads();
  }
}

// Sum of x over the threads before this one, and over all of them.
template <int THREADS>
__device__ __forceinline__ unsigned sum_before(unsigned x, unsigned* s_wave, unsigned* total) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  unsigned sum = x;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const unsigned y = __shfl_up(sum, o);
    if (lane >= o) sum += y;
  }
  if constexpr (THREADS == kWave) {
    *total = __builtin_amdgcn_readlane(sum, kWave - 1);
    return sum - x;
  }
  if (lane == kWave - 1) s_wave[wave] = sum;
  plan_sync<THREADS>();
  unsigned before = 0, all = 0;
  for (int w = 0; w < THREADS / kWave; ++w) {
    before += w < wave ? s_wave[w] : 0;
    all += s_wave[w];
  }
  plan_sync<THREADS>();
  *total = all;
  return before + sum - x;
}

// A thread to a group, and the sequences over the threads. Bounds of the groups are brought into [0, B] and in order, so that
// every sequence is in one group at most, whatever `first` holds.
template <bool C8, int THREADS>
__device__ __forceinline__ void make_plan(const SharedArgs& a, PlanScratch<THREADS>& s, SharedGroup* group, SharedSeq* seq, SharedTotals* totals) {
  auto sync = [] { plan_sync<THREADS>(); };
  const PagedCache& c = a.c;
  const int tid = threadIdx.x, ng = a.groups;
  s.f[tid] = tid < ng ? min(max(a.first[tid], 0), a.B) : 0;
  sync();
  for (int o = 1; o < ng; o <<= 1) {
    const int y = tid >= o ? s.f[tid - o] : 0;
    sync();
    s.f[tid] = max(s.f[tid], y);
    sync();
  }
  if (tid == 0) s.f[ng] = max(s.f[ng - 1], min(max(a.first[ng], 0), a.B));
  if (tid < ng) {
    s.base[tid] = min(max(a.rows[tid], 0), c.cap()) & ~(c.page - 1);
    s.lo[tid] = kMaxRows;
    s.hi[tid] = -1;
  }
  sync();
  unsigned own = 0, rows = 0;  // blocks and query rows of the sequences so far
  for (int b0 = 0; b0 < a.B; b0 += THREADS) {
    const int b = b0 + tid;
    SharedSeq q{0, 0, -1, 0, 0};
    unsigned blocks = 0, mine = 0;
    if (b < a.B) {
      if (b >= s.f[0] && b < s.f[ng]) {  // the last group that begins at or before b
        int g = 0, z = ng;
        while (z - g > 1) {
          const int m = (g + z) / 2;
          (s.f[m] <= b ? g : z) = m;
        }
        q.group = g;
        q.base = s.base[g];
      }
      const OwnRows o = own_rows<C8>(a, c.lens[b], c.n_valid ? c.n_valid[b] : c.n_new, q.base, a.own.unit_rows);
      if (q.group >= 0 && o.valid > 0) {
        atomicMin(&s.lo[q.group], o.start);
        atomicMax(&s.hi[q.group], o.len - 1);
      }
      q.nb = (o.all + a.own_block - 1) / a.own_block;
      blocks = (unsigned)(o.groups * a.L * a.Hkv) * (unsigned)q.nb;
      mine = (unsigned)o.valid << a.log_g;
    }
    unsigned all;
    q.block0 = own + sum_before<THREADS>(blocks, s.wave, &all);
    own += all;
    q.row0 = (int)(rows + sum_before<THREADS>(mine, s.wave, &all));
    rows += all;
    if (b < a.B) seq[b] = q;
  }
  sync();
  SharedGroup p{};
  if (tid < ng) {
    p.f0 = s.f[tid];
    p.f1 = s.f[tid + 1];
    p.base = s.base[tid];
    p.row0 = p.f0 < a.B ? seq[p.f0].row0 : (int)rows;
    p.query_rows = (p.f1 < a.B ? seq[p.f1].row0 : (int)rows) - p.row0;
    p.rt = (p.query_rows + a.shared.unit_rows - 1) / a.shared.unit_rows;
    const int all = (max(0, min(p.base, s.hi[tid] + 1)) + a.tile - 1) / a.tile;
    p.skip = p.at = all;
    if (a.window) {
      p.skip = min((a.sinks + a.tile - 1) / a.tile, all);
      p.at = max(p.skip, min(max(s.lo[tid] - a.window + 1, 0) / a.tile, all));
    }
    p.tiles = p.skip + all - p.at;
    p.nb = (p.tiles + a.shared_block - 1) / a.shared_block;
  }
  unsigned total;
  p.block0 = sum_before<THREADS>((unsigned)(p.rt * a.L * a.Hkv) * (unsigned)p.nb, s.wave, &total);
  if (tid < ng) group[tid] = p;
  if (tid == 0) *totals = SharedTotals{total, own};
}

// Where a workgroup finds the plan.
struct Plan {
  const SharedGroup* group;
  const SharedSeq* seq;
  unsigned shared, own;  // blocks
};
struct PlanSpace {
  PlanScratch<kPlanLanes> tmp;
  SharedGroup group[kPlanLanes];
  SharedSeq seq[kPlanLanes];
  SharedTotals total;
};
template <class T>
__device__ __forceinline__ T same(T x) { return (T)__builtin_amdgcn_readfirstlane((int)x); }
// The first workgroup's goes to memory, for the join.
template <bool C8>
__device__ __forceinline__ Plan plan_of(const SharedArgs& a, PlanSpace& s) {
  if (a.B > kPlanLanes) return Plan{a.group, a.seq, load_uniform(&a.total->shared), load_uniform(&a.total->own)};
  if (threadIdx.x < kPlanLanes) {
    make_plan<C8, kPlanLanes>(a, s.tmp, s.group, s.seq, &s.total);
    plan_sync<kPlanLanes>();
    if (blockIdx.x == 0) {
      const int i = threadIdx.x;
      if (i < a.groups) a.group[i] = s.group[i];
      if (i < a.B) a.seq[i] = s.seq[i];
      if (i == 0) *a.total = s.total;
    }
  }
  __syncthreads();
  return Plan{s.group, s.seq, same(s.total.shared), same(s.total.own)};
}

// A query row of a group: sequence, token and head of it, position. The rows of a group's sequences lie one after the other.
struct SharedRow {
  int b, in_seq, pos;
  bool live;
};
__device__ __forceinline__ SharedRow shared_row(const SharedArgs& a, const SharedSeq* seq, const SharedGroup* gp, int row) {
  const PagedCache& c = a.c;
  const int f0 = same(gp->f0), f1 = same(gp->f1);
  SharedRow r;
  r.live = row < same(gp->query_rows);
  r.b = f0;
  r.in_seq = 0;
  if (r.live) {
    if (!c.n_valid) {
      const int per = c.n_new << a.log_g, k = row / per;
      r.b += k;
      r.in_seq = row - k * per;
    } else {  // the last sequence that begins at or before the row
      const int at = same(gp->row0) + row;
      int z = f1;
      while (z - r.b > 1) {
        const int m = (r.b + z) / 2;
        (seq[m].row0 <= at ? r.b : z) = m;
      }
      r.in_seq = at - seq[r.b].row0;
    }
  }
  r.pos = c.len(r.b) - c.valid(r.b) + (r.in_seq >> a.log_g);
  return r;
}
// Row in_seq of (layer and kv head lh, sequence b) in a head array.
__device__ __forceinline__ long long part_row(const SharedArgs& a, int lh, int b, int in_seq) {
  return ((long long)lh * a.B + b) * ((long long)a.c.n_new << a.log_g) + in_seq;
}

// What a wave (one that holds the sums of its lanes' columns) has of its rows, written for the join: accumulators, the reference of
// their exponents (its lift taken off) and the weights' sum.
template <class DT, int D, int FMT, int RT>
__device__ __forceinline__ void write_part(const PagedWave<DT, D, FMT, RT>& w, int rt, float m, float sum, float* part) {
  using TL = PagedTile<DT, D, FMT, RT>;
  constexpr int NT = TL::NT;
  const int g = (threadIdx.x % kWave) / 16;
#pragma unroll
  for (int e = 0; e < 4; ++e)
#pragma unroll
    for (int n = 0; n < NT; n += 2) *(float2*)(part + (4 * g + e) * NT + n) = make_float2(w.o[rt][n][e], w.o[rt][n + 1][e]);
  if (g == 0) *(float2*)(part + D) = make_float2(m - TL::LIFT, sum);
}

template <class DT, int D, int FMT, int RT>
__device__ __forceinline__ void shared_rows(const SharedArgs& a, const Plan& plan) {
  using TL = PagedTile<DT, D, FMT, RT>;
  constexpr int NT = TL::NT, RW = 16 * RT, NW = paged_waves(RT);
  const PagedCache& c = a.c;
  const int lane = threadIdx.x % kWave, col = lane % 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  __shared__ __align__(16) f32x4 s_o[NW / 2][NT][kWave];
  __shared__ float s_ml[NW][RT][2][kWave];

  const unsigned total = plan.shared, id = by_die(blockIdx.x, gridDim.x);
  const unsigned per = (total + gridDim.x - 1) / gridDim.x;
  if ((unsigned long long)id * per >= total) return;
  const unsigned first = id * per, last = min(first + per, total);
  int gi = last_from(a.groups, first, [&](int i) { return plan.group[i].block0; });
  PagedWave<DT, D, FMT, RT> w;
  unsigned x = first;
  while (x < last) {
    while (gi + 1 < a.groups && x >= same(plan.group[gi + 1].block0)) ++gi;
    const SharedGroup* gp = plan.group + gi;
    const int f0 = same(gp->f0), nb = same(gp->nb), rts = same(gp->rt);
    const unsigned in = x - same(gp->block0);
    const int u = __builtin_amdgcn_readfirstlane(in / (unsigned)nb), blk = __builtin_amdgcn_readfirstlane(in - u * (unsigned)nb);
    const int blk_end = min(nb, blk + (int)(last - x));
    const int lh = u / rts, h = lh % a.Hkv, l = lh / a.Hkv, r0 = u % rts * RW;
    w.clear();
    SharedRow row[RT];
    int lo = kMaxRows, hi = -kMaxRows;  // positions of the unit's rows
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      row[rt] = shared_row(a, plan.seq, gp, r0 + 16 * rt + col);
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
        load_query_row<DT, D, FMT, RT>(w, rt, a.q.at(l, row[rt].b, hq, t), row[rt].live);
      }
    };
    const PageRows rows{same(gp->skip), same(gp->at), 0, 0, same(gp->base)};
    walk_pages<DT, D, FMT, RT, NW>(w, a, c, f0, l, h, rows, blk * a.shared_block + wave, min(blk_end * a.shared_block, same(gp->tiles)), lo, hi, load_queries);
    float M[RT], Lsum[RT];
    join_waves<DT, D, FMT, RT>(w, wave, s_ml, s_o, M, Lsum);
    if (wave == 0) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        if (!row[rt].live) continue;
        write_part(w, rt, M[rt], Lsum[rt], blk == 0 ? a.shared.head + part_row(a, lh, row[rt].b, row[rt].in_seq) * (D + kPartTail)
                                                    : a.shared.more + ((size_t)id * RW + 16 * rt + col) * (D + kPartTail));
      }
    }
    __syncthreads();  // the LDS buffers are free again
    x += blk_end - blk;
  }
}

// A wave to a run of blocks: nothing of it waits for another wave. Workgroups of WAVES waves.
template <class DT, int D, int FMT, int RT, int WAVES>
__device__ __forceinline__ void own_rows_of(const SharedArgs& a, const Plan& plan) {
  using TL = PagedTile<DT, D, FMT, RT>;
  constexpr int RW = 16 * RT;
  const PagedCache& c = a.c;
  const int lane = threadIdx.x % kWave, col = lane % 16;
  const unsigned id = by_die(blockIdx.x, gridDim.x) * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const unsigned total = plan.own, workers = gridDim.x * WAVES;
  const unsigned per = (total + workers - 1) / workers;
  if ((unsigned long long)id * per >= total) return;
  const unsigned first = id * per, last = min(first + per, total);
  int b = last_from(a.B, first, [&](int i) { return plan.seq[i].block0; });
  PagedWave<DT, D, FMT, RT> w;
  unsigned x = first;
  while (x < last) {
    while (b + 1 < a.B && x >= same(plan.seq[b + 1].block0)) ++b;
    const SharedSeq* sp = plan.seq + b;
    const int nb = same(sp->nb);
    const OwnRows s = own_rows<TL::C8>(a, load_uniform(c.lens + b), c.n_valid ? load_uniform(c.n_valid + b) : c.n_new, same(sp->base), RW);
    const unsigned in = x - same(sp->block0);
    const int u = __builtin_amdgcn_readfirstlane(in / (unsigned)nb), blk = __builtin_amdgcn_readfirstlane(in - u * (unsigned)nb);
    const int blk_end = min(nb, blk + (int)(last - x));
    const int rg = u % s.groups, lh = u / s.groups, h = lh % a.Hkv, l = lh / a.Hkv;
    const int r0 = rg * RW, r_end = min(s.valid << a.log_g, r0 + RW);
    const int lo = s.start + (r0 >> a.log_g), hi = s.start + ((r_end - 1) >> a.log_g);
    w.clear();
    auto load_queries = [&]() {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        const int r = r0 + 16 * rt + col;
        const bool ok = r < r_end;
        const int t = ok ? r >> a.log_g : 0, hq = (h << a.log_g) + (ok ? r - (t << a.log_g) : 0);
        w.pos[rt] = ok ? s.start + t : -kMaxRows;
        load_query_row<DT, D, FMT, RT>(w, rt, a.q.at(l, b, hq, t), ok);
      }
    };
    const int i = blk * a.own_block, i_end = min(blk_end * a.own_block, s.all);
    walk_pages<DT, D, FMT, RT, 1>(w, a, c, b, l, h, s.pages, i, min(i_end, s.tiles), lo, hi, load_queries);
    if constexpr (TL::C8) walk_tail<DT, D, RT, 1>(w, a, c, b, l, h, s.full, s.rows, max(i - s.tiles, 0), i_end - s.tiles, lo, hi);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const float sum = column_sum(w.l[rt]);
      const int r = 16 * rt + col;
      if (r0 + r >= r_end) continue;
      write_part(w, rt, w.m[rt], sum, blk == 0 ? a.own.head + part_row(a, lh, b, r0 + r) * (D + kPartTail)
                                               : a.own.more + ((size_t)id * RW + r) * (D + kPartTail));
    }
    x += blk_end - blk;
  }
}

// Shared rows, then own ones: a workgroup that is done with its run of the shared rows goes on with own rows.
template <class DT, int D, int FMT, int RT, int OWN_RT>
__global__ __launch_bounds__(paged_waves(RT) * kWave) void k_shared_rows(SharedArgs a) {
  __shared__ PlanSpace space;
  const Plan plan = plan_of<FMT == MPC_PAGE_E4M3>(a, space);
  shared_rows<DT, D, FMT, RT>(a, plan);
  own_rows_of<DT, D, FMT, OWN_RT, paged_waves(RT)>(a, plan);
}
template <class DT, int D, int FMT>
hipError_t launch_narrow(const SharedArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)a.shared.workers);
  if constexpr (FMT != MPC_PAGE_SAME) {
    if (a.shared.unit_rows == 16) {  // (then a sequence's rows fit 16 too)
      hipLaunchKernelGGL((k_shared_rows<DT, D, FMT, 1, 1>), grid, dim3(paged_waves(1) * kWave), 0, st, a);
      return hipGetLastError();
    }
  }
  if (a.own.unit_rows == 16)
    hipLaunchKernelGGL((k_shared_rows<DT, D, FMT, 2, 1>), grid, dim3(paged_waves(2) * kWave), 0, st, a);
  else
    hipLaunchKernelGGL((k_shared_rows<DT, D, FMT, 2, 2>), grid, dim3(paged_waves(2) * kWave), 0, st, a);
  return hipGetLastError();
}

}  // namespace dev
}  // namespace mpc
