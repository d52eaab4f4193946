// Attention behind shared rows: sizes, the plan of a call, made on the device from the groups and the lengths, and the join.
#include <algorithm>

#include "shared_attn_dev.h"

namespace mpc {
namespace {

using namespace dev;
constexpr int kPlanThreads = 1024, kJoinThreads = 256;

// Sum of x over the threads before this one, and over all of them.
__device__ __forceinline__ unsigned sum_before(unsigned x, unsigned* s_wave, unsigned* total) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  unsigned sum = x;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const unsigned y = __shfl_up(sum, o);
    if (lane >= o) sum += y;
  }
  if (lane == kWave - 1) s_wave[wave] = sum;
  __syncthreads();
  unsigned before = 0, all = 0;
  for (int w = 0; w < kPlanThreads / kWave; ++w) {
    before += w < wave ? s_wave[w] : 0;
    all += s_wave[w];
  }
  __syncthreads();
  *total = all;
  return before + sum - x;
}

// One workgroup: a thread to a group, and the sequences over the threads. Bounds of the groups are brought into [0, B] and in
// order, so that every sequence is in one group at most, whatever `first` holds.
template <bool C8>
__global__ __launch_bounds__(kPlanThreads) void k_shared_plan(SharedArgs a) {
  __shared__ int s_f[kMaxGroups + 1], s_base[kMaxGroups], s_lo[kMaxGroups], s_hi[kMaxGroups];
  __shared__ unsigned s_wave[kPlanThreads / kWave];
  const PagedCache& c = a.c;
  const int tid = threadIdx.x, ng = a.groups;
  s_f[tid] = tid < ng ? min(max(a.first[tid], 0), a.B) : 0;
  __syncthreads();
  for (int o = 1; o < ng; o <<= 1) {
    const int y = tid >= o ? s_f[tid - o] : 0;
    __syncthreads();
    s_f[tid] = max(s_f[tid], y);
    __syncthreads();
  }
  if (tid == 0) s_f[ng] = max(s_f[ng - 1], min(max(a.first[ng], 0), a.B));
  if (tid < ng) {
    s_base[tid] = min(max(a.rows[tid], 0), c.cap()) & ~(c.page - 1);
    s_lo[tid] = kMaxRows;
    s_hi[tid] = -1;
  }
  __syncthreads();
  unsigned own = 0;  // blocks of the sequences so far
  for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
    const int b = b0 + tid;
    SharedSeq q{0, -1, 0, 0};
    unsigned blocks = 0;
    if (b < a.B) {
      if (b >= s_f[0] && b < s_f[ng]) {  // the last group that begins at or before b
        int g = 0, z = ng;
        while (z - g > 1) {
          const int m = (g + z) / 2;
          (s_f[m] <= b ? g : z) = m;
        }
        q.group = g;
        q.base = s_base[g];
      }
      const OwnRows s = own_rows<C8>(a, c.lens[b], c.n_valid ? c.n_valid[b] : c.n_new, q.base, a.own.unit_rows);
      if (q.group >= 0 && s.valid > 0) {
        atomicMin(&s_lo[q.group], s.start);
        atomicMax(&s_hi[q.group], s.len - 1);
      }
      q.nb = (s.all + a.own_block - 1) / a.own_block;
      blocks = (unsigned)(s.groups * a.L * a.Hkv) * (unsigned)q.nb;
    }
    unsigned all;
    q.block0 = own + sum_before(blocks, s_wave, &all);
    own += all;
    if (b < a.B) a.seq[b] = q;
  }
  __syncthreads();
  SharedGroup p{};
  if (tid < ng) {
    p.f0 = s_f[tid];
    p.f1 = s_f[tid + 1];
    p.base = s_base[tid];
    const long long rows = (long long)(p.f1 - p.f0) * ((long long)c.n_new << a.log_g);
    p.rt = (int)((rows + a.shared.unit_rows - 1) / a.shared.unit_rows);
    const int all = (max(0, min(p.base, s_hi[tid] + 1)) + a.tile - 1) / a.tile;
    p.skip = p.at = all;
    if (a.window) {
      p.skip = min((a.sinks + a.tile - 1) / a.tile, all);
      p.at = max(p.skip, min(max(s_lo[tid] - a.window + 1, 0) / a.tile, all));
    }
    p.tiles = p.skip + all - p.at;
    p.nb = (p.tiles + a.shared_block - 1) / a.shared_block;
  }
  unsigned total;
  p.block0 = sum_before((unsigned)(p.rt * a.L * a.Hkv) * (unsigned)p.nb, s_wave, &total);
  if (tid < ng) a.group[tid] = p;
  if (tid == 0) *a.total = SharedTotals{total, own};
}

// The join: a wave to a query row, whose parts are those of its own rows and of the shared ones.
template <class DT, int D>
__global__ __launch_bounds__(kJoinThreads) void k_shared_join(SharedArgs a) {
  constexpr int PS = D + kPartTail;
  const PagedCache& c = a.c;
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int per = c.n_new << a.log_g;
  const long long row = (long long)blockIdx.x * (kJoinThreads / kWave) + wave;
  if (row >= (long long)a.L * a.Hkv * a.B * per) return;
  const int in_seq = (int)(row % per), lhb = (int)(row / per), b = lhb % a.B, lh = lhb / a.B;
  const int t = in_seq >> a.log_g, valid = c.n_valid ? min(max(load_uniform(c.n_valid + b), 0), c.n_new) : c.n_new;
  if (t >= valid) return;
  // the parts of a unit: its first worker's, then those of the workers that go on with it
  struct Side {
    const float *head, *more;
    int n;
  };
  auto side = [&](const Parts& p, unsigned total, unsigned x0, int nb, int in_unit) {
    Side s{p.head + row * PS, nullptr, 0};
    if (nb > 0) {
      const unsigned share = (total + p.workers - 1) / p.workers, w0 = x0 / share, w1 = (x0 + nb - 1) / share;
      s.more = p.more + ((size_t)w0 * p.unit_rows + in_unit) * PS;
      s.n = (int)(w1 - w0) + 1;
    }
    return s;
  };
  const SharedSeq* sp = a.seq + b;
  const int gi = load_uniform(&sp->group), nb = load_uniform(&sp->nb);
  const unsigned own_total = load_uniform(&a.total->own), shared_total = load_uniform(&a.total->shared);
  const int units = ((valid << a.log_g) + a.own.unit_rows - 1) / a.own.unit_rows;
  const Side o = side(a.own, own_total, load_uniform(&sp->block0) + (unsigned)(lh * units + in_seq / a.own.unit_rows) * (unsigned)nb, nb,
                      in_seq % a.own.unit_rows);
  Side s{nullptr, nullptr, 0};
  if (gi >= 0) {
    const SharedGroup* gp = a.group + gi;
    const int gb = load_uniform(&gp->nb), in_group = (b - load_uniform(&gp->f0)) * per + in_seq;
    const unsigned u = (unsigned)(lh * load_uniform(&gp->rt) + in_group / a.shared.unit_rows);
    s = side(a.shared, shared_total, load_uniform(&gp->block0) + u * (unsigned)gb, gb, in_group % a.shared.unit_rows);
  }
  const int all = o.n + s.n;
  auto at = [&](int n) {
    const bool own = n < o.n;
    const int k = own ? n : n - o.n;
    const Parts& p = own ? a.own : a.shared;
    return k == 0 ? (own ? o.head : s.head) : (own ? o.more : s.more) + (size_t)k * p.unit_rows * PS;
  };
  // a lane to a part: the row's reference and sum
  float mx = -INFINITY, sum = 0.f;
  for (int n = lane; n < all; n += kWave) {
    const float2 ml = *(const float2*)(at(n) + D);
    const float top = fmaxf(mx, ml.x), ref = top == -INFINITY ? 0.f : top;
    sum = sum * fast_exp2(mx - ref) + ml.y * fast_exp2(ml.x - ref);
    mx = top;
  }
  float top = mx;
#pragma unroll
  for (int i = 32; i > 0; i >>= 1) top = fmaxf(top, __shfl_xor(top, i));
  const float ref = top == -INFINITY ? 0.f : top;
  sum = wave_sum(sum * fast_exp2(mx - ref));
  // a lane to two channels, all parts; d 64: half of the lanes to every second part
  constexpr int WAYS = 128 / D, AHEAD = 8;
  const int way = lane / (D / 2), e = lane % (D / 2) * 2;
  float x0 = 0.f, x1 = 0.f;
  for (int c0 = 0; c0 < all; c0 += kWave) {
    const float f = c0 + lane < all ? fast_exp2(at(c0 + lane)[D] - ref) : 0.f;
    const int m = min(all - c0, kWave);
    for (int n0 = 0; n0 < m; n0 += AHEAD * WAYS) {
      float2 y[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) y[k] = *(const float2*)(at(c0 + min(n0 + k * WAYS + way, m - 1)) + e);
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        const int n = n0 + k * WAYS + way;
        const float fn = __shfl(f, min(n, kWave - 1));
        if (n < m) {
          x0 = fmaf(y[k].x, fn, x0);
          x1 = fmaf(y[k].y, fn, x1);
        }
      }
    }
  }
  if constexpr (WAYS == 2) {
    x0 += __shfl_xor(x0, 32);
    x1 += __shfl_xor(x1, 32);
  }
  if (way > 0) return;
  const int h = lh % a.Hkv, l = lh / a.Hkv, hq = (h << a.log_g) + in_seq - (t << a.log_g);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  char* out = a.out.at(l, b, hq, t) + e * DT::kElt;
  x0 = sum == 0.f ? 0.f : x0 * inv;
  x1 = sum == 0.f ? 0.f : x1 * inv;
  if constexpr (DT::kElt == 4)
    *(float2*)out = make_float2(x0, x1);
  else
    *(uint32_t*)out = pack2<DT>(x0, x1);
  if (e == 0 && a.lse)
    a.lse[(((size_t)l * a.B + b) * a.Hq + hq) * a.n + t] = sum == 0.f ? -INFINITY : (ref + __log2f(sum)) * 0.69314718055994531f;
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

template <class DT>
hipError_t launch_join(const SharedArgs& a, int D, hipStream_t st) {
  const long long rows = (long long)a.L * a.Hkv * a.B * ((long long)a.c.n_new << a.log_g);
  const dim3 grid((unsigned)((rows + kJoinThreads / kWave - 1) / (kJoinThreads / kWave)));
  if (D == 64)
    hipLaunchKernelGGL((k_shared_join<DT, 64>), grid, dim3(kJoinThreads), 0, st, a);
  else
    hipLaunchKernelGGL((k_shared_join<DT, 128>), grid, dim3(kJoinThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace

// Units of as many query rows as a group has on average, up to 32, and of 128 in 16-bit types beyond that; own rows in units of 16 where a sequence's fit, else 32. Blocks
// are a tile to each wave of a workgroup (shared rows), and 128 keys to a wave (own rows).
SharedPlan shared_plan(int dtype, int D, int L, int B, int Hq, int Hkv, int n, int cap, int groups) {
  SharedPlan p{};
  const long long each_seq = (long long)n * (Hq / Hkv), rows = B * each_seq, each = (rows + groups - 1) / groups, lh = (long long)L * Hkv;
  p.wide = dtype != MPC_FP32 && each > 32;
  p.shared_rows = p.wide ? 128 : each <= 16 ? 16 : 32;
  p.own_rows = each_seq <= 16 ? 16 : 32;
  p.tile = dtype == MPC_FP32 ? 16 : 32;
  p.shared_block = p.wide ? 4 * kWideGroups : paged_waves(p.shared_rows / 16);
  p.own_block = 128 / p.tile;
  p.shared_workers = p.wide ? kNumCU * 2 / kWideGroups : kNumCU;
  p.own_workers = kNumCU * kOwnWaves * (p.own_rows == 16 ? 2 : 1);
  auto blocks = [&](long long units, long long block) {
    const double nb = cap / (p.tile * block) + 2;  // complete pages' tiles and the ring's may each be cut short
    return (double)units * nb >= 2147483648.0 ? 1ll << 31 : units * (long long)nb;
  };
  p.blocks = std::max(blocks((rows / p.shared_rows + groups) * lh, p.shared_block),
                      blocks(B * ((each_seq + p.own_rows - 1) / p.own_rows) * lh, p.own_block));
  const size_t row = (D + kPartTail) * sizeof(float), heads = align256((size_t)lh * rows * row);
  p.total = kPagedCntBytes;  // behind the counters of the paged attention, which a workspace of this serves too
  p.group = p.total + align256(sizeof(SharedTotals));
  p.seq = p.group + align256((size_t)groups * sizeof(SharedGroup));
  p.shared_head = p.seq + align256((size_t)B * sizeof(SharedSeq));
  p.shared_more = p.shared_head + heads;
  p.own_head = p.shared_more + align256((size_t)p.shared_workers * p.shared_rows * row);
  p.own_more = p.own_head + heads;
  p.ws_bytes = std::max(p.own_more + (size_t)p.own_workers * p.own_rows * row, paged_plan(dtype, D, L, B, Hq, Hkv, n, cap).ws_bytes);
  return p;
}

hipError_t launch_shared_attn(const SharedArgs& a, int dtype, int D, hipStream_t st) {
  if (a.c.format == MPC_PAGE_E4M3)
    hipLaunchKernelGGL(k_shared_plan<true>, dim3(1), dim3(kPlanThreads), 0, st, a);
  else
    hipLaunchKernelGGL(k_shared_plan<false>, dim3(1), dim3(kPlanThreads), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  e = a.c.format == MPC_PAGE_MX4 ? launch_shared_mx4(a, dtype, D, st)
      : dtype == MPC_FP32        ? launch_shared_fp32(a, D, st)
      : dtype == MPC_FP16        ? launch_shared_fp16(a, D, st)
                                 : launch_shared_bf16(a, D, st);
  if (e != hipSuccess) return e;
  if (dtype == MPC_FP32) return launch_join<F32>(a, D, st);
  return dtype == MPC_FP16 ? launch_join<F16>(a, D, st) : launch_join<BF16>(a, D, st);
}

}  // namespace mpc
