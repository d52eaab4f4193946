// Attention behind shared rows: sizes, and the plan of a call, made on the device from the groups and the lengths.
#include <algorithm>

#include "paged_dev.h"

namespace mpc {
namespace {

using namespace dev;
constexpr int kPlanThreads = 1024;

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
__global__ __launch_bounds__(kPlanThreads) void k_shared_plan(PagedAttnArgs a) {
  __shared__ int s_f[kMaxGroups + 1], s_base[kMaxGroups], s_lo[kMaxGroups], s_hi[kMaxGroups];
  __shared__ unsigned s_wave[kPlanThreads / kWave];
  const PagedCache& c = a.c;
  const SharedArgs& sh = a.sh;
  const int tid = threadIdx.x, ng = sh.groups;
  const int mine = tid < ng ? min(max(sh.first[tid], 0), a.B) : 0;
  s_f[tid] = mine;
  __syncthreads();
  for (int o = 1; o < ng; o <<= 1) {
    const int y = tid >= o ? s_f[tid - o] : 0;
    __syncthreads();
    s_f[tid] = max(s_f[tid], y);
    __syncthreads();
  }
  if (tid == 0) s_f[ng] = max(s_f[ng - 1], min(max(sh.first[ng], 0), a.B));
  if (tid < ng) {
    s_base[tid] = min(max(sh.rows[tid], 0), c.cap()) & ~(c.page - 1);
    s_lo[tid] = kMaxRows;
    s_hi[tid] = -1;
  }
  __syncthreads();
  for (int b = tid; b < a.B; b += kPlanThreads) {
    int g = -1;
    if (b >= s_f[0] && b < s_f[ng]) {  // the last group that begins at or before b
      int z = ng;
      for (g = 0; z - g > 1;) {
        const int m = (g + z) / 2;
        (s_f[m] <= b ? g : z) = m;
      }
      const int valid = c.valid(b), len = c.len(b);
      if (valid > 0) {
        atomicMin(&s_lo[g], len - valid);
        atomicMax(&s_hi[g], len - 1);
      }
    }
    sh.seq[b] = make_int2(g < 0 ? 0 : s_base[g], g);
  }
  __syncthreads();
  SharedGroup p{};
  if (tid < ng) {
    p.f0 = s_f[tid];
    p.f1 = s_f[tid + 1];
    p.base = s_base[tid];
    const long long rows = (long long)(p.f1 - p.f0) * ((long long)c.n_new << a.log_g);
    p.rt = (int)((rows + sh.unit_rows - 1) / sh.unit_rows);
    const int all = (max(0, min(p.base, s_hi[tid] + 1)) + sh.tile - 1) / sh.tile;
    p.skip = p.at = all;
    if (a.window) {
      p.skip = min((a.sinks + sh.tile - 1) / sh.tile, all);
      p.at = max(p.skip, min(max(s_lo[tid] - a.window + 1, 0) / sh.tile, all));
    }
    p.tiles = p.skip + all - p.at;
    p.nb = (p.tiles + sh.per_block - 1) / sh.per_block;
  }
  const unsigned units = p.nb > 0 ? (unsigned)(p.rt * a.L * a.Hkv) : 0;
  unsigned total, n;
  p.block0 = sum_before(units * (unsigned)p.nb, s_wave, &total);
  p.unit0 = sum_before(units, s_wave, &n);
  if (tid < ng) sh.plan[tid] = p;
  if (tid == 0) *sh.total = total;
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

// Units of as many query rows as a group has on average, up to 32.
SharedPlan shared_plan(int dtype, int D, int L, int B, int Hq, int Hkv, int n, int cap, int groups) {
  SharedPlan p{};
  p.own = paged_plan(dtype, D, L, B, Hq, Hkv, n, cap);
  const long long rows = (long long)B * n * (Hq / Hkv), each = (rows + groups - 1) / groups;
  p.unit_rows = each <= 16 ? 16 : 32;
  p.tile = dtype == MPC_FP32 ? 16 : 32;
  p.per_block = paged_waves(p.unit_rows / 16);
  p.grid = kNumCU;
  const long long units = ((long long)rows / p.unit_rows + groups) * L * Hkv;
  const long long nb = cap / (p.tile * p.per_block) + 1;
  p.blocks = (double)units * (double)nb >= 2147483648.0 || p.own.blocks >= 1ll << 31 ? 1ll << 31 : units * nb;
  p.total = align256(p.own.ws_bytes);
  p.plan = p.total + 256;
  p.seq = p.plan + align256((size_t)groups * sizeof(SharedGroup));
  p.unit = p.seq + align256((size_t)B * sizeof(int2));
  p.head = p.unit + align256((size_t)units * sizeof(int2));
  p.more = p.head + align256((size_t)L * Hkv * rows * (D + 2) * sizeof(float));
  p.ws_bytes = p.more + (size_t)p.grid * p.unit_rows * (D + 2) * sizeof(float);
  return p;
}

hipError_t launch_shared_attn(const PagedAttnArgs& a, int dtype, int D, hipStream_t st) {
  hipLaunchKernelGGL(k_shared_plan, dim3(1), dim3(kPlanThreads), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.c.format == MPC_PAGE_MX4) return launch_shared_mx4(a, dtype, D, st);
  if (dtype == MPC_FP32) return launch_shared_fp32(a, D, st);
  return dtype == MPC_FP16 ? launch_shared_fp16(a, D, st) : launch_shared_bf16(a, D, st);
}

}  // namespace mpc
