// Attention of new tokens over a paged cache: how the work is laid out (paged_attn_dev.h has the kernel).
#include <algorithm>

#include "paged.h"

namespace mpc {

// Units of one 16-row tile where the rows fit, else of two. The grid is one workgroup to a compute unit (eight waves, what
// the registers allow), or fewer where even the longest sequences have fewer blocks. Runs of a single block are taken too: a
// wave's second tile costs as much as joining the parts (one sequence of 500 rows, 12 heads of 64: 11.5 us, with runs of at
// least four blocks 12.0; 32 heads over 8 behind a window of 1024: 13.5 and 22.8; four sequences of drafts behind it: 20.2
// and 33.0).
PagedPlan paged_plan(int dtype, int D, int L, int B, int Hq, int Hkv, int n, int cap) {
  PagedPlan p{};
  const long long rows = (long long)(Hq / Hkv) * n;
  p.row_tiles = rows > 16 ? 2 : 1;
  const int unit_rows = 16 * p.row_tiles;
  const long long groups = (rows + unit_rows - 1) / unit_rows;
  p.part_rows = (int)std::min<long long>(rows, unit_rows);
  const int tile = dtype == MPC_FP32 ? 16 : 32;
  const long long nb = cap / (tile * paged_waves(p.row_tiles)) + 2;  // complete pages' tiles and the tail's may each be cut short
  const long long units = (long long)L * B * Hkv * groups;
  p.blocks = (double)units * (double)nb >= 2147483648.0 ? 1ll << 31 : units * nb;
  p.grid = (int)std::min<long long>(kNumCU, p.blocks);
  // for the largest grid, so that a workspace made for the most rows serves calls of fewer, and every cache
  p.ws_bytes = kPagedCntBytes + (size_t)kNumCU * 2 * p.part_rows * (D + 2) * sizeof(float);
  return p;
}

hipError_t launch_paged_attn(const PagedAttnArgs& a, int dtype, int D, hipStream_t st) {
  if (a.c.format == MPC_PAGE_MX4) return launch_paged_attn_mx4(a, dtype, D, st);
  if (dtype == MPC_FP32) return launch_paged_attn_fp32(a, D, st);
  return dtype == MPC_FP16 ? launch_paged_attn_fp16(a, D, st) : launch_paged_attn_bf16(a, D, st);
}

}  // namespace mpc
