// Launch interface of the paged-cache append and of the attention over paged or plain keys.
#pragma once
#include "common.h"

namespace mpc {

constexpr int kMaxRows = 1 << 30;  // rows of a sequence, and new tokens of a call
constexpr int kMx4Block = 32;      // channels to a scale of 4-bit codes

// A tensor [L][B][H][n][d]: byte strides of the first four axes.
struct Rows {
  char* p;
  int64_t layer, batch, head, token;
  __host__ __device__ char* at(int l, int b, int h, int t) const {
    return p + l * layer + b * batch + h * head + t * token;
  }
};

// The cache of a call, with the sequence lengths and the new tokens of each sequence.
struct PagedCache {
  char *k, *v;            // pages
  float *ks, *vs;         // page scales (8-bit codes), or null
  uint8_t *kx, *vx;       // exponents of a row's scales (4-bit codes), or null
  char *k_tail, *v_tail;  // rings, or null
  const int32_t *table, *lens, *n_valid;
  int page, log_page, n_pages, max_pages, format;
  int L, B, Hkv, n_new;

  __device__ int cap() const { return max_pages * page; }
  __device__ int valid(int b) const { return n_valid ? min(max(n_valid[b], 0), n_new) : n_new; }
  // rows of sequence b, clamped so that sums with row counts stay in 32 bits
  __device__ int len(int b) const { return min(max(lens[b], 0), kMaxRows); }
};

struct RopeArgs {
  const float2* table;  // null: no rotation
  int n_pos, rot, half;
};

struct PagedAppendArgs {
  PagedCache c;
  RopeArgs rope;
  const int32_t* pos0;
  Rows k, v, q, q_out, k_out;  // k_out.p null: not asked for
  int Hq;        // 0 without queries
  int np;        // pages that the new tokens of one sequence can touch
};
hipError_t launch_paged_append(const PagedAppendArgs& a, int dtype, int D, hipStream_t st);

// Rows first[b] + t (null: the newest ones) of the cache, as rows of the element type.
struct PagedReadArgs {
  PagedCache c;
  const int32_t* first;
  Rows k, v;  // p null: not asked for
};
hipError_t launch_paged_read(const PagedReadArgs& a, int dtype, int D, hipStream_t st);

struct AttnArgs {
  Rows q, out;
  float* lse;  // [L][B][Hq][n] or null
  int L, B, Hq, Hkv, n;
  int window, sinks;
  float qscale;  // sm_scale * log2(e)
};

// Waves of a workgroup of the paged attention: eight where a wave may take half of a SIMD's registers, four where it takes
// all of them.
__host__ __device__ constexpr int paged_waves(int row_tiles) { return row_tiles == 1 ? 8 : 4; }

// Attention behind shared rows: the sequences of a group look at the first rows of the group's first sequence, which a kernel of
// its own takes for all of them (k_shared_rows); each sequence's other rows, and the join, are the paged attention's.
// What the first launch (k_shared_plan) makes of a group: sequences [f0, f1), shared rows [0, base), their tiles [0, skip) and
// from `at` on, blocks of keys nb (0: nothing to look at), units of query rows rt to a (layer, kv head); the blocks and units
// of the groups before it.
struct SharedGroup {
  int f0, f1, base, skip, at, tiles, nb, rt;
  unsigned block0, unit0;
};
constexpr int kMaxGroups = 1024;
struct SharedArgs {
  const int32_t *first, *rows;
  int groups;
  SharedGroup* plan;
  unsigned* total;   // blocks of all groups
  int2* seq;         // of each sequence: shared rows, group
  int2* unit;        // of each unit of the shared rows: its first workgroup, and how many share it
  float* head;       // [L][Hkv][B][n G][D + 2]: what a unit's first workgroup has of each row: accumulator, maximum, sum
  float* more;       // [grid][unit rows][D + 2]: and each of its other workgroups
  int unit_rows, grid, tile, per_block;  // tile: keys; per_block: tiles of a block
};

struct PagedAttnArgs : AttnArgs {
  PagedCache c;
  SharedArgs sh;
  int* cnt;       // arrivals at a shared unit, by its first workgroup; zero between launches
  float* part;    // [grid][2][part_rows][D + 2]: accumulator, maximum and sum of a unit's part
  int row_tiles;  // 16-row tiles of a unit
  int log_g;      // G = 2^log_g
  int part_rows, grid;
};
struct PagedPlan {
  int row_tiles, part_rows, grid;
  long long blocks;  // at most, for sequences as long as the table
  size_t ws_bytes;   // counters, then parts
};
// Bytes of the arrival counters: a workgroup is the first one of at most one unit that others share (one that goes on behind
// its run), so there is a counter to each, at the same place in every call.
constexpr size_t kPagedCntBytes = kNumCU * sizeof(int);
PagedPlan paged_plan(int dtype, int D, int L, int B, int Hq, int Hkv, int n, int cap);
hipError_t launch_paged_attn_fp32(const PagedAttnArgs& a, int D, hipStream_t st);
hipError_t launch_paged_attn_fp16(const PagedAttnArgs& a, int D, hipStream_t st);
hipError_t launch_paged_attn_bf16(const PagedAttnArgs& a, int D, hipStream_t st);
hipError_t launch_paged_attn_mx4(const PagedAttnArgs& a, int dtype, int D, hipStream_t st);
hipError_t launch_paged_attn(const PagedAttnArgs& a, int dtype, int D, hipStream_t st);

// Sizes of a call behind shared rows, and its workspace: that of the paged attention, then plan, sequences, units and parts.
struct SharedPlan {
  PagedPlan own;
  int unit_rows, grid, tile, per_block;
  long long blocks;
  size_t total, plan, seq, unit, head, more, ws_bytes;
};
SharedPlan shared_plan(int dtype, int D, int L, int B, int Hq, int Hkv, int n, int cap, int groups);
hipError_t launch_shared_fp32(const PagedAttnArgs& a, int D, hipStream_t st);
hipError_t launch_shared_fp16(const PagedAttnArgs& a, int D, hipStream_t st);
hipError_t launch_shared_bf16(const PagedAttnArgs& a, int D, hipStream_t st);
hipError_t launch_shared_mx4(const PagedAttnArgs& a, int dtype, int D, hipStream_t st);
hipError_t launch_shared_attn(const PagedAttnArgs& a, int dtype, int D, hipStream_t st);

struct PromptAttnArgs : AttnArgs {
  Rows k, v;
  const int32_t *q_lens, *k_lens;
  int T;
};
hipError_t launch_prompt_attn(const PromptAttnArgs& a, int dtype, int D, hipStream_t st);

}  // namespace mpc
