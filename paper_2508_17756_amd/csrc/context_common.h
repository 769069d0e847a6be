// Shared by the kernels of sg_tile_cross_attention and sg_tile_prefix_attention: what a call attends, how the work is numbered, and the
// addressing of queries and keys.
//
//     o[a][n] = sum_m p_m V[a'][m],   p = softmax over m of scale * <Q[a][n], K[a'][m]>,   a' = a / group
//
// over one or two segments of keys: segment 0 is the prefix that all tiles share, segment 1 the tile's own keys (of a cross attention:
// its context).  The group = heads / kv_heads query heads that read the same keys are stacked: a "row" is a (head of the group, token)
// pair of one tile and one head of keys, rows = group * tokens of them, so that grouped heads fill the tiles of the matrix instruction.
//
// A key that does not count (at or behind the segment's length, or masked) has its score set to -inf, and its key and value rows
// are never read: the transfer takes zeros in their place, so that a NaN or an infinity there does not become 0 * inf.
// A row without any key ends with a sum of 0 and gives zeros.
#pragma once
#include "attention_common.h"

namespace sg {

constexpr int kCtxTilesPerLaunch = 64;
struct CtxTable {
  const void* q[kCtxTilesPerLaunch];
  const void* k[kCtxTilesPerLaunch];   // segment 1
  const void* v[kCtxTilesPerLaunch];
  void* out[kCtxTilesPerLaunch];
};

// One way of numbering (rows, shares of the keys): `items` workgroups.  Stacked: the rows of all tiles behind one another over segment 0 alone.
struct CtxPart {
  int32_t items;
  int32_t batches;       // tiles, or 1 if stacked
  int32_t rows;          // rows of a batch and head of keys
  int32_t row_blocks;    // groups of row blocks (what one workgroup takes) of a batch and head of keys
  int32_t splits;        // shares of the keys taken by different workgroups
  int32_t ways;          // shares of the keys inside a workgroup (its other wavefronts take other row blocks): 1, 2, 4
  int32_t first_share;   // place of its first share among the shares that are joined
  int32_t seg0, seg1;    // segments it attends
  int32_t stacked;
};

struct CtxArgs {
  int64_t q_token, q_head, o_token, o_head;   // strides in elements
  int64_t kv_token[2], kv_head[2];            // of the segments
  const void* k0;
  const void* v0;
  const int32_t* len0;    // device, 1 or nullptr
  const int32_t* len1;    // device, n_tiles or nullptr
  const uint8_t* mask1;   // device, [n_tiles][cap1] or nullptr
  const uint8_t* run;     // device, n_tiles or nullptr
  float* shares;          // workspace: [row][share][head_dim] sums of p v, then [row][share][2] (reference, sum of p)
  int32_t cap0, cap1;     // rows in the buffers
  int32_t heads, kv_heads, group, tokens, n_tiles;
  int32_t n_shares;       // per row; 1: the result is written directly
  float scale;
  CtxPart part[2];
};

// Rows that no key transfer may read: the source of what is not to count.
static __device__ const uint4 g_ctx_zeros[16] = {};

__device__ __forceinline__ int ctx_length(const int32_t* len, int i, int cap) {
  if (!len) return cap;
  const int n = len[i];
  return n < 0 ? 0 : (n > cap ? cap : n);
}
// Workgroups are dealt round-robin to the 8 XCDs; renumbered so that each XCD walks a contiguous range of the work and what reads the
// same keys shares one L2.  -1: nothing left.
__device__ __forceinline__ int ctx_xcd_order(int block, int total) {
  const int per = (total + 7) / 8, id = (block & 7) * per + (block >> 3);
  return (block >> 3) < per && id < total ? id : -1;
}
// index of the a-th set bit of mask (a < popcount(mask))
__device__ __forceinline__ int ctx_nth_tile(uint64_t mask, int a) {
  for (int i = 0; i < a; ++i) mask &= mask - 1;
  return __builtin_ctzll(mask);
}

struct CtxRow {
  int tile, head, token;   // head: of the queries
  int rid;                 // row among the launch's rows: its place in the workspace
  bool there;              // a row of the batch whose tile runs
};
__device__ __forceinline__ CtxRow ctx_row(const CtxArgs& a, const CtxPart& p, int batch, int kvh, int row) {
  CtxRow r;
  r.there = row < p.rows;
  const int c = r.there ? row : p.rows - 1;
  const int per = a.group * a.tokens;
  r.tile = p.stacked ? c / per : batch;
  const int in = p.stacked ? c - r.tile * per : c;
  const int g = in / a.tokens;
  r.token = in - g * a.tokens;
  r.head = kvh * a.group + g;
  r.rid = (r.tile * a.kv_heads + kvh) * per + in;
  if (p.stacked && a.run) r.there = r.there && a.run[r.tile] != 0;
  return r;
}

// ---------------------------------------------------------------------------------------------------- host side
// The launches of one call (at most kCtxTilesPerLaunch tiles each) and what they need of the workspace.
struct CtxPlan {
  bool wide;             // workgroups of 128 rows share their keys in LDS, nothing is split
  int32_t wave_rows;     // otherwise rows of a wavefront: 32 (fp32: or 16)
  int32_t n_shares;
  CtxPart part[2];
  size_t bytes;          // workspace
};
CtxPlan plan_context(const sg_context_problem& p, bool prefix, int n_tiles);
int launch_context_bf16_wide(const CtxArgs& a, const CtxTable& tab, int head_dim, hipStream_t s);
int launch_context_bf16_split(const CtxArgs& a, const CtxTable& tab, int head_dim, hipStream_t s);
int launch_context_f32(const CtxArgs& a, const CtxTable& tab, const CtxPlan& plan, int head_dim, hipStream_t s);
int launch_context_join(const CtxArgs& a, const CtxTable& tab, int head_dim, int dtype, hipStream_t s);

}  // namespace sg
