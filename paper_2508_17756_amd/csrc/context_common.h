// Shared by the kernels of sg_tile_cross_attention and sg_tile_prefix_attention: what a call attends, how the work is numbered, and the
// addressing of queries and keys.
//
//     o[a][n] = sum_m p_m V[a'][m],   p = softmax over m of scale * <Q[a][n], K[a'][m]>,   a' = a / group
//
// over one or two segments of keys: segment 0 is the prefix that all tiles share, segment 1 the tile's own keys (of a cross attention:
// its context).  The group = heads / kv_heads query heads that read the same keys are stacked: a "row" is a (head of the group, token)
// pair of one tile and one head of keys, rows = group * tokens of them, so that grouped heads fill the tiles of the matrix instruction.
//
// A key that does not count (at or behind the segment's length, or masked) has its score set to -inf.  Its value row is never read: the transfer
// takes zeros in its place, so that a NaN or an infinity there does not become 0 * inf; nor is its key row, but for masked keys inside
// the length in the bf16 kernel of shared stages, which come along with the others (a score that is replaced may be anything).
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

// One launch's work: (rows, shares of the keys) in `items` workgroups.
struct CtxPart {
  int32_t items;
  int32_t rows;          // of a batch and head of keys; a batch is a tile, or all tiles if stacked
  int32_t row_blocks;    // what one workgroup takes of them
  int32_t splits;        // shares of the keys taken by different workgroups
  int32_t ways;          // shares of the keys inside a workgroup (its other wavefronts take other row blocks): 1, 2, 4
  int32_t first_share;   // place of its first share among a row's shares in the workspace
  int32_t prior;         // shares of a row that an earlier launch left there and this one joins with its own: its results are final
  int32_t seg0, seg1;    // segments it attends
  int32_t stacked;       // the rows of all tiles behind one another
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
  int32_t n_shares;       // per row, in the workspace; 0: none, results are written directly
  float scale;
  Divisor by_tokens, by_rows;   // tokens, group * tokens
  CtxPart part;
};

// Rows that no key transfer may read: the source of what is not to count.
static __device__ const uint4 g_ctx_zeros[16] = {};

__device__ __forceinline__ int ctx_length(const int32_t* len, int i, int cap) {
  if (!len) return cap;
  const int n = len[i];
  return n < 0 ? 0 : (n > cap ? cap : n);
}
// The keys of one segment, of one tile and head of keys, as stages are taken from them; BYTES: of an element.
struct CtxSegment {
  const char* k;    // head's first key
  const char* v;
  uint32_t token;   // bytes between keys
  int len;
  const uint8_t* mask;
};
template <int BYTES>
__device__ __forceinline__ CtxSegment ctx_segment(const CtxArgs& a, const CtxTable& tab, int which, int tile, int kvh) {
  CtxSegment g;
  const void* const k = which == 0 ? a.k0 : tab.k[tile];
  const void* const v = which == 0 ? a.v0 : tab.v[tile];
  const int64_t head = (int64_t)kvh * a.kv_head[which] * BYTES;
  g.k = (const char*)k + head;
  g.v = (const char*)v + head;
  g.token = (uint32_t)(a.kv_token[which] * BYTES);
  g.len = which == 0 ? ctx_length(a.len0, 0, a.cap0) : ctx_length(a.len1, tile, a.cap1);
  g.mask = (which == 1 && a.mask1) ? a.mask1 + (int64_t)tile * a.cap1 : nullptr;
  return g;
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

// What a workgroup of the kernels with shared stages takes.  Only the tiles that run are numbered, so that the work is spread evenly whichever they
// are and the rest of the grid exits at once.  False: nothing.
struct CtxItem {
  int tile, kvh, split, row_block;
};
__device__ __forceinline__ bool ctx_shared_item(const CtxArgs& a, const CtxPart& p, CtxItem& item) {
  const int lane = threadIdx.x & 63;
  uint64_t active = p.stacked ? 1 : a.n_tiles >= 64 ? ~0ull : (1ull << a.n_tiles) - 1;
  if (a.run && !p.stacked) active = __ballot(lane < a.n_tiles && a.run[lane < a.n_tiles ? lane : 0] != 0);
  const int per_head = p.splits * p.row_blocks, per_tile = a.kv_heads * per_head;
  const int id = ctx_xcd_order((int)blockIdx.x, __builtin_popcountll(active) * per_tile);
  if (id < 0) return false;
  const int nth = id / per_tile, in_tile = id - nth * per_tile;
  item.tile = __builtin_amdgcn_readfirstlane(ctx_nth_tile(active, nth));
  item.kvh = __builtin_amdgcn_readfirstlane(in_tile / per_head);
  const int in_head = in_tile - item.kvh * per_head;
  item.split = __builtin_amdgcn_readfirstlane(in_head / p.row_blocks);
  item.row_block = in_head - item.split * p.row_blocks;
  return true;
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
  r.tile = p.stacked ? (int)divide((uint32_t)c, a.by_rows) : batch;
  const int in = p.stacked ? c - r.tile * per : c;
  const int g = (int)divide((uint32_t)in, a.by_tokens);
  r.token = in - g * a.tokens;
  r.head = kvh * a.group + g;
  r.rid = (r.tile * a.kv_heads + kvh) * per + in;
  if (p.stacked && a.run) r.there = r.there && a.run[r.tile] != 0;
  return r;
}
// What the end of a call needs of a row: found once (divisions), kept in registers over the keys, then passed on in LDS.
struct CtxRowEnd {
  uint64_t out;   // address of its output; 0: it is not there
  int rid;
};
template <typename T>
__device__ __forceinline__ CtxRowEnd ctx_row_end(const CtxArgs& a, const CtxTable& tab, const CtxRow& r) {
  T* const o = (T*)tab.out[r.tile] + (int64_t)r.head * a.o_head + (int64_t)r.token * a.o_token;
  return {r.there ? (uint64_t)(uintptr_t)o : 0, r.rid};
}

// What a share whose reference is `ref` counts against one of `top` >= ref.  bf16 keeps references in the log2 domain.  fp32 keeps the scores'
// own, of which only differences are multiplied by log2(e), so that scores up to the largest number stay finite, and takes the function that returns
// results below 2^-126: times a value near the largest number they still count.
constexpr float kLog2e = 1.4426950408889634f;
template <typename OUT>
__device__ __forceinline__ float ctx_weight(float ref, float top) {
  if constexpr (sizeof(OUT) == 4) return exp2f((ref - top) * kLog2e);
  else return __builtin_amdgcn_exp2f(ref - top);
}

// A row's shares in the workspace, (reference, sum of probabilities) and sums of p v, joined to what (top, sum, acc) holds: four
// channels a lane.  The loads of 16 shares are in flight together; one share after the other, 32 of them took 25 us.
template <typename OUT>
__device__ __forceinline__ void ctx_add_shares(const f32x2* ml, const float* sums, int64_t stride, int n, float& top, float& sum, f32x4& acc) {
  constexpr int kBatch = 16;
  for (int k = 0; k < n; k += kBatch) {
    f32x2 x[kBatch];
    f32x4 v[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int i = k + u < n ? k + u : n - 1;
      x[u] = ml[i];
      v[u] = *(const f32x4*)(sums + i * stride);
    }
    float most = top;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) most = fmaxf(most, x[u][0]);
    const float keep = sum == 0.f ? 0.f : ctx_weight<OUT>(top, most);
    top = most;
    sum *= keep;
    acc *= keep;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      // a share without keys counts for nothing (one whose scores are all NaN has a reference of -inf as well, but a sum)
      const float e = k + u >= n || x[u][1] == 0.f ? 0.f : ctx_weight<OUT>(x[u][0], top);
      sum += e * x[u][1];
      acc += e * v[u];
    }
  }
}

// The end of a call whose wavefronts attended shares of the keys.  A wavefront's LDS holds its sums, ROWS x D floats (16-byte chunk c of row r at chunk
// c ^ (r & 15)), at `sums` (reference, sum) of the rows and at `ends` their CtxRowEnd.  The WAYS wavefronts of a row block join
// their shares, and those of an earlier launch, and write the results or, for a later join, their share.  Four rows at a time, so that their reads
// overlap: one after the other, 32 rows took 5 us.
template <typename OUT, int D, int ROWS, int WAYS>
__device__ __forceinline__ void ctx_finish(const CtxArgs& a, const CtxPart& p, uint32_t group, uint32_t wave_bytes, uint32_t sums, uint32_t ends,
                                           int way, int split, int row0) {
  constexpr int kLanes = D / 4, kAtOnce = 64 * WAYS / kLanes, kSteps = ROWS / kAtOnce > 0 ? ROWS / kAtOnce : 1, kBatch = kSteps < 4 ? kSteps : 4;
  const int tg = way * 64 + (threadIdx.x & 63), chunk = tg % kLanes, first = tg / kLanes;
  const int64_t all = (int64_t)a.n_tiles * a.heads * a.tokens * a.n_shares;
  for (int step = 0; step < kSteps && row0 + step * kAtOnce < p.rows; step += kBatch) {
    u32x4 end[kBatch];
    f32x2 ml[kBatch][WAYS];
    f32x4 o[kBatch][WAYS];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int r = first + (step + i) * kAtOnce;
      if (ROWS >= kAtOnce || r < ROWS) {
        end[i] = *(const SG_LDS u32x4*)(uintptr_t)(group + ends + r * 16);
#pragma unroll
        for (int w = 0; w < WAYS; ++w) {
          ml[i][w] = *(const SG_LDS f32x2*)(uintptr_t)(group + w * wave_bytes + sums + r * 8);
          o[i][w] = *(const SG_LDS f32x4*)(uintptr_t)(group + w * wave_bytes + r * (D * 4) + ((chunk ^ (r & 15)) << 4));
        }
      } else {
        end[i] = u32x4{0, 0, 0, 0};
      }
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const uint64_t to = (uint64_t)end[i][1] << 32 | end[i][0];
      if (!to) continue;
      float top = ml[i][0][0], sum = 0.f;
#pragma unroll
      for (int w = 1; w < WAYS; ++w) top = fmaxf(top, ml[i][w][0]);
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < WAYS; ++w) {
        const float e = ml[i][w][1] == 0.f ? 0.f : ctx_weight<OUT>(ml[i][w][0], top);   // 0: no keys (NaN scores leave a sum)
        sum += e * ml[i][w][1];
        acc += e * o[i][w];
      }
      const int64_t shares = (int64_t)(int)end[i][2] * a.n_shares;
      if (p.prior) ctx_add_shares<OUT>((const f32x2*)(a.shares + all * D) + shares, a.shares + shares * D + 4 * chunk, D, p.prior, top, sum, acc);
      if (a.n_shares == p.prior) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        if constexpr (sizeof(OUT) == 4) *(f32x4*)((OUT*)(uintptr_t)to + 4 * chunk) = acc * inv;
        else *(u32x2*)((OUT*)(uintptr_t)to + 4 * chunk) = u32x2{pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
      } else {
        const int64_t at = shares + p.first_share + split;
        *(f32x4*)(a.shares + at * D + 4 * chunk) = acc;
        if (chunk == 0) *(f32x2*)(a.shares + all * D + at * 2) = f32x2{top, sum};
      }
    }
  }
}

// ---------------------------------------------------------------------------------------------------- host side
// The launches for at most kCtxTilesPerLaunch tiles and what they need of the workspace.
constexpr int kCtxResidentBytes = 128 * 1024;
enum { kCtxWide, kCtxSplit, kCtxSplit16, kCtxResident };   // workgroups of 128 (fp32: 64) rows that share their keys; wavefronts of 32 (fp32: or 16) rows with keys of their own;
                                                         // bf16: all keys stay in LDS
struct CtxPlan {
  int32_t n_launches;
  int32_t kind[2];
  CtxPart part[2];
  bool join;             // a last launch joins the shares
  int32_t n_shares;
  size_t bytes;          // workspace
};
CtxPlan plan_context(const sg_context_problem& p, bool prefix, int n_tiles);
int launch_context_bf16_wide(const CtxArgs& a, const CtxTable& tab, int head_dim, hipStream_t s);
int launch_context_bf16_resident(const CtxArgs& a, const CtxTable& tab, int head_dim, hipStream_t s);
int launch_context_bf16_split(const CtxArgs& a, const CtxTable& tab, int head_dim, hipStream_t s);
int launch_context_f32(const CtxArgs& a, const CtxTable& tab, int kind, int head_dim, hipStream_t s);
int launch_context_join(const CtxArgs& a, const CtxTable& tab, int head_dim, int dtype, hipStream_t s);

}  // namespace sg
