// How a call of sg_tile_cross_attention / sg_tile_prefix_attention is cut into work, and the join of the shares of a row that
// different workgroups attended:
//     M = max m_s,   o = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s     over the shares s of (reference m, sum l, sums O of p v)
// in the order of the shares, so that a call gives the same bits every time.
#include "context_common.h"

namespace sg {
namespace {

template <typename OUT, int D>
__global__ __launch_bounds__(256) void context_join_kernel(const CtxArgs a, const CtxTable tab, const int64_t n_rows) {
  constexpr int kLanes = D / 4;   // lanes per row: 4 channels each
  const int64_t rid = (int64_t)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;
  if (rid >= n_rows) return;
  const int chunk = threadIdx.x % kLanes;
  const int head_row = (int)(rid / a.tokens), token = (int)(rid - (int64_t)head_row * a.tokens);
  const int tile = head_row / a.heads, head = head_row - tile * a.heads;   // rows: [tile][head of keys][head of its group][token]
  if (a.run && a.run[tile] == 0) return;
  const float* const sums = a.shares + rid * a.n_shares * D + 4 * chunk;
  const f32x2* const ml = (const f32x2*)(a.shares + n_rows * a.n_shares * D) + rid * a.n_shares;
  float top = -__builtin_inff();
  for (int i = 0; i < a.n_shares; ++i) top = fmaxf(top, ml[i][0]);
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float sum = 0.f;
  for (int i = 0; i < a.n_shares; ++i) {
    const f32x2 x = ml[i];
    if (x[1] == 0.f) continue;   // a share without keys (one whose scores are NaN has a reference of -inf too)
    const float e = __builtin_amdgcn_exp2f(x[0] - top);
    sum += e * x[1];
    acc += e * *(const f32x4*)(sums + (int64_t)i * D);
  }
  const f32x4 y = sum == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : acc / sum;
  OUT* const out = (OUT*)tab.out[tile] + (int64_t)head * a.o_head + (int64_t)token * a.o_token + 4 * chunk;
  if constexpr (sizeof(OUT) == 4) *(f32x4*)out = y;
  else *(u32x2*)out = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
}

// Wavefronts that the split kernels keep at work: 4 on each of the 256 compute units.
constexpr int64_t kWaves = 1024;

// Cuts the keys of `rows` rows into shares, so that about `waves` wavefronts have work.
void cut(CtxPart& p, int batches, int rows, int kv_heads, int64_t stages, int wave_rows, int64_t waves) {
  const int64_t blocks = (rows + wave_rows - 1) / wave_rows, base = (int64_t)batches * kv_heads * blocks;
  int64_t shares = waves / base;
  shares = shares > stages ? stages : (shares < 1 ? 1 : shares);
  // the wavefronts of a workgroup that no row block needs take shares
  p.ways = (shares >= 4 || blocks == 1) ? 4 : (shares >= 2 || blocks == 2) ? 2 : 1;
  // a share that goes through memory to be joined is worth its while from two stages per wavefront on
  const int64_t most = stages / (2 * p.ways) > 1 ? stages / (2 * p.ways) : 1;
  p.splits = (int32_t)(shares / p.ways < 1 ? 1 : (shares / p.ways > most ? most : shares / p.ways));
  p.batches = batches;
  p.rows = rows;
  p.row_blocks = (int32_t)((blocks + 4 / p.ways - 1) / (4 / p.ways));
  const int64_t items = (int64_t)batches * kv_heads * p.row_blocks * p.splits;
  p.items = items > (1 << 30) ? -1 : (int32_t)items;
}

}  // namespace

CtxPlan plan_context(const sg_context_problem& p, bool prefix, int n_tiles) {
  CtxPlan plan = {};
  plan.n_shares = 1;
  const int group = p.heads / p.kv_heads;
  const int64_t rows = (int64_t)group * p.tokens;   // per tile and head of keys
  const bool bf16 = p.dtype == SG_BF16;
  const int keys = bf16 ? (p.head_dim == 128 ? 32 : 64) : (p.head_dim == 128 ? 16 : 32);   // of a wavefront's stage
  const int64_t seg0 = prefix ? (p.ctx_tokens + keys - 1) / keys : 0;
  const int64_t seg1 = ((prefix ? p.own_tokens : p.ctx_tokens) + keys - 1) / keys;
  plan.part[0].seg0 = prefix;
  plan.part[0].seg1 = 1;
  const int64_t wide_blocks = (rows + 127) / 128, wide_items = (int64_t)n_tiles * p.kv_heads * wide_blocks;
  if (wide_items >= 256) {
    plan.wide = true;
    plan.wave_rows = 32;
    plan.part[0].items = wide_items > (1 << 30) ? -1 : (int32_t)wide_items;
    plan.part[0].batches = n_tiles;
    plan.part[0].rows = (int32_t)rows;
    plan.part[0].row_blocks = (int32_t)wide_blocks;
    plan.part[0].splits = plan.part[0].ways = 1;
    return plan;
  }
  // Few rows per tile: those of all tiles are stacked over the prefix, which is then read once for all, and each tile's own keys are a
  // work item beside it.
  const bool stacked = prefix && n_tiles > 1 && rows <= 16 && p.ctx_tokens >= 128;
  plan.wave_rows = (!bf16 && (stacked ? n_tiles * rows : rows) <= 16) ? 16 : 32;
  if (stacked) {
    CtxPart &all = plan.part[0], &each = plan.part[1];
    const int64_t blocks = (n_tiles * rows + plan.wave_rows - 1) / plan.wave_rows;
    const int64_t w0 = blocks * seg0, w1 = (int64_t)n_tiles * seg1;   // stages, per head of keys
    int64_t waves0 = kWaves * w0 / (w0 + w1), waves1 = kWaves - waves0;
    cut(all, 1, (int)(n_tiles * rows), p.kv_heads, seg0, plan.wave_rows, waves0 < 1 ? 1 : waves0);
    all.seg1 = 0;
    all.stacked = 1;
    plan.n_shares = all.splits;
    if (p.own_tokens > 0) {
      cut(each, n_tiles, (int)rows, p.kv_heads, seg1, plan.wave_rows, waves1 < 1 ? 1 : waves1);
      each.seg1 = 1;
      each.first_share = all.splits;
      plan.n_shares += each.splits;
    }
  } else {
    cut(plan.part[0], n_tiles, (int)rows, p.kv_heads, seg0 + seg1 > 0 ? seg0 + seg1 : 1, plan.wave_rows, kWaves);
    plan.n_shares = plan.part[0].splits;
  }
  if (plan.n_shares > 1) plan.bytes = ((size_t)n_tiles * p.heads * p.tokens * plan.n_shares * (p.head_dim + 2) * 4 + 255) / 256 * 256;
  return plan;
}

int launch_context_join(const CtxArgs& a, const CtxTable& tab, int head_dim, int dtype, hipStream_t s) {
  const int64_t n_rows = (int64_t)a.n_tiles * a.heads * a.tokens, per = 256 / (head_dim / 4), grid = (n_rows + per - 1) / per;
  if (grid > (1ll << 31) - 1) return SG_ERR_UNSUPPORTED;
  if (dtype == SG_F32) {
    if (head_dim == 128) context_join_kernel<float, 128><<<dim3((unsigned)grid), 256, 0, s>>>(a, tab, n_rows);
    else context_join_kernel<float, 64><<<dim3((unsigned)grid), 256, 0, s>>>(a, tab, n_rows);
  } else {
    if (head_dim == 128) context_join_kernel<uint16_t, 128><<<dim3((unsigned)grid), 256, 0, s>>>(a, tab, n_rows);
    else context_join_kernel<uint16_t, 64><<<dim3((unsigned)grid), 256, 0, s>>>(a, tab, n_rows);
  }
  SG_HIP_TRY(hipGetLastError());
  return SG_OK;
}

}  // namespace sg
