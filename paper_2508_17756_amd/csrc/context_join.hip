// How a call of sg_tile_cross_attention / sg_tile_prefix_attention is cut into work, and the join of the shares of a row that
// different workgroups attended:
//     M = max m_s,   o = sum_s e^(m_s - M) O_s / sum_s e^(m_s - M) l_s     over the shares s of (reference m, sum l, sums O of p v)
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
  float top = -__builtin_inff(), sum = 0.f;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  ctx_add_shares<OUT>(ml, sums, D, a.n_shares, top, sum, acc);
  const f32x4 y = sum == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : acc / sum;
  OUT* const out = (OUT*)tab.out[tile] + (int64_t)head * a.o_head + (int64_t)token * a.o_token + 4 * chunk;
  if constexpr (sizeof(OUT) == 4) *(f32x4*)out = y;
  else *(u32x2*)out = u32x2{pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3])};
}

constexpr int64_t kCus = 256;

// Cuts the keys of `rows` rows into shares for wavefronts with keys of their own, so that about `waves` of them have work.
void cut(CtxPart& p, int batches, int64_t rows, int kv_heads, int64_t stages, int wave_rows, int64_t waves) {
  const int64_t blocks = (rows + wave_rows - 1) / wave_rows, base = batches * kv_heads * blocks;
  int64_t shares = waves / base;
  shares = shares > stages ? stages : (shares < 1 ? 1 : shares);
  // the wavefronts of a workgroup that no row block needs take shares
  p.ways = (shares >= 4 || blocks == 1) ? 4 : (shares >= 2 || blocks == 2) ? 2 : 1;
  // a share that goes through memory to be joined is worth its while from two stages per wavefront on
  const int64_t most = stages / (2 * p.ways) > 1 ? stages / (2 * p.ways) : 1;
  p.splits = (int32_t)(shares / p.ways < 1 ? 1 : (shares / p.ways > most ? most : shares / p.ways));
  p.rows = (int32_t)rows;
  p.row_blocks = (int32_t)((blocks + 4 / p.ways - 1) / (4 / p.ways));
  const int64_t items = (int64_t)batches * kv_heads * p.row_blocks * p.splits;
  p.items = items > (1 << 30) ? -1 : (int32_t)items;
}
// The same for workgroups that share stages of keys: of 128 rows in bf16, of which there should be one for each compute unit (100 rows over a prefix of
// 32,760 keys, 8 heads x 128: 47.6 us, with two for each 52.7), of 64 in fp32, two for each (16 x 600 rows x 128 over 2,000 keys 110 us; 128 rows
// and one for each 119, 64 and three 118); of at least eight stages (bf16, 64 blocks x 128 over 500 keys: 14.5 us, with four 19.4).
int64_t shared_rows(bool bf16) { return bf16 ? 128 : 64; }
void cut_wide(CtxPart& p, int batches, int64_t rows, int kv_heads, int64_t stages, bool bf16, int head_dim) {
  const int64_t of = shared_rows(bf16), blocks = (rows + of - 1) / of, base = batches * kv_heads * blocks;
  int64_t splits = (bf16 ? kCus : 2 * kCus) / base;
  const int64_t most = stages / 8 > 1 ? stages / 8 : 1;
  splits = splits < 1 ? 1 : (splits > most ? most : splits);
  // head_dim 64: two groups of wavefronts share a workgroup's keys where it has its compute unit alone and eight stages (256 blocks over 2,000 keys
  // 33.4 -> 27.1 us, over 500 12.2 -> 11.5, over 77 7.2 and 7.6; head_dim 128, whose stages are bound by more than one wavefront's chain, 42.4 and 40.5,
  // 16.0 and 16.4)
  p.ways = bf16 && head_dim == 64 && base * splits <= kCus && stages / splits >= 8 ? 2 : 1;
  p.splits = (int32_t)splits;
  p.rows = (int32_t)rows;
  p.row_blocks = (int32_t)blocks;
  p.items = base * splits > (1 << 24) - 8 ? -1 : (int32_t)(base * splits);   // a grid has less than 2^32 threads, 256 a workgroup
}

}  // namespace

CtxPlan plan_context(const sg_context_problem& p, bool prefix, int n_tiles) {
  CtxPlan plan = {};
  const int group = p.heads / p.kv_heads;
  const int64_t rows = (int64_t)group * p.tokens;   // per tile and head of keys
  const bool bf16 = p.dtype == SG_BF16;
  const int keys = (bf16 ? 32 : 16) * (p.head_dim == 128 ? 1 : 2), wide_keys = bf16 ? 64 : keys;   // of a wavefront's, of a shared stage
  auto stages = [](int tokens, int of) -> int64_t { return (tokens + of - 1) / of; };
  const int tile_keys = prefix ? p.own_tokens : p.ctx_tokens, shared_keys = prefix ? p.ctx_tokens : 0;
  // fp32, 16 rows per wavefront instead of 32: where there are no more, and where wavefronts of 32 would have less than four stages each (4 tiles
  // of 300 queries, 2 heads x 64, over 377 keys: 17.6 -> 11.5 us; 64 rows over 16,000 keys, the other way round: 37 and 46 us)
  auto split_kind = [&](int64_t batches, int64_t n, int64_t of) {
    return !bf16 && (n <= 16 || batches * p.kv_heads * ((n + 31) / 32) * of < 16 * kCus) ? kCtxSplit16 : kCtxSplit;
  };
  auto wave_rows = [](int kind) { return kind == kCtxSplit16 ? 16 : 32; };
  plan.n_launches = 1;
  CtxPart &first = plan.part[0], &second = plan.part[1];
  // Few rows per tile: those of all tiles are stacked over the prefix, which is then read once for all, and each tile's own keys are attended
  // by a second launch, which joins the shares.
  if (prefix && n_tiles > 1 && rows <= 16 && shared_keys >= 128) {
    const int64_t all = n_tiles * rows;
    if (all > 64) {
      plan.kind[0] = kCtxWide;
      cut_wide(first, 1, all, p.kv_heads, stages(shared_keys, wide_keys), bf16, p.head_dim);
    } else {
      plan.kind[0] = split_kind(1, all, stages(shared_keys, keys));
      cut(first, 1, all, p.kv_heads, stages(shared_keys, keys), wave_rows(plan.kind[0]), 4 * kCus);
    }
    first.seg0 = first.stacked = 1;
    if (tile_keys > 0) {
      plan.n_launches = 2;
      plan.kind[1] = split_kind(n_tiles, rows, stages(tile_keys, keys));
      cut(second, n_tiles, rows, p.kv_heads, stages(tile_keys, keys), wave_rows(plan.kind[1]), 4 * kCus);
      second.seg1 = 1;
      second.first_share = first.splits;
      plan.n_shares = first.splits + second.splits;
      plan.join = second.splits > 1;
      if (!plan.join) {
        second.prior = first.splits;
        plan.n_shares = first.splits;
      }
    } else if (first.splits > 1) {
      plan.n_shares = first.splits;
      plan.join = true;
    }
  } else {
    const int64_t of = shared_rows(bf16), blocks = (int64_t)n_tiles * p.kv_heads * ((rows + of - 1) / of);
    const int64_t row_blocks = (rows + 31) / 32, all = n_tiles * p.kv_heads * row_blocks;
    const int64_t units = stages(shared_keys, 64) + stages(tile_keys, 64), wide_stages = stages(shared_keys, wide_keys) + stages(tile_keys, wide_keys);
    // Keys that fit stay in LDS where its wavefronts, 8 for each compute unit, have two row blocks each: head_dim 64, 500 keys, 8,192 row blocks
    // 47.4 us (shared stages: 54.8), 4,096 28.0 (30.0), 2,048 16.5 (16.4); head_dim 128, 250 keys 49.8 (59.5), 27.4 (31.5), 17.9 (17.6).
    if (bf16 && units * 64 * p.head_dim * 4 <= kCtxResidentBytes && all >= 16 * kCus && all < (1 << 30)) {
      plan.kind[0] = kCtxResident;
      first.rows = (int32_t)rows;
      first.row_blocks = (int32_t)row_blocks;
      first.splits = first.ways = first.items = 1;
    } else if (blocks >= (bf16 ? kCus / 2 : 2 * kCus) || blocks * wide_stages * wide_keys * p.head_dim >= (bf16 ? 10 : 9) * kCus * 64 * 64) {
      // Shared stages read a key from memory once for 128 rows (fp32: 64), wavefronts with keys of their own once for 32, but those need no barriers and
      // start and join sooner.  128 blocks of 128 rows, head_dim 128, 500 keys: 14.8 us (own keys: 19.1), 64 the same: 14.5 and 16.2, head_dim 64
      // 11.6 and 10.7.  Fewer blocks over more keys: 16 blocks, 8,000 keys x 128 23.2 (30.6), 2,000 20.0 (15.8).
      // fp32, blocks of 64 rows: 512 blocks, 500 keys x 128 80.7 us (95.5), 256 the same 56.2 (52.0); 80 blocks, 2,000 keys x 64 36.7 (47.5), 40 the same 30.6
      // (27.1).
      plan.kind[0] = kCtxWide;
      cut_wide(first, n_tiles, rows, p.kv_heads, wide_stages > 0 ? wide_stages : 1, bf16, p.head_dim);
    } else {
      const int64_t n = stages(shared_keys, keys) + stages(tile_keys, keys);
      plan.kind[0] = split_kind(n_tiles, rows, n);
      cut(first, n_tiles, rows, p.kv_heads, n > 0 ? n : 1, wave_rows(plan.kind[0]), 4 * kCus);
    }
    first.seg0 = prefix;
    first.seg1 = 1;
    if (first.splits > 1) {
      plan.n_shares = first.splits;
      plan.join = true;
    }
  }
  if (plan.n_shares > 0) plan.bytes = ((size_t)n_tiles * p.heads * p.tokens * plan.n_shares * (p.head_dim + 2) * 4 + 255) / 256 * 256;
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
