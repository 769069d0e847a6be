// C ABI of the operators beside a tile's self-attention: host-side argument checks and the order of launches.
#include <algorithm>
#include <cmath>
#include <utility>
#include "context_common.h"

namespace sg {

static bool aligned16(const void* p) { return (((uintptr_t)p) & 15u) == 0; }

static bool stride_ok(int64_t token, int64_t head, int d) {
  return token >= d && head > 0 && !(token & 7) && !(head & 7) && token < (1ll << 40) && head < (1ll << 40);
}

static int validate(const sg_context_problem* p) {
  if (!p) return SG_ERR_INVALID_ARG;
  if (p->heads <= 0 || p->kv_heads <= 0 || p->heads % p->kv_heads != 0 || p->head_dim <= 0 || p->tokens <= 0 || p->ctx_tokens < 0 ||
      p->own_tokens < 0)
    return SG_ERR_INVALID_ARG;
  if (p->dtype != SG_F32 && p->dtype != SG_BF16) return SG_ERR_INVALID_ARG;
  if (!std::isfinite(p->scale) || p->scale <= 0.f) return SG_ERR_INVALID_ARG;
  const int d = p->head_dim;
  if (!stride_ok(p->q_stride_token, p->q_stride_head, d) || !stride_ok(p->out_stride_token, p->out_stride_head, d) ||
      (p->ctx_tokens > 0 && !stride_ok(p->ctx_stride_token, p->ctx_stride_head, d)) ||
      (p->own_tokens > 0 && !stride_ok(p->own_stride_token, p->own_stride_head, d)))
    return SG_ERR_INVALID_ARG;
  // outputs that overlap: heads lie behind all tokens of the one before, or inside a token (in quotients: the products can pass 64 bits)
  if (p->heads > 1) {
    if (p->out_stride_head < d) return SG_ERR_INVALID_ARG;
    if ((p->out_stride_head - d) / p->out_stride_token < p->tokens - 1 && (p->out_stride_token - d) / p->out_stride_head < p->heads - 1)
      return SG_ERR_INVALID_ARG;
  }
  if (d != 64 && d != 128) return SG_ERR_UNSUPPORTED;
  // offsets inside a stage of 64 keys are 32-bit; rows and items are numbered in 32 bits, for 64 tiles a launch
  if ((p->ctx_tokens > 0 && p->ctx_stride_token >= (1ll << 22)) || (p->own_tokens > 0 && p->own_stride_token >= (1ll << 22)))
    return SG_ERR_UNSUPPORTED;
  if ((int64_t)p->heads * p->tokens >= (1ll << 25) || p->kv_heads > 65535) return SG_ERR_UNSUPPORTED;
  if (p->ctx_tokens >= (1 << 30) || p->own_tokens >= (1 << 30)) return SG_ERR_UNSUPPORTED;
  return SG_OK;
}

static int check_tiles(const void* const* a, int n) {
  if (!a) return SG_ERR_INVALID_ARG;
  for (int i = 0; i < n; ++i)
    if (!a[i] || !aligned16(a[i])) return SG_ERR_INVALID_ARG;
  return SG_OK;
}

// In-place sums: sum[i] may be x[i] or residual[i], with its stride, and nothing of another tile, whose rows other workgroups read and write meanwhile.
static bool sums_apart(const sg_norm_problem& p, int n, const void* const* x, const void* const* residual, void* const* sum) {
  std::pair<const void*, int> at[SG_MAX_TILES];
  for (int i = 0; i < n; ++i) at[i] = {sum[i], i};
  std::sort(at, at + n);
  for (int i = 1; i < n; ++i)
    if (at[i].first == at[i - 1].first) return false;
  auto reads = [&](const void* from, int i, int64_t stride) {
    const auto found = std::lower_bound(at, at + n, std::make_pair(from, 0));
    return found == at + n || found->first != from || (found->second == i && stride == p.sum_stride);
  };
  for (int i = 0; i < n; ++i)
    if (!reads(x[i], i, p.x_stride) || (residual && !reads(residual[i], i, p.residual_stride))) return false;
  return true;
}

static size_t workspace_bytes(const sg_context_problem& p, bool prefix, int n_tiles) {
  size_t most = 0;
  const int sizes[2] = {n_tiles < kCtxTilesPerLaunch ? n_tiles : kCtxTilesPerLaunch, n_tiles % kCtxTilesPerLaunch};
  for (int n : sizes) {
    if (n == 0) continue;
    const size_t b = plan_context(p, prefix, n).bytes;
    most = b > most ? b : most;
  }
  return most;
}

static int attend(const sg_context_problem& p, bool prefix, int n_tiles, const void* const* q, const void* const* k, const void* const* v,
                  const void* pk, const void* pv, const int32_t* tile_len, const int32_t* prefix_len, const uint8_t* mask,
                  const uint8_t* run, void* const* out, void* ws, size_t ws_bytes, hipStream_t s) {
  if (n_tiles < 0) return SG_ERR_INVALID_ARG;
  if (n_tiles > SG_MAX_TILES) return SG_ERR_UNSUPPORTED;
  if (n_tiles == 0) return SG_OK;
  const int tile_keys = prefix ? p.own_tokens : p.ctx_tokens;
  if (check_tiles(q, n_tiles) != SG_OK || check_tiles((const void* const*)out, n_tiles) != SG_OK) return SG_ERR_INVALID_ARG;
  if (tile_keys > 0 && (check_tiles(k, n_tiles) != SG_OK || check_tiles(v, n_tiles) != SG_OK)) return SG_ERR_INVALID_ARG;
  if (prefix && p.ctx_tokens > 0 && (!pk || !pv || !aligned16(pk) || !aligned16(pv))) return SG_ERR_INVALID_ARG;
  for (int n : {n_tiles < kCtxTilesPerLaunch ? n_tiles : kCtxTilesPerLaunch, n_tiles % kCtxTilesPerLaunch}) {
    if (n == 0) continue;
    const CtxPlan plan = plan_context(p, prefix, n);
    if (plan.part[0].items < 0 || plan.part[1].items < 0) return SG_ERR_UNSUPPORTED;
  }
  const size_t need = workspace_bytes(p, prefix, n_tiles);
  if (need > 0 && (!ws || (((uintptr_t)ws) & 255u) || ws_bytes < need)) return SG_ERR_WORKSPACE;
  for (int t0 = 0; t0 < n_tiles; t0 += kCtxTilesPerLaunch) {
    const int n = n_tiles - t0 < kCtxTilesPerLaunch ? n_tiles - t0 : kCtxTilesPerLaunch;
    const CtxPlan plan = plan_context(p, prefix, n);
    CtxTable tab = {};
    for (int i = 0; i < n; ++i) {
      tab.q[i] = q[t0 + i];
      tab.out[i] = out[t0 + i];
      tab.k[i] = tile_keys > 0 ? k[t0 + i] : nullptr;
      tab.v[i] = tile_keys > 0 ? v[t0 + i] : nullptr;
    }
    CtxArgs a = {};
    a.q_token = p.q_stride_token; a.q_head = p.q_stride_head;
    a.o_token = p.out_stride_token; a.o_head = p.out_stride_head;
    a.kv_token[0] = p.ctx_stride_token; a.kv_head[0] = p.ctx_stride_head;
    a.kv_token[1] = prefix ? p.own_stride_token : p.ctx_stride_token;
    a.kv_head[1] = prefix ? p.own_stride_head : p.ctx_stride_head;
    a.k0 = pk; a.v0 = pv;
    a.len0 = prefix_len;
    a.len1 = tile_len ? tile_len + t0 : nullptr;
    a.mask1 = mask ? mask + (int64_t)t0 * p.ctx_tokens : nullptr;
    a.run = run ? run + t0 : nullptr;
    a.shares = (float*)ws;
    a.cap0 = prefix ? p.ctx_tokens : 0;
    a.cap1 = tile_keys;
    a.heads = p.heads; a.kv_heads = p.kv_heads; a.group = p.heads / p.kv_heads; a.tokens = p.tokens; a.n_tiles = n;
    a.n_shares = plan.n_shares;
    a.by_tokens = make_divisor((uint32_t)a.tokens);
    a.by_rows = make_divisor((uint32_t)(a.group * a.tokens));
    a.scale = p.scale;
    for (int i = 0; i < plan.n_launches; ++i) {
      a.part = plan.part[i];
      const int st = p.dtype == SG_F32                ? launch_context_f32(a, tab, plan.kind[i], p.head_dim, s)
                     : plan.kind[i] == kCtxResident ? launch_context_bf16_resident(a, tab, p.head_dim, s)
                     : plan.kind[i] == kCtxWide     ? launch_context_bf16_wide(a, tab, p.head_dim, s)
                                                    : launch_context_bf16_split(a, tab, p.head_dim, s);
      if (st != SG_OK) return st;
    }
    if (plan.join) {
      const int st = launch_context_join(a, tab, p.head_dim, p.dtype, s);
      if (st != SG_OK) return st;
    }
  }
  return SG_OK;
}

}  // namespace sg

using namespace sg;

extern "C" {

int sg_context_validate(const sg_context_problem* p) { return validate(p); }

int sg_context_workspace_bytes(const sg_context_problem* p, int32_t n_tiles, size_t* out_bytes) {
  int st = validate(p);
  if (st != SG_OK) return st;
  if (!out_bytes || n_tiles < 0) return SG_ERR_INVALID_ARG;
  if (n_tiles > SG_MAX_TILES) return SG_ERR_UNSUPPORTED;
  const size_t a = workspace_bytes(*p, false, n_tiles), b = workspace_bytes(*p, true, n_tiles);
  *out_bytes = a > b ? a : b;
  return SG_OK;
}

int sg_tile_cross_attention(const sg_context_problem* p, int32_t n_tiles, const void* const* q, const void* const* k,
                            const void* const* v, const int32_t* ctx_len, const uint8_t* key_mask, const uint8_t* run,
                            void* const* out, void* workspace, size_t ws_bytes, void* stream) {
  const int st = validate(p);
  if (st != SG_OK) return st;
  return attend(*p, false, n_tiles, q, k, v, nullptr, nullptr, ctx_len, nullptr, key_mask, run, out, workspace, ws_bytes, (hipStream_t)stream);
}

int sg_tile_prefix_attention(const sg_context_problem* p, int32_t n_tiles, const void* const* q, const void* const* k,
                             const void* const* v, const void* prefix_k, const void* prefix_v, const int32_t* own_len,
                             const int32_t* prefix_len, const uint8_t* run, void* const* out, void* workspace, size_t ws_bytes,
                             void* stream) {
  const int st = validate(p);
  if (st != SG_OK) return st;
  return attend(*p, true, n_tiles, q, k, v, prefix_k, prefix_v, own_len, prefix_len, nullptr, run, out, workspace, ws_bytes,
                (hipStream_t)stream);
}

int sg_tile_residual_norm(const sg_norm_problem* p, int32_t n_tiles, const void* const* x, const void* const* residual,
                          const void* weight, const uint8_t* run, void* const* sum, void* const* out, float* const* out_scale,
                          void* stream) {
  if (!p || n_tiles < 0 || p->rows < 0 || p->channels <= 0 || (p->channels & 7)) return SG_ERR_INVALID_ARG;
  if (p->dtype != SG_F32 && p->dtype != SG_BF16) return SG_ERR_INVALID_ARG;
  if (p->out_dtype != p->dtype && p->out_dtype != SG_F8_E4M3) return SG_ERR_INVALID_ARG;
  if (p->scale_group != 0 && (p->out_dtype != SG_F8_E4M3 || p->scale_group < 0 || p->channels % p->scale_group != 0)) return SG_ERR_INVALID_ARG;
  if (!std::isfinite(p->eps) || p->eps < 0.f) return SG_ERR_INVALID_ARG;
  const int64_t strides[4] = {p->x_stride, residual ? p->residual_stride : p->channels, sum ? p->sum_stride : p->channels, p->out_stride};
  for (int64_t st : strides)
    if (st < p->channels || (st & 7) || st >= (1ll << 40)) return SG_ERR_INVALID_ARG;
  if (p->channels > 32768 || (p->scale_group != 0 && p->scale_group != 128) || n_tiles > SG_MAX_TILES) return SG_ERR_UNSUPPORTED;
  if (n_tiles == 0 || p->rows == 0) return SG_OK;
  if (check_tiles(x, n_tiles) != SG_OK || check_tiles((const void* const*)out, n_tiles) != SG_OK) return SG_ERR_INVALID_ARG;
  if (residual && check_tiles(residual, n_tiles) != SG_OK) return SG_ERR_INVALID_ARG;
  if (sum && (check_tiles((const void* const*)sum, n_tiles) != SG_OK || !sums_apart(*p, n_tiles, x, residual, sum))) return SG_ERR_INVALID_ARG;
  if (weight && !aligned16(weight)) return SG_ERR_INVALID_ARG;
  if ((p->out_dtype == SG_F8_E4M3) != (out_scale != nullptr)) return SG_ERR_INVALID_ARG;
  if (out_scale)
    for (int i = 0; i < n_tiles; ++i)
      if (!out_scale[i] || (((uintptr_t)out_scale[i]) & 3u)) return SG_ERR_INVALID_ARG;
  return launch_residual_norm(*p, n_tiles, x, residual, weight, run, sum, out, out_scale, (hipStream_t)stream);
}

}  // extern "C"
