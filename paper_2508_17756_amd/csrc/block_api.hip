// C ABI of the rotary positions, the gated norm and the 8-bit integer linear layer: host-side argument checks.
#include <algorithm>
#include <cmath>
#include "block_api.h"

namespace sg {

static bool aligned16(const void* p) { return (((uintptr_t)p) & 15u) == 0; }

static bool tiles_ok(const void* const* a, int n, uintptr_t mask = 15u) {
  if (!a) return false;
  for (int i = 0; i < n; ++i)
    if (!a[i] || (((uintptr_t)a[i]) & mask)) return false;
  return true;
}

// Buffers that a call writes: no two tiles write one, and none is what another tile reads or what the call reads in another place.
class Written {
 public:
  Written(void* const* written, int n) : written_(written), n_(n) {
    std::copy(written, written + n, at_);
    if (!std::is_sorted(at_, at_ + n)) std::sort(at_, at_ + n);
  }
  bool different() const { return std::adjacent_find(at_, at_ + n_) == at_ + n_; }
  // read[i] may be written[i] where both have the same strides: in place.
  bool apart_from(const void* const* read, bool same_strides = false) const {
    if (!read) return true;
    for (int i = 0; i < n_; ++i)
      if (read[i] >= at_[0] && read[i] <= at_[n_ - 1] && std::binary_search(at_, at_ + n_, read[i]) && !(same_strides && written_[i] == read[i])) return false;
    return true;
  }
  bool not_at(const void* read) const { return !read || !std::binary_search(at_, at_ + n_, read); }

 private:
  void* const* written_;
  int n_;
  const void* at_[SG_MAX_TILES];
};

static bool row_stride_ok(int64_t stride, int64_t channels, int64_t unit) { return stride >= channels && !(stride % unit) && stride < (1ll << 40); }

// Heads of an output: behind all tokens of the one before, or inside a token (in quotients: the products can pass 64 bits).
static bool heads_apart(int64_t token, int64_t head, int64_t tokens, int64_t heads, int64_t d) {
  if (heads <= 1) return true;
  if (head < d) return false;
  return (head - d) / token >= tokens - 1 || (token - d) / head >= heads - 1;
}

static bool head_strides_ok(int64_t token, int64_t head, int64_t d) {
  return token >= d && head > 0 && !(token & 7) && !(head & 7) && token < (1ll << 40) && head < (1ll << 40);
}

static int validate(const sg_rotary_problem* p, bool keys) {
  if (!p) return SG_ERR_INVALID_ARG;
  if (p->T <= 0 || p->H <= 0 || p->W <= 0 || p->heads <= 0 || (keys && p->kv_heads <= 0) || p->head_dim <= 0 || (p->head_dim & 7)) return SG_ERR_INVALID_ARG;
  if (p->dtype != SG_F32 && p->dtype != SG_BF16) return SG_ERR_INVALID_ARG;
  if (p->layout != SG_ROTARY_INTERLEAVED && p->layout != SG_ROTARY_HALF) return SG_ERR_INVALID_ARG;
  const int32_t axes[3] = {p->axis_t, p->axis_y, p->axis_x}, canvas[3] = {p->canvas_t, p->canvas_h, p->canvas_w};
  int64_t turned = 0;
  for (int i = 0; i < 3; ++i) {
    if (axes[i] < 0 || (axes[i] & 1) || canvas[i] < 0) return SG_ERR_INVALID_ARG;
    turned += axes[i];
  }
  if (turned < 2 || turned > p->head_dim) return SG_ERR_INVALID_ARG;
  if (p->position_axes != 1 && p->position_axes != 3) return SG_ERR_INVALID_ARG;
  if (!std::isfinite(p->eps) || p->eps < 0.f) return SG_ERR_INVALID_ARG;
  const int64_t plane = (int64_t)p->H * p->W;
  if (plane >= (1ll << 24) || plane * p->T >= (1ll << 24)) return SG_ERR_UNSUPPORTED;
  const int64_t tokens = plane * p->T, d = p->head_dim;
  if (!head_strides_ok(p->q_stride_token, p->q_stride_head, d) || !head_strides_ok(p->q_out_stride_token, p->q_out_stride_head, d) ||
      !heads_apart(p->q_out_stride_token, p->q_out_stride_head, tokens, p->heads, d))
    return SG_ERR_INVALID_ARG;
  if (keys && (!head_strides_ok(p->k_stride_token, p->k_stride_head, d) || !head_strides_ok(p->k_out_stride_token, p->k_out_stride_head, d) ||
               !heads_apart(p->k_out_stride_token, p->k_out_stride_head, tokens, p->kv_heads, d)))
    return SG_ERR_INVALID_ARG;
  if (p->head_dim > 512 || (p->layout == SG_ROTARY_HALF && (turned & 15)) || p->heads > 65535 || (keys && p->kv_heads > 65535)) return SG_ERR_UNSUPPORTED;
  return SG_OK;
}

static int validate(const sg_int8_linear_problem* p) {
  if (!p) return SG_ERR_INVALID_ARG;
  if (p->rows < 0 || p->channels <= 0 || (p->channels & 15) || p->outputs <= 0 || (p->outputs & 7)) return SG_ERR_INVALID_ARG;
  if (p->dtype != SG_F32 && p->dtype != SG_BF16) return SG_ERR_INVALID_ARG;
  if (p->activation != SG_ACT_NONE && p->activation != SG_ACT_GELU) return SG_ERR_INVALID_ARG;
  if (!row_stride_ok(p->x_stride, p->channels, 16) || !row_stride_ok(p->w_stride, p->channels, 16) || !row_stride_ok(p->out_stride, p->outputs, 8))
    return SG_ERR_INVALID_ARG;
  if (p->channels > 131056 || p->outputs > (1 << 26)) return SG_ERR_UNSUPPORTED;
  return SG_OK;
}

}  // namespace sg

using namespace sg;

extern "C" {

int sg_rotary_validate(const sg_rotary_problem* p) { return validate(p, p && p->kv_heads != 0); }

int sg_rotary_frequencies(const sg_rotary_problem* p, double base, int32_t scaling, double factor, double length, double slow, double fast, double* out) {
  const int st = validate(p, false);
  if (st != SG_OK) return st;
  if (!out || !std::isfinite(base) || base <= 0.0) return SG_ERR_INVALID_ARG;
  if (scaling < SG_ROTARY_PLAIN || scaling > SG_ROTARY_RAMP) return SG_ERR_INVALID_ARG;
  if (scaling != SG_ROTARY_PLAIN && (!std::isfinite(factor) || factor <= 0.0)) return SG_ERR_INVALID_ARG;
  if (scaling == SG_ROTARY_RAMP &&
      (!std::isfinite(length) || length <= 0.0 || !std::isfinite(slow) || slow < 0.0 || !std::isfinite(fast) || fast <= slow))
    return SG_ERR_INVALID_ARG;
  const int32_t axes[3] = {p->axis_t, p->axis_y, p->axis_x};
  for (int32_t n : axes) {
    const double b = scaling == SG_ROTARY_NTK && n > 2 ? base * std::pow(factor, n / (n - 2.0)) : base;
    for (int i = 0; i < n / 2; ++i) {
      double f = std::pow(b, -2.0 * i / n);
      if (scaling == SG_ROTARY_LINEAR) f /= factor;
      if (scaling == SG_ROTARY_RAMP) {
        const double turns = length * f / 6.283185307179586;
        const double stays = std::min(std::max((turns - slow) / (fast - slow), 0.0), 1.0);
        f = f * stays + f / factor * (1.0 - stays);
      }
      *out++ = f;
    }
  }
  return SG_OK;
}

int sg_tile_rotary(const sg_rotary_problem* p, int32_t n_tiles, const void* const* q, const void* const* k, const double* frequencies,
                   const int32_t* origin, const int32_t* const* positions, const void* q_weight, const void* k_weight, const uint8_t* run,
                   void* const* q_out, void* const* k_out, void* stream) {
  const int st = validate(p, k != nullptr || k_out != nullptr);
  if (st != SG_OK) return st;
  if (n_tiles < 0) return SG_ERR_INVALID_ARG;
  if (n_tiles > SG_MAX_TILES) return SG_ERR_UNSUPPORTED;
  if (n_tiles == 0) return SG_OK;
  if (!tiles_ok(q, n_tiles) || !tiles_ok((const void* const*)q_out, n_tiles) || (k != nullptr) != (k_out != nullptr)) return SG_ERR_INVALID_ARG;
  if (k && (!tiles_ok(k, n_tiles) || !tiles_ok((const void* const*)k_out, n_tiles))) return SG_ERR_INVALID_ARG;
  if (!frequencies || (((uintptr_t)frequencies) & 7u) || (origin != nullptr) == (positions != nullptr)) return SG_ERR_INVALID_ARG;
  if (positions && !tiles_ok((const void* const*)positions, n_tiles, 3u)) return SG_ERR_INVALID_ARG;
  if ((q_weight && !aligned16(q_weight)) || (k_weight && !aligned16(k_weight))) return SG_ERR_INVALID_ARG;
  if (origin) {
    const int32_t canvas[3] = {p->canvas_t, p->canvas_h, p->canvas_w}, size[3] = {p->T, p->H, p->W};
    for (int i = 0; i < 3 * n_tiles; ++i)
      if (canvas[i % 3] == 0 && (int64_t)origin[i] + size[i % 3] - 1 > INT32_MAX) return SG_ERR_INVALID_ARG;
  }
  const bool q_same = p->q_stride_token == p->q_out_stride_token && p->q_stride_head == p->q_out_stride_head;
  const Written qw(q_out, n_tiles);
  if (!qw.different() || !qw.apart_from(q, q_same)) return SG_ERR_INVALID_ARG;
  if (k) {
    const bool k_same = p->k_stride_token == p->k_out_stride_token && p->k_stride_head == p->k_out_stride_head;
    const Written kw(k_out, n_tiles);
    if (!kw.different() || !kw.apart_from(k, k_same) || !kw.apart_from(q) || !qw.apart_from(k) || !qw.apart_from((const void* const*)k_out))
      return SG_ERR_INVALID_ARG;
  }
  return launch_rotary(*p, n_tiles, q, k, frequencies, origin, positions, q_weight, k_weight, run, q_out, k_out, (hipStream_t)stream);
}

int sg_tile_gated_norm(const sg_gated_norm_problem* p, int32_t n_tiles, const void* const* x, const void* const* residual, const void* const* gate,
                       const void* post_weight, const void* weight, const void* const* scale, const void* const* shift, const uint8_t* run,
                       void* const* sum, void* const* out, float* const* out_scale, void* stream) {
  if (!p || n_tiles < 0 || p->rows < 0 || p->channels <= 0 || (p->channels & 7)) return SG_ERR_INVALID_ARG;
  if (p->dtype != SG_F32 && p->dtype != SG_BF16) return SG_ERR_INVALID_ARG;
  const bool eight = p->out_dtype == SG_F8_E4M3 || p->out_dtype == SG_I8;
  if (p->out_dtype != p->dtype && !eight) return SG_ERR_INVALID_ARG;
  if (p->mod_dtype != p->dtype && p->mod_dtype != SG_F32) return SG_ERR_INVALID_ARG;
  if (p->scale_group != 0 && (!eight || p->scale_group < 0 || p->channels % p->scale_group != 0)) return SG_ERR_INVALID_ARG;
  if (p->norm != SG_NORM_RMS && p->norm != SG_NORM_LAYER) return SG_ERR_INVALID_ARG;
  if (p->post_norm != SG_NORM_NONE && p->post_norm != SG_NORM_RMS && p->post_norm != SG_NORM_LAYER) return SG_ERR_INVALID_ARG;
  if (!std::isfinite(p->eps) || p->eps < 0.f || !std::isfinite(p->post_eps) || p->post_eps < 0.f) return SG_ERR_INVALID_ARG;
  if (p->mod_rows < 0 || (residual && !std::isfinite(p->residual_scale))) return SG_ERR_INVALID_ARG;
  if (!row_stride_ok(p->x_stride, p->channels, 8) || !row_stride_ok(p->out_stride, p->channels, 8) ||
      (residual && !row_stride_ok(p->residual_stride, p->channels, 8)) || (sum && !row_stride_ok(p->sum_stride, p->channels, 8)))
    return SG_ERR_INVALID_ARG;
  const bool vectors = (gate || scale || shift) && p->mod_rows > 0 && p->mod_rows < p->rows;
  if (vectors && !row_stride_ok(p->mod_stride, p->channels, 8)) return SG_ERR_INVALID_ARG;
  if (post_weight && p->post_norm == SG_NORM_NONE) return SG_ERR_INVALID_ARG;
  if (p->channels > 32768 || (p->scale_group != 0 && p->scale_group != 128) || n_tiles > SG_MAX_TILES) return SG_ERR_UNSUPPORTED;
  if (n_tiles == 0 || p->rows == 0) return SG_OK;
  if (!tiles_ok(x, n_tiles) || !tiles_ok((const void* const*)out, n_tiles)) return SG_ERR_INVALID_ARG;
  const void* const* const lists[4] = {residual, gate, scale, shift};
  for (const void* const* list : lists)
    if (list && !tiles_ok(list, n_tiles)) return SG_ERR_INVALID_ARG;
  if (!aligned16(weight) || !aligned16(post_weight)) return SG_ERR_INVALID_ARG;
  if (eight != (out_scale != nullptr) || (eight && !tiles_ok((const void* const*)out_scale, n_tiles, 3u))) return SG_ERR_INVALID_ARG;
  auto alone = [&](const Written& w) { return w.different() && w.not_at(weight) && w.not_at(post_weight); };
  auto aliases_nothing = [&](const Written& w) {
    if (!alone(w) || !w.apart_from(x)) return false;
    for (const void* const* list : lists)
      if (!w.apart_from(list)) return false;
    return w.apart_from((const void* const*)sum);
  };
  const Written ow(out, n_tiles);
  if (!aliases_nothing(ow)) return SG_ERR_INVALID_ARG;
  if (eight && (!aliases_nothing(Written((void* const*)out_scale, n_tiles)) || !ow.apart_from((const void* const*)out_scale))) return SG_ERR_INVALID_ARG;
  if (sum) {
    if (!tiles_ok((const void* const*)sum, n_tiles)) return SG_ERR_INVALID_ARG;
    const Written sw(sum, n_tiles);
    if (!alone(sw) || !sw.apart_from(x, p->x_stride == p->sum_stride) || !sw.apart_from(residual, p->residual_stride == p->sum_stride) ||
        !sw.apart_from(gate) || !sw.apart_from(scale) || !sw.apart_from(shift))
      return SG_ERR_INVALID_ARG;
  }
  return launch_gated_norm(*p, n_tiles, x, residual, gate, post_weight, weight, scale, shift, run, sum, out, out_scale, (hipStream_t)stream);
}

int sg_int8_linear_validate(const sg_int8_linear_problem* p) { return validate(p); }

int sg_tile_int8_linear(const sg_int8_linear_problem* p, int32_t n_tiles, const void* const* x, const float* const* x_scale, const void* w,
                        const float* w_scale, const void* bias, const uint8_t* run, void* const* out, void* stream) {
  const int st = validate(p);
  if (st != SG_OK) return st;
  if (n_tiles < 0) return SG_ERR_INVALID_ARG;
  if (n_tiles > SG_MAX_TILES) return SG_ERR_UNSUPPORTED;
  if (n_tiles == 0 || p->rows == 0) return SG_OK;
  if (!tiles_ok(x, n_tiles) || !tiles_ok((const void* const*)x_scale, n_tiles, 3u) || !tiles_ok((const void* const*)out, n_tiles)) return SG_ERR_INVALID_ARG;
  if (!w || !aligned16(w) || !w_scale || !aligned16(w_scale) || !aligned16(bias)) return SG_ERR_INVALID_ARG;
  const Written ow(out, n_tiles);
  if (!ow.different() || !ow.apart_from(x) || !ow.apart_from((const void* const*)x_scale) || !ow.not_at(w) || !ow.not_at(w_scale) || !ow.not_at(bias))
    return SG_ERR_INVALID_ARG;
  // rows are numbered in 31 bits; the largest calls are cut into blocks of 256 x 256, a workgroup of 512 threads each, for 64 tiles a launch
  const int64_t rows = (int64_t)p->rows * std::min(n_tiles, 64);
  if ((int64_t)p->rows * n_tiles >= (1ll << 31) || (rows + 255) / 256 * ((p->outputs + 255ll) / 256) >= (1ll << 23)) return SG_ERR_UNSUPPORTED;
  return launch_int8_linear(*p, n_tiles, x, x_scale, w, w_scale, bias, run, out, (hipStream_t)stream);
}

}  // extern "C"
