// The norms of a block with what stands between them (sg_tile_gated_norm), one pass over the rows:
//     s = residual_scale * residual + gate * post(x) * post_weight,   y = norm(s) * weight * (1 + scale) + shift
// in the tensors' type or in 8 bits with scales.  Everything between the loads and the stores is fp32 and stays in registers: one read of x and the
// residual, one write of s and out.  Bound by memory.
//
// Rows of up to 512 channels share a wavefront (the lanes of a row are a power of two), up to 2,048 take a wavefront each, up to 8,192 a
// workgroup of 4 and beyond that one of 16 wavefronts, so that a lane never holds more than 4 vectors of 8 channels.
#include "block_api.h"
#include "row_common.h"

namespace sg {
namespace {

constexpr int kGatedTilesPerLaunch = 32;
struct GatedTable {
  const void* x[kGatedTilesPerLaunch];
  const void* residual[kGatedTilesPerLaunch];
  const void* gate[kGatedTilesPerLaunch];
  const void* scale[kGatedTilesPerLaunch];
  const void* shift[kGatedTilesPerLaunch];
  void* sum[kGatedTilesPerLaunch];
  void* out[kGatedTilesPerLaunch];
  float* out_scale[kGatedTilesPerLaunch];
};
struct GatedArgs {
  const void* post_weight;
  const void* weight;
  const uint8_t* run;
  int64_t x_stride, r_stride, s_stride, o_stride, m_stride;
  uint32_t n_rows;     // of all tiles of the launch, below 2^31
  int32_t rows, channels, n_vec, lanes, group_vecs;
  Divisor by_rows, by_mod;   // rows of a tile; rows that share a vector
  int32_t norm, post_norm, out_dtype;
  bool has_residual, has_gate, has_scale, has_shift, has_sum;
  float residual_scale, eps, post_eps;
};

// T: stored type; M: type of gate, scale and shift; VPL: vectors per lane; WAVES: wavefronts per row (1: four wavefronts of a workgroup take rows
// of their own)
template <typename T, typename M, int VPL, int WAVES>
__global__ __launch_bounds__(WAVES == 16 ? 1024 : 256) void gated_norm_kernel(const GatedArgs a, const GatedTable tab) {
  constexpr int kThreads = WAVES == 16 ? 1024 : 256;
  __shared__ float shared[2][WAVES][2];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int lanes = WAVES > 1 ? 64 * WAVES : a.lanes;             // per row
  const int first = WAVES > 1 ? (int)threadIdx.x : lane & (lanes - 1);
  const int rows_per_wg = kThreads / lanes;
  const float by_channels = 1.f / (float)a.channels;
  int slot = 0;
  // One barrier per reduction: the slots alternate, so that one is written again behind the barrier of the reduction between.
  auto join = [&](float& u, float& v, auto op) {
    if constexpr (WAVES > 1) {
      if (lane == 0) { shared[slot][wave][0] = u; shared[slot][wave][1] = v; }
      __syncthreads();
      u = shared[slot][0][0]; v = shared[slot][0][1];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) { u = op(u, shared[slot][w][0]); v = op(v, shared[slot][w][1]); }
      slot ^= 1;
    }
  };
  auto add = [](float x, float y) { return x + y; };
  auto row_sum = [&](float v) {
    float none = 0.f;
    v = sum_over_lanes(v, WAVES > 1 ? 64 : a.lanes);
    join(v, none, add);
    return v;
  };
  auto row_sums = [&](float& u, float& v) {
    u = sum_over_lanes(u, WAVES > 1 ? 64 : a.lanes);
    v = sum_over_lanes(v, WAVES > 1 ? 64 : a.lanes);
    join(u, v, add);
  };
  auto row_max = [&](float v) {
    float none = 0.f;
    v = max_over_lanes(v, WAVES > 1 ? 64 : a.lanes);
    join(v, none, larger_or_nan);
    return v;
  };
  auto on = [&](int i) { return first + i * lanes < a.n_vec; };

  // v <- norm(v); places behind the row's end hold 0 and are left at anything.
  // Layer: with m1 = mean(v), d = v - m1, m2 = mean(d): variance = mean(d^2) - m2^2, v - mean = d - m2.  m2 is what rounding left in m1.
  auto normalise = [&](float (&v)[VPL][8], int kind, float eps) {
    float m1 = 0.f, m2 = 0.f, sq = 0.f;
    const bool layer = kind == SG_NORM_LAYER;
    if (layer) {
#pragma unroll
      for (int i = 0; i < VPL; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) m1 += v[i][e];
      m1 = row_sum(m1) * by_channels;
#pragma unroll
      for (int i = 0; i < VPL; ++i)
        if (on(i)) {
#pragma unroll
          for (int e = 0; e < 8; ++e) { const float d = v[i][e] - m1; m2 += d; sq += d * d; }
        }
      row_sums(m2, sq);
      m2 *= by_channels;
      sq = sq * by_channels - m2 * m2;
      if (sq < 0.f) sq = 0.f;   // (a NaN stays)
    } else {
#pragma unroll
      for (int i = 0; i < VPL; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) sq += v[i][e] * v[i][e];
      sq = row_sum(sq) * by_channels;
    }
    const float mean = sq + eps;
    float norm = rsqrtf(mean);
    const bool odd = !(mean >= kLeastMean && mean <= kMostFloat);   // (a NaN too; the lanes of a row agree, rows that share a wavefront may not)
    if (WAVES > 1 ? odd : __any(odd)) {
      const bool grow = mean < kLeastMean;
      const float to = grow ? kGrowRow : kShrinkRow;
      float n1 = 0.f, n2 = 0.f, q = 0.f;
      auto at = [&](int i, int e) { return grow ? (v[i][e] - m1 - m2) * to : v[i][e] * to; };
      if (layer) {   // (a row that grows has lost its mean already)
#pragma unroll
        for (int i = 0; i < VPL; ++i)
          if (on(i)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) n1 += at(i, e);
          }
        n1 = row_sum(n1) * by_channels;
      }
#pragma unroll
      for (int i = 0; i < VPL; ++i)
        if (on(i)) {
#pragma unroll
          for (int e = 0; e < 8; ++e) { const float d = at(i, e) - n1; n2 += d; q += d * d; }
        }
      row_sums(n2, q);
      n2 = layer ? n2 * by_channels : 0.f;
      q = q * by_channels - n2 * n2;
      if (q < 0.f) q = 0.f;
      const float other = rsqrtf(q + eps * to * to);
#pragma unroll
      for (int i = 0; i < VPL; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = odd ? (at(i, e) - n1 - n2) * other : (v[i][e] - m1 - m2) * norm;
      return;
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = (v[i][e] - m1 - m2) * norm;
  };

  const uint32_t step = gridDim.x * rows_per_wg;
  for (uint32_t base = blockIdx.x * rows_per_wg; base < a.n_rows; base += step) {
    const uint32_t at = base + (WAVES > 1 ? 0 : threadIdx.x / lanes);
    const bool in = at < a.n_rows;
    const uint32_t at_in = in ? at : a.n_rows - 1;
    const int tile = (int)divide(at_in, a.by_rows);
    const int64_t row = at_in - (uint32_t)tile * (uint32_t)a.rows;
    const bool runs = in && (!a.run || a.run[tile] != 0);   // (the lanes of a row agree)
    if (WAVES > 1 ? !runs : !__any(runs)) continue;         // nothing to do for the workgroup, or for a wavefront that meets no others
    const bool there = WAVES > 1 || runs;
    const int64_t vec = (int64_t)divide((uint32_t)row, a.by_mod) * a.m_stride;
    const T* const x = (const T*)tab.x[tile] + row * a.x_stride;
    float s[VPL][8];
    Chan8<T> rv[VPL];
    {
      Chan8<T> xv[VPL];
#pragma unroll
      for (int i = 0; i < VPL; ++i)
        if (there && on(i)) xv[i].stream(x + 8 * (first + i * lanes));
      if (a.has_residual) {
        const T* const r = (const T*)tab.residual[tile] + row * a.r_stride;
#pragma unroll
        for (int i = 0; i < VPL; ++i)
          if (there && on(i)) rv[i].stream(r + 8 * (first + i * lanes));
      }
#pragma unroll
      for (int i = 0; i < VPL; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[i][e] = there && on(i) ? xv[i].get(e) : 0.f;
    }
    if (a.post_norm != SG_NORM_NONE) {
      normalise(s, a.post_norm, a.post_eps);
      if (a.post_weight) {
#pragma unroll
        for (int i = 0; i < VPL; ++i)
          if (on(i)) {
            Chan8<T> w;
            w.load((const T*)a.post_weight + 8 * (first + i * lanes));
#pragma unroll
            for (int e = 0; e < 8; ++e) s[i][e] *= w.get(e);
          }
      }
    }
    if (a.has_gate) {
      const M* const g = (const M*)tab.gate[tile] + vec;
#pragma unroll
      for (int i = 0; i < VPL; ++i)
        if (there && on(i)) {
          Chan8<M> w;
          w.load(g + 8 * (first + i * lanes));
#pragma unroll
          for (int e = 0; e < 8; ++e) s[i][e] *= w.get(e);
        }
    }
    if (a.has_residual) {
#pragma unroll
      for (int i = 0; i < VPL; ++i)
        if (there && on(i)) {
#pragma unroll
          for (int e = 0; e < 8; ++e) s[i][e] = fmaf(a.residual_scale, rv[i].get(e), s[i][e]);
        }
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) s[i][e] = there && on(i) ? s[i][e] : 0.f;
    if (a.has_sum) {
      T* const o = (T*)tab.sum[tile] + row * a.s_stride;
#pragma unroll
      for (int i = 0; i < VPL; ++i)
        if (there && on(i)) stream8(o + 8 * (first + i * lanes), s[i]);
    }
    normalise(s, a.norm, a.eps);
#pragma unroll
    for (int i = 0; i < VPL; ++i)
      if (there && on(i)) {
        const int c = 8 * (first + i * lanes);
        if (a.weight) {
          Chan8<T> w;
          w.load((const T*)a.weight + c);
#pragma unroll
          for (int e = 0; e < 8; ++e) s[i][e] *= w.get(e);
        }
        if (a.has_scale) {
          Chan8<M> w;
          w.load((const M*)tab.scale[tile] + vec + c);
#pragma unroll
          for (int e = 0; e < 8; ++e) s[i][e] = s[i][e] * (1.f + w.get(e));
        }
        if (a.has_shift) {
          Chan8<M> w;
          w.load((const M*)tab.shift[tile] + vec + c);
#pragma unroll
          for (int e = 0; e < 8; ++e) s[i][e] += w.get(e);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) s[i][e] = 0.f;
      }
    if (a.out_dtype == SG_F32 || a.out_dtype == SG_BF16) {
      T* const o = (T*)tab.out[tile] + row * a.o_stride;
#pragma unroll
      for (int i = 0; i < VPL; ++i)
        if (there && on(i)) stream8(o + 8 * (first + i * lanes), s[i]);
      continue;
    }
    uint8_t* const o = (uint8_t*)tab.out[tile] + row * a.o_stride;
    float* const scales = tab.out_scale[tile];
    const float top = a.out_dtype == SG_I8 ? 127.f : 448.f;
    float most[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      most[i] = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) most[i] = larger_or_nan(most[i], fabsf(s[i][e]));
    }
    // (an infinity becomes a NaN: no factor brings it into 8 bits)
    auto scale_of = [&](float m) { return m < kLeastMean ? 0.f : m <= kMostFloat ? m / top : __uint_as_float(0x7fc00000u); };
    if (a.group_vecs == 0) {
      float m = most[0];
#pragma unroll
      for (int i = 1; i < VPL; ++i) m = larger_or_nan(m, most[i]);
      m = row_max(m);
#pragma unroll
      for (int i = 0; i < VPL; ++i) most[i] = m;
      if (there && first == 0) scales[row] = scale_of(m);
    } else {   // 16 lanes side by side hold the 128 channels of a block
      const int groups = a.n_vec / a.group_vecs;
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        most[i] = max_over_lanes(most[i], 16);
        const int v = first + i * lanes;
        if (there && v < a.n_vec && (v & 15) == 0) scales[row * groups + (v >> 4)] = scale_of(most[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      const float inv = most[i] < kLeastMean ? 0.f : top / most[i];
      uint32_t lo = 0, hi = 0;
      if (a.out_dtype == SG_I8) {   // rounded to the nearest integer; the largest product rounds to 127
        auto four = [&](int e) {
          int b[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) b[j] = (int)__builtin_rintf(s[i][e + j] * inv) & 0xff;
          return (uint32_t)(b[0] | b[1] << 8 | b[2] << 16 | b[3] << 24);
        };
        lo = four(0);
        hi = four(4);
      } else {                      // rounded to the nearest 8-bit value; the largest product rounds to 448
        int l = 0, h = 0;
        l = __builtin_amdgcn_cvt_pk_fp8_f32(s[i][0] * inv, s[i][1] * inv, l, false);
        l = __builtin_amdgcn_cvt_pk_fp8_f32(s[i][2] * inv, s[i][3] * inv, l, true);
        h = __builtin_amdgcn_cvt_pk_fp8_f32(s[i][4] * inv, s[i][5] * inv, h, false);
        h = __builtin_amdgcn_cvt_pk_fp8_f32(s[i][6] * inv, s[i][7] * inv, h, true);
        lo = (uint32_t)l;
        hi = (uint32_t)h;
      }
      if (there && on(i)) __builtin_nontemporal_store(u32x2{lo, hi}, (u32x2*)(o + 8 * (first + i * lanes)));
    }
  }
}

template <typename T, typename M>
int launch(const GatedArgs& a, const GatedTable& tab, int vpl, int waves, uint32_t grid, hipStream_t s) {
#define SG_GATED(V, W) gated_norm_kernel<T, M, V, W><<<dim3(grid), W == 16 ? 1024 : 256, 0, s>>>(a, tab)
#define SG_GATED_VPL(W)                \
  do {                                 \
    if (vpl <= 1) SG_GATED(1, W);      \
    else if (vpl == 2) SG_GATED(2, W); \
    else if (vpl == 3) SG_GATED(3, W); \
    else SG_GATED(4, W);               \
  } while (0)
  if (waves == 1) SG_GATED_VPL(1);
  else if (waves == 4) SG_GATED_VPL(4);
  else SG_GATED_VPL(16);
#undef SG_GATED_VPL
#undef SG_GATED
  SG_HIP_TRY(hipGetLastError());
  return SG_OK;
}

}  // namespace

int launch_gated_norm(const sg_gated_norm_problem& p, int n_tiles, const void* const* x, const void* const* residual, const void* const* gate,
                      const void* post_weight, const void* weight, const void* const* scale, const void* const* shift, const uint8_t* run,
                      void* const* sum, void* const* out, float* const* out_scale, hipStream_t s) {
  GatedArgs a = {};
  a.post_weight = post_weight; a.weight = weight;
  a.x_stride = p.x_stride; a.r_stride = p.residual_stride; a.s_stride = p.sum_stride; a.o_stride = p.out_stride;
  a.rows = p.rows; a.channels = p.channels; a.n_vec = p.channels / 8;
  a.group_vecs = p.scale_group / 8;
  a.by_rows = make_divisor((uint32_t)p.rows);
  a.by_mod = make_divisor((uint32_t)(p.mod_rows > 0 ? p.mod_rows : p.rows));
  a.m_stride = p.mod_rows > 0 && p.mod_rows < p.rows ? p.mod_stride : 0;
  a.norm = p.norm; a.post_norm = p.post_norm; a.out_dtype = p.out_dtype;
  a.has_residual = residual != nullptr; a.has_gate = gate != nullptr; a.has_scale = scale != nullptr; a.has_shift = shift != nullptr;
  a.has_sum = sum != nullptr;
  a.residual_scale = p.residual_scale; a.eps = p.eps; a.post_eps = p.post_eps;
  const int waves = a.n_vec <= 64 * 4 ? 1 : a.n_vec <= 256 * 4 ? 4 : 16;
  a.lanes = 64 * waves;
  if (a.n_vec < 64) {
    a.lanes = 1;
    while (a.lanes < a.n_vec) a.lanes <<= 1;
  }
  const int vpl = (a.n_vec + a.lanes - 1) / a.lanes, rows_per_wg = waves == 1 ? 256 / a.lanes : 1;
  // rows of a launch are numbered in 31 bits (the last step of a workgroup passes their number by less than the grid)
  int most_tiles = (int)((1ll << 30) / p.rows);
  most_tiles = most_tiles < 1 ? 1 : most_tiles > kGatedTilesPerLaunch ? kGatedTilesPerLaunch : most_tiles;
  for (int t0 = 0; t0 < n_tiles; t0 += most_tiles) {
    const int n = n_tiles - t0 < most_tiles ? n_tiles - t0 : most_tiles;
    GatedTable tab = {};
    for (int i = 0; i < n; ++i) {
      tab.x[i] = x[t0 + i];
      tab.residual[i] = residual ? residual[t0 + i] : nullptr;
      tab.gate[i] = gate ? gate[t0 + i] : nullptr;
      tab.scale[i] = scale ? scale[t0 + i] : nullptr;
      tab.shift[i] = shift ? shift[t0 + i] : nullptr;
      tab.sum[i] = sum ? sum[t0 + i] : nullptr;
      tab.out[i] = out[t0 + i];
      tab.out_scale[i] = out_scale ? out_scale[t0 + i] : nullptr;
    }
    a.n_rows = (uint32_t)n * (uint32_t)p.rows;
    a.run = run ? run + t0 : nullptr;
    uint32_t grid = (a.n_rows + rows_per_wg - 1) / rows_per_wg;
    // As the residual norm: a workgroup per row of 4 wavefronts, 8,192 workgroups of a wavefront per row; shorter rows and rows of 16 wavefronts
    // fill the chip and walk.
    const uint32_t most = waves == 16 ? 512 : waves == 4 ? 1u << 22 : a.lanes == 64 ? 8192 : 2048;
    if (grid > most) grid = most;
    const int st = p.dtype == SG_F32      ? launch<float, float>(a, tab, vpl, waves, grid, s)
                   : p.mod_dtype == SG_F32 ? launch<uint16_t, float>(a, tab, vpl, waves, grid, s)
                                           : launch<uint16_t, uint16_t>(a, tab, vpl, waves, grid, s);
    if (st != SG_OK) return st;
  }
  return SG_OK;
}

}  // namespace sg
