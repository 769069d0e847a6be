// The norms of a block with what stands between them (sg_tile_gated_norm), one pass over the rows:
//     s = residual_scale * residual + gate * post(x) * post_weight,   y = norm(s) * weight * (1 + scale) + shift
// in the tensors' type or in 8 bits with scales.  Everything between the loads and the stores is fp32 and stays in registers: one read of x and the
// residual, one write of s and out.  Bound by memory.
//
// 75,600 rows of 5,120, bf16, layer norm with gate, scale and shift to e4m3 477 us (5.7 TB/s; a large copy runs at 4.9), with those in fp32 603; 4 tiles of
// 2,925 rows of 1,536 with a norm of x and fp32 vectors for each 225 rows 35 us (4.1); 10^6 rows of 128 190 us (5.4).
//
// What keeps it from the memory's rate is the arithmetic beside it (some 550 vector instructions for 24 channels of a wavefront, half of the time) and the
// chain of latencies of a row: loads, one or two reductions, loads of what the reductions stand in front of, stores.  So a lane holds 3 vectors of 8
// channels, which shares the reductions among more channels and still leaves room for 4 workgroups of 4 wavefronts (one vector a lane: 844 us at the first
// size; 2: 647; 4: 680 and more, with registers in memory), mean and variance come from one pass, and the vectors in 16 bits come along with the row.
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
  int32_t early;       // of gate, scale and shift, in this order: how many wait in LDS
  bool has_residual, has_gate, has_scale, has_shift, has_sum;
  float residual_scale, eps, post_eps, by_channels;
};

// T: stored type; M: type of gate, scale and shift; VPL: vectors per lane; LONG: a workgroup per row (else four wavefronts of rows of their own);
// POST: a norm of x first
template <typename T, typename M, int VPL, bool LONG, bool POST>
__global__ __launch_bounds__(LONG && VPL != 3 ? 1024 : 256, LONG && VPL == 3 && sizeof(M) == 2 && !POST ? 4 : 1) void gated_norm_kernel(const GatedArgs a, const GatedTable tab) {
  __shared__ float shared[2][2][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int lanes = LONG ? (int)blockDim.x : a.lanes;             // per row
  const int first = LONG ? (int)threadIdx.x : lane & (lanes - 1);
  const int rows_per_wg = LONG ? 1 : 256 / lanes;
  const int waves = LONG ? (int)(blockDim.x >> 6) : 1;
  const float by_channels = a.by_channels;
  [[maybe_unused]] int slot = 0;
  // One barrier per reduction: the slots alternate, so that one is written again behind the barrier of the reduction between.
  auto join = [&](auto& parts, int what, auto op) {
    float v = parts[what][0];
    for (int w = 1; w < waves; ++w) v = op(v, parts[what][w]);
    return v;
  };
  auto add = [](float x, float y) { return x + y; };
  auto row_sums = [&](float& u, float& v) {
    u = sum_over_lanes(u, LONG ? 64 : a.lanes);
    v = sum_over_lanes(v, LONG ? 64 : a.lanes);
    if (LONG && waves > 1) {
      if (lane == 0) { shared[slot][0][wave] = u; shared[slot][1][wave] = v; }
      __syncthreads();
      u = join(shared[slot], 0, add);
      v = join(shared[slot], 1, add);
      slot ^= 1;
    }
  };
  auto row_sum = [&](float v) {
    v = sum_over_lanes(v, LONG ? 64 : a.lanes);
    if (LONG && waves > 1) {
      if (lane == 0) shared[slot][0][wave] = v;
      __syncthreads();
      v = join(shared[slot], 0, add);
      slot ^= 1;
    }
    return v;
  };
  auto row_max = [&](float v) {
    v = max_over_lanes(v, LONG ? 64 : a.lanes);
    if (LONG && waves > 1) {
      if (lane == 0) shared[slot][0][wave] = v;
      __syncthreads();
      v = join(shared[slot], 0, larger_or_nan);
      slot ^= 1;
    }
    return v;
  };
  // Long rows: only the last vector of a lane may lie behind the row's end.
  auto on = [&](int i) { return (LONG && i < VPL - 1) || first + i * lanes < a.n_vec; };

  // v <- norm(v).  Places behind the row's end hold 0 before and anything afterwards.
  // mean and variance come from one pass, mean(v^2) - mean(v)^2, where that loses less than two bits, mean^2 <= variance / 4; rows farther from 0
  // take a second pass: with m1 = mean(v), d = v - m1, m2 = mean(d), which is what rounding left in m1: variance = mean(d^2) - m2^2, v - mean = d - m2.
  // Where rounding left more than half a deviation (rows of one value, or nearly one, whatever its size) nothing is left of that difference either, and
  // where a sum left fp32 there is none: a third pass takes the mean once more, of what the second leaves or of the row brought into range by a power of
  // two, and puts it between the least and the largest of those numbers, which no mean leaves: a row of one value has no deviations then, and in others they
  // are never larger than the row is wide.
  auto normalise = [&](float (&v)[VPL][8], int kind, float eps) {
    float m1 = 0.f, m2 = 0.f, sq = 0.f;
    const bool layer = kind == SG_NORM_LAYER;
#pragma unroll
    for (int i = 0; i < VPL; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) sq = fmaf(v[i][e], v[i][e], sq);
    if (layer) {
#pragma unroll
      for (int i = 0; i < VPL; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) m1 += v[i][e];
      row_sums(m1, sq);
      m1 *= by_channels;
    } else {
      sq = row_sum(sq);
    }
    sq = fmaf(-m1, m1, sq * by_channels);
    float mean = sq + eps;
    const float norm = rsqrtf(mean), back = -m1 * norm;
    // Another pass, too, where a sum leaves fp32 or the variance is next to nothing (a NaN too).  The lanes of a row agree; rows that share a wavefront may not.
    const bool again = !(mean >= kLeastMean && mean <= kMostFloat && m1 * m1 <= 0.25f * sq);
    if (LONG ? again : __any(again)) {
      const float m0 = m1;
      bool off = false;
      if (layer) {
        float q = 0.f;
#pragma unroll
        for (int i = 0; i < VPL; ++i)
          if (on(i)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) { const float d = v[i][e] - m0; m2 += d; q = fmaf(d, d, q); }
          }
        row_sums(m2, q);
        m2 *= by_channels;
        q = q * by_channels - m2 * m2;
        off = !(m2 * m2 <= 0.25f * q);
        mean = q + eps;
      }
      const bool odd = !(mean >= kLeastMean && mean <= kMostFloat), third = odd || off;
      const bool late = !odd || mean < kLeastMean;
      const float to = !odd ? 1.f : late ? kGrowRow : kShrinkRow;
      // `to` brings the row into the range: what is too small once its mean is gone, what is too large before it is taken
      auto at = [&](int i, int e) { return late ? (v[i][e] - m0 - m2) * to : v[i][e] * to; };
      float n1 = 0.f, n2 = 0.f;
      if (LONG ? third : __any(third)) {
        if (layer) {
          float least = __builtin_inff(), most = -__builtin_inff();
#pragma unroll
          for (int i = 0; i < VPL; ++i)
            if (on(i)) {
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const float u = at(i, e);
                n1 += u;
                least = __builtin_elementwise_minimum(least, u);
                most = larger_or_nan(most, u);
              }
            }
          n1 = row_sum(n1) * by_channels;
          least = -row_max(-least);
          most = row_max(most);
          n1 = __builtin_elementwise_minimum(larger_or_nan(n1, least), most);
        }
        float w = 0.f;
#pragma unroll
        for (int i = 0; i < VPL; ++i)
          if (on(i)) {
#pragma unroll
            for (int e = 0; e < 8; ++e) { const float d = at(i, e) - n1; n2 += d; w = fmaf(d, d, w); }
          }
        row_sums(n2, w);
        n2 = layer ? n2 * by_channels : 0.f;
        w = w * by_channels - n2 * n2;
        if (w < 0.f) w = 0.f;   // (a NaN stays)
        if (third) {
          mean = w + eps * to * to;
          if (mean == 0.f && eps > 0.f) mean = 1.f;   // no deviations; eps 2^-144 has left fp32, but it is there
        } else {
          n1 = n2 = 0.f;
        }
      }
      const float other = rsqrtf(mean);
#pragma unroll
      for (int i = 0; i < VPL; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = again ? (at(i, e) - n1 - n2) * other : fmaf(v[i][e], norm, back);
      return;
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[i][e] = fmaf(v[i][e], norm, back);
  };

  // What each lane asked for of gate, scale and shift: [3][VPL][parts of 16 bytes][lanes of the workgroup].
  extern __shared__ __align__(1024) char vectors[];
  constexpr int kParts = sizeof(M) / 2;
  auto bring = [&](int what, int i, const M* p) {
#pragma unroll
    for (int h = 0; h < kParts; ++h)
      dma16_addr(p + 4 * h, __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(SG_LDS char*)vectors + ((what * VPL + i) * kParts + h) * (int)blockDim.x * 16 + wave * 1024));
  };
  auto kept = [&](int what, int i) {
    const char* const at = vectors + ((what * VPL + i) * kParts * (int)blockDim.x + (int)threadIdx.x) * 16;
    Chan8<M> v;
    if constexpr (kParts == 1) v.w = *(const u32x4*)at;
    else { v.a = *(const f32x4*)at; v.b = *(const f32x4*)(at + (int)blockDim.x * 16); }
    return v;
  };
  const uint32_t step = gridDim.x * rows_per_wg;
  for (uint32_t base = blockIdx.x * rows_per_wg; base < a.n_rows; base += step) {
    const uint32_t at = base + (LONG ? 0 : threadIdx.x / lanes);
    const bool in = at < a.n_rows;
    const uint32_t at_in = in ? at : a.n_rows - 1;
    const int tile = (int)divide(at_in, a.by_rows);
    const int64_t row = at_in - (uint32_t)tile * (uint32_t)a.rows;
    const bool runs = in && (!a.run || a.run[tile] != 0);   // (the lanes of a row agree)
    if (LONG ? !runs : !__any(runs)) continue;         // nothing to do for the workgroup, or for a wavefront that meets no others
    const bool there = LONG || runs;
    const int64_t vec = (int64_t)divide((uint32_t)row, a.by_mod) * a.m_stride;
    const T* const x = (const T*)tab.x[tile] + row * a.x_stride;
    constexpr bool kInRegisters = !LONG;
    Chan8<M> near[3][VPL];   // short rows: in registers
    auto ask = [&](int what, const void* from, bool has) {
      if constexpr (kInRegisters) {
        if (has) {
#pragma unroll
          for (int i = 0; i < VPL; ++i) {
            near[what][i].clear();
            if (there && on(i)) near[what][i].load((const M*)from + vec + 8 * (first + i * lanes));
          }
        }
      }
    };
    auto vector_of = [&](int what, int i, const void* from) {
      if constexpr (kInRegisters) return near[what][i];
      if (what < a.early) return kept(what, i);
      Chan8<M> v;
      v.clear();
      if (there && on(i)) v.load((const M*)from + vec + 8 * (first + i * lanes));
      return v;
    };
    // Everything that the row needs is asked for at once.  Gate, scale and shift of long rows wait in LDS, each lane's in its own place, which takes no
    // registers and no barrier.
    if constexpr (kInRegisters) {
      ask(0, tab.gate[tile], a.has_gate);
    } else {
#pragma unroll
      for (int i = 0; i < VPL; ++i)
        if (on(i)) {
          const int c = 8 * (first + i * lanes);
          if (a.has_gate && a.early > 0) bring(0, i, (const M*)tab.gate[tile] + vec + c);
          if (a.has_scale && a.early > 1) bring(1, i, (const M*)tab.scale[tile] + vec + c);
          if (a.has_shift && a.early > 2) bring(2, i, (const M*)tab.shift[tile] + vec + c);
        }
    }
    float s[VPL][8];
    Chan8<T> xv[VPL], rv[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      xv[i].clear();
      if (there && on(i)) xv[i].stream(x + 8 * (first + i * lanes));
    }
    if (a.has_residual) {
      const T* const r = (const T*)tab.residual[tile] + row * a.r_stride;
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        rv[i].clear();
        if (there && on(i)) rv[i].stream(r + 8 * (first + i * lanes));
      }
    }
    if constexpr (!kInRegisters) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int i = 0; i < VPL; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) s[i][e] = xv[i].get(e);
    if constexpr (POST) {
      normalise(s, a.post_norm, a.post_eps);
#pragma unroll
      for (int i = 0; i < VPL; ++i)
        if (!on(i)) {
#pragma unroll
          for (int e = 0; e < 8; ++e) s[i][e] = 0.f;
        } else if (a.post_weight) {
          Chan8<T> w;
          w.load((const T*)a.post_weight + 8 * (first + i * lanes));
#pragma unroll
          for (int e = 0; e < 8; ++e) s[i][e] *= w.get(e);
        }
    }
    if (a.has_gate) {
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        Chan8<M> g = vector_of(0, i, tab.gate[tile]);
        if (!on(i)) g.clear();
#pragma unroll
        for (int e = 0; e < 8; ++e) s[i][e] *= g.get(e);
      }
    }
    if (a.has_residual) {
#pragma unroll
      for (int i = 0; i < VPL; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[i][e] = fmaf(a.residual_scale, rv[i].get(e), s[i][e]);
    }
    if (a.has_sum) {
      T* const o = (T*)tab.sum[tile] + row * a.s_stride;
#pragma unroll
      for (int i = 0; i < VPL; ++i)
        if (there && on(i)) stream8(o + 8 * (first + i * lanes), s[i]);
    }
    ask(1, tab.scale[tile], a.has_scale);
    ask(2, tab.shift[tile], a.has_shift);
    normalise(s, a.norm, a.eps);
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      if (a.weight && on(i)) {
        Chan8<T> w;
        w.load((const T*)a.weight + 8 * (first + i * lanes));
#pragma unroll
        for (int e = 0; e < 8; ++e) s[i][e] *= w.get(e);
      }
      if (a.has_scale && a.has_shift) {
        const Chan8<M> w = vector_of(1, i, tab.scale[tile]), b = vector_of(2, i, tab.shift[tile]);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[i][e] = fmaf(s[i][e], 1.f + w.get(e), b.get(e));
      } else if (a.has_scale) {
        const Chan8<M> w = vector_of(1, i, tab.scale[tile]);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[i][e] *= 1.f + w.get(e);
      } else if (a.has_shift) {
        const Chan8<M> b = vector_of(2, i, tab.shift[tile]);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[i][e] += b.get(e);
      }
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
      most[i] = fabsf(s[i][0]);
#pragma unroll
      for (int e = 1; e < 8; ++e) most[i] = larger_or_nan(most[i], fabsf(s[i][e]));
      if (!(there && on(i))) most[i] = 0.f;
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
    float inv_row = 0.f;
    if (a.group_vecs == 0) inv_row = most[0] < kLeastMean ? 0.f : top / most[0];
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      const float inv = a.group_vecs == 0 ? inv_row : most[i] < kLeastMean ? 0.f : top / most[i];
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

template <typename T, typename M, bool POST>
int launch(const GatedArgs& a, const GatedTable& tab, bool is_short, int vpl, int threads, uint32_t grid, hipStream_t s) {
  const size_t lds = is_short ? 0 : (size_t)a.early * vpl * threads * 8 * sizeof(M);
#define SG_GATED(V, L) gated_norm_kernel<T, M, V, L, POST><<<dim3(grid), threads, lds, s>>>(a, tab)
  if (is_short && vpl == 1) SG_GATED(1, false);
  else if (is_short) SG_GATED(2, false);
  else if (vpl == 1) SG_GATED(1, true);
  else if (vpl == 2) SG_GATED(2, true);
  else if (vpl == 3) SG_GATED(3, true);
  else SG_GATED(4, true);
#undef SG_GATED
  SG_HIP_TRY(hipGetLastError());
  return SG_OK;
}
template <typename T, typename M>
int launch(const GatedArgs& a, const GatedTable& tab, bool is_short, int vpl, int threads, uint32_t grid, hipStream_t s) {
  return a.post_norm != SG_NORM_NONE ? launch<T, M, true>(a, tab, is_short, vpl, threads, grid, s) : launch<T, M, false>(a, tab, is_short, vpl, threads, grid, s);
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
  a.by_channels = 1.f / (float)p.channels;
  // Up to 256 channels rows share a wavefront, 2 vectors a lane (10^6 rows of 128 channels 190 us, one vector 343 in an earlier form; with blocks of 128 channels always one,
  // which leaves a block to 16 lanes side by side).  512 channels: one wavefront with one vector a lane (400,000 rows 256 us; shared 313 when that took 270).  Then up to 3
  // vectors; beyond 6,144 channels 2 (30,000 rows of 8,192 324 us; 3: 450 when that took 340) up to 16 wavefronts and beyond 16,384 4.
  const bool is_short = a.n_vec <= 32;
  int vpl, threads = 256;
  if (is_short) {
    vpl = a.group_vecs == 0 && a.n_vec > 1 ? 2 : 1;
    a.lanes = 1;
    while (a.lanes * vpl < a.n_vec) a.lanes <<= 1;
  } else {
    const int want = a.n_vec > 2048 ? 4 : a.n_vec <= 768 ? 3 : 2;
    threads = (a.n_vec + 64 * want - 1) / (64 * want) * 64;
    a.lanes = threads;
    vpl = (a.n_vec + threads - 1) / threads;   // so that all but the last vector of every lane lie inside the row
  }
  // Four workgroups of 4 wavefronts are to fit beside one another, and 64 KiB need no raised limit.
  const int tensor_bytes = vpl * threads * 8 * (p.mod_dtype == SG_F32 ? 4 : 2), room = threads < 409 ? 160 * threads : 65536;
  a.early = p.mod_dtype == SG_F32 ? 0 : room / tensor_bytes < 3 ? room / tensor_bytes : 3;
  const int rows_per_wg = is_short ? 256 / a.lanes : 1;
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
    // New workgroups for new rows: walking them, 2,048 workgroups took 344 us instead of 205 for 10^6 rows of 128 channels (190 by now).  (2^21 a launch, then they walk.)
    if (grid > 1u << 21) grid = 1u << 21;
    const int st = p.dtype == SG_F32      ? launch<float, float>(a, tab, is_short, vpl, threads, grid, s)
                   : p.mod_dtype == SG_F32 ? launch<uint16_t, float>(a, tab, is_short, vpl, threads, grid, s)
                                           : launch<uint16_t, uint16_t>(a, tab, is_short, vpl, threads, grid, s);
    if (st != SG_OK) return st;
  }
  return SG_OK;
}

}  // namespace sg
