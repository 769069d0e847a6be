// Residual addition and root-mean-square norm of the rows of tiles, in the tensors' type or in 8 bits with scales (sg_tile_residual_norm):
//     s = x + r,   y = s * rsqrt(mean(s^2) + eps) * w,   out = y   or   out = e4m3(y * 448 / a), scale = a / 448, a = max|y| of a row or block
// Everything between the loads and the stores is fp32 and stays in registers: one read of x and r, one write of s and out.  Bound by
// memory: 75,600 rows of 5,120, bf16 + bf16 to bf16 and e4m3 437 us (6.2 TB/s; a large copy runs at 5.4), 9 tiles of 153,600 rows of 128 in bf16
// 131 us (5.4 TB/s).
//
// Rows of up to 512 channels share a wavefront (the lanes of a row are a power of two), up to 2,048 take a wavefront each, up to 8,192 a
// workgroup of 4 and beyond that one of 16 wavefronts, so that a lane never holds more than 4 vectors of 8 channels and enough
// wavefronts fit beside one another to keep the memory busy.
#include "sg_common.h"

namespace sg {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kNormTilesPerLaunch = 64;
struct NormTable {
  const void* x[kNormTilesPerLaunch];
  const void* residual[kNormTilesPerLaunch];
  void* sum[kNormTilesPerLaunch];
  void* out[kNormTilesPerLaunch];
  float* scale[kNormTilesPerLaunch];
};
struct NormArgs {
  const void* weight;
  const uint8_t* run;
  int64_t x_stride, r_stride, s_stride, o_stride;
  int64_t n_rows;      // of all tiles of the launch
  int32_t rows, channels, n_vec, lanes, group_vecs;
  bool has_residual, has_sum;
  float eps;
};

// 8 channels as they are stored.  Rows pass once and are not to stay in the caches (75,600 rows of 5,120, bf16 to e4m3: 454 -> 440 us; fp32, whose
// 32 bytes a lane take two accesses that meet in the cache, loses by it: 276 -> 323 us at 4,096 channels).
template <typename T> struct Vec8;
template <> struct Vec8<uint16_t> {
  u32x4 w;
  __device__ __forceinline__ void load(const uint16_t* p) { w = *(const u32x4*)p; }
  __device__ __forceinline__ void stream(const uint16_t* p) { w = __builtin_nontemporal_load((const u32x4*)p); }
  __device__ __forceinline__ float get(int i) const { return i & 1 ? __uint_as_float(w[i >> 1] & 0xffff0000u) : __uint_as_float(w[i >> 1] << 16); }
};
template <> struct Vec8<float> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = *(const f32x4*)p; b = *(const f32x4*)(p + 4); }
  __device__ __forceinline__ void stream(const float* p) { load(p); }
  __device__ __forceinline__ float get(int i) const { return i < 4 ? a[i] : b[i - 4]; }
};
__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
  __builtin_nontemporal_store(u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])}, (u32x4*)p);
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
  *(f32x4*)p = f32x4{v[0], v[1], v[2], v[3]};
  *(f32x4*)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}

// The larger of two numbers; NaN where one is (fmaxf gives the other one, and a block with a NaN would have a scale that hides it).
__device__ __forceinline__ float nan_max(float a, float b) { return __builtin_elementwise_maximum(a, b); }

constexpr float kE4m3Max = 448.f;
// Blocks whose largest value is below this are written as zeros with a scale of 0: 448 / a has to stay finite.
constexpr float kLeast = 7.888609052210118e-31f;   // 2^-100
// Mean squares outside kLeast .. the largest fp32 number are taken again of the row scaled by a power of two, so that neither a square nor their sum
// leaves the range: |s| 2^-72 is below 2^56, 32,768 squares of it below 2^127; and with a mean below 2^-100 and up to 32,768 channels |s| 2^100 is below
// 2^58, the square of the smallest fp32 number 2^-98.  (From kLeast on what squares below 2^-149 lack is below 2^-49 of the mean.)
constexpr float kShrink = 2.117582368135751e-22f, kGrow = 1.2676506002282294e30f;   // 2^-72, 2^100

// T: stored type; E4M3: output in 8 bits; VPL: vectors per lane; WAVES: wavefronts per row (1: four wavefronts of a workgroup take rows
// of their own)
template <typename T, bool E4M3, int VPL, int WAVES>
__global__ __launch_bounds__(WAVES == 16 ? 1024 : 256) void residual_norm_kernel(const NormArgs a, const NormTable tab) {
  constexpr int kThreads = WAVES == 16 ? 1024 : 256;
  __shared__ float shared[2][3][WAVES];   // [parity of the row][sum, maximum, sum of the scaled row]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int lanes = WAVES > 1 ? 64 * WAVES : a.lanes;             // per row
  const int first = WAVES > 1 ? (int)threadIdx.x : lane & (lanes - 1);
  const int rows_per_wg = kThreads / lanes;
  int parity = 0;
  // One barrier per reduction: a slot is written again two rows later, behind the barrier of the row between.
  auto across = [&](float v, int what, auto op) {
    if constexpr (WAVES == 1) {
      for (int d = 1; d < lanes; d <<= 1) v = op(v, __shfl_xor(v, d, 64));
    } else {
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) v = op(v, __shfl_xor(v, d, 64));
      if (lane == 0) shared[parity][what][wave] = v;
      __syncthreads();
      v = shared[parity][what][0];
#pragma unroll
      for (int w = 1; w < WAVES; ++w) v = op(v, shared[parity][what][w]);
    }
    return v;
  };
  auto row_sum = [&](float v, int what) { return across(v, what, [](float x, float y) { return x + y; }); };
  auto row_max = [&](float v) { return across(v, 1, [](float x, float y) { return nan_max(x, y); }); };
  // What a row has one of: of a row of whole wavefronts in a scalar register (fp32 rows of 20,480 channels to e4m3 254 -> 246 us).
  auto of_row = [](float v) { return WAVES > 1 ? __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))) : v; };
  Vec8<T> w[VPL];
#pragma unroll
  for (int i = 0; i < VPL; ++i)
    if (a.weight && first + i * lanes < a.n_vec) w[i].load((const T*)a.weight + 8 * (first + i * lanes));
  const int64_t step = (int64_t)gridDim.x * rows_per_wg;
  for (int64_t base = (int64_t)blockIdx.x * rows_per_wg; base < a.n_rows; base += step) {
    const int64_t at = base + (WAVES > 1 ? 0 : threadIdx.x / lanes);
    const bool in = at < a.n_rows;
    const int64_t at_in = in ? at : a.n_rows - 1;
    const int tile = (int)(at_in / a.rows);
    const int64_t row = at_in - (int64_t)tile * a.rows;
    const bool runs = in && (!a.run || a.run[tile] != 0);   // (the lanes of a row agree)
    // Nothing to do for the workgroup, or for a wavefront that meets no others (none of 8 tiles of 9,450 rows of 5,120 to e4m3: 190 -> 74 us, 4 of them
    // 313 -> 257, all 445 - 448).
    if (WAVES > 1 ? !runs : !__any(runs)) continue;
    const bool there = WAVES > 1 || runs;
    const T* const x = (const T*)tab.x[tile] + row * a.x_stride;
    const T* const r = a.has_residual ? (const T*)tab.residual[tile] + row * a.r_stride : nullptr;
    Vec8<T> xv[VPL], rv[VPL];
#pragma unroll
    for (int i = 0; i < VPL; ++i)
      if (there && first + i * lanes < a.n_vec) {
        xv[i].stream(x + 8 * (first + i * lanes));
        if (a.has_residual) rv[i].stream(r + 8 * (first + i * lanes));
      }
    float s[VPL][8];
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < VPL; ++i) {
      const bool on = there && first + i * lanes < a.n_vec;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s[i][e] = on ? xv[i].get(e) + (a.has_residual ? rv[i].get(e) : 0.f) : 0.f;
        sq += s[i][e] * s[i][e];
      }
    }
    const float mean = of_row(row_sum(sq, 0) / (float)a.channels + a.eps);
    float norm = of_row(rsqrtf(mean)), by = 1.f;   // y = s * by * norm * w
    const bool odd = !(mean >= kLeast && mean <= 3.402823466e38f);   // (a NaN too; the lanes of a row agree, rows that share a wavefront may not)
    const bool any_odd = WAVES > 1 ? odd : __any(odd);
    if (any_odd) {
      const float to = mean < kLeast ? kGrow : kShrink;
      float again = 0.f;
#pragma unroll
      for (int i = 0; i < VPL; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) again += (s[i][e] * to) * (s[i][e] * to);
      again = rsqrtf(row_sum(again, 2) / (float)a.channels + a.eps * to * to);
      if (odd) {
        by = to;
        norm = of_row(again);
      }
    }
    if (a.has_sum) {
      T* const o = (T*)tab.sum[tile] + row * a.s_stride;
#pragma unroll
      for (int i = 0; i < VPL; ++i)
        if (there && first + i * lanes < a.n_vec) store8(o + 8 * (first + i * lanes), s[i]);
    }
    if (any_odd) {
#pragma unroll
      for (int i = 0; i < VPL; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[i][e] *= by;
    }
#pragma unroll
    for (int i = 0; i < VPL; ++i)
      if (there && first + i * lanes < a.n_vec) {
#pragma unroll
        for (int e = 0; e < 8; ++e) s[i][e] = s[i][e] * norm * (a.weight ? w[i].get(e) : 1.f);
      }
    if constexpr (!E4M3) {
      T* const o = (T*)tab.out[tile] + row * a.o_stride;
#pragma unroll
      for (int i = 0; i < VPL; ++i)
        if (there && first + i * lanes < a.n_vec) store8(o + 8 * (first + i * lanes), s[i]);
    } else {
      uint8_t* const o = (uint8_t*)tab.out[tile] + row * a.o_stride;
      float* const scales = tab.scale[tile];
      float most[VPL];
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        most[i] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) most[i] = nan_max(most[i], fabsf(s[i][e]));
      }
      if (a.group_vecs == 0) {
        float m = most[0];
#pragma unroll
        for (int i = 1; i < VPL; ++i) m = nan_max(m, most[i]);
        m = row_max(m);
#pragma unroll
        for (int i = 0; i < VPL; ++i) most[i] = m;
        if (there && first == 0) scales[row] = m < kLeast ? 0.f : m / kE4m3Max;
      } else {   // 16 lanes side by side hold the 128 channels of a block
        const int groups = a.n_vec / a.group_vecs;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
#pragma unroll
          for (int d = 1; d < 16; d <<= 1) most[i] = nan_max(most[i], __shfl_xor(most[i], d, 64));
          const int v = first + i * lanes;
          if (there && v < a.n_vec && (v & 15) == 0) scales[row * groups + (v >> 4)] = most[i] < kLeast ? 0.f : most[i] / kE4m3Max;
        }
      }
#pragma unroll
      for (int i = 0; i < VPL; ++i) {
        const float inv = most[i] < kLeast ? 0.f : kE4m3Max / most[i];
        int lo = 0, hi = 0;   // rounded to the nearest 8-bit value; the largest product rounds to 448
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(s[i][0] * inv, s[i][1] * inv, lo, false);
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(s[i][2] * inv, s[i][3] * inv, lo, true);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(s[i][4] * inv, s[i][5] * inv, hi, false);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(s[i][6] * inv, s[i][7] * inv, hi, true);
        if (there && first + i * lanes < a.n_vec) __builtin_nontemporal_store(u32x2{(uint32_t)lo, (uint32_t)hi}, (u32x2*)(o + 8 * (first + i * lanes)));
      }
    }
    parity ^= 1;   // (of the rows that are worked on)
  }
}

template <typename T, bool E4M3>
int launch(const NormArgs& a, const NormTable& tab, int vpl, int waves, int64_t grid, hipStream_t s) {
  const dim3 g((unsigned)grid);
#define SG_NORM(V, W) residual_norm_kernel<T, E4M3, V, W><<<g, W == 16 ? 1024 : 256, 0, s>>>(a, tab)
#define SG_NORM_VPL(W)              \
  do {                              \
    if (vpl <= 1) SG_NORM(1, W);    \
    else if (vpl == 2) SG_NORM(2, W); \
    else if (vpl == 3) SG_NORM(3, W); \
    else SG_NORM(4, W);             \
  } while (0)
  if (waves == 1) SG_NORM_VPL(1);
  else if (waves == 4) SG_NORM_VPL(4);
  else SG_NORM_VPL(16);
#undef SG_NORM_VPL
#undef SG_NORM
  SG_HIP_TRY(hipGetLastError());
  return SG_OK;
}

}  // namespace

int launch_residual_norm(const sg_norm_problem& p, int n_tiles, const void* const* x, const void* const* residual, const void* weight,
                         const uint8_t* run, void* const* sum, void* const* out, float* const* scale, hipStream_t s) {
  NormArgs a = {};
  a.weight = weight;
  a.x_stride = p.x_stride; a.r_stride = p.residual_stride; a.s_stride = p.sum_stride; a.o_stride = p.out_stride;
  a.rows = p.rows; a.channels = p.channels; a.n_vec = p.channels / 8;
  a.group_vecs = p.scale_group / 8;
  a.has_residual = residual != nullptr; a.has_sum = sum != nullptr;
  a.eps = p.eps;
  const int waves = a.n_vec <= 64 * 4 ? 1 : a.n_vec <= 256 * 4 ? 4 : 16;
  a.lanes = 64 * waves;
  if (a.n_vec < 64) {
    a.lanes = 1;
    while (a.lanes < a.n_vec) a.lanes <<= 1;
  }
  const int vpl = (a.n_vec + a.lanes - 1) / a.lanes, rows_per_wg = waves == 1 ? 256 / a.lanes : 1;
  for (int t0 = 0; t0 < n_tiles; t0 += kNormTilesPerLaunch) {
    const int n = n_tiles - t0 < kNormTilesPerLaunch ? n_tiles - t0 : kNormTilesPerLaunch;
    NormTable tab = {};
    for (int i = 0; i < n; ++i) {
      tab.x[i] = x[t0 + i];
      tab.residual[i] = residual ? residual[t0 + i] : nullptr;
      tab.sum[i] = sum ? sum[t0 + i] : nullptr;
      tab.out[i] = out[t0 + i];
      tab.scale[i] = scale ? scale[t0 + i] : nullptr;
    }
    a.n_rows = (int64_t)n * p.rows;
    a.run = run ? run + t0 : nullptr;
    int64_t grid = (a.n_rows + rows_per_wg - 1) / rows_per_wg;
    // Workgroups that walk the rows load the weight once, new ones overlap their start with the others' end.  One per row of 4 wavefronts: 75,600 rows
    // of 5,120 454 us (2,048 that walk them: 536).  A wavefront per row: 8,192 workgroups, 768 channels 336 -> 297 us.  Shorter rows and
    // rows of 16 wavefronts fill the chip once and walk: 128 channels 136 us, with 8,192 workgroups 140 us; 30,720 303 us, with 2,048 319 us.
    const int64_t most = waves == 16 ? 512 : waves == 4 ? 1 << 22 : a.lanes == 64 ? 8192 : 2048;
    if (grid > most) grid = most;
    int st;
    if (p.dtype == SG_F32) st = p.out_dtype == SG_F8_E4M3 ? launch<float, true>(a, tab, vpl, waves, grid, s) : launch<float, false>(a, tab, vpl, waves, grid, s);
    else st = p.out_dtype == SG_F8_E4M3 ? launch<uint16_t, true>(a, tab, vpl, waves, grid, s) : launch<uint16_t, false>(a, tab, vpl, waves, grid, s);
    if (st != SG_OK) return st;
  }
  return SG_OK;
}

}  // namespace sg
