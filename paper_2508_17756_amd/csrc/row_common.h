// Shared by the kernels that work on rows of channels (gated norm, rotary positions): 8 channels of a stored type, reductions over the lanes of a row.
#pragma once
#include "attention_common.h"

namespace sg {

// 8 channels as they are stored.
template <typename T> struct Chan8;
template <> struct Chan8<uint16_t> {
  u32x4 w;
  __device__ __forceinline__ void clear() { w = u32x4{0, 0, 0, 0}; }
  __device__ __forceinline__ void load(const uint16_t* p) { w = *(const u32x4*)p; }
  __device__ __forceinline__ void stream(const uint16_t* p) { w = __builtin_nontemporal_load((const u32x4*)p); }   // rows that pass once
  __device__ __forceinline__ float get(int i) const { return i & 1 ? __uint_as_float(w[i >> 1] & 0xffff0000u) : __uint_as_float(w[i >> 1] << 16); }
};
template <> struct Chan8<float> {
  f32x4 a, b;
  __device__ __forceinline__ void clear() { a = b = f32x4{0.f, 0.f, 0.f, 0.f}; }
  __device__ __forceinline__ void load(const float* p) { a = *(const f32x4*)p; b = *(const f32x4*)(p + 4); }
  __device__ __forceinline__ void stream(const float* p) { load(p); }   // (the two halves of a lane's 32 bytes meet in the cache)
  __device__ __forceinline__ float get(int i) const { return i < 4 ? a[i] : b[i - 4]; }
};
__device__ __forceinline__ void stream8(uint16_t* p, const float (&v)[8]) {
  __builtin_nontemporal_store(u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])}, (u32x4*)p);
}
__device__ __forceinline__ void stream8(float* p, const float (&v)[8]) {
  *(f32x4*)p = f32x4{v[0], v[1], v[2], v[3]};
  *(f32x4*)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}

__device__ __forceinline__ void store8(uint16_t* p, const float (&v)[8]) {
  *(u32x4*)p = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) { stream8(p, v); }

// The larger of two numbers; NaN where one is.
__device__ __forceinline__ float larger_or_nan(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// op over the `lanes` lanes (a power of two, the same for all) that share a row; every lane gets the result.  Exchanges inside 16 lanes go with the
// operand of the instruction (swap in pairs, in fours, mirror 8 and 16), the others by the instructions that swap halves.
template <int CTRL> __device__ __forceinline__ float exchanged(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <typename Op> __device__ __forceinline__ float over_lanes(float v, int lanes, Op op) {
  if (lanes > 1) v = op(v, exchanged<0xb1>(v));
  if (lanes > 2) v = op(v, exchanged<0x4e>(v));
  if (lanes > 4) v = op(v, exchanged<0x141>(v));
  if (lanes > 8) v = op(v, exchanged<0x140>(v));
  if (lanes > 16) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  if (lanes > 32) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
  return v;
}
__device__ __forceinline__ float sum_over_lanes(float v, int lanes) { return over_lanes(v, lanes, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ float max_over_lanes(float v, int lanes) { return over_lanes(v, lanes, larger_or_nan); }

// Mean squares outside kLeastMean .. the largest fp32 number are taken again of the row scaled by a power of two, so that neither a square nor a sum leaves
// the range: |s| 2^-72 is below 2^56, 32,768 squares of it below 2^127; and with a mean below 2^-100 and up to 32,768 channels |s| 2^100 is below
// 2^58, the square of the smallest fp32 number 2^-98.  (From kLeastMean on what squares below 2^-149 lack is below 2^-49 of the mean.)
constexpr float kLeastMean = 7.888609052210118e-31f;   // 2^-100
constexpr float kMostFloat = 3.402823466e38f;
constexpr float kShrinkRow = 2.117582368135751e-22f, kGrowRow = 1.2676506002282294e30f;   // 2^-72, 2^100

}  // namespace sg
