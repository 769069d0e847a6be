// Linear layer of tiles in 8-bit integers (sg_tile_int8_linear):
//     out[r][o] = act(x_scale[r] * w_scale[o] * sum_c x[r][c] w[o][c] + bias[o])
// Rows of all tiles of a launch that run are numbered one behind the other; a workgroup computes BM of them times BN outputs.  Both operands have their
// channels side by side in memory, as the matrix instruction wants them (32x32x32: a lane gives 16 channels of one row), so 128 channels of the
// block's rows of x and w go straight into LDS, 16 bytes a lane, one stage ahead of the products.  The 16-byte pieces of a row
// are stored in the order piece ^ (row mod 8): 8 lanes that read the same piece of 8 rows then meet 8 different groups of banks.
// w is the instruction's first operand: a lane then holds 4 outputs side by side of one row, which it scales and stores together.
#include "block_api.h"
#include "row_common.h"

namespace sg {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

constexpr int kLinearTilesPerLaunch = 64;
struct LinearTable {
  const void* x[kLinearTilesPerLaunch];
  const float* x_scale[kLinearTilesPerLaunch];
  void* out[kLinearTilesPerLaunch];
};
struct LinearArgs {
  const char* w;
  const float* w_scale;
  const void* bias;
  const uint8_t* run;
  int64_t x_stride, w_stride, o_stride;
  int32_t n_tiles, rows, channels, outputs;
  uint32_t blocks_m, blocks_n;
  Divisor by_rows;
  bool gelu;
};

// What lanes read of places behind the channels' end.
__device__ const u32x4 kNoChannels = {0, 0, 0, 0};

constexpr int kStageBytes = 128;   // channels of a stage

__device__ __forceinline__ float gelu(float v) {   // v (1 + tanh(u)) / 2 = v / (1 + exp(-2 u)),  u = sqrt(2 / pi) (v + 0.044715 v^3)
  const float u = v * (-2.3022081983f - 0.1029432402f * v * v);   // -2 u log2(e)
  return v / (1.f + exp2f(u));
}

__device__ __forceinline__ void store4(uint16_t* p, const float (&v)[4]) { *(u32x2*)p = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])}; }
__device__ __forceinline__ void store4(float* p, const float (&v)[4]) { *(f32x4*)p = f32x4{v[0], v[1], v[2], v[3]}; }
__device__ __forceinline__ void load4(const uint16_t* p, float (&v)[4]) {
  const u32x2 w = *(const u32x2*)p;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = e & 1 ? __uint_as_float(w[e >> 1] & 0xffff0000u) : __uint_as_float(w[e >> 1] << 16);
}
__device__ __forceinline__ void load4(const float* p, float (&v)[4]) {
  const f32x4 w = *(const f32x4*)p;
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = w[e];
}

// The tiles of a launch that run, in their order; false if there are none.  list: LDS.  (All threads of the workgroup.)
__device__ __forceinline__ int running_tiles(const LinearArgs& a, int* list) {
  const int lane = threadIdx.x & 63;
  const bool runs = lane < a.n_tiles && (!a.run || a.run[lane] != 0);
  const uint64_t mask = __ballot(runs);
  if (threadIdx.x < 64 && runs) list[__popcll(mask & ((1ull << lane) - 1))] = lane;
  __syncthreads();
  return __popcll(mask);
}

// Workgroups go to the 8 XCDs in turn: each XCD takes a run of blocks, in columns of up to 8 blocks of rows, so that the 32 that run on it side by
// side share 8 parts of x and 4 of w in its L2.
__device__ __forceinline__ void block_of(uint32_t id, uint32_t gm, uint32_t gn, uint32_t& m, uint32_t& n) {
  const uint32_t all = gm * gn, xcd = id & 7, per = all >> 3, more = all & 7;
  const uint32_t at = xcd * per + (xcd < more ? xcd : more) + (id >> 3);
  const uint32_t group = at / (8 * gn), rest = at - group * 8 * gn, left = gm - group * 8, tall = left < 8 ? left : 8;
  n = rest / tall;
  m = group * 8 + rest - n * tall;
}

template <typename T, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void int8_linear_kernel(const LinearArgs a, const LinearTable tab) {
  constexpr int kWaves = WM * WN, kRows = BM + BN, kLoads = kRows / 8 / kWaves;
  constexpr int FM = BM / WM / 32, FN = BN / WN / 32;   // 32 x 32 results of a wavefront
  static_assert(kRows % (8 * kWaves) == 0 && FM * WM * 32 == BM && FN * WN * 32 == BN, "tiles");
  extern __shared__ __align__(1024) char lds[];   // [2 stages][BM rows of x, BN rows of w][128]
  __shared__ int list[kLinearTilesPerLaunch];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t total = (uint32_t)running_tiles(a, list) * (uint32_t)a.rows;
  uint32_t bm, bn;
  block_of(blockIdx.x, a.blocks_m, a.blocks_n, bm, bn);
  const uint32_t m0 = bm * BM;
  const int n0 = (int)bn * BN;
  if (m0 >= total) return;
  auto row_at = [&](uint32_t r, int& tile) {   // rows behind the last one: the last one
    r = r < total ? r : total - 1;
    const uint32_t i = divide(r, a.by_rows);
    tile = list[i];
    return (int64_t)(r - i * (uint32_t)a.rows);
  };

  // One 1 KiB piece of a stage, 8 rows, is a load of a wavefront: lane i fills place i mod 8 of row i / 8.
  const char* from[kLoads];
  const int channel = 16 * ((lane & 7) ^ (lane >> 3));
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    const int row = (wave + j * kWaves) * 8 + (lane >> 3);
    if (row < BM) {
      int tile;
      const int64_t at = row_at(m0 + row, tile);
      from[j] = (const char*)tab.x[tile] + at * a.x_stride + channel;
    } else {
      const int o = n0 + row - BM;
      from[j] = a.w + (int64_t)(o < a.outputs ? o : a.outputs - 1) * a.w_stride + channel;
    }
  }
  const uint32_t lds_at = (uint32_t)(uintptr_t)(SG_LDS char*)lds;
  auto load = [&](int stage, int buffer) {
    const bool there = stage * kStageBytes + channel < a.channels;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const char* const p = there ? from[j] + (int64_t)stage * kStageBytes : (const char*)&kNoChannels;
      dma16_addr(p, __builtin_amdgcn_readfirstlane(lds_at + buffer * (kRows * kStageBytes) + (wave + j * kWaves) * 1024));
    }
  };

  i32x16 acc[FN][FM] = {};
  const int wm = wave % WM, wn = wave / WM;
  const int r32 = lane & 31;
  const int stages = (a.channels + kStageBytes - 1) / kStageBytes;
  load(0, 0);
  for (int k = 0; k < stages; ++k) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (k + 1 < stages) load(k + 1, (k + 1) & 1);
    const char* const xs = lds + (k & 1) * (kRows * kStageBytes) + (wm * FM * 32 + r32) * kStageBytes;
    const char* const ws = lds + (k & 1) * (kRows * kStageBytes) + (BM + wn * FN * 32 + r32) * kStageBytes;
#pragma unroll
    for (int c = 0; c < kStageBytes / 32; ++c) {
      const int place = 16 * ((2 * c + (lane >> 5)) ^ (lane & 7));
      i32x4 xf[FM], wf[FN];
#pragma unroll
      for (int i = 0; i < FM; ++i) xf[i] = *(const i32x4*)(xs + i * 32 * kStageBytes + place);
#pragma unroll
      for (int i = 0; i < FN; ++i) wf[i] = *(const i32x4*)(ws + i * 32 * kStageBytes + place);
#pragma unroll
      for (int i = 0; i < FN; ++i)
#pragma unroll
        for (int j = 0; j < FM; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[i], xf[j], acc[i][j], 0, 0, 0);
    }
  }

  // Lane: row r32 of each 32 rows; outputs 8 g + 4 (lane / 32) + 0 .. 3 in registers 4 g + 0 .. 3.
#pragma unroll
  for (int j = 0; j < FM; ++j) {
    const uint32_t r = m0 + (wm * FM + j) * 32 + r32;
    if (r >= total) continue;
    int tile;
    const int64_t row = row_at(r, tile);
    const float xs = tab.x_scale[tile][row];
    T* const out = (T*)tab.out[tile] + row * a.o_stride;
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int o = n0 + (wn * FN + i) * 32 + 8 * g + 4 * (lane >> 5);
        if (o >= a.outputs) continue;
        const f32x4 ws = *(const f32x4*)(a.w_scale + o);
        float b[4] = {0.f, 0.f, 0.f, 0.f}, v[4];
        if (a.bias) load4((const T*)a.bias + o, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[e] = fmaf((float)acc[i][j][4 * g + e] * xs, ws[e], b[e]);
          if (a.gelu) v[e] = gelu(v[e]);
        }
        store4(out + o, v);
      }
  }
}

template <typename T, int BM, int BN, int WM, int WN>
int launch(LinearArgs& a, const LinearTable& tab, hipStream_t s) {
  const uint64_t rows = (uint64_t)a.n_tiles * (uint64_t)a.rows;
  a.blocks_m = (uint32_t)((rows + BM - 1) / BM);
  a.blocks_n = (uint32_t)((a.outputs + BN - 1) / BN);
  constexpr size_t kLds = 2 * (BM + BN) * kStageBytes;
  auto* const kernel = int8_linear_kernel<T, BM, BN, WM, WN>;
  if (kLds > 65536) SG_HIP_TRY(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)kLds));
  kernel<<<dim3(a.blocks_m * a.blocks_n), 64 * WM * WN, kLds, s>>>(a, tab);
  SG_HIP_TRY(hipGetLastError());
  return SG_OK;
}

}  // namespace

int launch_int8_linear(const sg_int8_linear_problem& p, int n_tiles, const void* const* x, const float* const* x_scale, const void* w,
                       const float* w_scale, const void* bias, const uint8_t* run, void* const* out, hipStream_t s) {
  LinearArgs a = {};
  a.w = (const char*)w; a.w_scale = w_scale; a.bias = bias;
  a.x_stride = p.x_stride; a.w_stride = p.w_stride; a.o_stride = p.out_stride;
  a.rows = p.rows; a.channels = p.channels; a.outputs = p.outputs;
  a.by_rows = make_divisor((uint32_t)p.rows);
  a.gelu = p.activation == SG_ACT_GELU;
  for (int t0 = 0; t0 < n_tiles; t0 += kLinearTilesPerLaunch) {
    const int n = n_tiles - t0 < kLinearTilesPerLaunch ? n_tiles - t0 : kLinearTilesPerLaunch;
    LinearTable tab = {};
    for (int i = 0; i < n; ++i) {
      tab.x[i] = x[t0 + i];
      tab.x_scale[i] = x_scale[t0 + i];
      tab.out[i] = out[t0 + i];
    }
    a.n_tiles = n;
    a.run = run ? run + t0 : nullptr;
    const int st = p.dtype == SG_F32 ? launch<float, 128, 128, 2, 2>(a, tab, s) : launch<uint16_t, 128, 128, 2, 2>(a, tab, s);
    if (st != SG_OK) return st;
  }
  return SG_OK;
}

}  // namespace sg
