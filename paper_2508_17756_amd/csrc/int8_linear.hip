// Linear layer of tiles in 8-bit integers (sg_tile_int8_linear):
//     out[r][o] = act(x_scale[r] * w_scale[o] * sum_c x[r][c] w[o][c] + bias[o])
// Rows of all tiles of a launch that run are numbered one behind the other; a workgroup computes BM of them times BN outputs.  Both operands have their
// channels side by side in memory, as the matrix instruction wants them (16x16x64: a lane gives 16 channels of one row), so 128 channels of the
// block's rows of x and w go straight into LDS, 16 bytes a lane, a stage or more ahead of the products.  The 16-byte pieces of a row
// are stored in the order piece ^ (row / 2 mod 8): 16 lanes that read the same piece of 16 rows then meet 16 different groups of the 64 banks.
// w is the instruction's first operand, its rows in an order that leaves a lane with outputs side by side of one row, which it scales and stores together.
//
// Large calls: held in registers, N(0, 32)-distributed integers pass the instruction at 3.9 POP/s, bound by power (zeros: 4.9; the form 32x32x32, which touches each
// sum twice as often, at 3.3).  Blocks of 256 x 256: 34,560 x 5,120 x 15,360 2.13 - 2.19 ms = 2.48 - 2.55 POP/s (all zeros: 1.74 ms), 75,600 x 5,120 x 20,480 with GELU
// 6.6 - 6.9 ms.  A block's 40 stages take seven eighths of its time, its start and its stores the last.  What the stages lose, timed with parts left out, are
// the loads from the L2 into LDS (64 KiB a stage; without them 1.76 ms, zeros 1.43), hardly the barriers (a further 0.02) and not the reads of LDS.
// 32x32x32 instead: 2.58 ms at the first size; all of a stage's loads behind its barrier: 2.23; factors and places of the rows looked up at the end: 2.35.
#include <atomic>
#include "block_api.h"
#include "row_common.h"

namespace sg {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr int kLinearTilesPerLaunch = 64, kMaxDevices = 64;
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

// What lanes read of places behind the channels' end: 16 bytes at a time, up to STAGES + 1 stages behind one another.
__device__ __align__(16) const char kNoChannels[2048] = {};

__device__ __forceinline__ float gelu(float v) {   // v (1 + tanh(u)) / 2 = v / (1 + exp(-2 u)),  u = sqrt(2 / pi) (v + 0.044715 v^3)
  const float u = v * (-2.3022081983f - 0.1029432402f * v * v);   // -2 u log2(e)
  return v * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(u));
}

__device__ __forceinline__ float to_float(uint16_t v) { return bf16_bits_to_f32(v); }
__device__ __forceinline__ float to_float(float v) { return v; }

// 8 outputs side by side of a row, from output o on.
template <typename T> __device__ __forceinline__ void finish8(const LinearArgs& a, const int (&sum)[8], float x_scale, int o, T* out) {
  Chan8<float> ws;
  ws.load(a.w_scale + o);
  Chan8<T> b;
  if (a.bias) b.load((const T*)a.bias + o);
  float v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    v[e] = (float)sum[e] * x_scale;
    v[e] = a.bias ? fmaf(v[e], ws.get(e), b.get(e)) : v[e] * ws.get(e);
    if (a.gelu) v[e] = gelu(v[e]);
  }
  store8(out, v);
}

// The tiles of a launch that run, in their order, into list (LDS); how many.  (All threads of the workgroup.)
__device__ __forceinline__ int running_tiles(const LinearArgs& a, int* list) {
  const int lane = threadIdx.x & 63;
  const bool runs = lane < a.n_tiles && (!a.run || a.run[lane] != 0);
  const uint64_t mask = __ballot(runs);
  if (threadIdx.x < 64 && runs) list[__popcll(mask & ((1ull << lane) - 1))] = lane;
  __syncthreads();
  return __popcll(mask);
}

// Workgroups go to the 8 XCDs in turn: each XCD takes a run of blocks, in columns of up to 4 blocks of rows, so that the 32 that run on it side by
// side share 4 parts of x and 8 of w in its L2 (75,600 x 5,120 x 20,480: 6.77 ms; columns of 8 6.95, of 16 7.10).  The runs are of all rows of the call: where tiles do not run, the blocks that are left meet
// on the first XCDs (9 tiles of 3,840 x 5,120 x 15,360 2.13 ms, 4 of them 1.96, one 1.64).
__device__ __forceinline__ void block_of(uint32_t id, uint32_t gm, uint32_t gn, uint32_t& m, uint32_t& n) {
  const uint32_t all = gm * gn, xcd = id & 7, per = all >> 3, more = all & 7;
  const uint32_t at = xcd * per + (xcd < more ? xcd : more) + (id >> 3);
  const uint32_t group = at / (4 * gn), rest = at - group * 4 * gn, left = gm - group * 4, tall = left < 4 ? left : 4;
  n = rest / tall;
  m = group * 4 + rest - n * tall;
}

template <typename T, int BM, int BN, int WM, int WN, int STAGES>
__global__ __launch_bounds__(64 * WM * WN) void int8_linear_kernel(const LinearArgs a, const LinearTable tab) {
  constexpr int BK = 128;   // channels of a stage
  constexpr int kWaves = WM * WN, kRows = BM + BN, kLoads = kRows / 8 / kWaves, kStageBytes = kRows * BK, kAhead = (STAGES - 2) * kLoads;
  constexpr int FM = BM / WM / 16, FN = BN / WN / 16;   // 16 x 16 results of a wavefront
  static_assert(kRows % (8 * kWaves) == 0 && kWaves % 2 == 0 && FM * WM * 16 == BM && FN * WN * 16 == BN && FM % 2 == 0 && FN % 2 == 0, "tiles");
  static_assert((STAGES + 1) * BK + 16 <= (int)sizeof(kNoChannels) && kAhead + kLoads < 64, "loads behind the end, loads in flight");
  extern __shared__ __align__(1024) char lds[];   // [STAGES][BM rows of x, BN rows of w][BK]
  struct Row { const char* x; T* out; };
  __shared__ Row rows[BM];
  __shared__ float x_scales[BM];
  __shared__ __align__(16) float w_scales[BN], biases[BN];
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

  // A thread finds the place of one row, for all that load or store it, and brings a row's and an output's factors for the end.
  static_assert(64 * kWaves >= BM && 64 * kWaves >= BN, "a row and an output a thread");
  float row_scale = 0.f, out_scale = 0.f, out_bias = 0.f;
  if (threadIdx.x < BM) {
    int tile;
    const int64_t at = row_at(m0 + threadIdx.x, tile);
    rows[threadIdx.x] = {(const char*)tab.x[tile] + at * a.x_stride, (T*)tab.out[tile] + at * a.o_stride};
    row_scale = tab.x_scale[tile][at];
  }
  if (threadIdx.x < BN) {
    const int o = n0 + (int)threadIdx.x < a.outputs ? n0 + (int)threadIdx.x : a.outputs - 1;
    out_scale = a.w_scale[o];
    if (a.bias) out_bias = to_float(((const T*)a.bias)[o]);
  }
  __syncthreads();

  // One 1 KiB piece of a stage, 8 rows, is a load of a wavefront: lane i fills the i-th 16 bytes.
  const char* from[kLoads];
  const int channel = 16 * ((lane & 7) ^ ((wave & 1) << 2 | lane >> 4));
  constexpr int kXLoads = BM / (8 * kWaves);
  static_assert(BM % (8 * kWaves) == 0, "a piece has rows of x or of w");
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    const int row = (wave + j * kWaves) * 8 + (lane >> 3);
    if (j < kXLoads) {
      from[j] = rows[row].x + channel;
    } else {
      // Row 16 i + r of a wavefront's outputs is output 4 FN (r / 4) + 4 i + r mod 4 of them: what a lane gets is then side by side.
      const int w = (row - BM) % (16 * FN), r = w & 15;
      const int o = n0 + row - BM - w + 4 * FN * (r >> 2) + 4 * (w >> 4) + (r & 3);
      from[j] = a.w + (int64_t)(o < a.outputs ? o : a.outputs - 1) * a.w_stride + channel;
    }
  }
  const int stages = (a.channels + BK - 1) / BK;
  const uint32_t lds_at = (uint32_t)(uintptr_t)(SG_LDS char*)lds + wave * 1024;
  auto load = [&](int j, int buffer) {
    dma16_addr(from[j], __builtin_amdgcn_readfirstlane(lds_at + buffer * kStageBytes + j * kWaves * 1024));
    from[j] += BK;
  };
  // The last stage may have fewer channels, and as many loads follow it as are in flight: zeros.
  auto check_end = [&](int stage) {
    if (stage == stages - 1 ? stage * BK + channel >= a.channels : stage == stages) {
#pragma unroll
      for (int j = 0; j < kLoads; ++j) from[j] = kNoChannels;
    }
  };

  // A stage is two steps of 64 channels, a step FM groups of products with 16 rows each.  xf: the rows, read for the next step as soon as their
  // group is out; wf: the outputs, of this step and the next.
  i32x4 acc[FN][FM] = {}, xf[FM], wf[2][FN];
  const int wm = wave % WM, wn = wave / WM;
  const int r16 = lane & 15, quarter = lane >> 4;
  // What the lane gives of 16 rows at steps 0 and 1.
  const char* const at[2] = {lds + r16 * BK + 16 * (quarter ^ (r16 >> 1)), lds + r16 * BK + 16 * ((4 + quarter) ^ (r16 >> 1))};
  const char* const x_at[2] = {at[0] + wm * FM * 16 * BK, at[1] + wm * FM * 16 * BK};
  const char* const w_at[2] = {at[0] + (BM + wn * FN * 16) * BK, at[1] + (BM + wn * FN * 16) * BK};
  auto read_x = [&](int buffer, int c, int j) { xf[j] = *(const i32x4*)(x_at[c] + buffer * kStageBytes + j * 16 * BK); };
  auto read_w = [&](int buffer, int c, int i) { wf[c][i] = *(const i32x4*)(w_at[c] + buffer * kStageBytes + i * 16 * BK); };
  // Group j of step c; what `between` reads or loads goes out in the shadow of its products.
  auto group = [&](int c, int j, auto between) {
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < FN; ++i) {
      acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[c][i], xf[j], acc[i][j], 0, 0, 0);
      if (i == FN / 2 - 1) {
        __builtin_amdgcn_sched_barrier(0);
        between();
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // The loads of a stage go out beside the second half of one step's groups and all of the next one's.
  constexpr int kHalf = FM / 2, kReads = (FN + FM - 1) / FM, kLoadsPer = (kLoads + kHalf + FM - 1) / (kHalf + FM);
  auto load_some = [&](int group, int buffer) {
#pragma unroll
    for (int l = group * kLoadsPer; l < (group + 1) * kLoadsPer; ++l)
      if (l < kLoads) load(l, buffer);
  };
  auto first_step = [&](int buffer, int read_out) {   // read_out: a buffer that is to be filled, or -1
#pragma unroll
    for (int j = 0; j < FM; ++j) {
      group(0, j, [&] {
#pragma unroll
        for (int i = j * kReads; i < (j + 1) * kReads; ++i)
          if (i < FN) read_w(buffer, 1, i);
        if (read_out >= 0) load_some(kHalf + j, read_out);
      });
      read_x(buffer, 1, j);
    }
  };
#pragma unroll
  for (int k = 0; k < STAGES; ++k) {
    check_end(k);
#pragma unroll
    for (int j = 0; j < kLoads; ++j) load(j, k);
  }
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"(kAhead + kLoads) : "memory");
#pragma unroll
  for (int i = 0; i < FN; ++i) read_w(0, 0, i);
#pragma unroll
  for (int j = 0; j < FM; ++j) read_x(0, 0, j);
  first_step(0, -1);
#pragma unroll
  for (int j = 0; j < kHalf; ++j) group(1, j, [] {});
  // The barrier stands in the middle of the second step: by then every read of the stage has long been issued, and the other half of the products covers
  // the first reads of the next stage.
  int buffer = 0;
  for (int k = 0; k + 1 < stages; ++k) {
    const int next = buffer + 1 == STAGES ? 0 : buffer + 1;
    check_end(k + STAGES);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(kAhead) : "memory");
    constexpr int kWPer = (FN + kHalf - 1) / kHalf;
#pragma unroll
    for (int j = 0; j < kHalf; ++j) {
      group(1, kHalf + j, [&] {
#pragma unroll
        for (int i = j * kWPer; i < (j + 1) * kWPer; ++i)
          if (i < FN) read_w(next, 0, i);
        read_x(next, 0, j);
        load_some(j, buffer);
      });
      read_x(next, 0, kHalf + j);
    }
    const int read_out = buffer;
    buffer = next;
    first_step(buffer, read_out);
#pragma unroll
    for (int j = 0; j < kHalf; ++j) group(1, j, [] {});
  }
#pragma unroll
  for (int j = kHalf; j < FM; ++j) group(1, j, [] {});
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // nothing arrives in LDS that is another workgroup's by then

  if (threadIdx.x < BM) x_scales[threadIdx.x] = row_scale;
  if (threadIdx.x < BN) { w_scales[threadIdx.x] = out_scale; biases[threadIdx.x] = out_bias; }
  __syncthreads();

  // Lane: row r16 of each 16 rows; 4 FN outputs side by side.
  const int o_in = (wn * 4 + quarter) * 4 * FN;
  Chan8<float> ws[FN / 2], bs[FN / 2];
#pragma unroll
  for (int i = 0; i < FN / 2; ++i) {
    ws[i].load(w_scales + o_in + 8 * i);
    bs[i].load(biases + o_in + 8 * i);
  }
#pragma unroll
  for (int j = 0; j < FM; ++j) {
    const int row = (wm * FM + j) * 16 + r16;
    const float xs = x_scales[row];
    T* const out = rows[row].out + n0 + o_in;
#pragma unroll
    for (int i = 0; i < FN; i += 2) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] = (float)acc[i + e / 4][j][e % 4] * xs;
        v[e] = a.bias ? fmaf(v[e], ws[i / 2].get(e), bs[i / 2].get(e)) : v[e] * ws[i / 2].get(e);
        if (a.gelu) v[e] = gelu(v[e]);
      }
      if (m0 + row < total && n0 + o_in + 4 * i < a.outputs) store8(out + 4 * i, v);
    }
  }
}

// Few rows: the weights' bytes are what counts.  A workgroup takes 16 MT rows and 16 NT outputs; its wavefronts take the channels in turn, 128 at a time, each
// through a ring of DEPTH stages in LDS that is its own, so that no wavefront waits for another before the end.  Their sums meet in LDS: integers, so the
// order does not matter.
template <typename T, int MT, int NT, int DEPTH, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void int8_linear_rows_kernel(const LinearArgs a, const LinearTable tab) {
  constexpr int BK = 128, kRows = 16 * (MT + NT), kLoads = kRows / 8, kStageBytes = kRows * BK, kPitch = 16 * NT + 4, kThreads = 64 * WAVES;
  static_assert((DEPTH - 1) * kLoads < 64, "loads in flight");
  extern __shared__ __align__(1024) char lds[];   // [WAVES][DEPTH][rows of x, rows of w][128]
  __shared__ int list[kLinearTilesPerLaunch];
  __shared__ int sums[16 * MT * kPitch];          // [row][output]
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t total = (uint32_t)running_tiles(a, list) * (uint32_t)a.rows;
  const uint32_t blocks_n = (uint32_t)(a.outputs + 16 * NT - 1) / (16 * NT), m = blockIdx.x / blocks_n;
  const uint32_t m0 = m * 16 * MT;
  const int n0 = (int)(blockIdx.x - m * blocks_n) * 16 * NT;
  if (m0 >= total) return;
  const int stages = (a.channels + BK - 1) / BK, n = (stages - wave + WAVES - 1) / WAVES;   // of the wavefront: stage k WAVES + wave
  const char* from[kLoads];
  int channel[2];   // of the pieces with even and odd numbers
#pragma unroll
  for (int j = 0; j < 2; ++j) channel[j] = 16 * ((lane & 7) ^ (j << 2 | lane >> 4));
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    const int row = 8 * j + (lane >> 3);
    if (row < 16 * MT) {
      uint32_t r = m0 + row;
      r = r < total ? r : total - 1;
      const uint32_t i = divide(r, a.by_rows);
      from[j] = (const char*)tab.x[list[i]] + (int64_t)(r - i * (uint32_t)a.rows) * a.x_stride;
    } else {
      const int o = n0 + row - 16 * MT;
      from[j] = a.w + (int64_t)(o < a.outputs ? o : a.outputs - 1) * a.w_stride;
    }
    from[j] += wave * BK + channel[j & 1];
  }
  const uint32_t lds_at = (uint32_t)(uintptr_t)(SG_LDS char*)lds + wave * (DEPTH * kStageBytes);
  auto load = [&](int k, int slot) {
    const bool last = k * WAVES + wave == stages - 1;   // zeros behind the channels' end
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      const char* const p = last && (stages - 1) * BK + channel[j & 1] >= a.channels ? kNoChannels : from[j];
      dma16_addr(p, __builtin_amdgcn_readfirstlane(lds_at + slot * kStageBytes + j * 1024));
      from[j] += WAVES * BK;
    }
  };
#pragma unroll
  for (int k = 0; k < DEPTH; ++k)
    if (k < n) load(k, k);
  for (int i = threadIdx.x; i < 16 * MT * kPitch; i += kThreads) sums[i] = 0;
  const int r16 = lane & 15, quarter = lane >> 4;
  i32x4 acc[NT][MT] = {};
  const char* const mine = lds + wave * (DEPTH * kStageBytes) + r16 * BK;
  int slot = 0;
  for (int k = 0; k < n; ++k) {
    if (k + DEPTH <= n) asm volatile("s_waitcnt vmcnt(%0)" : : "n"((DEPTH - 1) * kLoads) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    i32x4 xf[2][MT], wf[2][NT];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const char* const at = mine + slot * kStageBytes + 16 * ((4 * c + quarter) ^ (r16 >> 1));
#pragma unroll
      for (int i = 0; i < NT; ++i) wf[c][i] = *(const i32x4*)(at + (MT + i) * 16 * BK);
#pragma unroll
      for (int j = 0; j < MT; ++j) xf[c][j] = *(const i32x4*)(at + j * 16 * BK);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (k + DEPTH < n) load(k + DEPTH, slot);
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[c][i], xf[c][j], acc[i][j], 0, 0, 0);
    slot = slot + 1 == DEPTH ? 0 : slot + 1;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) atomicAdd(&sums[(16 * j + r16) * kPitch + 16 * i + 4 * quarter + e], acc[i][j][e]);
  __syncthreads();
  for (int t = threadIdx.x; t < 16 * MT * 2 * NT; t += kThreads) {
    const int row_in = t / (2 * NT), o = n0 + 8 * (t - row_in * 2 * NT);
    const uint32_t r = m0 + row_in;
    if (r >= total || o >= a.outputs) continue;
    const uint32_t i = divide(r, a.by_rows);
    const int tile = list[i];
    const int64_t row = r - i * (uint32_t)a.rows;
    const int* const sum = sums + row_in * kPitch + (o - n0);
    int v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = sum[e];
    finish8<T>(a, v, tab.x_scale[tile][row], o, (T*)tab.out[tile] + row * a.o_stride + o);
  }
}

// The kernel's dynamic-LDS limit, raised once on each device.
inline int raise_lds(const void* kernel, size_t bytes, std::atomic<bool>* raised) {
  int dev = -1;
  if (bytes <= 49152) return SG_OK;
  SG_HIP_TRY(hipGetDevice(&dev));
  if (dev < 0 || dev >= kMaxDevices || !raised[dev].load(std::memory_order_acquire)) {
    SG_HIP_TRY(hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    if (dev >= 0 && dev < kMaxDevices) raised[dev].store(true, std::memory_order_release);
  }
  return SG_OK;
}

template <typename T, int BM, int BN, int WM, int WN, int STAGES>
int launch(LinearArgs& a, const LinearTable& tab, hipStream_t s) {
  const uint64_t rows = (uint64_t)a.n_tiles * (uint64_t)a.rows;
  a.blocks_m = (uint32_t)((rows + BM - 1) / BM);
  a.blocks_n = (uint32_t)((a.outputs + BN - 1) / BN);
  constexpr size_t kLds = STAGES * (BM + BN) * 128;
  static std::atomic<bool> raised[kMaxDevices];
  auto* const kernel = int8_linear_kernel<T, BM, BN, WM, WN, STAGES>;
  const int st = raise_lds((const void*)kernel, kLds, raised);
  if (st != SG_OK) return st;
  kernel<<<dim3(a.blocks_m * a.blocks_n), 64 * WM * WN, kLds, s>>>(a, tab);
  SG_HIP_TRY(hipGetLastError());
  return SG_OK;
}

template <typename T, int MT, int NT, int DEPTH, int WAVES> int launch_rows(const LinearArgs& a, const LinearTable& tab, hipStream_t s) {
  const int64_t rows = (int64_t)a.n_tiles * a.rows;
  const dim3 grid((unsigned)(((a.outputs + 16 * NT - 1) / (16 * NT)) * ((rows + 16 * MT - 1) / (16 * MT))));
  constexpr size_t kLds = WAVES * DEPTH * 16 * (MT + NT) * 128;
  static std::atomic<bool> raised[kMaxDevices];
  auto* const kernel = int8_linear_rows_kernel<T, MT, NT, DEPTH, WAVES>;
  const int st = raise_lds((const void*)kernel, kLds, raised);
  if (st != SG_OK) return st;
  kernel<<<grid, 64 * WAVES, kLds, s>>>(a, tab);
  SG_HIP_TRY(hipGetLastError());
  return SG_OK;
}

// Which blocks: those whose rounds over the compute units take least.  us for 40 stages of 128 channels and so many blocks, on 256 compute units:
//   256 x 256   65 for each round of 256                                      (256 blocks 65, 480 142)
//   128 x 128   40 for up to 256, then 46 for each round of 512               (240: 39, 480: 47, 960: 88, 1,920: 167)
//    64 x 64    19 for up to 256, then 10 and 0.036 a block                   (320: 28, 960: 47, 2,560: 104)
//    32 x 32, wavefronts apart   8 and 0.015 a block                          (160: 10.7, 640: 18, 1,280: 27, 2,560: 45)
// and up to 16 rows: 16 x 32 with 8 wavefronts (5,120 channels and outputs, weights from memory: 8.2 - 9.4; 16 x 16 with 4 8.8 - 10.4, 32 x 32 8.7 - 9.6), or
// 16 x 16 where that leaves most compute units without work (20,480 channels, 512 outputs: 15.4 instead of 22).
template <typename T> int launch_best(LinearArgs& a, const LinearTable& tab, hipStream_t s) {
  const int64_t rows = (int64_t)a.n_tiles * a.rows, outputs = a.outputs;
  auto blocks = [&](int64_t bm, int64_t bn) { return ((rows + bm - 1) / bm) * ((outputs + bn - 1) / bn); };
  if (rows <= 16) return blocks(16, 32) >= 64 ? launch_rows<T, 1, 2, 3, 8>(a, tab, s) : launch_rows<T, 1, 1, 4, 4>(a, tab, s);
  const int64_t b256 = blocks(256, 256), b128 = blocks(128, 128), b64 = blocks(64, 64), b32 = blocks(32, 32);
  const int64_t t256 = (b256 + 255) / 256 * 65000, t128 = b128 <= 256 ? 40000 : (b128 + 511) / 512 * 46000, t64 = b64 <= 256 ? 19000 : 10000 + 36 * b64,
                t32 = 8000 + 15 * b32;
  // (a grid has less than 2^32 threads: 256 of a workgroup, 512 of the largest blocks, whose number the call's checks bound)
  constexpr int64_t kMost = (1ll << 24) - 1;
  if (b32 <= kMost && t32 <= t64 && t32 <= t128 && t32 <= t256) return launch_rows<T, 2, 2, 2, 4>(a, tab, s);
  if (b64 <= kMost && t64 <= t128 && t64 <= t256) return launch<T, 64, 64, 2, 2, 3>(a, tab, s);
  if (b128 <= kMost && t128 <= t256) return launch<T, 128, 128, 2, 2, 2>(a, tab, s);
  return launch<T, 256, 256, 2, 4, 2>(a, tab, s);
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
    const int st = p.dtype == SG_F32 ? launch_best<float>(a, tab, s) : launch_best<uint16_t>(a, tab, s);
    if (st != SG_OK) return st;
  }
  return SG_OK;
}

}  // namespace sg
