// Context attention (sg_tile_cross_attention, sg_tile_prefix_attention) of many rows over few keys, bf16: all keys and values of a head stay in
// LDS (up to 128 KiB: 512 keys of head_dim 64, 256 of 128) while its rows pass by.
//
// A workgroup of 8 wavefronts, one per compute unit, takes a run of row blocks (32 rows each) from the list of all of them; where the run enters
// another tile or head of keys the keys are exchanged.  Between two exchanges the wavefronts go their own ways, a row block each, without
// barriers and without transfers: rows in, all keys, rows out; the next block's rows are requested before this one's keys are attended.  No unit is
// busy all the time (vector ALU 60 % of the cycles, exponentials first, matrix pipe 26 %, LDS 15 %): products and softmax of a row block follow one
// another, and the two wavefronts of a SIMD hide part of each other.  4 tiles of 17,550 rows, 48 heads x 64, 226 keys 0.35 - 0.38 ms from device to
// device (2.3 - 2.5 TB/s, 0.51 - 0.56 PFLOP/s; with shared stages 0.41 where this took 0.36), 4 x 9,000 rows, 24 heads x 128, 256 keys 0.16 ms
// (2.8 TB/s; 0.18).  12 wavefronts a compute unit gain nothing, 16 spill.
#include <atomic>
#include "context_bf16.h"

namespace sg {
namespace {

constexpr int kWaves = 8, kThreads = 64 * kWaves;
constexpr int kKeysLds = 128 * 1024;
template <int D>
constexpr int kUnit = 64 * D * 2;                    // keys (or values) of 64 tokens
static_assert(kKeysLds == kCtxResidentBytes, "");

template <int D>
__global__ __launch_bounds__(kThreads, 2) void context_bf16_resident_kernel(const CtxArgs a, const CtxTable tab) {
  constexpr int kNB = D == 128 ? 1 : 2, kPer = D == 128 ? 2 : 1;   // score blocks at a time, times per unit
  constexpr bool kAhead = D == 64;   // the next rows are requested before this block's keys (head_dim 128 has no registers left for them)
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(SG_LDS uint8_t*)smem;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int lq = lane & 31, half = lane >> 5;
  const CtxPart& p = a.part;
  uint64_t active = a.n_tiles >= 64 ? ~0ull : (1ull << a.n_tiles) - 1;
  if (a.run) active = __ballot(lane < a.n_tiles && a.run[lane < a.n_tiles ? lane : 0] != 0);
  const int total = __builtin_popcountll(active) * a.kv_heads * p.row_blocks;
  const int me = ((int)blockIdx.x & 7) * ((int)gridDim.x >> 3) + ((int)blockIdx.x >> 3);   // neighbours share an XCD's L2
  int pos = (int)((int64_t)total * me / gridDim.x);
  const int end = (int)((int64_t)total * (me + 1) / gridDim.x);
  const float c_log2 = a.scale * 1.4426950408889634f;
  const Frags f = make_frags();
  while (pos < end) {
    const int pair = pos / p.row_blocks, base = pair * p.row_blocks;
    const int stop = (end < base + p.row_blocks ? end : base + p.row_blocks) - base;   // behind the last row block of this tile and head
    const int nth = pair / a.kv_heads, kvh = __builtin_amdgcn_readfirstlane(pair - nth * a.kv_heads);
    const int tile = __builtin_amdgcn_readfirstlane(ctx_nth_tile(active, nth));
    const CtxSegment g0 = ctx_segment<2>(a, tab, 0, tile, kvh), g1 = ctx_segment<2>(a, tab, 1, tile, kvh);
    const int n0 = p.seg0 ? (g0.len + 63) / 64 : 0, n = n0 + (p.seg1 ? (g1.len + 63) / 64 : 0);
    // which keys of a unit count
    auto counting = [&](int u) SG_INLINE -> uint64_t {
      const CtxSegment& g = u >= n0 ? g1 : g0;
      const int key = (u >= n0 ? u - n0 : u) * 64 + lane;
      bool on = key < g.len;
      if (g.mask && on) on = g.mask[key] != 0;
      return __ballot(on);
    };
    int rb = pos - base + wave;
    bf16x8 qf[D / 16], next[D / 16];
    uint64_t to = 0, to_next = 0;   // where row lq goes
    auto rows = [&](int block, bf16x8 (&q)[D / 16]) SG_INLINE -> uint64_t {
      const CtxRow row = ctx_row(a, p, tile, kvh, block * 32 + lq);
      load_query<D>(a, tab, row, q);
      return ctx_row_end<uint16_t>(a, tab, row).out;
    };
    __syncthreads();   // the keys before these have been attended
    for (int i = wave; i < 2 * n; i += kWaves) {
      const int u = i >> 1;
      const CtxSegment& g = u >= n0 ? g1 : g0;
      move_half<D, D / 8>((i & 1) ? g.v : g.k, g.token, (u >= n0 ? u - n0 : u) * 64, 0, counting(u), (i & 1) != 0, lds0 + i * kUnit<D>);
    }
    if (rb < stop) to = rows(rb, qf);
    uint32_t partial = 0;   // units with keys that do not count
    for (int u = 0; u < n; ++u)
      if (counting(u) != ~0ull) partial |= 1u << u;
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();
    for (; rb < stop; rb += kWaves) {
      if (kAhead && rb + kWaves < stop) to_next = rows(rb + kWaves, next);
      RowState<D> st;
      clear(st);
      for (int u = 0; u < n; ++u) {
        const uint64_t valid = (partial >> u) & 1 ? counting(u) : ~0ull;
        const uint32_t k_at = lds0 + 2 * u * kUnit<D>, v_at = k_at + kUnit<D>;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const uint64_t v = kPer == 1 ? valid : (valid >> (32 * i)) & 0xffffffffull;
          if (v != 0) attend_keys<D, kNB>(f, k_at + i * 32 * kSlot, v_at + i * 32 * kSlot, qf, c_log2, v, st);
        }
      }
      const uint32_t lu = __float_as_uint(st.l);
      const auto sw = __builtin_amdgcn_permlane32_swap(lu, lu, false, false);
      const float l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
      write_row<D>(st.o, l == 0.f ? 0.f : 1.f / l, to);
      if constexpr (kAhead) {
        to = to_next;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk) qf[kk] = next[kk];
      } else if (rb + kWaves < stop) {
        to = rows(rb + kWaves, qf);
      }
    }
    pos = base + stop;
  }
}

}  // namespace

int launch_context_bf16_resident(const CtxArgs& a, const CtxTable& tab, int head_dim, hipStream_t s) {
  int dev = 0, n_cu = 0;
  SG_HIP_TRY(hipGetDevice(&dev));
  SG_HIP_TRY(hipDeviceGetAttribute(&n_cu, hipDeviceAttributeMultiprocessorCount, dev));
  constexpr int kMaxDevices = 64;
  static std::atomic<bool> attr_set[kMaxDevices][2];   // the kernels' dynamic-LDS limit has been raised
  auto launch = [&](auto kern, int slot) -> int {
    if (dev < 0 || dev >= kMaxDevices || !attr_set[dev][slot].load(std::memory_order_acquire)) {
      SG_HIP_TRY(hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, kKeysLds));
      if (dev >= 0 && dev < kMaxDevices) attr_set[dev][slot].store(true, std::memory_order_release);
    }
    const int grid = n_cu / 8 > 0 ? n_cu / 8 * 8 : 8;
    kern<<<dim3((unsigned)grid), kThreads, kKeysLds, s>>>(a, tab);
    SG_HIP_TRY(hipGetLastError());
    return SG_OK;
  };
  return head_dim == 128 ? launch(context_bf16_resident_kernel<128>, 0) : launch(context_bf16_resident_kernel<64>, 1);
}

}  // namespace sg
