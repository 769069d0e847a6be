// Context attention (sg_tile_cross_attention, sg_tile_prefix_attention) of calls with few rows, bf16: every wavefront streams keys of its own
// through LDS of its own, 32 rows at a time, and the shares of a row are joined in LDS and, over workgroups, by the join kernel.
//
// Bound by latency: a wavefront waits for nobody but its own transfers.  One token of 8 heads x 64 over 77 keys 6.7 - 7.2 us, of one
// head over one key 7.0 (6.1 between the kernel's begin and end); 20 single tokens' own keys (up to 460, 8 heads of keys x 128) and the join of 32 shares of a prefix 14 us.
#include <atomic>
#include "context_bf16.h"

namespace sg {
namespace {

// A wavefront's LDS: two stages of 32 slots of K and V.  After the keys it holds the wavefront's sums: 32 rows x D floats (16-byte chunk c of
// row r at chunk c ^ (r & 15)), then (reference, sum) of the rows and where they go.
constexpr int kSplitStage = 2 * 32 * kSlot;              // 16 KiB
constexpr int kSplitWave = 2 * kSplitStage;
constexpr int kSplitLds = 4 * kSplitWave;
constexpr int kSumsAt = kSplitStage, kRowsAt = kSumsAt + 512;

template <int D>
__global__ __launch_bounds__(256, 1) void context_bf16_split_kernel(const CtxArgs a, const CtxTable tab) {
  constexpr int kKeys = D == 128 ? 32 : 64, kBlocks = D == 128 ? 1 : 2;
  constexpr uint64_t kFull = kKeys == 32 ? 0xffffffffull : ~0ull;
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(SG_LDS uint8_t*)smem;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int lq = lane & 31, half = lane >> 5;

  const CtxPart& p = a.part;
  // The grid names tile and head of keys, so that the table of tiles can be read without waiting for anything else.
  const int split = (int)blockIdx.x / p.row_blocks, row_block = (int)blockIdx.x - split * p.row_blocks, kvh = (int)blockIdx.y, batch = (int)blockIdx.z;
  if (!p.stacked && a.run && a.run[batch] == 0) return;
  const int way = wave & (p.ways - 1);
  const int row0 = (row_block * (4 / p.ways) + wave / p.ways) * 32;

  RowState<D> st;
  clear(st);
  CtxRowEnd end = {0, 0};   // of row lq
  if (row0 < p.rows) {
    const CtxSegment g0 = ctx_segment<2>(a, tab, 0, batch, kvh), g1 = ctx_segment<2>(a, tab, 1, batch, kvh);
    const int n0 = p.seg0 ? (g0.len + kKeys - 1) / kKeys : 0, n1 = p.seg1 ? (g1.len + kKeys - 1) / kKeys : 0;
    const int n = n0 + n1;
    const int from = (int)((int64_t)n * split / p.splits), to = (int)((int64_t)n * (split + 1) / p.splits);
    const uint32_t ring = lds0 + wave * kSplitWave;
    uint64_t valid_next = 0;
    auto issue = [&](int j, int at) SG_INLINE {
      const bool second = j >= n0;
      const CtxSegment& g = second ? g1 : g0;
      const int key0 = (second ? j - n0 : j) * kKeys;
      bool counts = lane < kKeys && key0 + lane < g.len;
      if (g.mask && counts) counts = g.mask[key0 + lane] != 0;
      const uint64_t v = __ballot(counts);
      valid_next = v;
      const uint32_t dst = ring + at * kSplitStage;
      move_half<D, 8>(g.k, g.token, key0, 0, v, false, dst, kFull);
      move_half<D, 8>(g.v, g.token, key0, 0, v, true, dst + 32 * kSlot, kFull);
    };
    int j = from + way;
    if (j < to) issue(j, 0);
    bf16x8 qf[D / 16];
    const CtxRow row = ctx_row(a, p, batch, kvh, row0 + lq);
    load_query<D>(a, tab, row, qf);
    end = ctx_row_end<uint16_t>(a, tab, row);
    const Frags f = make_frags();
    const float c_log2 = a.scale * 1.4426950408889634f;
    for (int at = 0; j < to; j += p.ways, at ^= 1) {
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");   // this stage is there, the other one has been read
      __builtin_amdgcn_sched_barrier(0);
      const uint64_t v = valid_next;
      if (j + p.ways < to) issue(j + p.ways, at ^ 1);
      const uint32_t base = ring + at * kSplitStage;
      if (v != 0) attend_keys<D, kBlocks>(f, base, base + 32 * kSlot, qf, c_log2, v, st);
    }
  }
  const uint32_t lu = __float_as_uint(st.l);
  const auto sw = __builtin_amdgcn_permlane32_swap(lu, lu, false, false);
  const float l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);

  // ---- join of the shares in this workgroup
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  const uint32_t mine = lds0 + wave * kSplitWave;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 x = {st.o[db][4 * g], st.o[db][4 * g + 1], st.o[db][4 * g + 2], st.o[db][4 * g + 3]};
      *(SG_LDS f32x4*)(uintptr_t)(mine + lq * (D * 4) + (((8 * db + 2 * g + half) ^ (lq & 15)) << 4)) = x;
    }
  if (half == 0) {
    *(SG_LDS f32x2*)(uintptr_t)(mine + kSumsAt + lq * 8) = f32x2{st.m, l};
    *(SG_LDS u32x4*)(uintptr_t)(mine + kRowsAt + lq * 16) = u32x4{(uint32_t)end.out, (uint32_t)(end.out >> 32), (uint32_t)end.rid, 0u};
  }
  __syncthreads();
  const uint32_t group = lds0 + (wave & ~(p.ways - 1)) * kSplitWave;
  if (p.ways == 4) ctx_finish<uint16_t, D, 32, 4>(a, p, group, kSplitWave, kSumsAt, kRowsAt, way, split, row0);
  else if (p.ways == 2) ctx_finish<uint16_t, D, 32, 2>(a, p, group, kSplitWave, kSumsAt, kRowsAt, way, split, row0);
  else ctx_finish<uint16_t, D, 32, 1>(a, p, group, kSplitWave, kSumsAt, kRowsAt, way, split, row0);
}

}  // namespace

int launch_context_bf16_split(const CtxArgs& a, const CtxTable& tab, int head_dim, hipStream_t s) {
  int dev = 0;
  SG_HIP_TRY(hipGetDevice(&dev));
  // the kernels need more dynamic LDS than the default limit; the attribute is set once per device and kernel
  constexpr int kMaxDevices = 64;
  static std::atomic<bool> attr_set[kMaxDevices][2];
  auto launch = [&](auto kern, int slot) -> int {
    if (a.part.items == 0) return SG_OK;
    const dim3 grid((unsigned)(a.part.row_blocks * a.part.splits), (unsigned)a.kv_heads, (unsigned)(a.part.stacked ? 1 : a.n_tiles));
    if (dev < 0 || dev >= kMaxDevices || !attr_set[dev][slot].load(std::memory_order_acquire)) {
      SG_HIP_TRY(hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, kSplitLds));
      if (dev >= 0 && dev < kMaxDevices) attr_set[dev][slot].store(true, std::memory_order_release);
    }
    kern<<<grid, 256, kSplitLds, s>>>(a, tab);
    SG_HIP_TRY(hipGetLastError());
    return SG_OK;
  };
  return head_dim == 128 ? launch(context_bf16_split_kernel<128>, 0) : launch(context_bf16_split_kernel<64>, 1);
}

}  // namespace sg
