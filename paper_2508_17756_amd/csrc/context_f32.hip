// Attention of tiles to tokens beside their own (sg_tile_cross_attention, sg_tile_prefix_attention), fp32: products on the fp32 matrix
// instruction (16 x 16 x 4), everything else in fp32 too.
//
// S^T = K Q^T puts one row (query) per lane column and four keys in a lane's registers, which are then the B operands of
// O^T = V^T P^T as they stand: step r of a block of 16 keys contracts the keys 4 g + r of the four lane groups g.
//
// Row i of block db of O^T is channel 64 (db / 4) + 4 i + db % 4, so that a lane reads its values of four blocks, and writes its results, 16
// bytes at a time.
//
// Two forms.  Shared: the 4 wavefronts of a workgroup take 16 rows each against the same stages of keys, for calls with rows to fill the
// chip (32 each read fewer fragments, which do not bind, and end less evenly: 116 us for 110).  Otherwise every wavefront streams keys of its own through LDS of its own; wavefronts of a workgroup take other row blocks or other
// shares of the keys, whichever there are more of (context_common.h).
//
// Bound by the fp32 matrix instruction where there are rows (4 tiles of 2,880, 8 heads x 128, 226 keys: 112 us, 95 TFLOP/s; a large product of
// the library 154), by latency where there are few (4 tiles of 300, 2 heads x 64, 377 keys: 10.4 us).
#include <atomic>
#include "context_common.h"

namespace sg {
namespace {

#define SG_INLINE __attribute__((always_inline))

// A wavefront's LDS: two stages of 8 KiB of keys and 8 KiB of values; after the keys its sums (rows x D floats), then (reference, sum) of the rows and where they go.
constexpr int kHalfStage = 8192, kStage = 2 * kHalfStage, kWaveLds = 2 * kStage, kLds = 4 * kWaveLds;
constexpr int kSumsAt = kStage, kRowsAt = kSumsAt + 512;

// max / sum over the four lane groups
__device__ __forceinline__ float group_max(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t v = __float_as_uint(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float group_sum(float x) {
  x += __shfl_xor(x, 16, 64);
  return x + __shfl_xor(x, 32, 64);
}

template <int D, int QB, bool SHARED>
__global__ __launch_bounds__(256, SHARED ? 3 : 1) void context_f32_kernel(const CtxArgs a, const CtxTable tab) {
  constexpr int kKeys = kHalfStage / (D * 4);   // 16 (head_dim 64: 32)
  constexpr int kBlocks = kKeys / 16;
  constexpr int kChunks = D / 4;                // 16-byte chunks of a row
  constexpr int kRowsPer = 64 / kChunks;        // rows one transfer moves
  constexpr int kRows = 16 * QB;
  constexpr int kTransfers = SHARED ? 2 : 8;    // of a wavefront, of keys and as many of values
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(SG_LDS uint8_t*)smem;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int lq = lane & 15, grp = lane >> 4;

  const CtxPart& p = a.part;
  int split, row_block, kvh, batch;
  if constexpr (SHARED) {
    CtxItem item;
    if (!ctx_shared_item(a, p, item)) return;
    batch = item.tile;
    kvh = item.kvh;
    split = item.split;
    row_block = item.row_block;
  } else {   // the grid names tile and head of keys, so that the table of tiles can be read without waiting for anything else
    split = (int)blockIdx.x / p.row_blocks;
    row_block = (int)blockIdx.x - split * p.row_blocks;
    kvh = (int)blockIdx.y;
    batch = (int)blockIdx.z;
    if (!p.stacked && a.run && a.run[batch] == 0) return;
  }
  const int way = wave & (p.ways - 1);
  const int row0 = (row_block * (4 / p.ways) + wave / p.ways) * kRows;
  const uint32_t mine = SHARED ? lds0 : lds0 + wave * kWaveLds;

  f32x4 o[QB][D / 16];
  float m[QB], l[QB];
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) {
#pragma unroll
    for (int db = 0; db < D / 16; ++db) o[qb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
    m[qb] = -__builtin_inff();
    l[qb] = 0.f;
  }
  CtxRowEnd end[QB];   // of the rows lq
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) end[qb] = {0, 0};
  if (SHARED || row0 < p.rows) {
    const CtxSegment g0 = ctx_segment<4>(a, tab, 0, batch, kvh), g1 = ctx_segment<4>(a, tab, 1, batch, kvh);
    const int n0 = p.seg0 ? (g0.len + kKeys - 1) / kKeys : 0, n1 = p.seg1 ? (g1.len + kKeys - 1) / kKeys : 0;
    const int n = n0 + n1;
    const int from = (int)((int64_t)n * split / p.splits), to = (int)((int64_t)n * (split + 1) / p.splits);
    constexpr uint32_t kFull = kKeys == 32 ? 0xffffffffu : 0xffffu;
    uint32_t valid_next = 0;
    // 16-byte chunk c of K row r sits at chunk c ^ (r & 15), so that the 16 rows that a fragment read touches lie on different banks; V rows
    // are read along and stay as they are
    auto issue = [&](int j, int at) SG_INLINE {
      const bool second = j >= n0;
      const CtxSegment& g = second ? g1 : g0;
      const int key0 = (second ? j - n0 : j) * kKeys;
      bool counts = lane < kKeys && key0 + lane < g.len;
      if (g.mask && counts) counts = g.mask[key0 + lane] != 0;
      const uint32_t valid = (uint32_t)__ballot(counts);
      valid_next = valid;
      const int first = SHARED ? wave * kTransfers : 0;
      const uint32_t dst = mine + at * kStage + first * 1024;
      const char* const kp = g.k + (int64_t)key0 * g.token;
      const char* const vp = g.v + (int64_t)key0 * g.token;
      const int sub = lane / kChunks, c = lane % kChunks;
      if (valid == kFull) {
#pragma unroll
        for (int u = 0; u < kTransfers; ++u) {
          const int r = kRowsPer * (first + u) + sub;
          dma16(kp, (uint32_t)r * g.token + (uint32_t)((c ^ (r & 15)) << 4), dst + u * 1024);
          dma16(vp, (uint32_t)r * g.token + (uint32_t)(c << 4), dst + kHalfStage + u * 1024);
        }
      } else {   // keys that do not count are read from the zeros
        const char* const zeros = (const char*)g_ctx_zeros + ((c & 15) << 4);
#pragma unroll
        for (int u = 0; u < kTransfers; ++u) {
          const int r = kRowsPer * (first + u) + sub;
          const bool on = (valid >> r) & 1;
          dma16_addr(on ? kp + ((uint32_t)r * g.token + (uint32_t)((c ^ (r & 15)) << 4)) : zeros, dst + u * 1024);
          dma16_addr(on ? vp + ((uint32_t)r * g.token + (uint32_t)(c << 4)) : zeros, dst + kHalfStage + u * 1024);
        }
      }
    };
    int j = from + way;
    if (j < to) issue(j, 0);
    // B operand of S^T: query lq, step 4 jj + e contracts channel 16 jj + 4 grp + e
    f32x4 q[QB][D / 16];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      const CtxRow row = ctx_row(a, p, batch, kvh, row0 + 16 * qb + lq);
      end[qb] = ctx_row_end<float>(a, tab, row);
      const float* const src = (const float*)tab.q[row.tile] + (int64_t)row.head * a.q_head + (int64_t)row.token * a.q_token;
#pragma unroll
      for (int jj = 0; jj < D / 16; ++jj) {
        const f32x4 x = *(const f32x4*)(src + 16 * jj + 4 * grp);
        q[qb][jj] = x * a.scale;
      }
    }
    uint32_t kfrag[D / 16];   // offsets inside a half stage: row lq, chunk 4 jj + grp
#pragma unroll
    for (int jj = 0; jj < D / 16; ++jj) kfrag[jj] = lq * (D * 4) + (((4 * jj + grp) ^ lq) << 4);
    const uint32_t vfrag = kHalfStage + 4 * grp * (D * 4) + lq * 16;   // rows 4 grp (+ r), channels 4 lq (+ 64)
    for (int at = 0; j < to; j += p.ways, at ^= 1) {
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");   // this stage is there, the other one has been read
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (SHARED) {
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
      }
      const uint32_t valid = valid_next;
      if (j + p.ways < to) issue(j + p.ways, at ^ 1);
      if (valid == 0) continue;
      const uint32_t base = mine + at * kStage;
      // Fragments are read a group of matrix instructions ahead: those of K before the first product, those of V before the softmax.
      f32x4 kf[kBlocks][D / 16], vf[kBlocks][4][D / 64];
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int jj = 0; jj < D / 16; ++jj) kf[b][jj] = *(const SG_LDS f32x4*)(uintptr_t)(base + kfrag[jj] + b * 16 * D * 4);
      __builtin_amdgcn_sched_barrier(0);
      f32x4 s[QB][kBlocks];
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) s[qb][b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int jj = 0; jj < D / 16; ++jj)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) s[qb][b] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[b][jj][e], q[qb][jj][e], s[qb][b], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int h = 0; h < D / 64; ++h) vf[b][r][h] = *(const SG_LDS f32x4*)(uintptr_t)(base + vfrag + (16 * b + r) * (D * 4) + h * 256);
      __builtin_amdgcn_sched_barrier(0);
      if (__builtin_expect(valid != kFull, 0)) {
        uint32_t own_keys = valid >> (4 * grp);
        asm volatile("" : "+v"(own_keys));
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int qb = 0; qb < QB; ++qb)
              if (!((own_keys >> (16 * b + r)) & 1)) s[qb][b][r] = -__builtin_inff();
      }
#pragma unroll
      for (int qb = 0; qb < QB; ++qb) {
        float mx = s[qb][0][0];
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[qb][b][r]);
        mx = group_max(mx);
        const float top = fmaxf(m[qb], mx);
        if (__any(top != m[qb])) {
          const float alpha = m[qb] == top ? 1.f : exp2f((m[qb] - top) * kLog2e);   // first keys: exp2(-inf) = 0
          m[qb] = top;
          l[qb] *= alpha;
#pragma unroll
          for (int db = 0; db < D / 16; ++db) o[qb][db] *= alpha;
        }
        const float ref = m[qb] == -__builtin_inff() ? 0.f : m[qb];   // no key so far: probabilities 0
        // The exponential instruction returns 0 for results below 2^-126.  Where a score lies that far below the reference (or at -inf), the
        // function that returns them is called: times a value near the largest number they still count.  (4 tiles of 2,880, 8 heads x 128, 226 keys
        // 110.3 -> 112.4 us, 4 of 300, 2 heads x 64, 377 keys 10.2 -> 10.4.)
        float mn = s[qb][0][0];
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) mn = fminf(mn, s[qb][b][r]);
        const bool far = __any(mn - ref < -87.f);
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) s[qb][b][r] = (s[qb][b][r] - ref) * kLog2e;
        if (__builtin_expect(far, 0)) {
#pragma unroll
          for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[qb][b][r] = exp2f(s[qb][b][r]);
        } else {
#pragma unroll
          for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[qb][b][r] = __builtin_amdgcn_exp2f(s[qb][b][r]);
        }
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) l[qb] += s[qb][b][r];
      }
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int db = 0; db < D / 16; ++db)
#pragma unroll
            for (int qb = 0; qb < QB; ++qb)
              o[qb][db] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[b][r][db >> 2][db & 3], s[qb][b][r], o[qb][db], 0, 0, 0);
    }
  }
#pragma unroll
  for (int qb = 0; qb < QB; ++qb) l[qb] = group_sum(l[qb]);
  // a lane's results: channels 64 h + 16 grp + 4 r .. + 3 of its query
  auto four = [&](int qb, int h, int r) SG_INLINE -> f32x4 {
    return f32x4{o[qb][4 * h][r], o[qb][4 * h + 1][r], o[qb][4 * h + 2][r], o[qb][4 * h + 3][r]};
  };
  if constexpr (SHARED) {
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
      if (!end[qb].out) continue;
      float* dst;
      float by = 1.f;
      if (a.n_shares == 0) {
        dst = (float*)(uintptr_t)end[qb].out + 16 * grp;
        by = l[qb] == 0.f ? 0.f : 1.f / l[qb];
      } else {
        const int64_t at = (int64_t)end[qb].rid * a.n_shares + p.first_share + split;
        const int64_t all = (int64_t)a.n_tiles * a.heads * a.tokens * a.n_shares;
        dst = a.shares + at * D + 16 * grp;
        if (grp == 0) *(f32x2*)(a.shares + all * D + at * 2) = f32x2{m[qb], l[qb]};
      }
#pragma unroll
      for (int h = 0; h < D / 64; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) *(f32x4*)(dst + 64 * h + 4 * r) = four(qb, h, r) * by;
    }
  } else {
    // ---- join of the shares in this workgroup; chunk c of row r at chunk c ^ (r & 15)
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
#pragma unroll
      for (int h = 0; h < D / 64; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          *(SG_LDS f32x4*)(uintptr_t)(mine + (16 * qb + lq) * (D * 4) + (((16 * h + 4 * grp + r) ^ lq) << 4)) = four(qb, h, r);
      if (grp == 0) {
        *(SG_LDS f32x2*)(uintptr_t)(mine + kSumsAt + (16 * qb + lq) * 8) = f32x2{m[qb], l[qb]};
        *(SG_LDS u32x4*)(uintptr_t)(mine + kRowsAt + (16 * qb + lq) * 16) = u32x4{(uint32_t)end[qb].out, (uint32_t)(end[qb].out >> 32), (uint32_t)end[qb].rid, 0u};
      }
    }
    __syncthreads();
    const uint32_t group = lds0 + (wave & ~(p.ways - 1)) * kWaveLds;
    if (p.ways == 4) ctx_finish<float, D, kRows, 4>(a, p, group, kWaveLds, kSumsAt, kRowsAt, way, split, row0);
    else if (p.ways == 2) ctx_finish<float, D, kRows, 2>(a, p, group, kWaveLds, kSumsAt, kRowsAt, way, split, row0);
    else ctx_finish<float, D, kRows, 1>(a, p, group, kWaveLds, kSumsAt, kRowsAt, way, split, row0);
  }
}

}  // namespace

int launch_context_f32(const CtxArgs& a, const CtxTable& tab, int kind, int head_dim, hipStream_t s) {
  int dev = 0;
  SG_HIP_TRY(hipGetDevice(&dev));
  constexpr int kMaxDevices = 64;
  static std::atomic<bool> attr_set[kMaxDevices][6];   // the kernels' dynamic-LDS limit has been raised
  auto launch = [&](auto kern, int slot, int lds) -> int {
    if (a.part.items == 0) return SG_OK;
    const dim3 grid = kind == kCtxWide ? dim3((unsigned)((a.part.items + 7) / 8 * 8))
                                       : dim3((unsigned)(a.part.row_blocks * a.part.splits), (unsigned)a.kv_heads, (unsigned)(a.part.stacked ? 1 : a.n_tiles));
    if (dev < 0 || dev >= kMaxDevices || !attr_set[dev][slot].load(std::memory_order_acquire)) {
      SG_HIP_TRY(hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
      if (dev >= 0 && dev < kMaxDevices) attr_set[dev][slot].store(true, std::memory_order_release);
    }
    kern<<<grid, 256, lds, s>>>(a, tab);
    SG_HIP_TRY(hipGetLastError());
    return SG_OK;
  };
  if (kind == kCtxWide)
    return head_dim == 128 ? launch(context_f32_kernel<128, 1, true>, 4, kWaveLds) : launch(context_f32_kernel<64, 1, true>, 5, kWaveLds);
  if (kind == kCtxSplit16)
    return head_dim == 128 ? launch(context_f32_kernel<128, 1, false>, 0, kLds) : launch(context_f32_kernel<64, 1, false>, 1, kLds);
  return head_dim == 128 ? launch(context_f32_kernel<128, 2, false>, 2, kLds) : launch(context_f32_kernel<64, 2, false>, 3, kLds);
}

}  // namespace sg
