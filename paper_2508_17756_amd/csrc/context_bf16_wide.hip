// Context attention (sg_tile_cross_attention, sg_tile_prefix_attention) of calls with rows to fill the chip, bf16: products on the matrix
// cores with fp32 accumulation, softmax in fp32, scores scaled in fp32 behind the product.
//
// A workgroup of 4 wavefronts takes 128 rows of one head of keys, 32 per wavefront, over both segments of keys in one pass; its wavefronts
// share stages of 64 keys in LDS, two of keys and two of values.  The loop is pipelined inside a wavefront: iteration j takes the softmax
// of stage j on the vector ALU between the products of its neighbours, PV of stage j - 1 and QK of stage j + 1, on the matrix pipe.  Two
// workgroups run beside one another on a compute unit, so that the start and the end of one (rows in, rows out) hide behind the other.
//
// Measured, from device to device: 9 tiles of 3,840 rows over 512 + 3,840 keys, 24 heads x 128, 1.74 - 1.91 ms = 0.97 - 1.06 PFLOP/s at 1.74 - 1.83 GHz
// (power), matrix pipe 51 - 53 % busy; where it took 1.80, the loop took 1.53 ms without transfers, 1.36 without the fragment reads, 1.08 without both: bound
// by waits for LDS.  8 stages (75,600 rows over 512 keys, 40 heads) 0.93 - 1.03 ms = 0.77 - 0.85 PFLOP/s: start and end.  head_dim 64 (48 heads,
// 4 x 2,925 rows over 226 + 2,925 keys) 0.57 - 0.62 ms = 0.73 - 0.80: exponentials.
#include <atomic>
#include <type_traits>
#include "context_bf16.h"

namespace sg {
namespace {

template <int D>
constexpr int kWideSlots = D == 128 ? 64 : 32;
template <int D>
constexpr int kWideHalf = kWideSlots<D> * kSlot;   // keys (or values) of a stage
template <int D>
constexpr int kWideLds = 4 * kWideHalf<D>;         // two stages of keys, two of values: of a group of 4 wavefronts

// WAYS groups of 4 wavefronts take the same rows and shares of the keys, each with LDS of its own.
template <int D, int WAYS>
__global__ __launch_bounds__(256 * WAYS, 2) void context_bf16_wide_kernel(const CtxArgs a, const CtxTable tab) {
  constexpr int kKeys = 64, kInstr = kWideSlots<D> / 16, kHalf = kWideHalf<D>;
  extern __shared__ __attribute__((aligned(1024))) uint8_t smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) & 3;
  const int way = WAYS == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 8);
  const uint32_t lds_all = (uint32_t)(uintptr_t)(SG_LDS uint8_t*)smem, lds0 = lds_all + way * kWideLds<D>;
  const int lq = lane & 31, half = lane >> 5;
  const CtxPart& p = a.part;
  CtxItem item;
  if (!ctx_shared_item(a, p, item)) return;
  const int tile = item.tile, kvh = item.kvh, split = item.split, row_block = item.row_block;
  const int row0 = row_block * 128 + wave * 32;

  const CtxSegment g0 = ctx_segment<2>(a, tab, 0, tile, kvh), g1 = ctx_segment<2>(a, tab, 1, tile, kvh);
  const int n0 = p.seg0 ? (g0.len + kKeys - 1) / kKeys : 0, n1 = p.seg1 ? (g1.len + kKeys - 1) / kKeys : 0;
  const int part = split * WAYS + way, parts = p.splits * WAYS;
  const int from = (int)((int64_t)(n0 + n1) * part / parts), n = (int)((int64_t)(n0 + n1) * (part + 1) / parts) - from;   // stages: j = 0 is `from`

  bool mask_next = true;   // of the stage whose keys are requested next: whether key key0 + lane is unmasked
  auto fetch_mask = [&](int j) SG_INLINE {
    const int key = (from + j - n0) * kKeys + lane;
    mask_next = !(from + j >= n0 && j < n && g1.mask) || (key < g1.len && g1.mask[key] != 0);
  };
  const int first = wave * (kWideSlots<D> / 4);
  auto request = [&](int j, uint64_t v, bool is_v) SG_INLINE {
    const bool second = from + j >= n0;
    const CtxSegment& g = second ? g1 : g0;
    const int key0 = (second ? from + j - n0 : from + j) * kKeys;
    const uint32_t dst = lds0 + (is_v ? 2 * kHalf : 0) + (j & 1) * kHalf + first * kSlot;
    // (masked keys inside the segment may come along, their scores are replaced; masked values may not: 0 times a NaN is a NaN)
    const uint64_t take = !is_v && key0 + kKeys <= g.len ? ~0ull : v;
    move_half<D, kInstr>(is_v ? g.v : g.k, g.token, key0, first, take, is_v, dst);
  };
  // which of its keys count
  auto counting = [&](int j) SG_INLINE -> uint64_t {
    const bool second = from + j >= n0;
    const int key0 = (second ? from + j - n0 : from + j) * kKeys;
    const uint64_t v = __ballot(mask_next && key0 + lane < (second ? g1.len : g0.len));
    if (g1.mask) fetch_mask(j + 1);
    return v;
  };
  uint64_t v_now = 0, v_next = 0, v_later = 0;   // of the stages j, j + 1, j + 2
  if (n > 0) {
    if (g1.mask) fetch_mask(0);
    v_now = counting(0);
    request(0, v_now, false);
  }
  bf16x8 qf[D / 16];
  load_query<D>(a, tab, ctx_row(a, p, tile, kvh, row0 + lq), qf);
  Frags f = make_frags();
#pragma unroll
  for (int i = 0; i < 8; ++i) f.k[i] += lds0;
#pragma unroll
  for (int i = 0; i < 4; ++i) f.v[i] += lds0;
  int side = kHalf;
  auto turn = [&]() SG_INLINE {   // fragments are read from the other one of the two stages
#pragma unroll
    for (int i = 0; i < 8; ++i) f.k[i] += side;
#pragma unroll
    for (int i = 0; i < 4; ++i) f.v[i] += side;
    side = -side;
  };
  const float c_log2 = a.scale * 1.4426950408889634f;
  f32x16 o[D / 32], s[2];
  bf16x8 pr[4];
  float m = -__builtin_inff(), l = 0.f;
#pragma unroll
  for (int db = 0; db < D / 32; ++db) o[db] = zero16();

  auto meet = [&]() SG_INLINE {   // own transfers have landed; behind the barrier everyone's, and nobody reads what is requested next
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  // Fragment reads run kAhead steps (matrix instructions) ahead of their use; the scheduling barriers keep the compiler from gathering
  // them behind one another.
  constexpr int kAhead = 2, kDb = D / 32, kPv = 4 * kDb, kQk = 2 * (D / 16);
  auto kfrag = [&](uint32_t at0, int u) SG_INLINE -> bf16x8 {   // step u: block u / (D / 16), channels 16 (u % (D / 16)) .. + 15
    const int kk = u % (D / 16), b = u / (D / 16);
    const uint32_t at = at0 + f.k[D == 128 ? kk : 4 * b + kk] + (D == 128 ? b * 32 * kSlot : 0);
    return __builtin_bit_cast(bf16x8, *(const SG_LDS u32x4*)(uintptr_t)at);
  };
  auto vfrag = [&](uint32_t at0, int t) SG_INLINE -> bf16x8 {   // step t: the 16 keys of pr[t / kDb], channels 32 (t % kDb) .. + 31
    const int i = t / kDb, db = t % kDb, b = i >> 1, h = i & 1;
    const uint32_t at = at0 + f.v[D == 128 ? db : 2 * b + db] + (D == 128 ? b * 32 * kSlot : 0) + h * 16 * kSlot;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SG_LDS s16x4*)(uintptr_t)at);
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SG_LDS s16x4*)(uintptr_t)(at + 8 * kSlot));
    const s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(bf16x8, both);
  };
  bf16x8 ka[kQk], va[kPv];
  float alpha = 1.f, neg = 0.f, sum0 = 0.f, sum1 = 0.f;
  bool rescale = false;
  // Step t of a stage's softmax: the reference first, then a share of the exponentials, each rounded into pr when the product before has used
  // what was there.
  auto softmax_step = [&](int t) SG_INLINE {
    if (t == 0) {
      float mx0 = s[0][0], mx1 = s[1][0];
#pragma unroll
      for (int r = 1; r < 15; r += 2) {
        mx0 = fmaxf(fmaxf(mx0, s[0][r]), s[0][r + 1]);
        mx1 = fmaxf(fmaxf(mx1, s[1][r]), s[1][r + 1]);
      }
      float mx = fmaxf(fmaxf(mx0, mx1), fmaxf(s[0][15], s[1][15]));
      const uint32_t mu = __float_as_uint(mx);
      const auto sw = __builtin_amdgcn_permlane32_swap(mu, mu, false, false);
      mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * c_log2;
      const float moved = mx > m + kSlack ? mx : m;
      rescale = __any(moved != m);
      alpha = __builtin_amdgcn_exp2f(moved == m ? 0.f : m - moved);   // first keys: exp2(-inf) = 0
      m = moved;
      neg = m == -__builtin_inff() ? 0.f : -m;   // no key so far: probabilities 0
      sum0 = sum1 = 0.f;
    }
    constexpr int kSteps = kPv + kQk / 2 - 1;
    const int lo = t == 0 ? 0 : (t - 1) * 32 / kSteps, hi = t * 32 / kSteps;
#pragma unroll
    for (int e = 0; e < 32; ++e)
      if (e >= lo && e < hi) {
        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 4][e & 15], c_log2, neg));
        s[e >> 4][e & 15] = x;
      }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (8 * i + 8 > lo && 8 * i + 8 <= hi) {
#pragma unroll
        for (int r = 0; r < 8; ++r) pr[i][r] = (__bf16)s[i >> 1][8 * (i & 1) + r];
        asm volatile("" : "+v"(pr[i]));
        const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
#pragma unroll
        for (int r = 0; r < 8; r += 2) {
          const bf16x2 two = {pr[i][r], pr[i][r + 1]};
          if (r & 2) sum1 = __builtin_amdgcn_fdot2_f32_bf16(two, ones, sum1, false);
          else sum0 = __builtin_amdgcn_fdot2_f32_bf16(two, ones, sum0, false);
        }
      }
  };
  auto qk = [&](uint32_t at0, bool begun, bool soft) SG_INLINE {
    if (!begun) {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) ka[u] = kfrag(at0, u);
    }
#pragma unroll
    for (int u = 0; u < kQk; ++u) {
      if (u + kAhead < kQk) ka[u + kAhead] = kfrag(at0, u + kAhead);
      __builtin_amdgcn_sched_barrier(0);
      const int b = u / (D / 16), kk = u % (D / 16);
      s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[u], qf[kk], kk == 0 ? zero16() : s[b], 0, 0, 0);
      if (soft && b == 0) softmax_step(kPv + u);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto iteration = [&](int j, auto has_before, auto has_after) SG_INLINE {
    constexpr bool BEFORE = decltype(has_before)::value, AFTER = decltype(has_after)::value;
    meet();
    if (AFTER && j + 2 < n) {
      v_later = counting(j + 2);
      request(j + 2, v_later, false);
    }
    request(j, v_now, true);
    __builtin_amdgcn_sched_barrier(0);
    constexpr uint32_t k_at = 0, v_at = 2 * kHalf;   // of the other stage (the addresses change sides)
    turn();
    if (BEFORE) {
#pragma unroll
      for (int t = 0; t < kAhead; ++t) va[t] = vfrag(v_at, t);
    }
#pragma unroll
    for (int t = 0; t < kPv; ++t) {
      if (BEFORE && t + kAhead < kPv) va[t + kAhead] = vfrag(v_at, t + kAhead);
      else if (AFTER && t + kAhead >= kPv) ka[t + kAhead - kPv] = kfrag(k_at, t + kAhead - kPv);
      __builtin_amdgcn_sched_barrier(0);
      if (BEFORE) o[t % kDb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[t], pr[t / kDb], o[t % kDb], 0, 0, 0);
      softmax_step(t);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (AFTER) {
      qk(k_at, true, true);
    } else {
#pragma unroll
      for (int t = kPv; t < kPv + kQk / 2; ++t) softmax_step(t);
    }
    l = l * alpha + (sum0 + sum1);
    if (rescale) {
#pragma unroll
      for (int db = 0; db < D / 32; ++db) o[db] *= alpha;
    }
    if (AFTER && v_next != ~0ull) mask_scores<D, 2>(s, v_next);
    v_now = v_next;
    v_next = v_later;
  };
  if (n > 0) {
    meet();
    if (n > 1) {
      v_next = counting(1);
      request(1, v_next, false);
    }
    qk(0, false, false);
    if (v_now != ~0ull) mask_scores<D, 2>(s, v_now);
    using T = std::true_type;
    using F = std::false_type;
    if (n == 1) iteration(0, F{}, F{});
    else {
      iteration(0, F{}, T{});
      for (int j = 1; j < n - 1; ++j) iteration(j, T{}, T{});
      iteration(n - 1, T{}, F{});
    }
    meet();
    constexpr uint32_t v_at = 2 * kHalf;
    turn();
#pragma unroll
    for (int t = 0; t < kAhead; ++t) va[t] = vfrag(v_at, t);
#pragma unroll
    for (int t = 0; t < kPv; ++t) {
      if (t + kAhead < kPv) va[t + kAhead] = vfrag(v_at, t + kAhead);
      __builtin_amdgcn_sched_barrier(0);
      o[t % kDb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[t], pr[t / kDb], o[t % kDb], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  const uint32_t lu = __float_as_uint(l);
  const auto sw = __builtin_amdgcn_permlane32_swap(lu, lu, false, false);
  l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  if constexpr (WAYS == 2) {
    // The second group passes its share on through LDS, a register of all lanes behind another: sums where its stages were, (reference, sum) where
    // the first group's were.
    const int other = way == 0 ? 1 : 0, there = (int)((int64_t)(n0 + n1) * (split * 2 + other + 1) / parts) - (int)((int64_t)(n0 + n1) * (split * 2 + other) / parts);
    for (int i = n > 0 ? n + 2 : 0; i < (there > 0 ? there + 2 : 0); ++i) meet();   // the other group's barriers
    meet();
    const uint32_t sums = lds_all + kWideLds<D> + (wave * 64 + lane) * 16, ml = lds_all + (wave * 64 + lane) * 8;
    if (way == 1) {
      *(SG_LDS f32x2*)(uintptr_t)ml = f32x2{m, l};
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *(SG_LDS f32x4*)(uintptr_t)(sums + (4 * db + g) * 4096) = f32x4{o[db][4 * g], o[db][4 * g + 1], o[db][4 * g + 2], o[db][4 * g + 3]};
    }
    __syncthreads();
    if (way == 1) return;
    const f32x2 x = *(const SG_LDS f32x2*)(uintptr_t)ml;
    const float top = fmaxf(m, x[0]);
    const float e0 = l == 0.f ? 0.f : __builtin_amdgcn_exp2f(m - top), e1 = x[1] == 0.f ? 0.f : __builtin_amdgcn_exp2f(x[0] - top);   // 0: no keys
    m = top;
    l = l * e0 + x[1] * e1;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 v = *(const SG_LDS f32x4*)(uintptr_t)(sums + (4 * db + g) * 4096);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[db][4 * g + e] = o[db][4 * g + e] * e0 + v[e] * e1;
      }
  }
  const CtxRow mine = ctx_row(a, p, tile, kvh, row0 + lq);
  if (a.n_shares > 0) {   // a share: sums and reference for the join
    if (!mine.there) return;
    const int64_t at = (int64_t)mine.rid * a.n_shares + p.first_share + split;
    const int64_t all = (int64_t)a.n_tiles * a.heads * a.tokens * a.n_shares;
    if (half == 0) *(f32x2*)(a.shares + all * D + at * 2) = f32x2{m, l};
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(f32x4*)(a.shares + at * D + 32 * db + 8 * g + 4 * half) = f32x4{o[db][4 * g], o[db][4 * g + 1], o[db][4 * g + 2], o[db][4 * g + 3]};
    return;
  }
  write_row<D>(o, l == 0.f ? 0.f : 1.f / l, ctx_row_end<uint16_t>(a, tab, mine).out);
}

}  // namespace

int launch_context_bf16_wide(const CtxArgs& a, const CtxTable& tab, int head_dim, hipStream_t s) {
  int dev = 0;
  SG_HIP_TRY(hipGetDevice(&dev));
  constexpr int kMaxDevices = 64;
  static std::atomic<bool> attr_set[kMaxDevices][3];   // the kernels' dynamic-LDS limit has been raised
  auto launch = [&](auto kern, int slot, int lds) -> int {
    const int64_t grid = ((int64_t)a.part.items + 7) / 8 * 8;
    if (grid == 0) return SG_OK;
    if (dev < 0 || dev >= kMaxDevices || !attr_set[dev][slot].load(std::memory_order_acquire)) {
      SG_HIP_TRY(hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
      if (dev >= 0 && dev < kMaxDevices) attr_set[dev][slot].store(true, std::memory_order_release);
    }
    kern<<<dim3((unsigned)grid), 256 * a.part.ways, lds, s>>>(a, tab);
    SG_HIP_TRY(hipGetLastError());
    return SG_OK;
  };
  if (a.part.ways == 2) return launch(context_bf16_wide_kernel<64, 2>, 2, 2 * kWideLds<64>);   // (head_dim 64 alone: plan_context)
  return head_dim == 128 ? launch(context_bf16_wide_kernel<128, 1>, 0, kWideLds<128>) : launch(context_bf16_wide_kernel<64, 1>, 1, kWideLds<64>);
}

}  // namespace sg
