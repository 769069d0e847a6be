// Shared by the bf16 kernels of context attention (context_bf16_wide.hip, context_bf16_split.hip, context_bf16_resident.hip): the layout of keys
// and values in LDS, the fragments read from it, masks, and the transfers that fill it.
//
// All of them form S^T = K Q^T, which puts one row (query) per lane column, so that the probabilities of a row stay in their lanes
// and are already the B operand of O^T = V^T P^T; V^T comes out of LDS through the transposing read.
#pragma once
#include "context_common.h"

namespace sg {
namespace {

#define SG_INLINE __attribute__((always_inline))

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// How far a score may pass a row's reference, log2, before the reference moves: any reference gives the same quotient, the sums of p v grow to at most
// 32 times what they are against the maximum, and the common path rescales nothing.  Probabilities are rounded to bf16 for the second product (half
// a step of each, which averages out over a row); their sum is taken of the rounded ones, so that the weights sum to one.
constexpr float kSlack = 5.f;

constexpr int kSlot = 256;   // LDS bytes of a "slot": one key of head_dim 128, two neighbouring ones of head_dim 64

__device__ __forceinline__ f32x16 zero16() {
  return f32x16{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
}

// Per-lane LDS offsets of the fragments.  16-byte chunk c of K slot r sits at chunk c ^ (r & 15), of V slot r at c ^ ((r & 3) << 2):
// both reads are then free of bank conflicts.
struct Frags {
  uint32_t k[8];   // slot lq, chunk 2 kk + half
  uint32_t v[4];   // transposing read: 64-byte piece db of 4 slots
};
__device__ __forceinline__ Frags make_frags() {
  const int lane = threadIdx.x & 63, lq = lane & 31, half = lane >> 5;
  Frags f;
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) f.k[kk] = lq * kSlot + (((2 * kk + half) ^ (lq & 15)) << 4);
  const int grp = lane >> 4, gi = lane & 15;
  const int row = 4 * (grp >> 1) + (gi >> 2), dbyte = (16 * (grp & 1) + 4 * (gi & 3)) * 2;
#pragma unroll
  for (int db = 0; db < 4; ++db) f.v[db] = row * kSlot + (((4 * db + (dbyte >> 4)) ^ ((row & 3) << 2)) << 4) + (dbyte & 15);
  return f;
}

// Scores of the keys that do not count become -inf.  Register r of block b is row 8 (r >> 2) + 4 half + (r & 3) of it: key 32 b + row
// (head_dim 128) or 2 row + b (64); bit i of valid is key i.
template <int D, int NB>
__device__ __forceinline__ void mask_scores(f32x16 (&s)[NB], const uint64_t valid) {
  const int half = (threadIdx.x & 63) >> 5;
  uint64_t mine = valid >> (D == 128 ? 4 * half : 8 * half);
  asm volatile("" : "+v"(mine));   // keeps the compiler from doing this for whole stages as well and selecting afterwards
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int row = 8 * (r >> 2) + (r & 3), bit = D == 128 ? 32 * b + row : 2 * row + b;
      const uint32_t w = bit < 32 ? (uint32_t)mine : (uint32_t)(mine >> 32);
      const uint32_t keep = (uint32_t)((int32_t)(w << (31 - (bit & 31))) >> 31);
      s[b][r] = __uint_as_float((__float_as_uint(s[b][r]) & keep) | (0xff800000u & ~keep));
    }
}

// (a row that is not there stands in for the last one; its results are not written)
template <int D>
__device__ __forceinline__ void load_query(const CtxArgs& a, const CtxTable& tab, const CtxRow& row, bf16x8 (&qf)[D / 16]) {
  const int half = (threadIdx.x & 63) >> 5;
  const uint16_t* const q = (const uint16_t*)tab.q[row.tile] + (int64_t)row.head * a.q_head + (int64_t)row.token * a.q_token;
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) qf[kk] = __builtin_bit_cast(bf16x8, *(const u32x4*)(q + 16 * kk + 8 * half));
}

// Transfers of a wavefront: instruction u moves the slots first + 4 u .. + 3; lane l fills chunk l & 15 of the (l >> 4)-th of them and
// so fetches the chunk that belongs there: chunk `chunk` of the key `key` behind the first key of these slots.
template <int D>
__device__ __forceinline__ void lane_source(int slot, int lane, bool is_v, int& key, int& chunk) {
  const int c = (lane & 15) ^ (is_v ? (slot & 3) << 2 : slot & 15);
  key = D == 128 ? slot : 2 * slot + (c >> 3);
  chunk = D == 128 ? c : c & 7;
}
// Moves N_INSTR x 4 slots of keys (or values) of a stage whose first key is key0, from slot `first` on, to LDS dst; bit i of valid: whether
// its key i counts (all 64 bits: whole).  A whole stage is addressed by a 64-bit base and 32-bit offsets; in others the keys that do not
// count are read from the zeros.
template <int D, int N_INSTR>
__device__ __forceinline__ void move_half(const char* base, const uint32_t token, const int key0, const int first, const uint64_t valid,
                                          const bool is_v, const uint32_t dst, const uint64_t whole = ~0ull) {
  const int lane = threadIdx.x & 63;
  const char* const from = base + (int64_t)key0 * token;
  if (valid == whole) {
#pragma unroll
    for (int u = 0; u < N_INSTR; ++u) {
      int key, chunk;
      lane_source<D>(first + 4 * u + (lane >> 4), lane, is_v, key, chunk);
      dma16(from, (uint32_t)key * token + (uint32_t)chunk * 16, dst + u * 1024);
    }
  } else {
    const char* const zeros = (const char*)g_ctx_zeros;
#pragma unroll
    for (int u = 0; u < N_INSTR; ++u) {
      int key, chunk;
      lane_source<D>(first + 4 * u + (lane >> 4), lane, is_v, key, chunk);
      dma16_addr((valid >> key) & 1 ? from + ((uint32_t)key * token + (uint32_t)chunk * 16) : zeros + chunk * 16, dst + u * 1024);
    }
  }
}

// One row's softmax (the same in lanes l and l ^ 32) and its output accumulators.
template <int D>
struct RowState {
  f32x16 o[D / 32];
  float m;   // running maximum, log2 domain
  float l;   // this lane's share of the sum
};
template <int D>
__device__ __forceinline__ void clear(RowState<D>& st) {
#pragma unroll
  for (int db = 0; db < D / 32; ++db) st.o[db] = zero16();
  st.m = -__builtin_inff();
  st.l = 0.f;
}

// NB blocks of 32 keys, K at LDS address kb0 and V at vb0.  head_dim 128: block b is the slots 32 b .. 32 b + 31; head_dim 64: the 32 slots
// hold two keys each and block b (of 2) is their b-th ones.
template <int D, int NB>
__device__ __forceinline__ void attend_keys(const Frags& f, const uint32_t kb0, const uint32_t vb0, const bf16x8 (&qf)[D / 16], const float c_log2,
                                            const uint64_t valid, RowState<D>& st) {
  // All fragments of a product are read at once, those of V before the softmax: one or two wavefronts on a SIMD hide little behind each other.
  static_assert(D == 128 || NB == 2, "");
  constexpr uint64_t kFull = (D == 128 && NB == 1) ? 0xffffffffull : ~0ull;
  bf16x8 kf[NB][D / 16], vf[2 * NB][D / 32];
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
    for (int b = 0; b < NB; ++b)
      kf[b][kk] = __builtin_bit_cast(bf16x8, *(const SG_LDS u32x4*)(uintptr_t)(kb0 + f.k[D == 128 ? kk : 4 * b + kk] + (D == 128 ? b * 32 * kSlot : 0)));
  __builtin_amdgcn_sched_barrier(0);
  f32x16 s[NB];
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk)
#pragma unroll
    for (int b = 0; b < NB; ++b) s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[b][kk], qf[kk], kk == 0 ? zero16() : s[b], 0, 0, 0);
#pragma unroll
  for (int i = 0; i < 2 * NB; ++i)
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      const int b = i >> 1, h = i & 1;
      const uint32_t at = vb0 + f.v[D == 128 ? db : 2 * b + db] + (D == 128 ? b * 32 * kSlot : 0) + h * 16 * kSlot;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SG_LDS s16x4*)(uintptr_t)at);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((SG_LDS s16x4*)(uintptr_t)(at + 8 * kSlot));
      const s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      vf[i][db] = __builtin_bit_cast(bf16x8, both);
    }
  __builtin_amdgcn_sched_barrier(0);
  if (valid != kFull) mask_scores<D, NB>(s, valid);
  float mx = s[0][0];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int r = 0; r < 16; r += 2) mx = fmaxf(fmaxf(mx, s[b][r]), s[b][r + 1]);
  const uint32_t mu = __float_as_uint(mx);
  const auto sw = __builtin_amdgcn_permlane32_swap(mu, mu, false, false);
  mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
  mx *= c_log2;
  if (__any(mx > st.m + kSlack)) {   // (the first keys, too: -inf + 5)
    const float top = mx > st.m + kSlack ? mx : st.m;
    const float alpha = __builtin_amdgcn_exp2f(top == st.m ? 0.f : st.m - top);   // first keys: exp2(-inf) = 0
    st.m = top;
    st.l *= alpha;
#pragma unroll
    for (int db = 0; db < D / 32; ++db) st.o[db] *= alpha;
  }
  const float neg = st.m == -__builtin_inff() ? 0.f : -st.m;   // no key so far: probabilities 0
  const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
  float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      bf16x8 p;
#pragma unroll
      for (int r = 0; r < 8; ++r) p[r] = (__bf16)__builtin_amdgcn_exp2f(__builtin_fmaf(s[b][8 * h + r], c_log2, neg));
#pragma unroll
      for (int r = 0; r < 8; r += 2) {
        const bf16x2 two = {p[r], p[r + 1]};
        if (r & 2) sum1 = __builtin_amdgcn_fdot2_f32_bf16(two, ones, sum1, false);
        else sum0 = __builtin_amdgcn_fdot2_f32_bf16(two, ones, sum0, false);
      }
#pragma unroll
      for (int db = 0; db < D / 32; ++db) st.o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[2 * b + h][db], p, st.o[db], 0, 0, 0);
    }
  st.l += sum0 + sum1;
}

// Row lq of lanes lq and lq + 32 to its place (0: none): the two exchange halves, so that each writes 16 bytes at a time.  (Through LDS a store
// writes whole rows, but the way there and back, with the rows' addresses, took 1,700 cycles; this takes 500.)
template <int D>
__device__ __forceinline__ void write_row(const f32x16 (&o)[D / 32], const float inv, const uint64_t to) {
  const int half = (threadIdx.x & 63) >> 5;
  uint16_t* const dst = (uint16_t*)(uintptr_t)to + 8 * half;
  u32x4 w[D / 16];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int r = 8 * k;   // registers r .. r + 3: channels 32 db + 16 k + 4 half + 0..3, r + 4 .. r + 7: 8 channels on
      const auto lo = __builtin_amdgcn_permlane32_swap(pack_bf16x2(o[db][r] * inv, o[db][r + 1] * inv), pack_bf16x2(o[db][r + 4] * inv, o[db][r + 5] * inv), false, false);
      const auto hi = __builtin_amdgcn_permlane32_swap(pack_bf16x2(o[db][r + 2] * inv, o[db][r + 3] * inv), pack_bf16x2(o[db][r + 6] * inv, o[db][r + 7] * inv), false, false);
      w[2 * db + k] = u32x4{(uint32_t)lo[0], (uint32_t)hi[0], (uint32_t)lo[1], (uint32_t)hi[1]};
    }
  if (to) {
#pragma unroll
    for (int i = 0; i < D / 16; ++i) *(u32x4*)(dst + 16 * i) = w[i];
  }
}

}  // namespace
}  // namespace sg
