// Shared by the two bf16 kernels of context attention (context_bf16_wide.hip, context_bf16_split.hip): the layout of keys and values in LDS,
// the fragments read from it, masks, and the transfers that fill it.
//
// Both kernels form S^T = K Q^T, which puts one row (query) per lane column, so that the probabilities of a row stay in their lanes
// and are already the B operand of O^T = V^T P^T; V^T comes out of LDS through the transposing read.
#pragma once
#include "context_common.h"

namespace sg {
namespace {

#define SG_INLINE __attribute__((always_inline))

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

template <int D>
__device__ __forceinline__ void load_query(const CtxArgs& a, const CtxTable& tab, const CtxRow& row, bf16x8 (&qf)[D / 16]) {
  const int half = (threadIdx.x & 63) >> 5;
  const uint16_t* const q = (const uint16_t*)tab.q[row.tile] + (int64_t)row.head * a.q_head + (int64_t)row.token * a.q_token;
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) {
    u32x4 x = *(const u32x4*)(q + 16 * kk + 8 * half);
    if (!row.there) x = u32x4{0, 0, 0, 0};
    qf[kk] = __builtin_bit_cast(bf16x8, x);
  }
}

// The keys of one segment as a stage of 64 (or 32) is taken from them.
struct Segment {
  const char* k;    // head's first key
  const char* v;
  uint32_t token;   // bytes between keys
  int len;
  const uint8_t* mask;
};
__device__ __forceinline__ Segment segment(const CtxArgs& a, const CtxTable& tab, int which, int tile, int kvh) {
  Segment g;
  const void* const k = which == 0 ? a.k0 : tab.k[tile];
  const void* const v = which == 0 ? a.v0 : tab.v[tile];
  const int64_t head = (int64_t)kvh * a.kv_head[which] * 2;
  g.k = (const char*)k + head;
  g.v = (const char*)v + head;
  g.token = (uint32_t)(a.kv_token[which] * 2);
  g.len = which == 0 ? ctx_length(a.len0, 0, a.cap0) : ctx_length(a.len1, tile, a.cap1);
  g.mask = (which == 1 && a.mask1) ? a.mask1 + (int64_t)tile * a.cap1 : nullptr;
  return g;
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

}  // namespace
}  // namespace sg
