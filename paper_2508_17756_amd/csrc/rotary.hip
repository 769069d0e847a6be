// Rotary positions of the queries and keys of tiles (sg_tile_rotary): pair (a, b) -> (a cos w - b sin w, b cos w + a sin w), w = frequency * position,
// with or without a root-mean-square norm of each head before it.
//
// A workgroup takes a few tokens of a tile with all their heads (or a part of them): it computes the tokens' sines and cosines once, into LDS, and then
// passes over the heads, each lane with 16 channels of one head as two vectors of 8 whose pairs lie in the lane.  The angle is a product in fp64
// (positions reach millions of turns), reduced to a part of one turn there, and only that is rounded to fp32.
//
// Bound by memory, every channel read and written once: 75,600 tokens of 40 + 40 heads x 128 in bf16, token-major, with or without the norm of the heads 510 us
// (6.1 TB/s; a large copy runs at 5.0), head-major 605; 9 x 4,000 tokens of 40 + 8 heads 153 us (5.8).  The arithmetic has to stay below it: with factors and
// places found anew for every head and each pair asked whether it turns, the vector units were 96 % busy and the first of these took 587 us.  So q and k are
// passes of their own with their weight in registers, offsets are 32 bits where they fit, and heads that turn whole have a form without questions.  Few short heads
// are bound by the sines: 9 tiles of 75,600 tokens, 1 + 1 heads x 64 97 us (3.6 TB/s).
#include "block_api.h"
#include "row_common.h"

namespace sg {
namespace {

constexpr int kRotaryTilesPerLaunch = 32;
struct RotaryTable {
  const void* q[kRotaryTilesPerLaunch];
  const void* k[kRotaryTilesPerLaunch];
  void* q_out[kRotaryTilesPerLaunch];
  void* k_out[kRotaryTilesPerLaunch];
  const int32_t* positions[kRotaryTilesPerLaunch];
  int32_t origin[kRotaryTilesPerLaunch][3];
};
struct RotaryArgs {
  const double* frequencies;
  const void* q_weight;
  const void* k_weight;
  const uint8_t* run;
  int64_t q_token, q_head, qo_token, qo_head, k_token, k_head, ko_token, ko_head;
  int32_t tokens, chunk, chunk_shift, chunks;   // of a tile; tokens of a workgroup (2^chunk_shift); workgroups of a tile
  int32_t heads, all_heads;                     // of q; of q and k
  int32_t head_step;                            // heads of a workgroup: blockIdx.y takes head_step of them
  int32_t channels, n_vec, lanes, lane_shift;   // of a head; vectors of 8; lanes of a head (a power of two)
  int32_t turned, first_y, first_x;             // channels that turn; first pair of the axes y and x
  int32_t H_W, W, position_axes;
  int32_t canvas[3];
  Divisor by_plane, by_row, by_chunks, by_heads, by_kv_heads;
  bool near;                                    // offsets inside a workgroup's tokens are below 2^32 elements
  bool by_token;                                // rows in the order of memory: heads of a token side by side
  float eps, by_channels;
};

// HALF: layout; LINES: a load of a head's lanes takes whole cache lines; FULL: every channel turns and every lane has two vectors
template <typename T, bool HALF, bool LINES, bool FULL>
__global__ __launch_bounds__(256) void rotary_kernel(const RotaryArgs a, const RotaryTable tab) {
  extern __shared__ __align__(16) float turns[];   // [chunk][pairs padded to 8] cosines, then sines
  const int tile = (int)divide(blockIdx.x, a.by_chunks);
  if (a.run && a.run[tile] == 0) return;
  const int token0 = (int)(blockIdx.x - (uint32_t)tile * (uint32_t)a.chunks) << a.chunk_shift;
  const int n_tokens = a.tokens - token0 < a.chunk ? a.tokens - token0 : a.chunk;
  const int pairs = a.turned >> 1, row_pairs = (pairs + 7) & ~7;
  float* const cosines = turns;
  float* const sines = turns + a.chunk * row_pairs;

  const int l = threadIdx.x & (a.lanes - 1);
  // The lane's vectors: HALF: those of the channels that turn meet their partners, half of them behind; the others two by two.
  const int half = a.turned >> 4;
  const bool has_a = FULL || 2 * l < a.n_vec || (!HALF && l < (a.n_vec + 1) / 2);
  int va, vb;
  if (HALF) {
    va = FULL || l < half ? l : 2 * l;
    vb = FULL || l < half ? l + half : 2 * l + 1;
  } else {
    va = l;
    vb = l + (a.n_vec + 1) / 2;
  }
  const bool has_b = FULL || (has_a && vb < a.n_vec);

  // The workgroup's heads: of q, then of k.
  const int step = 256 >> a.lane_shift;
  const int head0 = blockIdx.y * a.head_step, head1 = min(head0 + a.head_step, a.all_heads);
  const int q_heads = max(min(head1, a.heads) - head0, 0), k_heads = head1 - max(head0, a.heads);
  // Its row r of n heads as (token, head).
  struct Row { int t, head; };
  auto row_of = [&](int r, int n) {
    int t, head;
    if (a.by_token) {
      t = n == a.heads ? (int)divide((uint32_t)r, a.by_heads) : n == a.all_heads - a.heads ? (int)divide((uint32_t)r, a.by_kv_heads) : r / n;
      head = r - t * n;
    } else {
      head = n_tokens == a.chunk ? r >> a.chunk_shift : r / n_tokens;
      t = r - head * n_tokens;
    }
    return Row{t, head};
  };
  auto offset = [&](Row w, int64_t token, int64_t head) -> int64_t {
    return a.near ? (int64_t)((uint32_t)w.t * (uint32_t)token + (uint32_t)w.head * (uint32_t)head) : w.t * token + w.head * head;
  };
  Chan8<T> ra, rb;
  auto fetch = [&](const T* x) {
    if constexpr (LINES) {
      if (has_a) ra.stream(x + 8 * va);
      if (has_b) rb.stream(x + 8 * vb);
    } else {
      if (has_a) ra.load(x + 8 * va);
      if (has_b) rb.load(x + 8 * vb);
    }
  };
  // The first rows are on their way while the sines are computed, the next ones while a row is turned.
  const T* const q = (const T*)tab.q[tile] + token0 * a.q_token + head0 * a.q_head;
  if (q_heads > 0 && (int)(threadIdx.x >> a.lane_shift) < q_heads * n_tokens) fetch(q + offset(row_of(threadIdx.x >> a.lane_shift, q_heads), a.q_token, a.q_head));

  for (int i = threadIdx.x; i < n_tokens * row_pairs; i += 256) {
    const int t = i / row_pairs, pair = i - t * row_pairs;
    if (pair >= pairs) continue;
    const int token = token0 + t;
    const int axis = (pair >= a.first_y) + (pair >= a.first_x);
    int position;
    if (tab.positions[tile]) {
      position = a.position_axes == 1 ? tab.positions[tile][token] : tab.positions[tile][3 * (int64_t)token + axis];
    } else {
      const int frame = (int)divide((uint32_t)token, a.by_plane), rest = token - frame * a.H_W;
      const int y = (int)divide((uint32_t)rest, a.by_row);
      const int* const origin = tab.origin[tile];
      position = axis == 0 ? origin[0] + frame : axis == 1 ? origin[1] + y : origin[2] + rest - y * a.W;
      const int size = axis == 0 ? a.canvas[0] : axis == 1 ? a.canvas[1] : a.canvas[2];
      if (size > 0) position = (int)((uint32_t)position % (uint32_t)size);   // (the origin lies inside the canvas)
    }
    double turn = (double)position * (a.frequencies[pair] * 0.15915494309189535);   // 1 / (2 pi)
    turn -= __builtin_rint(turn);
    float sine, cosine;
    if constexpr (sizeof(T) == 2) {   // the instructions take parts of a turn and are off by 2^-22.9 at most over one (measured; sincospif in the fp32 form: 2^-24)
      sine = __builtin_amdgcn_sinf((float)turn);
      cosine = __builtin_amdgcn_cosf((float)turn);
    } else {
      sincospif(2.f * (float)turn, &sine, &cosine);
    }
    cosines[i] = cosine;
    sines[i] = sine;
  }
  __syncthreads();

  auto turn_heads = [&](const T* const x, T* const y, int heads, int64_t x_token, int64_t x_head, int64_t y_token, int64_t y_head, const T* const weight, bool fetched) {
    const int n_rows = heads * n_tokens;
    int r = threadIdx.x >> a.lane_shift;
    if (r >= n_rows) return;
    Row now = row_of(r, heads);
    if (!fetched) fetch(x + offset(now, x_token, x_head));
    Chan8<T> wa, wb;
    wa.clear();
    wb.clear();
    if (weight && has_a) wa.load(weight + 8 * va);
    if (weight && has_b) wb.load(weight + 8 * vb);
    for (; r < n_rows;) {
      float u[8], v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        u[e] = has_a ? ra.get(e) : 0.f;
        v[e] = has_b ? rb.get(e) : 0.f;
      }
      const int t = now.t;
      T* const to = y + offset(now, y_token, y_head);
      r += step;
      if (r < n_rows) {
        now = row_of(r, heads);
        fetch(x + offset(now, x_token, x_head));
      }
      if (weight) {
        float sq = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) sq = fmaf(u[e], u[e], fmaf(v[e], v[e], sq));
        const float mean = sum_over_lanes(sq, a.lanes) * a.by_channels + a.eps;
        float norm = rsqrtf(mean);
        const bool odd = !(mean >= kLeastMean && mean <= kMostFloat);
        if (__any(odd)) {
          const float to_range = !odd ? 1.f : mean < kLeastMean ? kGrowRow : kShrinkRow;
          sq = 0.f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            u[e] *= to_range;
            v[e] *= to_range;
            sq = fmaf(u[e], u[e], fmaf(v[e], v[e], sq));
          }
          const float other = rsqrtf(sum_over_lanes(sq, a.lanes) * a.by_channels + a.eps * to_range * to_range);
          if (odd) norm = other;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          u[e] = u[e] * norm * wa.get(e);
          v[e] = v[e] * norm * wb.get(e);
        }
      }
      const float* const c = cosines + t * row_pairs;
      const float* const s = sines + t * row_pairs;
      if (HALF) {
        if (FULL || l < half) {
          Chan8<float> cs, sn;
          cs.load(c + 8 * l);
          sn.load(s + 8 * l);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float p = u[e], q = v[e];
            u[e] = p * cs.get(e) - q * sn.get(e);
            v[e] = q * cs.get(e) + p * sn.get(e);
          }
        }
      } else {
        auto turn4 = [&](float (&w)[8], int first) {   // pairs first .. first + 3
          if (!FULL && first >= row_pairs) return;
          const f32x4 cs = *(const f32x4*)(c + first), sn = *(const f32x4*)(s + first);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (FULL || first + e < pairs) {
              const float p = w[2 * e], q = w[2 * e + 1];
              w[2 * e] = p * cs[e] - q * sn[e];
              w[2 * e + 1] = q * cs[e] + p * sn[e];
            }
        };
        turn4(u, 4 * va);
        turn4(v, 4 * vb);
      }
      if constexpr (LINES) {
        if (has_a) stream8(to + 8 * va, u);
        if (has_b) stream8(to + 8 * vb, v);
      } else {
        if (has_a) store8(to + 8 * va, u);
        if (has_b) store8(to + 8 * vb, v);
      }
    }
  };
  if (q_heads > 0)
    turn_heads(q, (T*)tab.q_out[tile] + token0 * a.qo_token + head0 * a.qo_head, q_heads, a.q_token, a.q_head, a.qo_token, a.qo_head, (const T*)a.q_weight, true);
  if (k_heads > 0) {
    const int first = max(head0, a.heads) - a.heads;
    turn_heads((const T*)tab.k[tile] + token0 * a.k_token + first * a.k_head, (T*)tab.k_out[tile] + token0 * a.ko_token + first * a.ko_head, k_heads, a.k_token, a.k_head,
               a.ko_token, a.ko_head, (const T*)a.k_weight, false);
  }
}

}  // namespace

int launch_rotary(const sg_rotary_problem& p, int n_tiles, const void* const* q, const void* const* k, const double* frequencies,
                  const int32_t* origin, const int32_t* const* positions, const void* q_weight, const void* k_weight, const uint8_t* run,
                  void* const* q_out, void* const* k_out, hipStream_t s) {
  RotaryArgs a = {};
  a.frequencies = frequencies; a.q_weight = q_weight; a.k_weight = k ? k_weight : nullptr;
  a.q_token = p.q_stride_token; a.q_head = p.q_stride_head; a.qo_token = p.q_out_stride_token; a.qo_head = p.q_out_stride_head;
  a.k_token = p.k_stride_token; a.k_head = p.k_stride_head; a.ko_token = p.k_out_stride_token; a.ko_head = p.k_out_stride_head;
  a.tokens = p.T * p.H * p.W;
  a.heads = p.heads; a.all_heads = p.heads + (k ? p.kv_heads : 0);
  a.channels = p.head_dim; a.n_vec = p.head_dim / 8;
  a.lanes = 1; a.lane_shift = 0;
  while (2 * a.lanes < a.n_vec) { a.lanes <<= 1; ++a.lane_shift; }
  a.turned = p.axis_t + p.axis_y + p.axis_x;
  a.first_y = p.axis_t / 2; a.first_x = (p.axis_t + p.axis_y) / 2;
  a.H_W = p.H * p.W; a.W = p.W; a.position_axes = p.position_axes;
  a.canvas[0] = p.canvas_t; a.canvas[1] = p.canvas_h; a.canvas[2] = p.canvas_w;
  a.by_plane = make_divisor((uint32_t)a.H_W); a.by_row = make_divisor((uint32_t)p.W);
  a.by_heads = make_divisor((uint32_t)a.heads);
  a.by_kv_heads = make_divisor((uint32_t)(k ? p.kv_heads : 1));
  a.by_token = p.q_stride_head < p.q_stride_token;
  a.eps = p.eps;
  a.by_channels = 1.f / (float)p.head_dim;
  // Tokens of a workgroup: rows for one pass of it at least, where that leaves 2,048 workgroups (2 x 36 x 40 tokens, 4 tiles, 8 + 8 heads of 128, fp32: 45 us, with 8
  // passes 49), and for few passes: 4 over heads of whole cache lines that lie side by side (75,600 tokens, 40 + 40 heads x 128 509 us; 2 523, 8 543, 16 569), 8 over
  // others (4 tiles, 5 + 5 heads x 96 244; 4 274).  Heads that lie apart: for runs of 4 KiB, up to 64 passes (605 us; 8 626, 2 677).  Its table within 32 KiB.
  const int rows_per_pass = 256 >> a.lane_shift, row_pairs = (a.turned / 2 + 7) & ~7;
  const int passes_most = !a.by_token ? 64 : p.head_dim % 128 == 0 ? 4 : 8;
  const int run_bytes = p.head_dim * (p.dtype == SG_F32 ? 4 : 2);
  a.chunk = 1; a.chunk_shift = 0;
  while (a.chunk < 64 && a.chunk < a.tokens && 2 * a.chunk * row_pairs * 8 <= 32768) {
    const int64_t rows = (int64_t)a.chunk * a.all_heads, wgs = (int64_t)n_tiles * a.tokens / (2 * a.chunk);
    if (rows >= rows_per_pass && (wgs < 2048 || rows >= passes_most * rows_per_pass || (rows >= 8 * rows_per_pass && a.chunk * run_bytes >= 4096))) break;
    a.chunk <<= 1; ++a.chunk_shift;
  }
  a.chunks = (a.tokens + a.chunk - 1) / a.chunk;
  a.by_chunks = make_divisor((uint32_t)a.chunks);
  const size_t lds = (size_t)a.chunk * row_pairs * 8;
  auto reach = [&](int64_t token, int64_t head, int64_t heads) {   // (in doubles: the products can pass 64 bits)
    return (double)(a.chunk - 1) * (double)token + (double)(heads - 1) * (double)head < 4294967296.0 && token < (1ll << 32) && head < (1ll << 32);
  };
  a.near = reach(a.q_token, a.q_head, a.heads) && reach(a.qo_token, a.qo_head, a.heads) &&
           (!k || (reach(a.k_token, a.k_head, p.kv_heads) && reach(a.ko_token, a.ko_head, p.kv_heads)));
  // A grid has less than 2^32 threads: 2^24 workgroups, times the parts of few tokens' heads.
  int most_tiles = ((1 << 24) - 1) / a.chunks;
  most_tiles = most_tiles < 1 ? 1 : most_tiles > kRotaryTilesPerLaunch ? kRotaryTilesPerLaunch : most_tiles;
  for (int t0 = 0; t0 < n_tiles; t0 += most_tiles) {
    const int n = n_tiles - t0 < most_tiles ? n_tiles - t0 : most_tiles;
    RotaryTable tab = {};
    for (int i = 0; i < n; ++i) {
      tab.q[i] = q[t0 + i];
      tab.q_out[i] = q_out[t0 + i];
      tab.k[i] = k ? k[t0 + i] : nullptr;
      tab.k_out[i] = k ? k_out[t0 + i] : nullptr;
      tab.positions[i] = positions ? positions[t0 + i] : nullptr;
      for (int j = 0; j < 3 && origin; ++j) {
        int64_t at = origin[3 * (t0 + i) + j];
        if (a.canvas[j] > 0) at = (at % a.canvas[j] + a.canvas[j]) % a.canvas[j];
        tab.origin[i][j] = (int32_t)at;
      }
    }
    a.run = run ? run + t0 : nullptr;
    // Few tokens: their heads go to several workgroups, one pass each.
    int splits = 1;
    const int64_t wgs = (int64_t)n * a.chunks;
    const int passes = (int)(((int64_t)a.chunk * a.all_heads + rows_per_pass - 1) / rows_per_pass);
    while (splits < passes && wgs * splits < 512) ++splits;
    a.head_step = (a.all_heads + splits - 1) / splits;
    splits = (a.all_heads + a.head_step - 1) / a.head_step;
    const dim3 grid((unsigned)wgs, (unsigned)splits);
    // Where a load of a head's lanes takes whole cache lines, they pass the caches by; other heads' lines are met twice (4 tiles of 75,600 tokens, 5 + 5 heads
    // x 96: past the caches a seventh more).
    const bool half = p.layout == SG_ROTARY_HALF, lines = p.head_dim % 128 == 0, full = a.turned == p.head_dim && a.n_vec == 2 * a.lanes;
#define SG_ROTARY(T, H, L, F) rotary_kernel<T, H, L, F><<<grid, 256, lds, s>>>(a, tab)
#define SG_ROTARY_FULL(T, H, L)             \
  do {                                      \
    if (full) SG_ROTARY(T, H, L, true);     \
    else SG_ROTARY(T, H, L, false);         \
  } while (0)
    if (p.dtype == SG_F32) {
      if (half) SG_ROTARY_FULL(float, true, false);
      else SG_ROTARY_FULL(float, false, false);
    } else if (lines) {
      if (half) SG_ROTARY_FULL(uint16_t, true, true);
      else SG_ROTARY_FULL(uint16_t, false, true);
    } else {
      if (half) SG_ROTARY_FULL(uint16_t, true, false);
      else SG_ROTARY_FULL(uint16_t, false, false);
    }
#undef SG_ROTARY_FULL
#undef SG_ROTARY
    SG_HIP_TRY(hipGetLastError());
  }
  return SG_OK;
}

}  // namespace sg
