// attend_masked.cuh - what the kernels of attention with masks share: tiles of rows, the tokens that they run
// through, and which of these a row sees.
#pragma once

#include <math_constants.h>

#include "convert.cuh"
#include "serve.h"

namespace emoe {

// The n lowest bits.
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? 0xffffffffu : (1u << max(n, 0)) - 1; }

// Rows of a KV head in a sequence: its query tokens times the query heads of the KV head, a token's rows one
// after the other.  A tile is up to R of them.
struct RowTile {
  int seq, row0, rows;   // rows 0: there is no such tile
  int first, count;      // the sequence's query tokens: the first one, and how many are computed
  int context;           // tokens before the query tokens (negative: more query tokens than tokens)
  int length;            // tokens
};

// Packed: sequence s has the tiles from floor(q_start[s] * group / R) + s on, which leaves it enough of them and can
// be said without a sum over the sequences before.  The whole warp looks for the sequence, 32 probes at a time.
template <int R>
__device__ __forceinline__ RowTile row_tile(const MaskedArgs &a, int tiles_a_seq, int tile) {
  RowTile t;
  int local;
  const auto start_of = [&](int s) { return max(0, min(a.q_start[s], a.n_tokens)); };
  if (tiles_a_seq) {
    t.seq = tile / tiles_a_seq;
    local = tile - t.seq * tiles_a_seq;
  } else {
    const auto tile_of = [&](int s) { return (int)((int64_t)start_of(s) * a.group / R) + s; };
    int lo = 0, hi = a.n_seqs;   // the last sequence whose first tile is not behind this one
    while (hi - lo > 1) {
      const int step = (hi - lo + 31) / 32, s = lo + (int)(threadIdx.x & 31) * step;
      const int found = __popc(__ballot_sync(0xffffffffu, s < hi && tile_of(s) <= tile));
      lo += max(0, found - 1) * step;
      hi = min(hi, lo + step);
    }
    t.seq = lo;
    local = tile - tile_of(lo);
  }
  t.first = start_of(t.seq);
  const int all = max(0, start_of(t.seq + 1) - t.first);
  t.count = min(all, a.max_q);
  t.length = max(0, min(a.own_lens[t.seq], a.max_blocks * a.c.block_tokens));
  t.context = t.length - all;
  t.row0 = local * R;
  t.rows = local < 0 ? 0 : max(0, min(R, t.count * a.group - t.row0));
  if (all > a.max_q && local == 0 && a.c.status) *a.c.status = EMOE_ERR_TOO_LARGE;
  return t;
}

// Blocks start in the order of their numbers: where not all of them run at once, sequences with many tokens come first, so that none
// of those is left for the end.  The tile whose sequence has the rank that `tile` asks for; one thread a sequence, all of the block: more
// sequences than a row kernel's block has threads stay as they come.  That costs the less the more there are: of trees of 5 to 13 nodes on 13 to
// 2750 tokens, 16 heads, e4m3, 129 took 267 us as they came and 239 the longest first, 256 490 and 460, 512 941 and 930.
constexpr int kMostRanked = 128;
__device__ __forceinline__ int ranked_tile(const MaskedArgs &a, int tiles_a_seq, int tile) {
  __shared__ int s_tokens[kMostRanked], s_seq;
  const int t = threadIdx.x, wanted = tile / tiles_a_seq;
  int mine = 0;
  if (t < a.n_seqs) {
    mine = max(0, min(a.own_lens[t], a.max_blocks * a.c.block_tokens));
    if (!a.mask) mine = (int)min((uint32_t)mine, (uint32_t)a.window + (uint32_t)a.sinks);   // (the two come to 2^31 where neither has a limit)
    s_tokens[t] = mine;
  }
  __syncthreads();
  int rank = 0;
  for (int i = 0; i < a.n_seqs; ++i) rank += s_tokens[i] > mine || (s_tokens[i] == mine && i < t);
  if (t < a.n_seqs && rank == wanted) s_seq = t;
  __syncthreads();
  return s_seq * tiles_a_seq + tile - wanted * tiles_a_seq;
}

// The tokens that some row of a tile may see, as one run: the first tokens, then those from `low` on.
struct Run {
  int count, sinks, low;
  int seen;   // those before are seen by all rows that come after them (the first tokens and what joins on)
  __device__ __forceinline__ int token(int u) const { return u < sinks ? u : u - sinks + low; }
};
__device__ __forceinline__ Run run_of(const MaskedArgs &a, const RowTile &t) {
  Run r{t.length, 0, 0, 0};
  if (a.mask) return r;
  const int earliest = t.context + t.row0 / a.group, latest = t.context + (t.row0 + t.rows - 1) / a.group;
  r.low = max(0, earliest - a.window + 1);
  r.sinks = min(a.sinks, r.low);
  r.seen = r.sinks + max(0, a.sinks - r.low);
  r.count = r.sinks + max(0, latest + 1 - r.low);
  return r;
}

// What one row of a tile sees of its run: a word of 32 tokens from u on.  (Tokens that the run does not have may be among them.)
struct Sight {
  int begin, end;        // window: the last tokens up to the row's own
  int64_t mask;          // tree: word of the row's mask
  __device__ __forceinline__ Sight(const MaskedArgs &a, const RowTile &t, const Run &r, int row) {
    const int token = (t.row0 + row) / a.group, place = t.context + token;
    begin = max(place - a.window + 1, r.low) - r.low + r.sinks;
    end = place + 1 - r.low + r.sinks;
    if (place < 0) end = 0;
    mask = (int64_t)(t.first + token) * a.mask_words;
  }
  __device__ __forceinline__ uint32_t word(const MaskedArgs &a, const RowTile &t, const Run &r, int u) const {
    if (!a.mask) return low_bits(end - u) & (low_bits(r.seen - u) | ~low_bits(begin - u));
    const int node = u - t.context;
    if (node <= -32) return 0xffffffffu;
    const int i = max(node, 0) >> 5;
    const uint32_t w0 = i < a.mask_words ? a.mask[mask + i] : 0;
    if (node < 0) return w0 << -node | low_bits(-node);
    const uint32_t w1 = i + 1 < a.mask_words ? a.mask[mask + i + 1] : 0;
    return __funnelshift_r(w0, w1, node & 31);
  }
};

// A token's column of the table and its place in the block there.  (The quotient by the floor of (2^32 - 1) / block_tokens is one too small
// at most: tokens are below 2^30.)
struct TokenPlace { uint32_t column, off; };
__device__ __forceinline__ TokenPlace place_of_token(const MaskedArgs &a, int token) {
  const uint32_t bt = (uint32_t)a.c.block_tokens;
  uint32_t q = __umulhi((uint32_t)token, a.per_token), off = (uint32_t)token - q * bt;
  if (off >= bt) ++q, off -= bt;
  return {q, off};
}
// Vector index of place `off` of `block`; -1 (and the status word) if that is outside the pool.
// (The table is read apart from this and well before: a branch on what it says waits for it.)
__device__ __forceinline__ int64_t masked_vector(const MaskedArgs &a, int block, uint32_t off, int head) {
  if (block < 0 || block >= a.num_blocks) {
    if (a.c.status) *a.c.status = EMOE_ERR_BLOCK_TABLE;
    return -1;
  }
  return a.c.head_major ? ((int64_t)block * a.c.n_heads + head) * a.c.block_tokens + off
                        : ((int64_t)block * a.c.block_tokens + off) * a.c.n_heads + head;
}

// Element offsets of a tile's row in q / out and in lse.
__device__ __forceinline__ int64_t row_at(const MaskedArgs &a, const RowTile &t, int head, int row, int64_t stride) {
  const int r = t.row0 + row, token = r / a.group;
  return (int64_t)(t.first + token) * stride + (int64_t)(head * a.group + r - token * a.group) * a.c.head_dim;
}
__device__ __forceinline__ void write_lse(const MaskedArgs &a, const RowTile &t, int head, int row, float m, float l) {
  const int r = t.row0 + row, token = r / a.group;
  if (a.lse)
    a.lse[(int64_t)(t.first + token) * a.n_q_heads + head * a.group + r - token * a.group] =
        l > 0.f || l != l ? (m + log2f(l)) * CUDART_LN2_F : -CUDART_INF_F;
}

// Whether a word of two 16-bit elements, or of four e4m3 codes, has one that is infinite or not a number.
template <typename T, bool FP8> __device__ __forceinline__ bool not_finite(uint32_t w) {
  if constexpr (FP8) return __vcmpeq4(w & 0x7f7f7f7fu, 0x7f7f7f7fu) != 0;
  constexpr uint32_t kTop = __is_same(T, __half) ? 0x7c007c00u : 0x7f807f80u;
  return __vcmpeq2(w & kTop, kTop) != 0;
}

// The end of a block of a row kernel, all threads: the parts of its WARPS warps - s_m, s_l, and in `joined` [warp][row][HD + 4] -
// become one, and the rows go out, or, where the tile's tokens are split, to the workspace for the join kernel.
template <typename IO, int HD, int R, int WARPS>
__device__ __forceinline__ void finish_rows(const MaskedArgs &a, const RowTile &tile, int head, int unit, int split, const float *joined,
                                            const float (&s_m)[WARPS][R], const float (&s_l)[WARPS][R]) {
  constexpr int kLanes = HD / 4 < 32 ? HD / 4 : 32;   // of a row, 4 columns each at a time
  const bool last = a.splits == 1;
  for (int row = threadIdx.x / kLanes; row < tile.rows; row += WARPS * 32 / kLanes) {
    float m = -CUDART_INF_F, l = 0.f, w[WARPS];
#pragma unroll
    for (int i = 0; i < WARPS; ++i) m = fmaxf(m, s_m[i][row]);
#pragma unroll
    for (int i = 0; i < WARPS; ++i) {
      w[i] = m == -CUDART_INF_F ? 0.f : exp2_fast(s_m[i][row] - m);
      l += w[i] * s_l[i][row];
      if (s_l[i][row] != s_l[i][row]) l = w[i] = CUDART_NAN_F;   // a maximum does not carry a NaN: the sum does
    }
    const int64_t part = ((int64_t)unit * a.splits + split) * R + row;
    const float by = last ? (l > 0.f || l != l ? 1.f / l : 0.f) : 1.f;
    IO *const out = (IO *)a.out + row_at(a, tile, head, row, a.out_stride);
    for (int col = threadIdx.x % kLanes * 4; col < HD; col += 128) {
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < WARPS; ++i) {
        const float4 y = *(const float4 *)&joined[(i * R + row) * (HD + 4) + col];
        x.x += w[i] * y.x;
        x.y += w[i] * y.y;
        x.z += w[i] * y.z;
        x.w += w[i] * y.w;
      }
      if (last)
        *(uint2 *)(out + col) = make_uint2(Pair<IO>::pack(x.x * by, x.y * by), Pair<IO>::pack(x.z * by, x.w * by));
      else
        *(float4 *)(a.part_o + part * HD + col) = x;
    }
    if (threadIdx.x % kLanes == 0) {
      if (last) write_lse(a, tile, head, row, m, l);
      else a.part_ml[part] = make_float2(m, l);
    }
  }
}

}  // namespace emoe
