// attend.cu - decode attention over a paged KV cache, a shared prefix computed once for the batch.
//
// o = sum_j p_j v_j / sum_j p_j with p_j = 2^(s_j - m), s_j = scale * log2(e) * q.k_j and m the
// largest s_j, in one pass over the tokens: each part of the work keeps its own m, sum and
// unnormalised o in 32 bits, and parts are joined by o = sum 2^(m_i - m) o_i.
//
// Work is cut into items (row tile, KV head, token range).  The rows of a KV head are its query
// heads times the query tokens - of the whole batch for the prefix, which is thereby read once, and
// of one sequence for that sequence's own tokens.  When there are few rows the token axis is split
// until the machine is full; a second kernel joins the splits.
#include <algorithm>
#include <cmath>

#include "attend_item.cuh"

namespace emoe {
namespace {

constexpr int kWarps = 4, kStages = 2;
// Tokens of one warp's step: the same bytes for both element sizes.
template <bool FP8> constexpr int kGroupOf = FP8 ? 32 : 16;

struct Item {
  bool prefix;
  int seq, head, row0, rows, slot;  // rows of this tile, first row inside the sequence or batch
  int t0, t1;                       // tokens
};

__device__ __forceinline__ Item item_of(const AttendArgs &a, uint32_t i) {
  Item it;
  const uint32_t heads = a.c.n_heads;
  if (i < a.prefix_items) {
    it.prefix = true;
    it.seq = 0;
    const uint32_t split = i % a.prefix_splits, j = i / a.prefix_splits;
    it.head = j % heads;
    it.row0 = (j / heads) * 16;
    it.rows = min(16, a.n_seqs * a.seq_rows - it.row0);
    it.slot = split;
    it.t0 = split * a.prefix_chunk;
    it.t1 = min(a.prefix_len, it.t0 + a.prefix_chunk);
  } else {
    i -= a.prefix_items;
    it.prefix = false;
    const uint32_t split = i % a.own_splits;
    uint32_t j = i / a.own_splits;
    it.head = j % heads;
    j /= heads;
    const uint32_t tiles = (a.seq_rows + 15) / 16;
    it.row0 = (j % tiles) * 16;
    it.seq = j / tiles;
    it.rows = min(16, a.seq_rows - it.row0);
    it.slot = a.prefix_splits + split;
    it.t0 = split * a.own_chunk;
    it.t1 = min(own_length(a, it.seq), it.t0 + a.own_chunk);
  }
  return it;
}

// 16-byte piece c of row r of a tile with CH pieces a row: rotated so that eight rows' equal pieces
// lie in different banks.
template <int CH> __device__ __forceinline__ int swizzled(int r, int c) {
  if constexpr (CH >= 8) return r * CH + (c ^ (r & 7));
  else if constexpr (CH == 4) return r * CH + (c ^ ((r >> 1) & 3));
  else return r * CH + (c ^ ((r >> 2) & 1));
}

__device__ __forceinline__ void write_row(const AttendArgs &a, int64_t row, int hd, float m, float l) {
  if (a.lse) a.lse[row] = l > 0.f || l != l ? (m + log2f(l)) * CUDART_LN2_F : -CUDART_INF_F;
}

// One warp's step covers 16 tokens (32 of an e4m3 cache): K and V rows come through a ring of its own in shared memory
// (no block barrier in the loop), scores and products on the tensor cores with the 16 rows of the
// item as the m side (rows that do not exist are zero), running maximum and sum in registers.  The
// four warps take every fourth group of tokens and are joined at the end.  Bound by the reads of K
// and V: 2 stages x 4 warps x 8 KB and three blocks an SM have 192 KB of ring there (head_dim 128).  Measured, 32 sequences
// of 3000 tokens, 16 heads: bf16 132 us, 6.0 TB/s; e4m3 132 us, 3.0 TB/s - there no pipe is full (issue slots 51%, integer
// pipe 42%, DRAM 37%): it is the chain of a step, with three warps a scheduler.  Short calls are bound by an item's start and end (48 x 625 tokens, 4 heads: 2.3 TB/s).
template <typename IO, int HD, bool FP8>
__global__ void __launch_bounds__(kWarps * 32, HD < 256 ? 3 : 1) attend_rows_kernel(const __grid_constant__ AttendArgs a) {
  using T = typename Operand<IO, FP8>::type;
  constexpr int kGroup = kGroupOf<FP8>;
  constexpr int ES = FP8 ? 1 : 2, CH = HD * ES / 16, kTile = kGroup * HD * ES, kStage = 2 * kTile;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint16_t s_scale[kWarps][kStages][kGroup];
  __shared__ uint32_t s_valid[kWarps][kStages];
  __shared__ float s_m[kWarps][16], s_l[kWarps][16];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const Item it = item_of(a, blockIdx.x);
  const int slots = a.prefix_splits + a.own_splits;

  let_next_start();
  if (it.t0 >= it.t1 && slots > 1) {   // nothing here: say so to the joining kernel
    wait_for_previous();
    if (threadIdx.x < it.rows)
      a.part_ml[output_row(a, it.seq, it.head, it.row0 + threadIdx.x) * slots + it.slot] = make_float2(-CUDART_INF_F, 0.f);
    return;
  }

  const int groups = it.t1 > it.t0 ? (it.t1 - it.t0 + kGroup - 1) / kGroup : 0;
  const int steps = groups > warp ? (groups - warp + kWarps - 1) / kWarps : 0;
  const int32_t *table = it.prefix ? a.prefix_table : a.block_table + (int64_t)it.seq * a.max_blocks;
  uint8_t *const ring = smem + warp * (kStages * kStage);
  const uint32_t ring_at = shared_address(ring);

  // this lane's token of step i (lanes beyond a group's tokens repeat them), -1 if there is none; its block; its vector index
  auto token_of = [&](int i) {
    const int t = it.t0 + (warp + kWarps * i) * kGroup + (lane & (kGroup - 1));
    return i >= steps || t >= it.t1 ? -1 : t;
  };
  auto block_of = [&](int i) {
    const int t = token_of(i);
    return t < 0 ? 0 : table[(uint32_t)t / (uint32_t)a.c.block_tokens];
  };
  auto vector_of = [&](int i, int block) {
    const int t = token_of(i);
    return t < 0 ? (int64_t)-1 : token_vector(a, block, t, it.head);
  };
  uint32_t held_scale = 0, held_valid = 0;
  auto issue = [&](int i, int64_t vec) {   // starts the copies of step i
    const uint32_t at = ring_at + (i % kStages) * kStage;
    held_valid = __ballot_sync(0xffffffffu, vec >= 0);
    if constexpr (FP8) held_scale = vec >= 0 ? a.c.k_scale[vec] | (uint32_t)a.c.v_scale[vec] << 8 : 0x007f;   // a token that is not there has no part in the largest scale of v
#pragma unroll
    for (int j = 0; j < (kGroup * CH + 31) / 32; ++j) {
      const int id = j * 32 + lane, row = id / CH, ch = id % CH;
      const int64_t v = __shfl_sync(0xffffffffu, vec, row & (kGroup - 1));
      if (kGroup * CH % 32 == 0 || id < kGroup * CH) {
        const int64_t src = v < 0 ? 0 : v * (HD * ES) + ch * 16;
        const uint32_t dst = at + swizzled<CH>(row, ch) * 16;
        copy_async_16(dst, a.c.k + src, v < 0 ? 0 : 16);
        copy_async_16(dst + kTile, a.c.v + src, v < 0 ? 0 : 16);
      }
    }
  };
  auto keep = [&](int i) {   // what the issue of step i found, for its use
    if (FP8) s_scale[warp][i % kStages][lane] = (uint16_t)held_scale;
    if (lane == 0) s_valid[warp][i % kStages] = held_valid;
  };

  // e4m3: the largest scale byte of v so far that a row (g, g + 8) sees, whose scale its o is relative to
  uint32_t v_ref[2] = {0, 0};
  constexpr int kTileGroup = FP8 ? 4 : 2;   // column tiles that are read together
  float o[HD / 8 / kTileGroup][kTileGroup][4] = {}, m[2] = {-CUDART_INF_F, -CUDART_INF_F}, l[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) {
    if (i < steps) {
      issue(i, vector_of(i, block_of(i)));
      keep(i);
    }
    copy_async_commit();
  }
  int block = block_of(kStages - 1);   // the table is read a step ahead

  // query rows g and g + 8 of the tile as matrix operands, from global memory
  uint32_t q[HD / 16][4];
  int limit[2];      // tokens that the row sees
  float by_row[2];   // scores to log2 weights
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int row = g + 8 * half;
    const bool real = row < it.rows;
    const int r = real ? it.row0 + row : 0;
    const int token = r / a.group;
    const IO *src = (const IO *)a.q + ((int64_t)it.seq * a.q_len + token) * a.q_stride + (it.head * a.group + r - token * a.group) * HD;
    limit[half] = !real ? 0 : it.prefix ? it.t1 : own_length(a, it.seq) - a.q_len + token + 1;
    by_row[half] = a.scale_log2;
#pragma unroll
    for (int ks = 0; ks < HD / 16; ++ks) {
      if constexpr (!FP8) {
        const uint32_t *p = (const uint32_t *)(src + ks * 16 + 2 * c);
        q[ks][half] = real ? p[0] : 0;
        q[ks][2 + half] = real ? p[4] : 0;
      } else {   // four neighbouring elements, as the codes of a word come
        const uint2 w = real ? *(const uint2 *)(src + (ks >> 1) * 32 + c * 8 + (ks & 1) * 4) : make_uint2(0, 0);
        q[ks][half] = w.x;
        q[ks][2 + half] = w.y;
      }
    }
    if constexpr (FP8) {
      uint32_t top = 0;
#pragma unroll
      for (int ks = 0; ks < HD / 16; ++ks)
#pragma unroll
        for (int k = 0; k < 4; k += 2) {
          const float2 f = Pair<IO>::unpack(q[ks][half + k]);
          top = max(top, max(__float_as_uint(f.x) & 0x7fffffffu, __float_as_uint(f.y) & 0x7fffffffu));
        }
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const float by = query_scale(top);
      by_row[half] = a.scale_log2 / by;
#pragma unroll
      for (int ks = 0; ks < HD / 16; ++ks)
#pragma unroll
        for (int k = 0; k < 4; k += 2) {
          const float2 f = Pair<IO>::unpack(q[ks][half + k]);
          q[ks][half + k] = Pair<T>::pack(f.x * by, f.y * by);
        }
    }
  }

  for (int i = 0; i < steps; ++i) {
    const int ahead = i + kStages - 1;
    if (ahead < steps) issue(ahead, vector_of(ahead, block));
    copy_async_commit();
    block = block_of(ahead + 1);
    copy_async_wait<kStages - 1>();
    __syncwarp();

    const uint32_t k_at = ring_at + (i % kStages) * kStage, v_at = k_at + kTile;
    const uint32_t valid = s_valid[warp][i % kStages];
    constexpr int kN = kGroup / 8, kP = kGroup / 16;   // column tiles of the scores, k steps of the second product
    float s[kN][4] = {};
    if constexpr (!FP8) {
#pragma unroll
      for (int ks = 0; ks < HD / 16; ++ks) {
        uint32_t b[4];
        ldmatrix_x4(b, k_at + swizzled<CH>((lane >> 4) * 8 + (lane & 7), ks * 2 + ((lane >> 3) & 1)) * 16);
        mma_16816<T>(s[0], q[ks], b[0], b[1]);
        mma_16816<T>(s[1], q[ks], b[2], b[3]);
      }
    } else {
#pragma unroll
      for (int kb = 0; kb < HD / 32; ++kb)
#pragma unroll
        for (int j = 0; j < kN; ++j) {
          const uint2 w = *(const uint2 *)(ring + (i % kStages) * kStage + swizzled<CH>(j * 8 + g, kb * 2 + (c >> 1)) * 16 + (c & 1) * 8);
          uint32_t b[4];
          codes_to_half(b[0], b[1], w.x);
          codes_to_half(b[2], b[3], w.y);
          mma_16816<T>(s[j], q[2 * kb], b[0], b[1]);
          mma_16816<T>(s[j], q[2 * kb + 1], b[2], b[3]);
        }
    }

    const int base = it.t0 + (warp + kWarps * i) * kGroup;
    // Query tokens of one sequence see different ends: in a ragged step some real row does not see all of its tokens.
    const int end = min(base + kGroup, it.t1);
    const auto is_ragged = [&]() {
      return a.q_len > 1 && __any_sync(0xffffffffu, (g < it.rows && limit[0] < end) || (g + 8 < it.rows && limit[1] < end));
    };
    const bool ragged_scales = FP8 && is_ragged();
    float k_by[kN][2], v_by[kN][2], v_raise[2] = {1.f, 1.f};
    if constexpr (FP8) {   // scales are powers of two; 255 is not a number and not counted in the largest of v so far
      uint32_t largest = v_ref[0];
      if (!ragged_scales) {   // no ragged step has been yet: all rows have the same largest scale
        const uint32_t mine = s_scale[warp][i % kStages][lane] >> 8;
        largest = max(v_ref[0], __reduce_max_sync(0xffffffffu, mine == 255 ? 0 : mine));
        v_raise[0] = v_raise[1] = v_relative(v_ref[0], largest);
        v_ref[0] = v_ref[1] = largest;
      }
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        const uint32_t two = *(const uint32_t *)&s_scale[warp][i % kStages][j * 8 + 2 * c];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          k_by[j][e] = scale_of(two >> (16 * e) & 255);
          v_by[j][e] = v_relative(two >> (16 * e + 8) & 255, largest);
        }
      }
      if (ragged_scales) {   // what a row does not see has no part in its largest scale: weights are scaled row by row below
#pragma unroll
        for (int j = 0; j < kN; ++j) v_by[j][0] = v_by[j][1] = 1.f;
      }
    }
    float top[2] = {m[0], m[1]};
#pragma unroll
    for (int j = 0; j < kN; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int t = j * 8 + 2 * c + e;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          float &x = s[j][2 * half + e];
          x = ((valid >> t) & 1) && base + t < limit[half] ? x * (FP8 ? k_by[j][e] * by_row[half] : by_row[half]) : -CUDART_INF_F;
          top[half] = fmaxf(top[half], x);
        }
      }
    float alpha[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      top[half] = fmaxf(top[half], __shfl_xor_sync(0xffffffffu, top[half], 1));
      top[half] = fmaxf(top[half], __shfl_xor_sync(0xffffffffu, top[half], 2));
      alpha[half] = exp2_fast(m[half] - (top[half] == -CUDART_INF_F ? 0.f : top[half]));
      const float safe = top[half] == -CUDART_INF_F ? 0.f : top[half] - kWeightLift<T>;
      m[half] = top[half];
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < kN; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float &x = s[j][2 * half + e];
          x = exp2_fast(x - safe);
          sum += x;
          // (what no row sees has a finite scale here; a NaN scale shows even where the weight has come to zero)
          if constexpr (FP8) x *= v_by[j][e];
        }
      l[half] = l[half] * alpha[half] + sum;
    }
    if constexpr (FP8)
      if (__builtin_expect(ragged_scales, 0)) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const auto scale_byte = [&](int t) { return (uint32_t)s_scale[warp][i % kStages][t] >> 8; };
          uint32_t largest = v_ref[half];
          const int seen = min(limit[half] - base, kGroup);
          for (int t = 0; t < seen; ++t) largest = max(largest, scale_byte(t) == 255 ? 0 : scale_byte(t));
          v_raise[half] = v_relative(v_ref[half], largest);
          v_ref[half] = largest;
#pragma unroll
          for (int j = 0; j < kN; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int t = j * 8 + 2 * c + e;
              if (t < seen) s[j][2 * half + e] *= v_relative(scale_byte(t), largest);
            }
        }
      }
    alpha[0] *= v_raise[0];
    alpha[1] *= v_raise[1];
    if (!__all_sync(0xffffffffu, alpha[0] == 1.f && alpha[1] == 1.f)) {
#pragma unroll
      for (int n = 0; n < HD / 8; ++n) {
        float(&d)[4] = o[n / kTileGroup][n % kTileGroup];
        d[0] *= alpha[0];
        d[1] *= alpha[0];
        d[2] *= alpha[1];
        d[3] *= alpha[1];
      }
    }
    // weights rounded to T, once, as the second product's operand: the result's own rounding is as large
    uint32_t p[kP][4];
#pragma unroll
    for (int k = 0; k < kP; ++k) {
      p[k][0] = Pair<T>::pack(s[2 * k][0], s[2 * k][1]);
      p[k][1] = Pair<T>::pack(s[2 * k][2], s[2 * k][3]);
      p[k][2] = Pair<T>::pack(s[2 * k + 1][0], s[2 * k + 1][1]);
      p[k][3] = Pair<T>::pack(s[2 * k + 1][2], s[2 * k + 1][3]);
    }
    // Products with the n-th 16 (e4m3: 32) columns of v, pieces read with ldmatrix: two column tiles of an e4m3
    // cache share 16-bit elements (two neighbouring columns) and are parted here.
    constexpr int kTiles = FP8 ? 4 : 2, kReads = HD / 8 / kTiles;   // column tiles a read, reads
    auto products = [&](float (&d)[kTiles][4], int n) {
#pragma unroll
      for (int k = 0; k < kP; ++k) {
        uint32_t b[4];
        ldmatrix_x4_trans(b, v_at + swizzled<CH>(16 * k + (lane & 15), 2 * n + (lane >> 4)) * 16);
        if constexpr (FP8) {
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            uint32_t x[4];   // column, column + 1 of tokens 2c, 2c + 1; of tokens 2c + 8, 2c + 9
            codes_to_half(x[0], x[1], __byte_perm(b[2 * t], 0, 0x3120));
            codes_to_half(x[2], x[3], __byte_perm(b[2 * t + 1], 0, 0x3120));
            mma_16816<T>(d[2 * t], p[k], x[0], x[2]);
            mma_16816<T>(d[2 * t + 1], p[k], x[1], x[3]);
          }
        } else {
          mma_16816<T>(d[0], p[k], b[0], b[1]);
          mma_16816<T>(d[1], p[k], b[2], b[3]);
        }
      }
    };
    // A value that some rows must not see may be infinite or not a number, and a weight of zero does not
    // silence it: a ragged step is done end by end, each row taking the pass of its own, with the values
    // behind that end cleared.
    if (FP8 ? ragged_scales : is_ragged()) {
      for (int stop = end; stop > base; --stop) {
        const bool now0 = min(limit[0], end) == stop, now1 = min(limit[1], end) == stop;
        if (__any_sync(0xffffffffu, now0 || now1)) {
#pragma unroll
          for (int n = 0; n < kReads; ++n) {
            float part[kTiles][4] = {};
            products(part, n);
#pragma unroll
            for (int k = 0; k < kTiles; ++k)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (e < 2 ? now0 : now1) o[n][k][e] += part[k][e];
          }
        }
        __syncwarp();
        for (int ch = lane; ch < CH; ch += 32)
          *(uint4 *)(ring + (i % kStages) * kStage + kTile + swizzled<CH>(stop - 1 - base, ch) * 16) = make_uint4(0, 0, 0, 0);
        __syncwarp();
      }
    } else {
#pragma unroll
      for (int n = 0; n < kReads; ++n) products(o[n], n);
    }
    if (ahead < steps) keep(ahead);
    __syncwarp();
  }
  copy_async_wait<0>();

  // the four warps' parts become one
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    l[half] += __shfl_xor_sync(0xffffffffu, l[half], 1);
    l[half] += __shfl_xor_sync(0xffffffffu, l[half], 2);
    if (c == 0) {
      s_m[warp][g + 8 * half] = m[half] - kWeightLift<T>;
      s_l[warp][g + 8 * half] = l[half];
    }
  }
  __syncthreads();
  constexpr int kPitch = HD + 4;
  float *const joined = (float *)smem;
#pragma unroll
  for (int n = 0; n < HD / 8; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int col = FP8 ? (n >> 1) * 16 + 4 * c + (n & 1) + 2 * (e & 1) : n * 8 + 2 * c + (e & 1);
      joined[(warp * 16 + g + 8 * (e >> 1)) * kPitch + col] = o[n / kTileGroup][n % kTileGroup][e] * (FP8 ? scale_of(v_ref[e >> 1]) : 1.f);
    }
  __syncthreads();
  // the prefix's own kernel may still be running: the joining one waits for this one alone
  wait_for_previous();
  const int row = threadIdx.x >> 3;
  if (row >= it.rows) return;
  float mm = -CUDART_INF_F, ll = 0.f, w[kWarps];
#pragma unroll
  for (int i = 0; i < kWarps; ++i) mm = fmaxf(mm, s_m[i][row]);
#pragma unroll
  for (int i = 0; i < kWarps; ++i) {
    w[i] = mm == -CUDART_INF_F ? 0.f : exp2_fast(s_m[i][row] - mm);
    ll += w[i] * s_l[i][row];
    if (s_l[i][row] != s_l[i][row]) ll = w[i] = CUDART_NAN_F;   // a maximum does not carry a NaN: the sum does
  }
  const int64_t orow = output_row(a, it.seq, it.head, it.row0 + row);
  const bool last = slots == 1;
  const float by = last ? (ll > 0.f || ll != ll ? 1.f / ll : 0.f) : 1.f;
  for (int col = (threadIdx.x & 7) * 4; col < HD; col += 32) {
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      const float4 y = *(const float4 *)&joined[(i * 16 + row) * kPitch + col];
      x.x += w[i] * y.x;
      x.y += w[i] * y.y;
      x.z += w[i] * y.z;
      x.w += w[i] * y.w;
    }
    if (last) {
      const int64_t token = orow / a.n_q_heads;
      *(uint2 *)((IO *)a.out + token * a.out_stride + (orow - token * a.n_q_heads) * HD + col) =
          make_uint2(Pair<IO>::pack(x.x * by, x.y * by), Pair<IO>::pack(x.z * by, x.w * by));
    } else {
      *(float4 *)(a.part_o + (orow * slots + it.slot) * HD + col) = x;
    }
  }
  if ((threadIdx.x & 7) == 0) {
    if (last) write_row(a, orow, HD, mm, ll);
    else a.part_ml[orow * slots + it.slot] = make_float2(mm, ll);
  }
}

// Joins the splits of an output row: a block of four warps a row, each with every fourth group of four splits (read
// without waiting for one another), joined in the order of the warps.  Bound by the latency of its reads: about 4 us behind the
// other kernels for 8 rows of many splits, 8 for 1536 rows of 10 (the grid starts while they end).
constexpr int kJoinWarps = 4;
template <typename T, int HD>
__global__ void __launch_bounds__(kJoinWarps * 32) attend_join_kernel(const __grid_constant__ AttendArgs a) {
  constexpr int N = HD / 32;
  __shared__ float s_x[kJoinWarps][HD], s_l[kJoinWarps];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t row = blockIdx.x;
  const int slots = a.prefix_splits + a.own_splits;
  const float2 *const ml = a.part_ml + row * slots;
  const float *const parts = a.part_o + row * slots * HD + lane * N;
  wait_for_previous();
  float m = -CUDART_INF_F;
  for (int i = lane; i < slots; i += 32) m = fmaxf(m, ml[i].x);
#pragma unroll
  for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
  float l = 0.f, x[N] = {};
  for (int first = warp * 4; first < slots; first += kJoinWarps * 4) {
    float w[4], y[4][N];
    bool there[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const float2 p = first + u < slots ? ml[first + u] : make_float2(-CUDART_INF_F, 0.f);
      // an empty part (sum 0) does not count: nothing was written there
      there[u] = p.y != 0.f;
      w[u] = p.y != p.y ? CUDART_NAN_F : exp2_fast(p.x - m);
      l += there[u] ? w[u] * p.y : 0.f;
      const float *const src = parts + (int64_t)min(first + u, slots - 1) * HD;
      if constexpr (N % 4 == 0) {
#pragma unroll
        for (int j = 0; j < N; j += 4) *(float4 *)&y[u][j] = *(const float4 *)(src + j);
      } else if constexpr (N == 2) {
        *(float2 *)y[u] = *(const float2 *)src;
      } else {
        y[u][0] = src[0];
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] += there[u] ? w[u] * y[u][j] : 0.f;
  }
#pragma unroll
  for (int j = 0; j < N; ++j) s_x[warp][lane * N + j] = x[j];
  if (lane == 0) s_l[warp] = l;
  __syncthreads();
  if (threadIdx.x * 2 >= HD) return;
  l = 0.f;
  float u = 0.f, v = 0.f;
#pragma unroll
  for (int w = 0; w < kJoinWarps; ++w) {
    l += s_l[w];
    u += s_x[w][threadIdx.x * 2];
    v += s_x[w][threadIdx.x * 2 + 1];
  }
  const float by = l == 0.f ? 0.f : 1.f / l;
  const int64_t token = row / a.n_q_heads;
  *(uint32_t *)((T *)a.out + token * a.out_stride + (row - token * a.n_q_heads) * HD + threadIdx.x * 2) = Pair<T>::pack(u * by, v * by);
  if (threadIdx.x == 0) write_row(a, row, HD, m, l);
}

template <typename K>
cudaError_t launch_after(K kernel, dim3 grid, int threads, size_t smem, cudaStream_t st, bool early, const AttendArgs &a) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = early ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <typename T, int HD, bool FP8>
cudaError_t launch_rows(const AttendArgs &a, cudaStream_t st) {
  constexpr size_t ring = (size_t)kWarps * kStages * 2 * kGroupOf<FP8> * HD * (FP8 ? 1 : 2);
  constexpr size_t join = (size_t)kWarps * 16 * (HD + 4) * 4;
  constexpr size_t smem = ring > join ? ring : join;
  cudaError_t e = allow_shared<attend_rows_kernel<T, HD, FP8>>();
  if (e != cudaSuccess) return e;
  AttendArgs rest = a;
  if (a.tensor) rest.prefix_items = 0;
  if (rest.prefix_items + rest.own_items) {
    e = launch_after(attend_rows_kernel<T, HD, FP8>, dim3(rest.prefix_items + rest.own_items), kWarps * 32, smem, st, a.tensor, rest);
    if (e != cudaSuccess) return e;
  }
  if (!a.tensor && a.prefix_splits + a.own_splits == 1) return e;
  const int64_t rows = (int64_t)a.n_seqs * a.q_len * a.n_q_heads;
  return launch_after(attend_join_kernel<T, HD>, dim3((unsigned)rows), kJoinWarps * 32, 0, st, true, a);
}

template <typename T, bool FP8>
cudaError_t by_head_dim(const AttendArgs &a, cudaStream_t st) {
  switch (a.c.head_dim) {
    case 32: return launch_rows<T, 32, FP8>(a, st);
    case 64: return launch_rows<T, 64, FP8>(a, st);
    case 128: return launch_rows<T, 128, FP8>(a, st);
    case 256: return launch_rows<T, 256, FP8>(a, st);
  }
  return cudaErrorInvalidValue;
}

}  // namespace

namespace {

constexpr int kMostSplits = 64;
// Whether the prefix goes to the tensor core kernel.  It starts later and ends earlier than the other one and takes 256 rows
// at once.  They meet at about 2^17 row tiles
// (of 16 rows) x tokens.  The whole call, this kernel and the other one, 4 KV heads, head_dim 128:
//   64 rows, 2000 tokens (2^15): bf16 21.5 and 15.4 us, e4m3 25.6 and 17.4
//   128 rows, 2000 tokens (2^16): 25.6 and 21.5, 31.7 and 25.6;  17 rows, 16000 (2^17): 27.6 and 27.8, 33.8 and 33.8
//   384 rows, 2000 (1.5 x 2^17): 27.6 and 29.7, 31.7 and 37.9;  384 rows, 16000: 42 and 120, 54 and 132
bool prefix_on_tensor(int n_heads, int64_t batch_rows, int head_dim, int prefix_len) {
  return (head_dim == 64 || head_dim == 128) && batch_rows > 16 && n_heads * ((batch_rows + 15) / 16) * prefix_len >= 1 << 17;
}

}  // namespace

AttendShape attend_shape(int n_heads, int n_seqs, int q_len, int n_q_heads, int head_dim, bool e4m3, int64_t own_max, int prefix_len) {
  AttendShape s{};
  s.seq_rows = q_len * (n_q_heads / n_heads);
  const int64_t unit = 4 * (e4m3 ? kGroupOf<true> : kGroupOf<false>);
  // Row tiles over up to `tokens` tokens (how many there really are is known on the device only): splits are whole
  // steps of the four warps, as many as make the sum of all the work over two blocks an SM, an item's start and
  // end counting as 96 tokens, and of the last item least.  (That is at about n = sqrt(3 tokens / tiles), and was never
  // met beyond sqrt(17 tokens / tiles): the bound is for attend_parts.)
  const auto cut = [&](int64_t tiles, int64_t tokens, int32_t &splits, int32_t &chunk) {
    int64_t best = unit * ((tokens + unit - 1) / unit), cost = INT64_MAX;
    for (int64_t n = 1; n <= kMostSplits && (n == 1 || ((n - 1) * unit < tokens && n * n * tiles <= 20 * tokens)); ++n) {
      const int64_t c = ((tokens + n - 1) / n + unit - 1) / unit * unit;
      const int64_t t = tiles * n * (c + 96) / (2 * kSms) + c;
      if (t < cost) cost = t, best = c;
    }
    chunk = (int32_t)(best ? best : unit);
    splits = tokens ? (int32_t)((tokens + chunk - 1) / chunk) : 1;
  };
  const int64_t batch_rows = (int64_t)n_seqs * s.seq_rows;
  if (prefix_on_tensor(n_heads, batch_rows, head_dim, prefix_len)) {
    // Blocks of up to 256 rows, one an SM: the number of splits with the fewest steps one after the
    // other, a block's start and end counting as two.  Beyond two blocks an SM 16 of them are enough: more would save 0.2%
    // of the steps on average and fill the workspace.
    s.tensor = 1;
    s.alternate = batch_rows <= 128;
    const int64_t units = n_heads * ((batch_rows + 255) / 256);
    const int64_t tiles = (prefix_len + 127) / 128, steps = s.alternate ? (tiles + 1) / 2 : tiles;
    int64_t best = 1, cost = INT64_MAX, most = s.alternate ? 8 : 16;   // two parts a block
    if (2 * kSms / units > most) most = 2 * kSms / units;
    for (int64_t n = 1; n <= kMostSplits && n <= steps && n <= most; ++n) {
      const int64_t c = ((units * n + kSms - 1) / kSms) * ((steps + n - 1) / n + 2);
      if (c < cost) cost = c, best = n;
    }
    const int64_t per = (steps + best - 1) / best * (s.alternate ? 2 : 1);   // tiles
    const int64_t blocks = (tiles + per - 1) / per;
    s.prefix_chunk = (int32_t)(per * 128);
    s.prefix_splits = (int32_t)(blocks * (s.alternate ? 2 : 1));
    s.prefix_items = units * blocks;
  } else if (prefix_len > 0) {
    const int64_t tiles = (int64_t)n_heads * ((batch_rows + 15) / 16);
    cut(tiles, prefix_len, s.prefix_splits, s.prefix_chunk);
    s.prefix_items = tiles * s.prefix_splits;
  }
  if (own_max > 0 || prefix_len == 0) {   // without any token there still is an (empty) item a row tile
    const int64_t tiles = (int64_t)n_heads * n_seqs * ((s.seq_rows + 15) / 16);
    cut(tiles, own_max, s.own_splits, s.own_chunk);
    s.own_items = tiles * s.own_splits;
  }
  const int64_t rows = (int64_t)n_seqs * q_len * n_q_heads, slots = s.prefix_splits + s.own_splits;
  s.parts = s.tensor || slots > 1 ? rows * slots : 0;
  return s;
}

int64_t attend_parts(int n_heads, int n_seqs, int q_len, int n_q_heads, int head_dim, bool e4m3, int64_t own_max, int prefix_len) {
  const int64_t rows = (int64_t)n_seqs * q_len * n_q_heads, unit = 4 * (e4m3 ? kGroupOf<true> : kGroupOf<false>);
  // The row kernel's splits n are 1, or at most sqrt(20 tokens / tiles) with tiles >= rows / 16.
  const auto most_splits = [&](int64_t tokens) { return std::min<int64_t>(kMostSplits, (tokens + unit - 1) / unit); };
  const auto of_rows_x_tokens = [](double n) { return (int64_t)std::sqrt(320.0 * n) + 1; };
  const auto on_rows = [&](int64_t r, int64_t tokens) {
    return tokens ? std::max(r, std::min(r * most_splits(tokens), of_rows_x_tokens((double)r * tokens))) : 0;
  };
  int64_t prefix = on_rows(rows, prefix_len), slots = most_splits(prefix_len) + most_splits(own_max);
  if (prefix_on_tensor(n_heads, (int64_t)n_seqs * q_len * (n_q_heads / n_heads), head_dim, prefix_len)) {
    // Smaller calls that stay with the row kernel have up to 16 rows a head, or up to 2^17 row tiles x tokens.
    const int64_t left = std::max(on_rows(std::min<int64_t>(rows, 16 * (int64_t)n_heads), prefix_len), of_rows_x_tokens(16 << 17));
    // The others have units >= rows / 256, a block each, and up to 16 splits or 2 kSms / units; with alternating tiles units
    // >= rows / 128, 8 splits or 2 kSms / units, and two parts a split.
    const int64_t tiles = (prefix_len + 127) / 128;
    const int64_t tensor = std::min(rows * std::min<int64_t>(2 * kMostSplits, tiles + 1), std::max<int64_t>(16 * rows, 2 * kSms * 256));
    prefix = std::max({rows, std::min(prefix, left), tensor});
    slots = 2;
  }
  return slots > 1 ? prefix + on_rows(rows, own_max) : 0;
}

cudaError_t launch_attend(const AttendArgs &a, int type, int io, cudaStream_t st) {
  if (a.tensor) {
    const cudaError_t e = launch_attend_prefix(a, type, io, st);
    if (e != cudaSuccess) return e;
  }
  if (type == EMOE_TYPE_E4M3)
    return io == EMOE_TYPE_BF16 ? by_head_dim<__nv_bfloat16, true>(a, st) : by_head_dim<__half, true>(a, st);
  return io == EMOE_TYPE_BF16 ? by_head_dim<__nv_bfloat16, false>(a, st) : by_head_dim<__half, false>(a, st);
}

}  // namespace emoe
