// attend_masked.cu - attention of packed query tokens over their own sequences' pages, each row with a mask: a window and
// the first tokens, or a tree of drafted tokens.
//
// o = sum_j p_j v_j / sum_j p_j with p_j = 2^(s_j - m), s_j = scale * log2(e) * q.k_j over the tokens that the row
// sees, m the largest s_j, in one pass: each part of the work keeps its own m, sum and unnormalised o in
// 32 bits, and parts are joined by o = sum 2^(m_i - m) o_i.
//
// A tile of rows has a run of tokens: those that some row of it may see.  What a row sees of 32 of them is a word of bits,
// made from two bounds or read from the tree's mask.  A step whose words are all ones - most of them: only the
// ends of a window and the nodes of a tree have others - is computed without looking at them.
#include <algorithm>

#include "attend_item.cuh"
#include "attend_masked.cuh"

namespace emoe {
namespace {

constexpr int kRows = kMaskedRows, kWarps = 4, kStages = 2;
// Tokens of one warp's step: the same bytes for both element sizes.
template <bool FP8> constexpr int kGroupOf = FP8 ? 32 : 16;

// One warp's step covers 16 tokens (32 of an e4m3 cache): K and V rows come through a ring of its own in shared
// memory, scores and products on the tensor cores with the 16 rows of the tile as the m side, running maximum
// and sum in registers.  The four warps take every fourth group of tokens and are joined at the end.  Three blocks an SM (registers, ring).
// Measured, 48 trees of up to 13 nodes on up to 2750 tokens, 16 heads of their own, e4m3, head_dim 128: 97 us, 2.6 TB/s; issue
// slots 46%, integer pipe 37%: what bounds it is the chain of a step, with three warps a scheduler.  (168 registers hold it but for 8 to 28 bytes
// that go to memory with e4m3 at 64 and 128; at 256 it has 255 registers, one block an SM, and 28 to 124 bytes go.)
template <typename IO, int HD, bool FP8>
__global__ void __launch_bounds__(kWarps * 32, HD < 256 ? 3 : 1) masked_rows_kernel(const __grid_constant__ MaskedArgs a) {
  using T = typename Operand<IO, FP8>::type;
  constexpr int kGroup = kGroupOf<FP8>;
  constexpr int ES = FP8 ? 1 : 2, CH = HD * ES / 16, kTile = kGroup * HD * ES, kStage = 2 * kTile;
  constexpr uint32_t kAll = kGroup == 32 ? 0xffffffffu : (1u << (kGroup & 31)) - 1;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ uint16_t s_scale[kWarps][kStages][kGroup];
  __shared__ uint32_t s_valid[kWarps][kStages];
  __shared__ float s_m[kWarps][kRows], s_l[kWarps][kRows];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const int split = blockIdx.x % a.splits, unit_rank = blockIdx.x / a.splits, head = unit_rank % a.c.n_heads;
  let_next_start();
  const int number = a.ranked ? ranked_tile(a, a.tiles_a_seq, unit_rank / a.c.n_heads) : unit_rank / a.c.n_heads, unit = number * a.c.n_heads + head;
  const RowTile tile = row_tile<kRows>(a, a.tiles_a_seq, number);
  if (tile.rows == 0 || (a.short_rows && tile.count * a.group > a.short_rows)) return;
  const Run run = run_of(a, tile);
  // tokens of this split: whole steps of a warp
  const int chunk = ((run.count + a.splits - 1) / a.splits + kGroup - 1) / kGroup * kGroup;
  const int u0 = min(run.count, split * chunk), u1 = min(run.count, u0 + chunk);

  const int groups = (u1 - u0 + kGroup - 1) / kGroup;
  const int steps = groups > warp ? (groups - warp + kWarps - 1) / kWarps : 0;
  const int32_t *const table = a.block_table + (int64_t)tile.seq * a.max_blocks;
  uint8_t *const ring = smem + warp * (kStages * kStage);
  const uint32_t ring_at = shared_address(ring);

  // this lane's place in the run in step i (lanes beyond a group's tokens repeat them), -1 if there is none
  auto place_of = [&](int i) {
    const int u = u0 + (warp + kWarps * i) * kGroup + (lane & (kGroup - 1));
    return i >= steps || u >= u1 ? -1 : u;
  };
  // What the table says of it: the block, and the place there (beyond any block: there is no token).
  constexpr uint32_t kNone = 0xffffffffu;
  struct Found { int block; uint32_t off; };
  auto find = [&](int i) {
    const int u = place_of(i);
    if (u < 0) return Found{0, kNone};
    const TokenPlace p = place_of_token(a, run.token(u));
    return Found{table[p.column], p.off};
  };
  auto vector_of = [&](const Found &f) { return f.off == kNone ? (int64_t)-1 : masked_vector(a, f.block, f.off, head); };
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
      issue(i, vector_of(find(i)));
      keep(i);
    }
    copy_async_commit();
  }
  Found next = find(kStages - 1);   // the table is read a step ahead

  // query rows g and g + 8 of the tile as matrix operands, from global memory; rows that do not exist are the last one again
  uint32_t q[HD / 16][4];
  float by_row[2];   // scores to log2 weights
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const IO *const src = (const IO *)a.q + row_at(a, tile, head, min(g + 8 * half, tile.rows - 1), a.q_stride);
    by_row[half] = a.scale_log2;
#pragma unroll
    for (int ks = 0; ks < HD / 16; ++ks) {
      if constexpr (!FP8) {
        const uint32_t *p = (const uint32_t *)(src + ks * 16 + 2 * c);
        q[ks][half] = p[0];
        q[ks][2 + half] = p[4];
      } else {   // four neighbouring elements, as the codes of a word come
        const uint2 w = *(const uint2 *)(src + (ks >> 1) * 32 + c * 8 + (ks & 1) * 4);
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
  const Sight sight[2] = {Sight(a, tile, run, min(g, tile.rows - 1)), Sight(a, tile, run, min(g + 8, tile.rows - 1))};

  for (int i = 0; i < steps; ++i) {
    const int ahead = i + kStages - 1;
    if (ahead < steps) issue(ahead, vector_of(next));
    copy_async_commit();
    next = find(ahead + 1);
    const int base = u0 + (warp + kWarps * i) * kGroup;
    uint32_t seen[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) seen[half] = sight[half].word(a, tile, run, base);
    copy_async_wait<kStages - 1>();
    __syncwarp();

    const uint32_t k_at = ring_at + (i % kStages) * kStage, v_at = k_at + kTile;
    const uint32_t valid = s_valid[warp][i % kStages] & kAll;
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

    seen[0] &= valid;
    seen[1] &= valid;
    const bool mixed = !__all_sync(0xffffffffu, (seen[0] & seen[1]) == kAll);
    float k_by[kN][2], v_by[kN][2], v_raise[2] = {1.f, 1.f}, v_rest[2] = {1.f, 1.f};
    if constexpr (FP8) {   // scales are powers of two; 255 is not a number and not counted in the largest of v so far
      uint32_t largest[2];
      uint32_t all_largest = 0;
      if (!mixed) {
        const uint32_t mine = s_scale[warp][i % kStages][lane] >> 8;
        all_largest = largest[0] = largest[1] = __reduce_max_sync(0xffffffffu, mine == 255 ? 0 : mine);
      } else {
        largest[0] = largest[1] = 0;
      }
      uint32_t two[kN];
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        two[j] = *(const uint32_t *)&s_scale[warp][i % kStages][j * 8 + 2 * c];
#pragma unroll
        for (int e = 0; e < 2; ++e) k_by[j][e] = scale_of(two[j] >> (16 * e) & 255);
        if (mixed) {   // what a row does not see has no part in its largest scale
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t byte = two[j] >> (16 * e + 8) & 255;
#pragma unroll
            for (int half = 0; half < 2; ++half)
              if (byte != 255 && (seen[half] >> (j * 8 + 2 * c + e) & 1)) largest[half] = max(largest[half], byte);
          }
        }
      }
      if (mixed) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          largest[half] = max(largest[half], __shfl_xor_sync(0xffffffffu, largest[half], 1));
          largest[half] = max(largest[half], __shfl_xor_sync(0xffffffffu, largest[half], 2));
        }
      }
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const uint32_t now = max(v_ref[half], largest[half]);
        v_raise[half] = v_relative(v_ref[half], now);
        v_ref[half] = now;
        v_rest[half] = mixed ? 1.f : v_relative(all_largest, now);
      }
#pragma unroll
      for (int j = 0; j < kN; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) v_by[j][e] = mixed ? 1.f : v_relative(two[j] >> (16 * e + 8) & 255, all_largest);
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
          x *= FP8 ? k_by[j][e] * by_row[half] : by_row[half];
          if (mixed && !(seen[half] >> t & 1)) x = -CUDART_INF_F;
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
          // (a NaN scale shows even where the weight has come to zero)
          if constexpr (FP8) x *= v_by[j][e] * v_rest[half];
        }
      l[half] = l[half] * alpha[half] + sum;
    }
    uint32_t bad = 0;   // tokens of a mixed step with a value that is infinite or not a number
    if (mixed) {
      if constexpr (FP8) {
#pragma unroll
        for (int j = 0; j < kN; ++j) {
          const uint32_t two = *(const uint32_t *)&s_scale[warp][i % kStages][j * 8 + 2 * c];
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int half = 0; half < 2; ++half)
              if (seen[half] >> (j * 8 + 2 * c + e) & 1) s[j][2 * half + e] *= v_relative(two >> (16 * e + 8) & 255, v_ref[half]);
        }
      }
#pragma unroll
      for (int j = 0; j < (kGroup * CH + 31) / 32; ++j) {
        const int id = j * 32 + lane, row = id / CH;
        if (kGroup * CH % 32 == 0 || id < kGroup * CH) {
          const uint4 w = *(const uint4 *)(ring + (i % kStages) * kStage + kTile + swizzled<CH>(row, id % CH) * 16);
          if (not_finite<T, FP8>(w.x) || not_finite<T, FP8>(w.y) || not_finite<T, FP8>(w.z) || not_finite<T, FP8>(w.w)) bad |= 1u << row;
        }
      }
      bad = __reduce_or_sync(0xffffffffu, bad);
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
    // A weight of zero does not silence such a value: its token goes, element by element, to the rows that see
    // it, and is then cleared for the product.
    while (__builtin_expect(bad != 0, 0)) {
      const int t = __ffs(bad) - 1;
      bad &= bad - 1;
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        uint32_t word = 0;
#pragma unroll
        for (int k = 0; k < kP; ++k)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (t >> 3 == 2 * k + e) word = p[k][2 * e + half];
        const float2 two = Pair<T>::unpack(__shfl_sync(0xffffffffu, word, (lane & ~3) | (t >> 1 & 3)));
        if (seen[half] >> t & 1) {
          const float weight = t & 1 ? two.y : two.x;
#pragma unroll
          for (int n = 0; n < HD / 8; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int col = FP8 ? (n >> 1) * 16 + 4 * c + (n & 1) + 2 * e : n * 8 + 2 * c + e;
              const uint8_t *const at = ring + (i % kStages) * kStage + kTile + swizzled<CH>(t, col * ES / 16) * 16 + col * ES % 16;
              float v;
              if constexpr (FP8) {
                uint32_t lo, hi;
                codes_to_half(lo, hi, *at);
                v = Pair<__half>::unpack(lo).x;
              } else {
                v = Pair<T>::unpack(*(const uint16_t *)at).x;
              }
              o[n / kTileGroup][n % kTileGroup][2 * half + e] += weight * v;
            }
        }
      }
      __syncwarp();
      for (int ch = lane; ch < CH; ch += 32)
        *(uint4 *)(ring + (i % kStages) * kStage + kTile + swizzled<CH>(t, ch) * 16) = make_uint4(0, 0, 0, 0);
      __syncwarp();
    }
    // Products with the n-th 16 (e4m3: 32) columns of v, pieces read with ldmatrix: two column tiles of an e4m3
    // cache share 16-bit elements (two neighbouring columns) and are parted here.
    constexpr int kReads = HD / 8 / kTileGroup;
#pragma unroll
    for (int n = 0; n < kReads; ++n) {
      float(&d)[kTileGroup][4] = o[n];
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
      joined[(warp * kRows + g + 8 * (e >> 1)) * kPitch + col] = o[n / kTileGroup][n % kTileGroup][e] * (FP8 ? scale_of(v_ref[e >> 1]) : 1.f);
    }
  __syncthreads();
  finish_rows<IO, HD, kRows, kWarps>(a, tile, head, unit, split, joined, s_m, s_l);
}

// Joins the parts of the rows of a tile of R: TEAM warps a row, four parts read without waiting for one another.  Bound by the latency
// of its reads: 5 to 7 us alone, about 3 behind a kernel that is still ending.
constexpr int kJoinWarps = 16;
struct JoinArgs {
  MaskedArgs a;
  const float2 *ml;          // [tile][head][part][row]
  const float *o;
  int32_t parts, tiles_a_seq;
  int32_t least, most;       // rows of the sequences that count
};
template <typename T, int HD, int R, int TEAM>
__global__ void __launch_bounds__(kJoinWarps * 32) masked_join_kernel(const __grid_constant__ JoinArgs j) {
  constexpr int N = HD / 32, kMine = kJoinWarps / TEAM, kBlocks = (R + kMine - 1) / kMine;   // rows of a block, blocks of a tile
  __shared__ float s_x[kJoinWarps][HD], s_l[kJoinWarps];
  const MaskedArgs &a = j.a;
  const int unit = blockIdx.x / kBlocks, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, head = unit % a.c.n_heads, n = j.parts;
  const int row = blockIdx.x % kBlocks * kMine + warp / TEAM;
  const RowTile tile = row_tile<R>(a, j.tiles_a_seq, unit / a.c.n_heads);
  wait_for_previous();
  const int all = tile.count * a.group;
  if (all < j.least || all > j.most) return;
  const bool mine = row < tile.rows;
  const int64_t first = (int64_t)unit * n * R + row;
  float m = -CUDART_INF_F, l = 0.f, x[N] = {};
  if (mine) {
    for (int i = lane; i < n; i += 32) m = fmaxf(m, j.ml[first + (int64_t)i * R].x);
#pragma unroll
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    for (int i = warp % TEAM * 4; i < n; i += TEAM * 4) {
      float w[4], y[4][N];
      bool there[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int64_t at = first + (int64_t)min(i + u, n - 1) * R;
        const float2 p = i + u < n ? j.ml[at] : make_float2(-CUDART_INF_F, 0.f);
        // an empty part (sum 0) does not count
        there[u] = p.y != 0.f;
        w[u] = p.y != p.y ? CUDART_NAN_F : exp2_fast(p.x - m);
        l += there[u] ? w[u] * p.y : 0.f;
        const float *const src = j.o + at * HD + lane * N;
        if constexpr (N % 4 == 0) {
#pragma unroll
          for (int k = 0; k < N; k += 4) *(float4 *)&y[u][k] = *(const float4 *)(src + k);
        } else if constexpr (N == 2) {
          *(float2 *)y[u] = *(const float2 *)src;
        } else {
          y[u][0] = src[0];
        }
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] += there[u] ? w[u] * y[u][k] : 0.f;
    }
  }
  if constexpr (TEAM > 1) {   // in the order of the warps
#pragma unroll
    for (int k = 0; k < N; ++k) s_x[warp][lane * N + k] = x[k];
    if (lane == 0) s_l[warp] = l;
    __syncthreads();
    if (warp % TEAM == 0)
#pragma unroll
      for (int t = 1; t < TEAM; ++t) {
        l += s_l[warp + t];
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] += s_x[warp + t][lane * N + k];
      }
  }
  if (!mine || warp % TEAM) return;
  const float by = l == 0.f ? 0.f : 1.f / l;
  T *const out = (T *)a.out + row_at(a, tile, head, row, a.out_stride) + lane * N;
  if constexpr (N >= 2) {
#pragma unroll
    for (int k = 0; k < N; k += 2) *(uint32_t *)(out + k) = Pair<T>::pack(x[k] * by, x[k + 1] * by);
  } else {
    out[0] = (T)(x[0] * by);
  }
  if (lane == 0) write_lse(a, tile, head, row, m, l);
}

template <typename T, int HD, bool FP8>
cudaError_t launch_rows(const MaskedArgs &a, cudaStream_t st) {
  constexpr size_t ring = (size_t)kWarps * kStages * 2 * kGroupOf<FP8> * HD * (FP8 ? 1 : 2);
  constexpr size_t join = (size_t)kWarps * kRows * (HD + 4) * 4;
  constexpr size_t smem = ring > join ? ring : join;
  const cudaError_t e = allow_shared<masked_rows_kernel<T, HD, FP8>>();
  if (e != cudaSuccess) return e;
  masked_rows_kernel<T, HD, FP8><<<(unsigned)a.tiles * a.c.n_heads * a.splits, kWarps * 32, smem, st>>>(a);
  return cudaGetLastError();
}

template <typename T, int HD, int R, int TEAM>
cudaError_t launch_join_by(const JoinArgs &j, int tiles, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)tiles * j.a.c.n_heads * ((R * TEAM + kJoinWarps - 1) / kJoinWarps));
  cfg.blockDim = dim3(kJoinWarps * 32);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, masked_join_kernel<T, HD, R, TEAM>, j);
}
template <typename T, int HD, int R>
cudaError_t launch_join(const JoinArgs &j, int tiles, cudaStream_t st) {   // more than two groups of four parts go to four warps
  return j.parts > 8 ? launch_join_by<T, HD, R, 4>(j, tiles, st) : launch_join_by<T, HD, R, 1>(j, tiles, st);
}

// The row kernel, the tensor core kernel, the joins: each may start while the one before still runs and waits for it
// before it ends, so that the last one ends last.
template <typename T, int HD, bool FP8>
cudaError_t launch_all(const MaskedArgs &a, int type, int io, cudaStream_t st) {
  cudaError_t e = !a.tiles ? cudaSuccess : a.few ? launch_masked_few(a, type, io, st) : launch_rows<T, HD, FP8>(a, st);
  if constexpr (HD == 64 || HD == 128) {
    if (e == cudaSuccess && a.tensor_tiles) e = launch_masked_tensor(a, type, io, a.tiles != 0, st);
    if (e == cudaSuccess && a.tensor_tiles && a.tensor_splits > 1)
      e = launch_join<T, HD, kMaskedTensorRows>({a, a.tensor_ml, a.tensor_o, a.tensor_splits, a.tensor_tiles_a_seq, a.short_rows + 1, 1 << 30}, a.tensor_tiles, st);
  }
  if (e == cudaSuccess && a.tiles && a.splits > 1) {
    const JoinArgs j{a, a.part_ml, a.part_o, a.splits, a.tiles_a_seq, 1, a.short_rows ? a.short_rows : 1 << 30};
    e = a.few ? launch_join<T, HD, kMaskedFewRows>(j, a.tiles, st) : launch_join<T, HD, kRows>(j, a.tiles, st);
  }
  return e;
}

template <typename T, bool FP8>
cudaError_t by_head_dim(const MaskedArgs &a, int type, int io, cudaStream_t st) {
  switch (a.c.head_dim) {
    case 32: return launch_all<T, 32, FP8>(a, type, io, st);
    case 64: return launch_all<T, 64, FP8>(a, type, io, st);
    case 128: return launch_all<T, 128, FP8>(a, type, io, st);
    case 256: return launch_all<T, 256, FP8>(a, type, io, st);
  }
  return cudaErrorInvalidValue;
}

constexpr int64_t kMostSplits = 64, kMostUnits = 8 * kSms, kMostTensorSplits = 64, kMostTensorUnits = 2 * kSms;   // splits of a unit, units with their splits

// Row tiles of R rows: as many for every sequence, or as the packed tokens make, what leaves fewer of them empty.
void count_tiles(MaskedShape &s, const MaskedSizes &n, int64_t rows) {
  const int64_t group = n.n_q_heads / n.n_heads, each = (n.max_q * group + rows - 1) / rows, packed = n.n_tokens * group / rows + n.n_seqs;
  s.tiles_a_seq = each * n.n_seqs <= packed ? (int32_t)each : 0;
  s.tiles = (int32_t)std::min(each * n.n_seqs, packed);
}

// Whether sequences with more than 16 rows a head go to the tensor core kernel, which has head_dim 64 and 128 only (at 256, O of two slots alone
// would fill tensor memory).  It takes 128 rows at least at once, so that it
// pays from about 2^17 row tiles (of 16 rows) x heads x tokens on, with few rows later.  Measured, 4 heads, us of the row kernel and of
// the other one, bf16 and e4m3:
//   64 and more rows: 1 x 128 rows x 2000 tokens (2^16) 18.9, 20.2 and 20.9, 20.9;  4 x 128 x 1000 (2^17) 22.3, 18.0 and 27.0, 21.0;
//     16 x 128 x 500 (2^18) 35.3, 23.0 and 42.6, 27.8;  64 x 128 x 250 (2^19) 62.5, 31.3 and 76.5, 43.4
//   32 rows: 16 x 1000 (2^17) 21.9, 23.5 and 25.0, 30.7;  16 x 2000 (2^18) 33.3, 29.2 and 36.5, 40.3;  64 x 1000 (2^19) 62.2, 60.9 and 70.5, 76.4
bool on_tensor(const MaskedSizes &n) {
  MaskedShape s;
  count_tiles(s, n, kRows);
  const int64_t rows = (int64_t)n.max_q * (n.n_q_heads / n.n_heads), least = rows >= 64 ? 1 << 17 : n.e4m3 ? 1 << 20 : 1 << 18;
  return (n.head_dim == 64 || n.head_dim == 128) && rows > kRows && (int64_t)s.tiles * n.n_heads * n.most_tokens >= least;
}

}  // namespace

MaskedShapes masked_shapes(const MaskedSizes &n) {
  MaskedShapes s{};
  const bool tensor = on_tensor(n);
  const int64_t group = n.n_q_heads / n.n_heads;
  if (tensor) {
    // Blocks of up to 256 rows, one an SM: the number of splits with the fewest tiles one after the other, a block's
    // start and end counting as three.
    count_tiles(s.tensor, n, kMaskedTensorRows);
    const int64_t units = (int64_t)s.tensor.tiles * n.n_heads, tiles = (n.most_tokens + 127) / 128;
    int64_t best = 1, cost = INT64_MAX;
    for (int64_t k = 1; k <= kMostTensorSplits && k <= tiles && (k == 1 || k * units <= kMostTensorUnits); ++k) {
      const int64_t c = ((units * k + kSms - 1) / kSms) * ((tiles + k - 1) / k + 3);
      if (c < cost) cost = c, best = k;
    }
    s.tensor.splits = (int32_t)best;
    s.tensor.parts = best > 1 ? units * best * kMaskedTensorRows : 0;
    // (as below: 64 trees of 24 nodes on 26 to 2750 tokens, 4 heads, 98 us as they come, 79 the longest first)
    s.tensor_ranked = n.by_length && s.tensor.tiles_a_seq && n.n_seqs > 1 && n.n_seqs <= kMostRanked && units * best > kSms;
  }
  // Beside the tensor core kernel a row kernel takes sequences with few rows, unless there are so few that they do not matter there.
  if (tensor && n.n_seqs * (int64_t)n.n_heads <= kSms / 2) return s;
  s.few = tensor ? group <= kMaskedFewRows : n.max_q * group <= kMaskedFewRows;
  const int rows = s.few ? kMaskedFewRows : kRows;
  count_tiles(s.rows, n, rows);
  if (tensor) s.rows.tiles = n.n_seqs, s.rows.tiles_a_seq = 1;
  // Splits.  Three blocks an SM run at once; while they do 64 tokens of a block take 2.4 us, with fewer of them down to 1 us (what a
  // step's chain waits for; e4m3 2.0 and 1.3); a block's start and end count as 64 tokens, the join, a launch, as
  // 5 us and 1 us for 16 parts.  Times in tenths of a us and 64ths.  Measured, 64 sequences in a window of 1024, 4 heads: 1 split 28 us, 2 37,
  // 3 33, 8 42; 128 in a window of 4095, 2 heads, e4m3: 92, 82, 80, 89; one sequence of 2375 tokens, 64 rows: 1 split 50 us, 4 21, 8 16, 16 14.
  const int64_t units = (int64_t)s.rows.tiles * n.n_heads, full = n.e4m3 ? 20 : 24, least = n.e4m3 ? 13 : 10;
  int64_t cost = INT64_MAX;
  for (int64_t k = 1; k <= kMostSplits && (k == 1 || ((k - 1) * 16 < n.most_tokens && k * units <= kMostUnits)); ++k) {
    const int64_t c = (n.most_tokens + k - 1) / k + 64, waves = units * k / (3 * kSms), rest = units * k % (3 * kSms);
    const int64_t t = c * (full * waves + (rest ? std::max(least, full * rest / (3 * kSms)) : 0)) + (k > 1 ? 3200 + 40 * k : 0);
    if (t < cost) cost = t, s.rows.splits = (int32_t)k;
  }
  s.rows.parts = s.rows.splits > 1 ? units * s.rows.splits * rows : 0;
  // Finding a rank costs a block about 1 us; it pays where blocks wait for others to end, if lengths differ.  Measured, 48 trees on 13 to
  // 2750 tokens, 16 heads: e4m3 130 us as they come, 97 the longest first, bf16 106 and 88; 128 single tokens in a window of 512 that
  // nearly all of them fill: 56 and 60.
  s.ranked = n.by_length && s.rows.tiles_a_seq && n.n_seqs > 1 && n.n_seqs <= kMostRanked && units * s.rows.splits > 3 * kSms;
  return s;
}

void masked_parts(const MaskedSizes &n, int64_t &rows, int64_t &tensor) {
  // Only calls whose units come to kMostUnits (kMostTensorUnits) at most with their splits have any parts.
  MaskedShape s;
  const auto most = [&](int tile_rows, int64_t step, int64_t most_splits, int64_t most_units) {
    count_tiles(s, n, tile_rows);
    const int64_t splits = std::min(most_splits, (n.most_tokens + step - 1) / step);
    return splits > 1 ? std::min(most_units, (int64_t)s.tiles * n.n_heads * splits) * tile_rows : 0;
  };
  rows = std::max(most(kMaskedFewRows, 16, kMostSplits, kMostUnits), most(kRows, 16, kMostSplits, kMostUnits));
  tensor = on_tensor(n) ? most(kMaskedTensorRows, 128, kMostTensorSplits, kMostTensorUnits) : 0;
}

cudaError_t launch_attend_masked(const MaskedArgs &a, int type, int io, cudaStream_t st) {
  if (type == EMOE_TYPE_E4M3)
    return io == EMOE_TYPE_BF16 ? by_head_dim<__nv_bfloat16, true>(a, type, io, st) : by_head_dim<__half, true>(a, type, io, st);
  return io == EMOE_TYPE_BF16 ? by_head_dim<__nv_bfloat16, false>(a, type, io, st) : by_head_dim<__half, false>(a, type, io, st);
}

}  // namespace emoe
