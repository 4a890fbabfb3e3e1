// attend_masked_few.cu - attention with masks for up to 8 rows a sequence and KV head: one token of a decoding sequence with
// up to 8 query heads a KV head, a few drafted tokens.
//
// The row kernel's matrices turned round: S^T = K Q^T and O^T = V^T P^T, so that tokens (and columns of v) lie along the 16 rows of
// a matrix instruction and the query rows along its 8 columns.  Against 16 query rows as the long side that is half the
// products, half the scores a lane holds and half the registers of O.  P^T comes out of the scores' layout by transposing 8 x 8
// matrices of 16 bits in registers.
//
// Measured, head_dim 128: 64 sequences x 1028 tokens x 4 heads, bf16, 28.7 us, 4.2 TB/s over the call (the row kernel with three splits and
// their join 36.9): 256 blocks, fewer than two an SM, which is less than splitting and joining costs.  128 x up to 4099 tokens x
// 2 heads, e4m3, 78 us, 2.8 TB/s (97.9): DRAM at 43%, issue slots 46%, integer pipe 41% - widening codes, and a step's chain.
#include "attend_item.cuh"
#include "attend_masked.cuh"

namespace emoe {
namespace {

constexpr int kRows = kMaskedFewRows, kWarps = 4, kStages = 2;
template <bool FP8> constexpr int kGroupOf = FP8 ? 32 : 16;   // tokens of one warp's step: the same bytes for both element sizes

__device__ __forceinline__ uint32_t transposed(uint32_t x) {   // of an 8 x 8 matrix of 16 bits, two neighbours of a row a lane
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

template <typename IO, int HD, bool FP8>
__global__ void __launch_bounds__(kWarps * 32, HD < 256 ? 3 : 1) masked_few_kernel(const __grid_constant__ MaskedArgs a) {
  using T = typename Operand<IO, FP8>::type;
  constexpr int kGroup = kGroupOf<FP8>, kBlocks = kGroup / 8;   // 8-token blocks of a step
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

  // Lane (g, c): rows 2 c and 2 c + 1, tokens g of each block of 8.  O^T: rows 2 c, 2 c + 1 of columns g and g + 8 of each 16 (e4m3:
  // 2 g and 2 g + 1).  v_ref: the largest scale byte of v so far that a row sees, whose scale its o is relative to.
  uint32_t v_ref[2] = {0, 0};
  float o[HD / 16][4] = {}, m[2] = {-CUDART_INF_F, -CUDART_INF_F}, l[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) {
    if (i < steps) {
      issue(i, vector_of(find(i)));
      keep(i);
    }
    copy_async_commit();
  }
  Found next = find(kStages - 1);   // the table is read a step ahead

  // Query row g as a matrix operand, from global memory; rows that do not exist are the last one again.
  uint32_t q[HD / 16][2];
  float by_row[2] = {a.scale_log2, a.scale_log2};   // scores to log2 weights
  {
    const IO *const src = (const IO *)a.q + row_at(a, tile, head, min(g, tile.rows - 1), a.q_stride);
#pragma unroll
    for (int ks = 0; ks < HD / 16; ++ks) {
      if constexpr (!FP8) {
        const uint32_t *p = (const uint32_t *)(src + ks * 16 + 2 * c);
        q[ks][0] = p[0];
        q[ks][1] = p[4];
      } else {   // four neighbouring elements, as the codes of a word come
        const uint2 w = *(const uint2 *)(src + (ks >> 1) * 32 + c * 8 + (ks & 1) * 4);
        q[ks][0] = w.x;
        q[ks][1] = w.y;
      }
    }
    if constexpr (FP8) {
      uint32_t top = 0;
#pragma unroll
      for (int ks = 0; ks < HD / 16; ++ks)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const float2 f = Pair<IO>::unpack(q[ks][k]);
          top = max(top, max(__float_as_uint(f.x) & 0x7fffffffu, __float_as_uint(f.y) & 0x7fffffffu));
        }
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const float by = query_scale(top);
#pragma unroll
      for (int ks = 0; ks < HD / 16; ++ks)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const float2 f = Pair<IO>::unpack(q[ks][k]);
          q[ks][k] = Pair<T>::pack(f.x * by, f.y * by);
        }
#pragma unroll
      for (int e = 0; e < 2; ++e) by_row[e] = a.scale_log2 / __shfl_sync(0xffffffffu, by, (2 * c + e) * 4);   // row 2 c + e is lane group 2 c + e's
    }
  }
  const Sight sight[2] = {Sight(a, tile, run, min(2 * c, tile.rows - 1)), Sight(a, tile, run, min(2 * c + 1, tile.rows - 1))};

  for (int i = 0; i < steps; ++i) {
    const int ahead = i + kStages - 1;
    if (ahead < steps) issue(ahead, vector_of(next));
    copy_async_commit();
    next = find(ahead + 1);
    const int base = u0 + (warp + kWarps * i) * kGroup;
    uint32_t seen[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) seen[e] = sight[e].word(a, tile, run, base);
    copy_async_wait<kStages - 1>();
    __syncwarp();

    uint8_t *const k_tile = ring + (i % kStages) * kStage, *const v_tile = k_tile + kTile;
    const uint32_t k_at = ring_at + (i % kStages) * kStage, v_at = k_at + kTile;
    const uint32_t valid = s_valid[warp][i % kStages] & kAll;
    float s[kBlocks / 2][4] = {};   // of 16 tokens: (token g, rows 2 c, 2 c + 1), (token g + 8, ...)
#pragma unroll
    for (int t = 0; t < kBlocks / 2; ++t) {
      if constexpr (!FP8) {
#pragma unroll
        for (int ks = 0; ks < HD / 16; ++ks) {
          uint32_t k[4];
          ldmatrix_x4(k, k_at + swizzled<CH>(t * 16 + (lane & 15), ks * 2 + (lane >> 4)) * 16);
          mma_16816<T>(s[t], k, q[ks][0], q[ks][1]);
        }
      } else {
#pragma unroll
        for (int kb = 0; kb < HD / 32; ++kb) {
          const uint2 lo = *(const uint2 *)(k_tile + swizzled<CH>(t * 16 + g, kb * 2 + (c >> 1)) * 16 + (c & 1) * 8);
          const uint2 hi = *(const uint2 *)(k_tile + swizzled<CH>(t * 16 + 8 + g, kb * 2 + (c >> 1)) * 16 + (c & 1) * 8);
          uint32_t k[4], n[4];
          codes_to_half(k[0], k[2], lo.x);
          codes_to_half(n[0], n[2], lo.y);
          codes_to_half(k[1], k[3], hi.x);
          codes_to_half(n[1], n[3], hi.y);
          mma_16816<T>(s[t], k, q[2 * kb][0], q[2 * kb][1]);
          mma_16816<T>(s[t], n, q[2 * kb + 1][0], q[2 * kb + 1][1]);
        }
      }
    }

    seen[0] &= valid;
    seen[1] &= valid;
    const bool mixed = !__all_sync(0xffffffffu, (seen[0] & seen[1]) == kAll);
    uint32_t scales[kBlocks];   // e4m3: scale bytes of k and v of this lane's token of each block
    float v_by[kBlocks], v_raise[2] = {1.f, 1.f}, v_rest[2] = {1.f, 1.f};
    if constexpr (FP8) {   // scales are powers of two; 255 is not a number and not counted in the largest of v so far
      uint32_t largest[2] = {0, 0};
#pragma unroll
      for (int j = 0; j < kBlocks; ++j) {
        scales[j] = s_scale[warp][i % kStages][j * 8 + g];
        const uint32_t byte = scales[j] >> 8;
#pragma unroll
        for (int e = 0; e < 2; ++e)   // what a row does not see has no part in its largest scale
          if (byte != 255 && (!mixed || (seen[e] >> (j * 8 + g) & 1))) largest[e] = max(largest[e], byte);
      }
      const uint32_t both = largest[0] | largest[1] << 16;   // (bytes: two maxima at once)
      uint32_t top = both;
#pragma unroll
      for (int d = 4; d < 32; d *= 2) top = __vmaxu2(top, __shfl_xor_sync(0xffffffffu, top, d));
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t step_top = e ? top >> 16 : top & 0xffffu, now = max(v_ref[e], step_top);
        v_raise[e] = v_relative(v_ref[e], now);
        v_ref[e] = now;
        v_rest[e] = mixed ? 1.f : v_relative(step_top, now);   // without masks both rows have the same step_top
      }
#pragma unroll
      for (int j = 0; j < kBlocks; ++j) v_by[j] = mixed ? 1.f : v_relative(scales[j] >> 8, top & 0xffffu);
    }
    float top[2] = {m[0], m[1]};
#pragma unroll
    for (int j = 0; j < kBlocks; ++j) {
      const float k_by = FP8 ? scale_of(scales[j] & 255) : 1.f;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float &x = s[j >> 1][2 * (j & 1) + e];
        x *= FP8 ? k_by * by_row[e] : by_row[e];
        if (mixed && !(seen[e] >> (j * 8 + g) & 1)) x = -CUDART_INF_F;
        top[e] = fmaxf(top[e], x);
      }
    }
    float alpha[2], sum[2] = {0.f, 0.f}, safe[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int d = 4; d < 32; d *= 2) top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], d));
      alpha[e] = exp2_fast(m[e] - (top[e] == -CUDART_INF_F ? 0.f : top[e]));
      safe[e] = top[e] == -CUDART_INF_F ? 0.f : top[e] - kWeightLift<T>;
      m[e] = top[e];
    }
    uint32_t w[kBlocks];   // weights of a block's token, both rows, rounded to T, once, as the second product's operand
#pragma unroll
    for (int j = 0; j < kBlocks; ++j) {
      float p[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        p[e] = exp2_fast(s[j >> 1][2 * (j & 1) + e] - safe[e]);
        sum[e] += p[e];
        // (a NaN scale shows even where the weight has come to zero)
        if constexpr (FP8) {
          if (!mixed) p[e] *= v_by[j] * v_rest[e];
          else if (seen[e] >> (j * 8 + g) & 1) p[e] *= v_relative(scales[j] >> 8, v_ref[e]);
        }
      }
      w[j] = Pair<T>::pack(p[0], p[1]);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      l[e] = l[e] * alpha[e] + sum[e];
      alpha[e] *= v_raise[e];
    }
    uint32_t bad = 0;   // tokens of a mixed step with a value that is infinite or not a number
    if (mixed) {
#pragma unroll
      for (int j = 0; j < (kGroup * CH + 31) / 32; ++j) {
        const int id = j * 32 + lane, row = id / CH;
        if (kGroup * CH % 32 == 0 || id < kGroup * CH) {
          const uint4 x = *(const uint4 *)(v_tile + swizzled<CH>(row, id % CH) * 16);
          if (not_finite<T, FP8>(x.x) || not_finite<T, FP8>(x.y) || not_finite<T, FP8>(x.z) || not_finite<T, FP8>(x.w)) bad |= 1u << row;
        }
      }
      bad = __reduce_or_sync(0xffffffffu, bad);
    }
    if (!__all_sync(0xffffffffu, alpha[0] == 1.f && alpha[1] == 1.f)) {
#pragma unroll
      for (int n = 0; n < HD / 16; ++n) {
        o[n][0] *= alpha[0];
        o[n][1] *= alpha[1];
        o[n][2] *= alpha[0];
        o[n][3] *= alpha[1];
      }
    }
    // A weight of zero does not silence such a value: its token goes, element by element, to the rows that see
    // it, and is then cleared for the product.
    while (__builtin_expect(bad != 0, 0)) {
      const int t = __ffs(bad) - 1;
      bad &= bad - 1;
      uint32_t mine = 0;
#pragma unroll
      for (int j = 0; j < kBlocks; ++j)
        if (t >> 3 == j) mine = w[j];
      const float2 two = Pair<T>::unpack(__shfl_sync(0xffffffffu, mine, (t & 7) * 4 + c));
#pragma unroll
      for (int n = 0; n < HD / 16; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int col = n * 16 + (FP8 ? 2 * g + h : g + 8 * h);
          const uint8_t *const at = v_tile + swizzled<CH>(t, col * ES / 16) * 16 + col * ES % 16;
          float v;
          if constexpr (FP8) {
            uint32_t lo, hi;
            codes_to_half(lo, hi, *at);
            v = Pair<__half>::unpack(lo).x;
          } else {
            v = Pair<T>::unpack(*(const uint16_t *)at).x;
          }
          if (seen[0] >> t & 1) o[n][2 * h] += two.x * v;
          if (seen[1] >> t & 1) o[n][2 * h + 1] += two.y * v;
        }
      __syncwarp();
      for (int ch = lane; ch < CH; ch += 32) *(uint4 *)(v_tile + swizzled<CH>(t, ch) * 16) = make_uint4(0, 0, 0, 0);
      __syncwarp();
    }
#pragma unroll
    for (int j = 0; j < kBlocks; ++j) w[j] = transposed(w[j]);
#pragma unroll
    for (int t = 0; t < kBlocks / 2; ++t) {
      if constexpr (!FP8) {
#pragma unroll
        for (int n = 0; n < HD / 16; ++n) {
          uint32_t v[4];
          ldmatrix_x4_trans(v, v_at + swizzled<CH>(t * 16 + (lane & 7) + (lane >> 4) * 8, 2 * n + (lane >> 3 & 1)) * 16);
          mma_16816<T>(o[n], v, w[2 * t], w[2 * t + 1]);
        }
      } else {   // 16-bit elements are two neighbouring columns, which are parted here
#pragma unroll
        for (int n = 0; n < HD / 32; ++n) {
          uint32_t b[4];
          ldmatrix_x4_trans(b, v_at + swizzled<CH>(t * 16 + (lane & 15), 2 * n + (lane >> 4)) * 16);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t v[4];   // columns 2 g and 2 g + 1 of tokens 2 c, 2 c + 1; of tokens 2 c + 8, 2 c + 9
            codes_to_half(v[0], v[1], __byte_perm(b[2 * h], 0, 0x3120));
            codes_to_half(v[2], v[3], __byte_perm(b[2 * h + 1], 0, 0x3120));
            mma_16816<T>(o[2 * n + h], v, w[2 * t], w[2 * t + 1]);
          }
        }
      }
    }
    if (ahead < steps) keep(ahead);
    __syncwarp();
  }
  copy_async_wait<0>();

  // the four warps' parts become one
#pragma unroll
  for (int e = 0; e < 2; ++e) {
#pragma unroll
    for (int d = 4; d < 32; d *= 2) l[e] += __shfl_xor_sync(0xffffffffu, l[e], d);
    if (g == 0) {
      s_m[warp][2 * c + e] = m[e] - kWeightLift<T>;
      s_l[warp][2 * c + e] = l[e];
    }
  }
  __syncthreads();
  constexpr int kPitch = HD + 4;
  float *const joined = (float *)smem;
#pragma unroll
  for (int n = 0; n < HD / 16; ++n)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int col = n * 16 + (FP8 ? 2 * g + (k >> 1) : g + 8 * (k >> 1));
      joined[(warp * kRows + 2 * c + (k & 1)) * kPitch + col] = o[n][k] * (FP8 ? scale_of(v_ref[k & 1]) : 1.f);
    }
  __syncthreads();
  finish_rows<IO, HD, kRows, kWarps>(a, tile, head, unit, split, joined, s_m, s_l);
}

template <typename T, int HD, bool FP8>
cudaError_t launch(const MaskedArgs &a, cudaStream_t st) {
  constexpr size_t ring = (size_t)kWarps * kStages * 2 * kGroupOf<FP8> * HD * (FP8 ? 1 : 2);
  constexpr size_t join = (size_t)kWarps * kRows * (HD + 4) * 4;
  constexpr size_t smem = ring > join ? ring : join;
  const cudaError_t e = allow_shared<masked_few_kernel<T, HD, FP8>>();
  if (e != cudaSuccess) return e;
  masked_few_kernel<T, HD, FP8><<<(unsigned)a.tiles * a.c.n_heads * a.splits, kWarps * 32, smem, st>>>(a);
  return cudaGetLastError();
}

template <typename T, bool FP8>
cudaError_t by_head_dim(const MaskedArgs &a, cudaStream_t st) {
  switch (a.c.head_dim) {
    case 32: return launch<T, 32, FP8>(a, st);
    case 64: return launch<T, 64, FP8>(a, st);
    case 128: return launch<T, 128, FP8>(a, st);
    case 256: return launch<T, 256, FP8>(a, st);
  }
  return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_masked_few(const MaskedArgs &a, int type, int io, cudaStream_t st) {
  if (type == EMOE_TYPE_E4M3)
    return io == EMOE_TYPE_BF16 ? by_head_dim<__nv_bfloat16, true>(a, st) : by_head_dim<__half, true>(a, st);
  return io == EMOE_TYPE_BF16 ? by_head_dim<__nv_bfloat16, false>(a, st) : by_head_dim<__half, false>(a, st);
}

}  // namespace emoe
