// moe.cu - a whole mixture-of-experts layer for a few tokens: routing, gate and up products,
// activation, down product, weighted sum.
//
//   y_t = sum over the experts e chosen by t of w_te * Wd_e (silu(Wg_e x_t) * (Wu_e x_t))
//
// With a few tokens the layer is bound by reading the chosen experts' weights once, so everything
// is arranged around that stream: each lane owns a ring of 16-byte slots in shared memory that it
// fills with asynchronous copies and reads back itself (no barrier between a warp's copies and its
// use of them), weights are the 16-row side of the tensor-core product straight from those slots,
// tokens its 8-column side, and the order of the k axis inside a block is the order in which the
// slots hold it.  Three launches, chained so that each one's prologue overlaps the tail of the one before:
//   route: one block; top-k and softmax by warps, the list of experts in use, the pairs (expert, token)
//   up:    items of 8 gate and 8 up rows of one expert (one product gives both, in the same thread)
//   down:  16 rows of the output over ALL experts in use: every token's sum stays in registers, in
//          the order of the slots - no partial results, no atomics.
#include <math_constants.h>

#include "convert.cuh"
#include "serve.h"

namespace emoe {
namespace {

constexpr int kRouteThreads = 1024, kWarps = 8;

// Order of logits: larger value first, then the smaller index; NaN as minus infinity.
__device__ __forceinline__ uint64_t rank_key(float v, int e) {
  if (v != v) v = -CUDART_INF_F;
  const uint32_t b = __float_as_uint(v);
  const uint32_t ordered = b & 0x80000000u ? ~b : b | 0x80000000u;
  return (uint64_t)ordered << 32 | (uint32_t)~e;
}
constexpr uint32_t kLowest = 0x007fffffu;   // minus infinity's place in that order

__global__ void __launch_bounds__(kRouteThreads) moe_route_kernel(const __grid_constant__ MoeArgs a) {
  extern __shared__ unsigned long long s_tokens[];   // [n_slots]
  int32_t *const s_base = (int32_t *)(s_tokens + a.n_slots);
  __shared__ int32_t s_scan[2][32];
  __shared__ int32_t s_total[2];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  let_next_start();
  for (int i = threadIdx.x; i < a.n_slots; i += kRouteThreads) s_tokens[i] = 0;
  if (threadIdx.x < 2) s_total[threadIdx.x] = 0;
  __syncthreads();

  int my_slot[2] = {-1, -1};   // of pair number `lane` (routed, then shared) of tokens warp and warp + 32
  float my_weight[2] = {};
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int t = warp + 32 * half;
    if (t >= a.n_tokens) continue;
    const float *row = a.logits + t * a.logits_stride;
    uint32_t taken = 0;   // of this lane's experts lane + 32 j
    float top = 0.f, chosen_sum = 0.f, mine = 0.f;
    int my_id = -1;
    for (int k = 0; k < a.top_k; ++k) {
      uint64_t best = 0;
      for (int j = 0; j * 32 < a.n_experts; ++j) {
        const int e = j * 32 + lane;
        if (e < a.n_experts && !(taken >> j & 1)) {
          const uint64_t key = rank_key(row[e], e);
          best = key > best ? key : best;
        }
      }
#pragma unroll
      for (int d = 16; d; d >>= 1) {
        const uint64_t other = __shfl_xor_sync(0xffffffffu, best, d);
        best = other > best ? other : best;
      }
      if ((uint32_t)(best >> 32) <= kLowest) break;   // nothing above minus infinity is left
      const int e = (int)~(uint32_t)best;
      const float v = row[e];
      if (k == 0) top = v;
      const float p = expf(v - top);
      chosen_sum += p;
      if (lane == (e & 31)) taken |= 1u << (e >> 5);
      if (lane == k) {
        my_id = e;
        mine = p;
      }
    }
    float total = chosen_sum;
    if (!a.renormalize) {
      total = 0.f;
      for (int e = lane; e < a.n_experts; e += 32) {
        const float v = row[e];
        total += v != v ? 0.f : expf(v - top);
      }
#pragma unroll
      for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
    }
    const float w = my_id >= 0 ? mine / total * a.routed_scale : 0.f;
    if (lane < a.top_k) {
      if (a.ids_out) a.ids_out[t * a.top_k + lane] = my_id;
      if (a.weights_out) a.weights_out[t * a.top_k + lane] = w;
    }
    int expert = -1;
    my_weight[half] = w;
    if (lane < a.top_k) expert = my_id;
    else if (lane < a.top_k + a.n_shared) {
      expert = a.n_experts + lane - a.top_k;
      my_weight[half] = 1.f;
    }
    int slot = expert >= 0 ? a.slot_of_expert[expert] : -1;
    if (slot >= a.n_slots) {
      if (a.status) *a.status = EMOE_ERR_PLACEMENT;
      slot = -1;
    }
    my_slot[half] = slot;
    if (slot >= 0) atomicOr(&s_tokens[slot], 1ull << t);
  }
  __syncthreads();

  // experts in use, in the order of their slots, and the number of pairs before each
  for (int first = 0; first < a.n_slots; first += kRouteThreads) {
    const int slot = first + threadIdx.x;
    const uint64_t tokens = slot < a.n_slots ? s_tokens[slot] : 0;
    int used = tokens != 0, pairs = __popcll(tokens), u = used, p = pairs;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int x = __shfl_up_sync(0xffffffffu, u, d), y = __shfl_up_sync(0xffffffffu, p, d);
      if (lane >= d) u += x, p += y;
    }
    if (lane == 31) s_scan[0][warp] = u, s_scan[1][warp] = p;
    __syncthreads();
    int before_u = s_total[0], before_p = s_total[1];
    for (int i = 0; i < warp; ++i) before_u += s_scan[0][i], before_p += s_scan[1][i];
    if (slot < a.n_slots) s_base[slot] = before_p + p - pairs;
    if (used) a.active[before_u + u - 1] = MoeActive{tokens, slot, before_p + p - pairs};
    __syncthreads();
    if (threadIdx.x == kRouteThreads - 1) s_total[0] = before_u + u, s_total[1] = before_p + p;
    __syncthreads();
  }
  if (threadIdx.x == 0) *a.n_active = s_total[0];
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    if (my_slot[half] < 0) continue;
    const int t = warp + 32 * half;
    const int at = s_base[my_slot[half]] + __popcll(s_tokens[my_slot[half]] & ((1ull << t) - 1));
    a.pair_token[at] = t;
    a.pair_weight[at] = my_weight[half];
  }
}

// ---- the weight stream --------------------------------------------------------------------

template <bool FP8> struct Block;           // of the k axis: four lanes' 16 bytes of a row
template <> struct Block<false> { static constexpr int kElems = 32, kProducts = 2; };
template <> struct Block<true> { static constexpr int kElems = 64, kProducts = 4; };

// Weight rows g and g + 8 of a block, 16 bytes each, as the 16-row operand of product j.
template <typename T, bool FP8>
__device__ __forceinline__ void weight_operand(uint32_t (&r)[4], const uint4 &lo, const uint4 &hi, int j) {
  if constexpr (FP8) {
    const uint32_t x = j == 0 ? lo.x : j == 1 ? lo.y : j == 2 ? lo.z : lo.w;
    const uint32_t y = j == 0 ? hi.x : j == 1 ? hi.y : j == 2 ? hi.z : hi.w;
    r[0] = even_codes<T>(x);
    r[1] = even_codes<T>(y);
    r[2] = odd_codes<T>(x);
    r[3] = odd_codes<T>(y);
  } else {
    r[0] = j ? lo.z : lo.x;
    r[1] = j ? hi.z : hi.x;
    r[2] = j ? lo.w : lo.y;
    r[3] = j ? hi.w : hi.y;
  }
}
// This lane's part of a token's block (16 or 32 bytes), and the operand of product j from it.
template <bool FP8> struct TokenPart { uint4 x; };
template <> struct TokenPart<true> { uint4 x, y; };
template <bool FP8>
__device__ __forceinline__ TokenPart<FP8> load_token(const uint8_t *p, bool there) {
  TokenPart<FP8> r = {};
  if (there) {
    r.x = *(const uint4 *)p;
    if constexpr (FP8) r.y = *(const uint4 *)(p + 16);
  }
  return r;
}
template <bool FP8>
__device__ __forceinline__ void token_operand(uint32_t &b0, uint32_t &b1, const TokenPart<FP8> &t, int j) {
  if constexpr (FP8) {   // the codes of a word come out as (0, 2) and (1, 3)
    const uint32_t lo = j == 0 ? t.x.x : j == 1 ? t.x.z : j == 2 ? t.y.x : t.y.z;
    const uint32_t hi = j == 0 ? t.x.y : j == 1 ? t.x.w : j == 2 ? t.y.y : t.y.w;
    b0 = __byte_perm(lo, hi, 0x5410);
    b1 = __byte_perm(lo, hi, 0x7632);
  } else {
    b0 = j ? t.x.z : t.x.x;
    b1 = j ? t.x.w : t.x.y;
  }
}

constexpr int kStages = 12;
constexpr int kStageBytes = 2 * 32 * 16;   // rows g and g + 8, 16 bytes a lane
constexpr int kRingBytes = kWarps * kStages * kStageBytes;

// One lane's ring.
struct Ring {
  uint8_t *base;
  uint32_t at;
  __device__ __forceinline__ explicit Ring(uint8_t *smem) {
    base = smem + (threadIdx.x >> 5) * (kStages * kStageBytes) + (threadIdx.x & 31) * 16;
    at = shared_address(base);
  }
  __device__ __forceinline__ void fill(int stage, const uint8_t *lo, const uint8_t *hi, bool there) {
    copy_async_16(at + stage * kStageBytes, lo, there ? 16 : 0);
    copy_async_16(at + stage * kStageBytes + 512, hi, there ? 16 : 0);
  }
  __device__ __forceinline__ uint4 lo(int stage) const { return *(const uint4 *)(base + stage * kStageBytes); }
  __device__ __forceinline__ uint4 hi(int stage) const { return *(const uint4 *)(base + stage * kStageBytes + 512); }
};

__device__ __forceinline__ MoeActive read_active(const MoeArgs &a, int i) {
  const longlong2 raw = __ldcg((const longlong2 *)(a.active + i));
  MoeActive r;
  r.tokens = (uint64_t)raw.x;
  r.slot = (int32_t)raw.y;
  r.base = (int32_t)(raw.y >> 32);
  return r;
}

// h[pair] = w silu(gate) up, rounded once to T.  NT: column tiles of 8 tokens that an expert may have.
// The k axis is split over the warps, joined in shared memory in the order of the warps.
template <typename T, bool FP8, int NT>
__global__ void __launch_bounds__(kWarps * 32) moe_up_kernel(const __grid_constant__ MoeArgs a) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float s_part[2][kWarps][16][9];
  constexpr int kElems = Block<FP8>::kElems, kES = FP8 ? 1 : 2;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  wait_for_previous();
  let_next_start();
  const int tiles = a.d_ff / 8;
  const int items = *a.n_active * tiles;
  const int blocks = (a.d_model + kElems - 1) / kElems;
  const int kb0 = blocks * warp / kWarps, kb1 = blocks * (warp + 1) / kWarps, steps = kb1 - kb0;
  const int64_t row_bytes = (int64_t)a.d_model * kES;
  const int lane_k = c * (16 / kES);   // this lane's first element inside a block

  Ring ring(smem);
  // the copies run ahead of the products over (item, block)
  int fill_item = blockIdx.x, fill_kb = kb0, fill_stage = 0;
  const uint8_t *fill_lo = nullptr, *fill_hi = nullptr;
  auto enter = [&](int item) {
    if (item >= items) return;
    const int slot = read_active(a, item / tiles).slot, row = (item % tiles) * 8 + g;
    fill_lo = a.gate + slot * a.gate_stride + row * row_bytes + c * 16;
    fill_hi = a.up + slot * a.gate_stride + row * row_bytes + c * 16;
  };
  auto fill = [&]() {
    if (steps && fill_item < items) {
      const int64_t off = (int64_t)fill_kb * (kElems * kES);
      const bool there = fill_kb * kElems + lane_k < a.d_model;
      ring.fill(fill_stage, there ? fill_lo + off : fill_lo, there ? fill_hi + off : fill_hi, there);
      if (++fill_kb == kb1) {
        fill_kb = kb0;
        fill_item += gridDim.x;
        enter(fill_item);
      }
    }
    copy_async_commit();
    fill_stage = fill_stage + 1 == kStages ? 0 : fill_stage + 1;
  };
  enter(fill_item);
  for (int i = 0; i < kStages - 1; ++i) fill();

  int stage = 0, buffer = 0;
  for (int item = blockIdx.x; item < items; item += gridDim.x) {
    const MoeActive e = read_active(a, item / tiles);
    const int count = __popcll(e.tokens), row0 = (item % tiles) * 8;
    const uint8_t *x[NT];
    float acc[NT][4] = {};
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int j = n * 8 + g;
      x[n] = j < count ? (const uint8_t *)a.x + (a.pair_token[e.base + j] * a.x_stride + lane_k) * 2 : nullptr;
    }
    const float *scale_g = nullptr, *scale_u = nullptr;
    if constexpr (FP8) {
      scale_g = a.gate_scale + (int64_t)e.slot * a.scale_stride + (row0 / 128) * ((a.d_model + 127) / 128);
      scale_u = a.up_scale + (int64_t)e.slot * a.scale_stride + (row0 / 128) * ((a.d_model + 127) / 128);
    }
    for (int kb = kb0; kb < kb1; ++kb) {
      fill();
      copy_async_wait<kStages - 1>();
      const uint4 lo = ring.lo(stage), hi = ring.hi(stage);
      stage = stage + 1 == kStages ? 0 : stage + 1;
      const bool there = kb * kElems + lane_k < a.d_model;
      float sg = 1.f, su = 1.f;
      if constexpr (FP8) {
        sg = scale_g[kb >> 1];
        su = scale_u[kb >> 1];
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        if (n && n * 8 >= count) break;
        const TokenPart<FP8> tp = load_token<FP8>(x[n] + (int64_t)kb * (kElems * 2), there && x[n]);
        float part[4] = {};
#pragma unroll
        for (int j = 0; j < Block<FP8>::kProducts; ++j) {
          uint32_t w[4], b0, b1;
          weight_operand<T, FP8>(w, lo, hi, j);
          token_operand<FP8>(b0, b1, tp, j);
          if constexpr (FP8) mma_16816<T>(part, w, b0, b1);
          else mma_16816<T>(acc[n], w, b0, b1);
        }
        if constexpr (FP8) {   // one scale for 128 of the k axis: two blocks
          acc[n][0] += part[0] * sg;
          acc[n][1] += part[1] * sg;
          acc[n][2] += part[2] * su;
          acc[n][3] += part[3] * su;
        }
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (n * 8 >= count) break;
      float(*part)[16][9] = s_part[buffer];
      buffer ^= 1;
      part[warp][g][2 * c] = acc[n][0];
      part[warp][g][2 * c + 1] = acc[n][1];
      part[warp][g + 8][2 * c] = acc[n][2];
      part[warp][g + 8][2 * c + 1] = acc[n][3];
      __syncthreads();   // the other buffer is written next: one barrier a tile is enough
      if (threadIdx.x < 64) {
        const int f = threadIdx.x & 7, j = threadIdx.x >> 3;
        float gate = 0.f, up = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          gate += part[w][f][j];
          up += part[w][f + 8][j];
        }
        if (n * 8 + j < count) {
          const int pair = e.base + n * 8 + j;
          float h = gate / (1.f + expf(-gate)) * up * a.pair_weight[pair];
          // f16 ends at 65504: the largest value stands for what is beyond (bf16 reaches as far as 32 bits)
          if constexpr (__is_same(T, __half)) h = fminf(fmaxf(h, -65504.f), 65504.f);
          ((T *)a.h)[(int64_t)pair * a.d_ff + row0 + f] = T(h);
        }
      }
    }
  }
  copy_async_wait<0>();
}

// y for 16 output rows a block: the (expert, block of k) steps of all experts in use are dealt to the
// warps in equal runs.  The columns are the tokens themselves, so that every expert adds to the same
// accumulators; column tiles without a token of the expert are left out.
template <typename T, bool FP8, int NT, bool F32_OUT>
__global__ void __launch_bounds__(kWarps * 32) moe_down_kernel(const __grid_constant__ MoeArgs a) {
  extern __shared__ __align__(128) uint8_t smem[];
  constexpr int kElems = Block<FP8>::kElems, kES = FP8 ? 1 : 2;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const int row0 = blockIdx.x * 16;
  const int blocks = (a.d_ff + kElems - 1) / kElems;
  const int64_t row_bytes = (int64_t)a.d_ff * kES;
  const int lane_k = c * (16 / kES);
  wait_for_previous();
  const int n_active = *a.n_active;
  const int64_t total = (int64_t)n_active * blocks;
  const int64_t s0 = total * warp / kWarps, s1 = total * (warp + 1) / kWarps;

  Ring ring(smem);
  int64_t fill_step = s0;
  int fill_expert = (int)(s0 / blocks), fill_kb = (int)(s0 % blocks), fill_stage = 0;
  const uint8_t *fill_lo = nullptr;
  auto enter = [&](int i) {
    if (i < n_active) fill_lo = a.down + read_active(a, i).slot * a.down_stride + (row0 + g) * row_bytes + c * 16;
  };
  auto fill = [&]() {
    if (fill_step < s1) {
      const bool there = fill_kb * kElems + lane_k < a.d_ff;
      const uint8_t *p = fill_lo + (there ? (int64_t)fill_kb * (kElems * kES) : 0);
      ring.fill(fill_stage, p, p + 8 * row_bytes, there);
      ++fill_step;
      if (++fill_kb == blocks) {
        fill_kb = 0;
        enter(++fill_expert);
      }
    }
    copy_async_commit();
    fill_stage = fill_stage + 1 == kStages ? 0 : fill_stage + 1;
  };
  enter(fill_expert);
  for (int i = 0; i < kStages - 1; ++i) fill();

  float acc[NT][4] = {};
  int expert = (int)(s0 / blocks), kb = (int)(s0 % blocks), stage = 0;
  uint64_t tokens = 0;
  const uint8_t *h[NT];
  const float *scale = nullptr;
  auto take = [&](int i) {
    const MoeActive e = read_active(a, i);
    tokens = e.tokens;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int t = n * 8 + g;
      const int pair = e.base + __popcll(tokens & ((1ull << t) - 1));
      h[n] = tokens >> t & 1 ? (const uint8_t *)a.h + ((int64_t)pair * a.d_ff + lane_k) * 2 : nullptr;
    }
    if constexpr (FP8) scale = a.down_scale + (int64_t)e.slot * a.scale_stride + (row0 / 128) * ((a.d_ff + 127) / 128);
  };
  if (s0 < s1) take(expert);
  for (int64_t s = s0; s < s1; ++s) {
    fill();
    copy_async_wait<kStages - 1>();
    const uint4 lo = ring.lo(stage), hi = ring.hi(stage);
    stage = stage + 1 == kStages ? 0 : stage + 1;
    const bool there = kb * kElems + lane_k < a.d_ff;
    float by = 1.f;
    if constexpr (FP8) by = scale[kb >> 1];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (!(tokens >> (n * 8) & 0xff)) continue;
      const TokenPart<FP8> tp = load_token<FP8>(h[n] + (int64_t)kb * (kElems * 2), there && h[n]);
      float part[4] = {};
#pragma unroll
      for (int j = 0; j < Block<FP8>::kProducts; ++j) {
        uint32_t w[4], b0, b1;
        weight_operand<T, FP8>(w, lo, hi, j);
        token_operand<FP8>(b0, b1, tp, j);
        if constexpr (FP8) mma_16816<T>(part, w, b0, b1);
        else mma_16816<T>(acc[n], w, b0, b1);
      }
      if constexpr (FP8) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[n][e] += part[e] * by;
      }
    }
    if (++kb == blocks) {
      kb = 0;
      if (s + 1 < s1) take(++expert);
    }
  }
  copy_async_wait<0>();
  __syncthreads();   // every warp is done with its ring: the sums meet there
  float *const sums = (float *)smem;   // [warp][token][row], 17 floats a token against bank conflicts
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int e = 0; e < 4; ++e)
      sums[(warp * (NT * 8) + n * 8 + 2 * c + (e & 1)) * 17 + g + 8 * (e >> 1)] = acc[n][e];
  __syncthreads();
  for (int i = threadIdx.x; i < NT * 8 * 16; i += kWarps * 32) {
    const int t = i >> 4, r = i & 15;
    if (t >= a.n_tokens) break;
    float y = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) y += sums[(w * (NT * 8) + t) * 17 + r];
    if constexpr (F32_OUT) ((float *)a.out)[t * a.out_stride + row0 + r] = y;
    else ((T *)a.out)[t * a.out_stride + row0 + r] = T(y);
  }
}

template <typename K>
cudaError_t launch(K kernel, unsigned grid, int threads, size_t smem, bool early, const MoeArgs &a, cudaStream_t st) {
  if (smem > 40 * 1024) {   // with the static part more than a launch may have unasked
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
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

template <typename T, bool FP8, int NT>
cudaError_t launch_layer(const MoeArgs &a, bool f32_out, cudaStream_t st) {
  cudaError_t e = launch(moe_route_kernel, 1, kRouteThreads, (size_t)a.n_slots * 12, false, a, st);
  if (e != cudaSuccess) return e;
  const int64_t pairs = (int64_t)a.n_tokens * (a.top_k + a.n_shared);
  const int64_t most = (pairs < a.n_slots ? pairs : a.n_slots) * (a.d_ff / 8);
  e = launch(moe_up_kernel<T, FP8, NT>, (unsigned)(most < 2 * kSms ? most : 2 * kSms), kWarps * 32, kRingBytes, true, a, st);
  if (e != cudaSuccess) return e;
  constexpr size_t sums = (size_t)kWarps * NT * 8 * 17 * 4;
  constexpr size_t smem = sums > kRingBytes ? sums : kRingBytes;
  return f32_out ? launch(moe_down_kernel<T, FP8, NT, true>, a.d_model / 16, kWarps * 32, smem, true, a, st)
                 : launch(moe_down_kernel<T, FP8, NT, false>, a.d_model / 16, kWarps * 32, smem, true, a, st);
}

template <typename T, bool FP8>
cudaError_t by_tokens(const MoeArgs &a, bool f32_out, cudaStream_t st) {
  if (a.n_tokens <= 8) return launch_layer<T, FP8, 1>(a, f32_out, st);
  if (a.n_tokens <= 16) return launch_layer<T, FP8, 2>(a, f32_out, st);
  if (a.n_tokens <= 32) return launch_layer<T, FP8, 4>(a, f32_out, st);
  return launch_layer<T, FP8, 8>(a, f32_out, st);
}

}  // namespace

MoeShape moe_shape(int n_slots, int d_ff, int n_tokens, int top_k, int n_shared) {
  MoeShape s{};
  const int64_t pairs = (int64_t)n_tokens * (top_k + n_shared), most = pairs < n_slots ? pairs : n_slots;
  const auto up = [](int64_t n) { return (n + 255) / 256 * 256; };
  s.active = 256;                       // the number of experts in use lies at the start
  s.token = s.active + up(most * (int64_t)sizeof(MoeActive));
  s.weight = s.token + up(pairs * 4);
  s.h = s.weight + up(pairs * 4);
  s.bytes = s.h + up(pairs * d_ff * 2);
  return s;
}

cudaError_t launch_moe(const MoeArgs &a, int type, int io, bool f32_out, cudaStream_t st) {
  if (type == EMOE_TYPE_E4M3)
    return io == EMOE_TYPE_BF16 ? by_tokens<__nv_bfloat16, true>(a, f32_out, st) : by_tokens<__half, true>(a, f32_out, st);
  return io == EMOE_TYPE_BF16 ? by_tokens<__nv_bfloat16, false>(a, f32_out, st) : by_tokens<__half, false>(a, f32_out, st);
}

}  // namespace emoe
