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

constexpr int kRouteThreads = 1024, kUpWarps = 8;

// Logits as unsigned numbers in the same order; NaN counts as minus infinity, and minus infinity and
// what has been chosen already as 0.
__device__ __forceinline__ uint32_t ordered(float v) {
  if (!(v > -CUDART_INF_F)) return 0;
  const uint32_t b = __float_as_uint(v);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

// One block.  A warp takes tokens warp and warp + 32: its lanes hold the token's logits in registers,
// each choice is a maximum over the lanes and then the smallest index that has it.  N: experts a lane.
template <int N>
__global__ void __launch_bounds__(kRouteThreads) moe_route_kernel(const __grid_constant__ MoeArgs a) {
  extern __shared__ unsigned long long s_tokens[];   // [n_slots]: which tokens an expert has
  int32_t *const s_base = (int32_t *)(s_tokens + a.n_slots);
  __shared__ int32_t s_scan[2][32];
  __shared__ int32_t s_total[2];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  let_next_start();
  for (int i = threadIdx.x; i < a.n_slots; i += kRouteThreads) s_tokens[i] = 0;
  if (threadIdx.x < 2) s_total[threadIdx.x] = 0;
  __syncthreads();

  int my_slot[2] = {-1, -1};   // of pair number `lane` (routed, then shared) of the two tokens
  float my_weight[2] = {};
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int t = warp + 32 * half;
    if (t >= a.n_tokens) continue;
    const float *row = a.logits + t * a.logits_stride;
    uint32_t key[N];
#pragma unroll
    for (int j = 0; j < N; ++j) key[j] = j * 32 + lane < a.n_experts ? ordered(row[j * 32 + lane]) : 0;
    float total = 0.f, top = 0.f, mine = 0.f;
    int my_id = -1;
    if (!a.renormalize) {
      uint32_t best = 0;
#pragma unroll
      for (int j = 0; j < N; ++j) best = max(best, key[j]);
      top = value_of(__reduce_max_sync(0xffffffffu, best));
#pragma unroll
      for (int j = 0; j < N; ++j) total += key[j] ? expf(value_of(key[j]) - top) : 0.f;
#pragma unroll
      for (int d = 16; d; d >>= 1) total += __shfl_xor_sync(0xffffffffu, total, d);
    }
    for (int k = 0; k < a.top_k; ++k) {
      uint32_t best = 0;
#pragma unroll
      for (int j = 0; j < N; ++j) best = max(best, key[j]);
      best = __reduce_max_sync(0xffffffffu, best);
      if (best == 0) break;   // nothing above minus infinity is left
      uint32_t e = 0xffffffffu;
#pragma unroll
      for (int j = N - 1; j >= 0; --j)
        if (key[j] == best) e = j * 32 + lane;
      e = __reduce_min_sync(0xffffffffu, e);
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (e == (uint32_t)(j * 32 + lane)) key[j] = 0;
      const float v = value_of(best);
      if (k == 0) top = v;
      const float p = expf(v - top);
      if (a.renormalize) total += p;
      if (lane == k) {
        my_id = (int)e;
        mine = p;
      }
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
    const int pairs = slot < a.n_slots ? __popcll(s_tokens[slot]) : 0, used = pairs != 0;
    int u = used, p = pairs;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int x = __shfl_up_sync(0xffffffffu, u, d), y = __shfl_up_sync(0xffffffffu, p, d);
      if (lane >= d) u += x, p += y;
    }
    if (lane == 31) s_scan[0][warp] = u, s_scan[1][warp] = p;
    __syncthreads();
    const int below = lane < warp ? -1 : 0;
    u += __reduce_add_sync(0xffffffffu, s_scan[0][lane] & below) + s_total[0];
    p += __reduce_add_sync(0xffffffffu, s_scan[1][lane] & below) + s_total[1];
    if (slot < a.n_slots) s_base[slot] = p - pairs;
    if (used) a.active[u - 1] = make_int2(slot, p - pairs);
    __syncthreads();
    if (threadIdx.x == kRouteThreads - 1) s_total[0] = u, s_total[1] = p;
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    *a.n_active = s_total[0];
    a.active[s_total[0]] = make_int2(-1, s_total[1]);   // the end of the last expert's pairs
  }
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

// A block of the k axis: 16 bytes of weights a lane and row, four lanes a row; kTok 16-byte parts of the
// matching token elements a lane.
template <bool FP8> struct Block {
  static constexpr int kElems = FP8 ? 64 : 32, kProducts = FP8 ? 4 : 2, kTok = FP8 ? 2 : 1, kES = FP8 ? 1 : 2;
  static constexpr int kStageBytes = (2 + kTok) * 512;
};

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
// This lane's part of a token's block, and the operand of product j from it.
template <bool FP8> struct TokenPart { uint4 v[Block<FP8>::kTok]; };
template <bool FP8>
__device__ __forceinline__ void token_operand(uint32_t &b0, uint32_t &b1, const TokenPart<FP8> &t, int j) {
  if constexpr (FP8) {   // the codes of a word come out as (0, 2) and (1, 3)
    const uint4 &v = t.v[j >> 1];
    const uint32_t lo = j & 1 ? v.z : v.x, hi = j & 1 ? v.w : v.y;
    b0 = __byte_perm(lo, hi, 0x5410);
    b1 = __byte_perm(lo, hi, 0x7632);
  } else {
    b0 = j ? t.v[0].z : t.v[0].x;
    b1 = j ? t.v[0].w : t.v[0].y;
  }
}
template <bool FP8>
__device__ __forceinline__ TokenPart<FP8> load_token(const uint8_t *p, bool there) {
  TokenPart<FP8> r = {};
  if (there) {
#pragma unroll
    for (int i = 0; i < Block<FP8>::kTok; ++i) r.v[i] = ((const uint4 *)p)[i];
  }
  return r;
}

// One lane's ring: what it copies there it reads back itself.
template <bool FP8, int STAGES>
struct Ring {
  static constexpr int kStage = Block<FP8>::kStageBytes;
  uint8_t *base;
  uint32_t at;
  __device__ __forceinline__ explicit Ring(uint8_t *smem) {
    base = smem + (threadIdx.x >> 5) * (STAGES * kStage) + (threadIdx.x & 31) * 16;
    at = shared_address(base);
  }
  __device__ __forceinline__ void fill(int stage, const uint8_t *lo, const uint8_t *hi, const uint8_t *tok, bool there, bool tok_there) {
    const uint32_t dst = at + stage * kStage;
    copy_async_16(dst, lo, there ? 16 : 0);
    copy_async_16(dst + 512, hi, there ? 16 : 0);
#pragma unroll
    for (int i = 0; i < Block<FP8>::kTok; ++i) copy_async_16(dst + 1024 + i * 512, tok + i * 16, tok_there ? 16 : 0);
  }
  __device__ __forceinline__ uint4 lo(int stage) const { return *(const uint4 *)(base + stage * kStage); }
  __device__ __forceinline__ uint4 hi(int stage) const { return *(const uint4 *)(base + stage * kStage + 512); }
  __device__ __forceinline__ TokenPart<FP8> token(int stage) const {
    TokenPart<FP8> r;
#pragma unroll
    for (int i = 0; i < Block<FP8>::kTok; ++i) r.v[i] = *(const uint4 *)(base + stage * kStage + 1024 + i * 512);
    return r;
  }
};

// acc += weights x tokens over one block; e4m3 blocks come with the scales of rows g and g + 8.
template <typename T, bool FP8>
__device__ __forceinline__ void block_product(float (&acc)[4], const uint4 &lo, const uint4 &hi, const TokenPart<FP8> &tok,
                                              float scale_lo, float scale_hi) {
  float part[4] = {};
#pragma unroll
  for (int j = 0; j < Block<FP8>::kProducts; ++j) {
    uint32_t w[4], b0, b1;
    weight_operand<T, FP8>(w, lo, hi, j);
    token_operand<FP8>(b0, b1, tok, j);
    if constexpr (FP8) mma_16816<T>(part, w, b0, b1);
    else mma_16816<T>(acc, w, b0, b1);
  }
  if constexpr (FP8) {
    acc[0] += part[0] * scale_lo;
    acc[1] += part[1] * scale_lo;
    acc[2] += part[2] * scale_hi;
    acc[3] += part[3] * scale_hi;
  }
}

// What the routing found, in shared memory: (slot, first pair) of each expert in use and one more
// entry for the end, and each pair's token.
struct Routed {
  int2 *active;
  uint8_t *token;
  int n_active;
  __device__ __forceinline__ void read(const MoeArgs &a, uint8_t *at) {
    n_active = __ldcg(a.n_active);
    active = (int2 *)at;
    for (int i = threadIdx.x; i <= n_active; i += blockDim.x) active[i] = __ldcg(a.active + i);
    __syncthreads();
    token = at + (n_active + 1) * 8;
    const int pairs = active[n_active].y;
    for (int i = threadIdx.x; i < pairs; i += blockDim.x) token[i] = (uint8_t)__ldcg(a.pair_token + i);
    __syncthreads();
  }
};
int routed_bytes(const MoeArgs &a) {
  const int pairs = a.n_tokens * (a.top_k + a.n_shared);
  return ((pairs < a.n_slots ? pairs : a.n_slots) + 1) * 8 + pairs;
}

// h[pair] = w silu(gate) up, rounded once to T.  An item is 8 rows of gate and the same 8 of up as one
// 16-row operand, so a thread gets both sums of its outputs.  The k axis is split over the warps,
// joined in shared memory in the order of the warps.  NT: column tiles of 8 tokens an expert may have;
// the first comes through the ring, the others (more than 8 tokens of one expert) straight from L2.
template <typename T, bool FP8, int NT, int STAGES>
__global__ void __launch_bounds__(kUpWarps * 32) moe_up_kernel(const __grid_constant__ MoeArgs a) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float s_part[2][kUpWarps][16][9];
  using B = Block<FP8>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  wait_for_previous();
  let_next_start();
  Routed routed;
  routed.read(a, smem + kUpWarps * STAGES * B::kStageBytes);
  const int tiles = a.d_ff / 8;
  const int items = routed.n_active * tiles;
  const int blocks = (a.d_model + B::kElems - 1) / B::kElems;
  const int kb0 = blocks * warp / kUpWarps, kb1 = blocks * (warp + 1) / kUpWarps;
  const int64_t row_bytes = (int64_t)a.d_model * B::kES;
  const int lane_k = c * (16 / B::kES);   // this lane's first element inside a block
  const uint8_t *const x_lane = (const uint8_t *)a.x + lane_k * 2;

  Ring<FP8, STAGES> ring(smem);
  // the copies run ahead of the products over (item, block)
  int fill_item = kb0 < kb1 ? blockIdx.x : items, fill_kb = kb0, fill_stage = 0;
  const uint8_t *fill_lo = nullptr, *fill_hi = nullptr, *fill_tok = nullptr;
  bool fill_col = false;
  auto enter = [&]() {
    if (fill_item >= items) return;
    const int i = fill_item / tiles, row = (fill_item - i * tiles) * 8 + g;
    const int2 e = routed.active[i];
    fill_lo = a.gate + e.x * a.gate_stride + row * row_bytes + c * 16;
    fill_hi = a.up + e.x * a.gate_stride + row * row_bytes + c * 16;
    fill_col = g < routed.active[i + 1].y - e.y;
    fill_tok = fill_col ? x_lane + routed.token[e.y + g] * a.x_stride * 2 : x_lane;
  };
  auto fill = [&]() {
    if (fill_item < items) {
      const bool there = fill_kb * B::kElems + lane_k < a.d_model;
      const int off = there ? fill_kb * 64 : 0;
      ring.fill(fill_stage, fill_lo + off, fill_hi + off, fill_tok + off * B::kTok, there, there && fill_col);
      if (++fill_kb == kb1) {
        fill_kb = kb0;
        fill_item += gridDim.x;
        enter();
      }
    }
    copy_async_commit();
    fill_stage = fill_stage + 1 == STAGES ? 0 : fill_stage + 1;
  };
  enter();
  for (int i = 0; i < STAGES - 1; ++i) fill();

  int stage = 0, buffer = 0;
  for (int item = blockIdx.x; item < items; item += gridDim.x) {
    const int i = item / tiles, row0 = (item - i * tiles) * 8;
    const int2 e = routed.active[i];
    const int count = routed.active[i + 1].y - e.y;
    float acc[NT][4] = {};
    const uint8_t *more[NT];   // this lane's column of the further tiles
#pragma unroll
    for (int n = 1; n < NT; ++n)
      more[n] = n * 8 + g < count ? x_lane + routed.token[e.y + n * 8 + g] * a.x_stride * 2 : nullptr;
    const float *scale_g = nullptr, *scale_u = nullptr;
    float sg = 1.f, su = 1.f;
    if constexpr (FP8) {
      const int64_t at = e.x * a.scale_stride + (row0 / 128) * ((a.d_model + 127) / 128);
      scale_g = a.gate_scale + at;
      scale_u = a.up_scale + at;
      if (kb0 < kb1) {
        sg = scale_g[kb0 >> 1];
        su = scale_u[kb0 >> 1];
      }
    }
    for (int kb = kb0; kb < kb1; ++kb) {
      fill();
      float next_g = 1.f, next_u = 1.f;
      if constexpr (FP8) {   // one scale for two blocks, read a block ahead
        if (kb + 1 < kb1) {
          next_g = scale_g[(kb + 1) >> 1];
          next_u = scale_u[(kb + 1) >> 1];
        }
      }
      copy_async_wait<STAGES - 1>();
      const uint4 lo = ring.lo(stage), hi = ring.hi(stage);
      block_product<T, FP8>(acc[0], lo, hi, ring.token(stage), sg, su);
      stage = stage + 1 == STAGES ? 0 : stage + 1;
      if (NT > 1 && count > 8) {
        const bool there = kb * B::kElems + lane_k < a.d_model;
        const int64_t off = (int64_t)kb * (B::kElems * 2);
#pragma unroll
        for (int n = 1; n < NT; n += 2) {
          if (n * 8 >= count) break;
          const TokenPart<FP8> x0 = load_token<FP8>(more[n] + off, there && more[n]);
          const TokenPart<FP8> x1 = load_token<FP8>(more[n + 1 < NT ? n + 1 : n] + off, n + 1 < NT && there && more[n + 1 < NT ? n + 1 : n]);
          block_product<T, FP8>(acc[n], lo, hi, x0, sg, su);
          if (n + 1 < NT) block_product<T, FP8>(acc[n + 1 < NT ? n + 1 : n], lo, hi, x1, sg, su);
        }
      }
      sg = next_g;
      su = next_u;
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
        for (int w = 0; w < kUpWarps; ++w) {
          gate += part[w][f][j];
          up += part[w][f + 8][j];
        }
        if (n * 8 + j < count) {
          const int pair = e.y + n * 8 + j;
          float h = gate / (1.f + expf(-gate)) * up * a.pair_weight[pair];
          // f16 ends at 65504: the largest value stands for what is beyond (bf16 reaches as far as 32 bits)
          if constexpr (__is_same(T, __half)) h = h != h ? h : fminf(fmaxf(h, -65504.f), 65504.f);
          ((T *)a.h)[(int64_t)pair * a.d_ff + row0 + f] = T(h);
        }
      }
    }
  }
  copy_async_wait<0>();
}

// y for 16 output rows a block: the (expert, block of k) steps of all experts in use are dealt to the
// warps in equal runs.  At the end of its part of an expert a warp adds the expert's columns to its
// own sums of the tokens in shared memory; the warps' sums are joined at the end, in their order.
template <typename T, bool FP8, int NT, int STAGES, int WARPS, bool F32_OUT>
__global__ void __launch_bounds__(WARPS * 32) moe_down_kernel(const __grid_constant__ MoeArgs a) {
  extern __shared__ __align__(128) uint8_t smem[];
  using B = Block<FP8>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  const int row0 = blockIdx.x * 16;
  const int blocks = (a.d_ff + B::kElems - 1) / B::kElems;
  const int64_t row_bytes = (int64_t)a.d_ff * B::kES;
  const int lane_k = c * (16 / B::kES);
  float *const sums = (float *)(smem + WARPS * STAGES * B::kStageBytes);   // [warp][token][17]
  for (int i = threadIdx.x; i < WARPS * a.n_tokens * 17; i += WARPS * 32) sums[i] = 0.f;
  wait_for_previous();
  Routed routed;
  routed.read(a, (uint8_t *)(sums + (WARPS * a.n_tokens * 17 + 3) / 4 * 4));
  const int total = routed.n_active * blocks;   // at most 4096 experts x 32768 blocks
  const int s0 = (int)((int64_t)total * warp / WARPS), s1 = (int)((int64_t)total * (warp + 1) / WARPS);
  const uint8_t *const h_lane = (const uint8_t *)a.h + lane_k * 2;

  Ring<FP8, STAGES> ring(smem);
  int fill_step = s0, fill_expert = s0 / blocks, fill_kb = s0 - fill_expert * blocks, fill_stage = 0;
  const uint8_t *fill_lo = nullptr, *fill_tok = nullptr;
  bool fill_col = false;
  auto enter = [&]() {
    if (fill_expert >= routed.n_active) return;
    const int2 e = routed.active[fill_expert];
    fill_lo = a.down + e.x * a.down_stride + (row0 + g) * row_bytes + c * 16;
    fill_col = g < routed.active[fill_expert + 1].y - e.y;
    fill_tok = h_lane + (fill_col ? (int64_t)(e.y + g) * a.d_ff * 2 : 0);
  };
  auto fill = [&]() {
    if (fill_step < s1) {
      const bool there = fill_kb * B::kElems + lane_k < a.d_ff;
      const int off = there ? fill_kb * 64 : 0;
      ring.fill(fill_stage, fill_lo + off, fill_lo + 8 * row_bytes + off, fill_tok + off * B::kTok, there, there && fill_col);
      ++fill_step;
      if (++fill_kb == blocks) {
        fill_kb = 0;
        ++fill_expert;
        enter();
      }
    }
    copy_async_commit();
    fill_stage = fill_stage + 1 == STAGES ? 0 : fill_stage + 1;
  };
  enter();
  for (int i = 0; i < STAGES - 1; ++i) fill();

  int stage = 0, s = s0;
  for (int expert = s0 / blocks; s < s1; ++expert) {
    const int2 e = routed.active[expert];
    const int count = routed.active[expert + 1].y - e.y;
    const int first = s - expert * blocks, last = min(blocks, s1 - expert * blocks);
    s += last - first;
    const float *scale = nullptr;
    float by = 1.f;
    if constexpr (FP8) {
      scale = a.down_scale + (int64_t)e.x * a.scale_stride + (row0 / 128) * ((a.d_ff + 127) / 128);
      by = scale[first >> 1];
    }
    const uint8_t *const h0 = h_lane + (int64_t)(e.y + g) * a.d_ff * 2;
    float acc[NT][4] = {};
    for (int kb = first; kb < last; ++kb) {
      fill();
      float next = 1.f;
      if constexpr (FP8) {
        if (kb + 1 < last) next = scale[(kb + 1) >> 1];
      }
      copy_async_wait<STAGES - 1>();
      const uint4 lo = ring.lo(stage), hi = ring.hi(stage);
      block_product<T, FP8>(acc[0], lo, hi, ring.token(stage), by, by);
      stage = stage + 1 == STAGES ? 0 : stage + 1;
      if (NT > 1 && count > 8) {
        const bool there = kb * B::kElems + lane_k < a.d_ff;
        const uint8_t *const p = h0 + (int64_t)kb * (B::kElems * 2);
#pragma unroll
        for (int n = 1; n < NT; n += 2) {
          if (n * 8 >= count) break;
          const TokenPart<FP8> x0 = load_token<FP8>(p + (int64_t)n * 8 * a.d_ff * 2, there && n * 8 + g < count);
          const TokenPart<FP8> x1 = load_token<FP8>(p + (int64_t)(n + 1) * 8 * a.d_ff * 2, n + 1 < NT && there && (n + 1) * 8 + g < count);
          block_product<T, FP8>(acc[n], lo, hi, x0, by, by);
          if (n + 1 < NT) block_product<T, FP8>(acc[n + 1 < NT ? n + 1 : n], lo, hi, x1, by, by);
        }
      }
      by = next;
    }
    float *const mine = sums + warp * a.n_tokens * 17;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (n * 8 >= count) break;
#pragma unroll
      for (int k = 0; k < 2; ++k) {   // columns 2c and 2c + 1: no two lanes have the same token and row
        const int j = n * 8 + 2 * c + k;
        if (j < count) {
          float *const y = mine + routed.token[e.y + j] * 17;
          y[g] += acc[n][k];
          y[g + 8] += acc[n][2 + k];
        }
      }
    }
    __syncwarp();   // the next expert may have the same tokens in other lanes
  }
  copy_async_wait<0>();
  __syncthreads();
  for (int i = threadIdx.x; i < a.n_tokens * 16; i += WARPS * 32) {
    const int t = i >> 4, r = i & 15;
    float y = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) y += sums[(w * a.n_tokens + t) * 17 + r];
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

template <typename T, bool FP8, int NT, int STAGES, int WARPS>
cudaError_t launch_down(const MoeArgs &a, bool f32_out, cudaStream_t st) {
  const size_t smem = (size_t)WARPS * STAGES * Block<FP8>::kStageBytes + (size_t)(WARPS * a.n_tokens * 17 + 3) / 4 * 16 + routed_bytes(a);
  return f32_out ? launch(moe_down_kernel<T, FP8, NT, STAGES, WARPS, true>, a.d_model / 16, WARPS * 32, smem, true, a, st)
                 : launch(moe_down_kernel<T, FP8, NT, STAGES, WARPS, false>, a.d_model / 16, WARPS * 32, smem, true, a, st);
}

template <typename T, bool FP8, int NT>
cudaError_t launch_layer(const MoeArgs &a, bool f32_out, cudaStream_t st) {
  cudaError_t e = a.n_experts <= 256 ? launch(moe_route_kernel<8>, 1, kRouteThreads, (size_t)a.n_slots * 12, false, a, st)
                                     : launch(moe_route_kernel<32>, 1, kRouteThreads, (size_t)a.n_slots * 12, false, a, st);
  if (e != cudaSuccess) return e;
  constexpr int kStages = FP8 ? 6 : 8;   // 96 KB: two blocks an SM
  const int64_t pairs = (int64_t)a.n_tokens * (a.top_k + a.n_shared);
  const int64_t most = (pairs < a.n_slots ? pairs : a.n_slots) * (a.d_ff / 8);
  e = launch(moe_up_kernel<T, FP8, NT, kStages>, (unsigned)(most < 2 * kSms ? most : 2 * kSms), kUpWarps * 32,
             (size_t)kUpWarps * kStages * Block<FP8>::kStageBytes + routed_bytes(a), true, a, st);
  if (e != cudaSuccess) return e;
  // Up to about one block an SM: 8 warps each; more: 4 warps, four blocks an SM, all of them at once.
  if (a.d_model / 16 <= kSms) return launch_down<T, FP8, NT, FP8 ? 8 : 10, 8>(a, f32_out, st);
  return launch_down<T, FP8, NT, FP8 ? 5 : 6, 4>(a, f32_out, st);
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
  s.token = s.active + up((most + 1) * 8);
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
