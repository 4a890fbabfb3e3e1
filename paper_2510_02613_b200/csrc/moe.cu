// moe.cu - a whole mixture-of-experts layer for a few tokens: routing, gate and up products,
// activation, down product, weighted sum.
//
//   y_t = sum over the experts e chosen by t of w_te * Wd_e (silu(Wg_e x_t) * (Wu_e x_t))
//
// With a few tokens the layer is bound by reading the chosen experts' weights once, so everything
// is arranged around that stream: each lane owns a ring of 16-byte slots in shared memory that it
// fills with asynchronous copies and reads back itself (no barrier between a warp's copies and its
// use of them), weights are the 16-row side of the tensor-core product straight from those slots,
// tokens its 8-column side, and the order of the k axis inside a step is the order in which the
// slots hold it.  Three launches, chained so that each one's prologue overlaps the tail of the one before:
//   route: a block a token; top-k and softmax by one warp
//   up:    items of 8 gate and 8 up rows of one expert (one product gives both, in the same thread)
//   down:  16 rows of the output over ALL experts in use: the tokens' sums stay in shared memory, in
//          the order of the slots - no partial results in memory, no atomics.
#include <math_constants.h>

#include "convert.cuh"
#include "serve.h"

namespace emoe {
namespace {

constexpr int kRouteThreads = 256, kUpWarps = 8;
constexpr size_t kMaxShared = 226 * 1024;   // of 227 KB: a kernel's own variables have the rest

// Where element k of a token lies in the order that moved e4m3 operands want.
__device__ __forceinline__ int moved_place(int k) { return (k & ~3) | (k & 1) << 1 | (k & 2) >> 1; }

// The gate and up products of an e4m3 arena run on f16 operands whatever the type of x: cvt widens four
// codes in two instructions (to bf16 it takes seven, on a pipe half as wide).  bf16 tokens are brought to f16 by the
// power of two that puts their largest element below 2^15 - exact but for elements 2^29 times smaller, whose
// error is far below that of a 32-bit sum.  The hidden vectors'
// largest element is not known when they are written, so the down product keeps them in bf16.
template <typename IO, bool FP8> struct UpOperand { using type = IO; };
template <typename IO> struct UpOperand<IO, true> { using type = __half; };

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

// A block a token.  The first warp holds the token's logits in registers, N experts a lane; each
// choice is a maximum over the lanes and then the smallest index that has it.  The other warps bring a bf16
// token to f16 where the weights are e4m3.  Bound by latency: 4 to 7 us, most of it under the next kernel's start.
template <int N, bool MOVED>
__global__ void __launch_bounds__(kRouteThreads) moe_route_kernel(const __grid_constant__ MoeArgs a) {
  const int t = blockIdx.x, lane = threadIdx.x & 31;
  let_next_start();
  if (threadIdx.x >= 32) {
    if constexpr (MOVED) {
      __shared__ uint32_t s_top[kRouteThreads / 32];
      const uint2 *const x = (const uint2 *)((const __nv_bfloat16 *)a.x + t * a.x_stride);
      uint2 *const to = (uint2 *)((__half *)a.moved_x + (int64_t)t * a.d_model);
      constexpr int kThreads = kRouteThreads - 32;
      uint32_t top = 0;   // two magnitudes a word compare as their bits do
      for (int i = threadIdx.x - 32; i < a.d_model / 4; i += kThreads) {
        const uint2 w = x[i];
        top = __vmaxu2(top, __vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu));
      }
      top = __reduce_max_sync(0xffffffffu, max(top >> 16, top & 0xffffu));
      if (lane == 0) s_top[threadIdx.x >> 5] = top;
      asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory");
      for (int i = 1; i < kRouteThreads / 32; ++i) top = max(top, s_top[i]);
      // 2^(14 - exponent); 1 for a zero token and one that is not finite
      const uint32_t e = top >> 7;
      const float by = top == 0 || e == 255 ? 1.f : __uint_as_float((uint32_t)min(254, 268 - max(1, (int)e)) << 23);
      for (int i = threadIdx.x - 32; i < a.d_model / 4; i += kThreads) {
        const uint2 w = x[i];
        const float2 p = Pair<__nv_bfloat16>::unpack(w.x), q = Pair<__nv_bfloat16>::unpack(w.y);
        to[i] = make_uint2(Pair<__half>::pack(p.x * by, p.y * by), Pair<__half>::pack(q.x * by, q.y * by));
      }
      if (threadIdx.x == 32) a.token_scale[t] = 1.f / by;
    }
    return;
  }
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
  float w = my_id >= 0 ? mine / total * a.routed_scale : 0.f;
  if (lane < a.top_k) {
    if (a.ids_out) a.ids_out[t * a.top_k + lane] = my_id;
    if (a.weights_out) a.weights_out[t * a.top_k + lane] = w;
  }
  const int chosen = a.top_k + a.n_shared;
  if (lane >= chosen) return;
  int expert = my_id;
  if (lane >= a.top_k) {
    expert = a.n_experts + lane - a.top_k;
    w = 1.f;
  }
  int slot = expert >= 0 ? a.slot_of_expert[expert] : -1;
  if (slot >= a.n_slots) {
    if (a.status) *a.status = EMOE_ERR_PLACEMENT;
    slot = -1;
  }
  a.choice[t * chosen + lane] = make_int2(slot < 0 ? -1 : slot, __float_as_int(w));
}

template <bool FP8, int NT> __device__ __forceinline__ int stages_of(int count);

// The choices grouped by expert, built by each block for itself: (slot, first pair) of each expert in
// use in the order of the slots, one more entry for the end, and each pair's token and weight, in the
// order of the tokens.  `scratch` is free again afterwards.
struct Routed {
  int2 *active;
  float *weight;
  uint8_t *token;
  int n_active;

  __device__ __forceinline__ void build(const MoeArgs &a, uint8_t *at, uint8_t *scratch) {
    __shared__ int s_scan[2][32], s_total[2];
    unsigned long long *const tokens = (unsigned long long *)scratch;   // [n_slots]
    int *const base = (int *)(tokens + a.n_slots);                      // [n_slots]
    const int chosen = a.top_k + a.n_shared, pairs = a.n_tokens * chosen;
    const int most = min(pairs, a.n_slots);
    active = (int2 *)at;
    weight = (float *)(active + most + 1);
    token = (uint8_t *)(weight + pairs);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    for (int i = threadIdx.x; i < a.n_slots; i += blockDim.x) tokens[i] = 0;
    if (threadIdx.x < 2) s_total[threadIdx.x] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < pairs; i += blockDim.x) {
      const int slot = __ldcg(&a.choice[i].x);
      if (slot < 0) continue;
      const unsigned long long bit = 1ull << (i / chosen);
      if ((atomicOr(&tokens[slot], bit) & bit) && a.status) *a.status = EMOE_ERR_PLACEMENT;   // one slot for two experts
    }
    __syncthreads();
    for (int first = 0; first < a.n_slots; first += blockDim.x) {
      const int slot = first + threadIdx.x;
      const int n = slot < a.n_slots ? __popcll(tokens[slot]) : 0, used = n != 0;
      int u = used, p = n;
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const int x = __shfl_up_sync(0xffffffffu, u, d), y = __shfl_up_sync(0xffffffffu, p, d);
        if (lane >= d) u += x, p += y;
      }
      if (lane == 31) s_scan[0][warp] = u, s_scan[1][warp] = p;
      __syncthreads();
      for (int i = 0; i < warp; ++i) u += s_scan[0][i], p += s_scan[1][i];
      u += s_total[0];
      p += s_total[1];
      if (slot < a.n_slots) base[slot] = p - n;
      if (used) active[u - 1] = make_int2(slot, p - n);
      __syncthreads();
      if (warp == warps - 1 && lane == 31) s_total[0] = u, s_total[1] = p;
      __syncthreads();
    }
    n_active = s_total[0];
    if (threadIdx.x == 0) active[n_active] = make_int2(-1, s_total[1]);
    for (int i = threadIdx.x; i < pairs; i += blockDim.x) {
      const int2 c = __ldcg(a.choice + i);
      if (c.x < 0) continue;
      const int t = i / chosen, pair = base[c.x] + __popcll(tokens[c.x] & ((1ull << t) - 1));
      token[pair] = (uint8_t)t;
      weight[pair] = __int_as_float(c.y);
    }
    __syncthreads();
  }

  // The step - of all experts' steps in a row - at which share `i` of `n` equal shares begins, equal in the
  // stages that the steps take.
  template <bool FP8, int NT>
  __device__ __forceinline__ int share(int steps, int i, int n) const {
    if constexpr (NT == 1) return (int)((int64_t)n_active * steps * i / n);
    const int lane = threadIdx.x & 31;
    int parts = 0;
    for (int e = lane; e < n_active; e += 32) parts += stages_of<FP8, NT>(active[e + 1].y - active[e].y);
    int64_t target = (int64_t)__reduce_add_sync(0xffffffffu, parts) * steps * i / n;
    for (int first = 0; first < n_active; first += 32) {
      const int e = first + lane, own = e < n_active ? stages_of<FP8, NT>(active[e + 1].y - active[e].y) : 0;
      int sum = own;
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const int x = __shfl_up_sync(0xffffffffu, sum, d);
        if (lane >= d) sum += x;
      }
      // the first expert that ends beyond the target
      const uint32_t beyond = __ballot_sync(0xffffffffu, (int64_t)sum * steps > target);
      if (beyond) {
        const int at = __ffs(beyond) - 1;
        const int own_at = __shfl_sync(0xffffffffu, own, at), before = __shfl_sync(0xffffffffu, sum, at) - own_at;
        return (first + at) * steps + (int)((target - (int64_t)before * steps) / own_at);
      }
      target -= (int64_t)__shfl_sync(0xffffffffu, sum, 31) * steps;
    }
    return n_active * steps;
  }
};
size_t routed_bytes(const MoeArgs &a) {
  const int pairs = a.n_tokens * (a.top_k + a.n_shared);
  return ((size_t)(pairs < a.n_slots ? pairs : a.n_slots) + 1) * 8 + (size_t)pairs * 5;
}
size_t scratch_bytes(const MoeArgs &a) { return (size_t)a.n_slots * 12; }

// ---- the weight stream --------------------------------------------------------------------

// A step of the k axis: 128 bytes of each of 16 weight rows, a lane having bytes 16c.. and 64 + 16c.. of
// rows g and g + 8 (g = lane / 4, c = lane % 4), and the same elements of token g.
template <bool FP8> struct Step {
  static constexpr int kES = FP8 ? 1 : 2, kElems = 128 / kES, kHalf = kElems / 2, kLane = 16 / kES;
  static constexpr int kTok = FP8 ? 2 : 1;              // 16-byte parts of a token a lane and half
  static constexpr int kBytes = (4 + 2 * kTok) * 512;   // of a warp's ring
  static constexpr int kMore = FP8 ? 2 : 3;             // column tiles that a stage holds without weights
};
template <bool FP8> struct TokenPart { uint4 v[2 * Step<FP8>::kTok]; };

template <bool FP8, int STAGES>
struct Ring {
  using S = Step<FP8>;
  uint8_t *base;
  uint32_t at;
  __device__ __forceinline__ explicit Ring(uint8_t *smem) {
    base = smem + (threadIdx.x >> 5) * (STAGES * S::kBytes) + (threadIdx.x & 31) * 16;
    at = shared_address(base);
  }
  // n0, n1: 16 where the halves lie inside the row, else 0
  __device__ __forceinline__ void fill_weights(int stage, const uint8_t *lo, const uint8_t *hi, uint32_t n0, uint32_t n1) {
    const uint32_t dst = at + stage * S::kBytes;
    copy_async_16(dst, lo, n0);
    copy_async_16(dst + 512, hi, n0);
    copy_async_16(dst + 1024, lo + (n1 ? 64 : 0), n1);
    copy_async_16(dst + 1536, hi + (n1 ? 64 : 0), n1);
  }
  __device__ __forceinline__ void put(uint32_t dst, const uint8_t *tok, uint32_t n0, uint32_t n1) {
#pragma unroll
    for (int i = 0; i < S::kTok; ++i) {
      copy_async_16(dst + i * 512, tok + i * 16, n0);
      copy_async_16(dst + (S::kTok + i) * 512, tok + (n1 ? S::kHalf * 2 : 0) + i * 16, n1);
    }
  }
  // (Columns without a token are left as they are: they only make sums that nobody looks at.)
  __device__ __forceinline__ void fill_token(int stage, const uint8_t *tok, uint32_t n0, uint32_t n1) {
    put(at + stage * S::kBytes + 2048, tok, n0, n1);
  }
  __device__ __forceinline__ void fill_more(int stage, int tile, const uint8_t *tok, uint32_t n0, uint32_t n1) {
    put(at + stage * S::kBytes + tile * (S::kTok * 1024), tok, n0, n1);
  }
  __device__ __forceinline__ uint4 get(int stage, int i) const { return *(const uint4 *)(base + stage * S::kBytes + i * 512); }
};

template <bool FP8>
__device__ __forceinline__ TokenPart<FP8> load_token(const uint8_t *p, bool in0, bool in1) {
  using S = Step<FP8>;
  TokenPart<FP8> r = {};
#pragma unroll
  for (int i = 0; i < S::kTok; ++i) {
    if (in0) r.v[i] = *(const uint4 *)(p + i * 16);
    if (in1) r.v[S::kTok + i] = *(const uint4 *)(p + S::kHalf * 2 + i * 16);
  }
  return r;
}

__device__ __forceinline__ uint32_t word(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// acc += 16 weight rows x 8 tokens over one step; e4m3 steps come with the scales of rows g and g + 8.
template <typename T, bool FP8>
__device__ __forceinline__ void step_product(float (&acc)[4], const uint4 (&w)[4], const TokenPart<FP8> &tok, float scale_lo,
                                             float scale_hi) {
  if constexpr (FP8) {
    float part[4] = {};
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t r[4];
        word_of_codes<T>(r[0], r[2], word(w[2 * half], j));
        word_of_codes<T>(r[1], r[3], word(w[2 * half + 1], j));
        const uint4 &v = tok.v[2 * half + (j >> 1)];
        mma_16816<T>(part, r, j & 1 ? v.z : v.x, j & 1 ? v.w : v.y);
      }
    acc[0] += part[0] * scale_lo;
    acc[1] += part[1] * scale_lo;
    acc[2] += part[2] * scale_hi;
    acc[3] += part[3] * scale_hi;
  } else {
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const uint32_t r[4] = {word(w[2 * half], 2 * j), word(w[2 * half + 1], 2 * j), word(w[2 * half], 2 * j + 1), word(w[2 * half + 1], 2 * j + 1)};
        mma_16816<T>(acc, r, word(tok.v[half], 2 * j), word(tok.v[half], 2 * j + 1));
      }
  }
}

// With e4m3 weights and up to 16 tokens the second tile's tokens are read straight from L2 ahead of the wait
// for the step's weights: in a stage of the ring (three of 4 KB) they would halve the steps that the weights run
// ahead (16 tokens, 14 experts of 7168 x 2048: 144 us, through the ring 159).  Everywhere else they come through the ring
// (64 tokens, about 108 bf16 experts of 2048 x 768: 189 us, straight from L2 207; 20 of 7168 x 2048, two of them with all
// tokens: 341 and 527).
template <bool FP8, int NT> constexpr bool kDirect = FP8 && NT == 2;

// Stages that a step takes: its weights with the first 8 tokens, then the further column tiles, kMore at a time.
template <bool FP8, int NT>
__device__ __forceinline__ int stages_of(int count) {
  if constexpr (NT == 1 || kDirect<FP8, NT>) return 1;
  else return 1 + (max(count - 1, 0) / 8 + Step<FP8>::kMore - 1) / Step<FP8>::kMore;
}

// The products of one step for all column tiles of an expert.  fill() starts the copies of the stage that was
// consumed last; second() reads this lane's token of the second tile.  top: moved_top of this lane's codes in rows g
// and g + 8.
template <typename T, bool FP8, int NT, int STAGES, typename F, typename G>
__device__ __forceinline__ void step_products(float (&acc)[NT][4], const Ring<FP8, STAGES> &ring, int &stage, int count,
                                              float scale_lo, float scale_hi, uint32_t (&top)[2], F fill, G second) {
  using S = Step<FP8>;
  const auto next = [&]() { stage = stage + 1 == STAGES ? 0 : stage + 1; };
  uint4 w[4];
  TokenPart<FP8> tok, tok2 = {};
  if constexpr (kDirect<FP8, NT>)
    if (count > 8) tok2 = second();
  copy_async_wait<STAGES - 1>();
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = ring.get(stage, i);
  if constexpr (kMoved<T, FP8>) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) top[i & 1] = moved_top(top[i & 1], word(w[i], j));
  }
#pragma unroll
  for (int i = 0; i < 2 * S::kTok; ++i) tok.v[i] = ring.get(stage, 4 + i);
  step_product<T, FP8>(acc[0], w, tok, scale_lo, scale_hi);
  next();
  if constexpr (kDirect<FP8, NT>) {
    if (count > 8) step_product<T, FP8>(acc[1], w, tok2, scale_lo, scale_hi);
  } else {
#pragma unroll
    for (int n = 1; n < NT; n += S::kMore) {
      if (n * 8 >= count) break;
      fill();
      copy_async_wait<STAGES - 1>();
#pragma unroll
      for (int m = 0; m < S::kMore; ++m) {
        if (n + m >= NT || (n + m) * 8 >= count) break;
#pragma unroll
        for (int i = 0; i < 2 * S::kTok; ++i) tok.v[i] = ring.get(stage, m * (2 * S::kTok) + i);
        step_product<T, FP8>(acc[n + m < NT ? n + m : 0], w, tok, scale_lo, scale_hi);
      }
      next();
    }
  }
}

// Up to 8 tokens: what rounding takes from a hidden vector goes to columns 4 to 7 of the down product where an
// expert has at most 4 tokens - those columns cost nothing, and where few values make an output their rounding would
// show (one token, two experts of 224: 1.6 times the error of the output's own rounding; with it, none).
template <int NT> constexpr bool kWithRest = NT == 1;

// h[pair] = w silu(gate) up, rounded once to IO.  An item is 8 rows of gate and the same 8 of up as one
// 16-row operand, so a thread gets both sums of its outputs.  The k axis is split over the warps,
// joined in shared memory in the order of the warps.  NT: column tiles of 8 tokens an expert may have.  Two blocks
// an SM with 64 KB of weights and 32 KB of tokens in their rings each; bound by the weights: 680 MB (108 bf16 experts of
// 2 x 768 x 2048, 64 tokens) in 120 us, 5.7 TB/s, 69% of the memory's nominal rate.  e4m3 weights:
// 25 experts of 2 x 2048 x 7168, 16 tokens, 734 MB in 154 us, 4.8 TB/s (DRAM 59%, issue slots 43%, integer pipe 40%); 20 with
// 28 tokens each, 701 us, waiting for the tokens' operands from shared memory (DRAM 10%, issue slots 22%).  Items dealt
// by a counter in memory instead of in turn: 2% faster for the bf16 ones, 8% slower for 14 e4m3 experts.
template <typename IO, bool FP8, int NT, int STAGES>
__global__ void __launch_bounds__(kUpWarps * 32) moe_up_kernel(const __grid_constant__ MoeArgs a) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float s_part[2][kUpWarps][16][9];
  using S = Step<FP8>;
  using T = typename UpOperand<IO, FP8>::type;
  constexpr bool kOnePart = NT == 1 || kDirect<FP8, NT>;
  constexpr bool kScaled = !__is_same(T, IO);   // tokens in f16, by a power of two each
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  wait_for_previous();
  let_next_start();
  Routed routed;
  routed.build(a, smem + a.ring_bytes, smem);
  const int tiles = a.d_ff / 8;
  const int items = routed.n_active * tiles;
  const int steps = (a.d_model + S::kElems - 1) / S::kElems;
  const int k0 = steps * warp / kUpWarps, k1 = steps * (warp + 1) / kUpWarps;
  const int64_t row_bytes = (int64_t)a.d_model * S::kES;
  // the step at which this lane's half leaves the row: only the last one can
  const int end0 = (a.d_model - c * S::kLane + S::kElems - 1) / S::kElems;
  const int end1 = (a.d_model - c * S::kLane - S::kHalf + S::kElems - 1) / S::kElems;
  const uint8_t *const x_lane = (const uint8_t *)(kScaled ? a.moved_x : a.x) + c * S::kLane * 2;
  const int64_t x_stride = (kScaled ? a.d_model : a.x_stride) * 2;

  Ring<FP8, STAGES> ring(smem);
  // the copies run ahead of the products over (item, step)
  int fill_item = k0 < k1 ? blockIdx.x : items, fill_k = k0, fill_part = 0, fill_parts = 1, fill_stage = 0;
  const uint8_t *fill_lo = nullptr, *fill_hi = nullptr, *fill_tok = nullptr;
  bool fill_col = false;
  auto enter = [&]() {
    if (fill_item >= items) return;
    const int i = fill_item / tiles, row = (fill_item - i * tiles) * 8 + g;
    const int2 e = routed.active[i];
    const int64_t at = e.x * a.gate_stride + row * row_bytes + c * 16 + k0 * 128;
    fill_lo = a.gate + at;
    fill_hi = a.up + at;
    const int count = routed.active[i + 1].y - e.y;
    fill_parts = stages_of<FP8, NT>(count);
    fill_col = g < count;
    fill_tok = x_lane + (fill_col ? routed.token[e.y + g] * x_stride : 0) + k0 * (S::kElems * 2);
  };
  auto fill = [&]() {
    if (fill_item < items) {
      const uint32_t n0 = fill_k < end0 ? 16 : 0, n1 = fill_k < end1 ? 16 : 0;
      if (kOnePart || fill_part == 0) {
        ring.fill_weights(fill_stage, n0 ? fill_lo : a.gate, n0 ? fill_hi : a.gate, n0, n1);
        if (fill_col) ring.fill_token(fill_stage, n0 ? fill_tok : x_lane, n0, n1);
      } else {
        const int i = fill_item / tiles, first = routed.active[i].y, end = routed.active[i + 1].y;
#pragma unroll
        for (int m = 0; m < S::kMore; ++m) {
          const int pair = first + (1 + (fill_part - 1) * S::kMore + m) * 8 + g;
          if (pair < end)
            ring.fill_more(fill_stage, m, x_lane + (n0 ? routed.token[pair] * x_stride + fill_k * (S::kElems * 2) : 0), n0, n1);
        }
      }
      if (kOnePart || ++fill_part == fill_parts) {
        fill_part = 0;
        fill_lo += 128;
        fill_hi += 128;
        fill_tok += S::kElems * 2;
        if (++fill_k == k1) {
          fill_k = k0;
          fill_item += gridDim.x;
          enter();
        }
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
    uint32_t top[2] = {0, 0};
    const uint8_t *const second = 8 + g < count ? x_lane + routed.token[e.y + 8 + g] * x_stride : x_lane;
    const float *scale_g = nullptr, *scale_u = nullptr;
    float sg = 1.f, su = 1.f;
    if constexpr (FP8) {
      const int64_t at = e.x * a.scale_stride + (row0 / 128) * ((a.d_model + 127) / 128);
      scale_g = a.gate_scale + at;
      scale_u = a.up_scale + at;
      if (k0 < k1) {
        sg = scale_g[k0];
        su = scale_u[k0];
      }
    }
    for (int k = k0; k < k1; ++k) {
      fill();
      float next_g = 1.f, next_u = 1.f;
      if constexpr (FP8) {   // a step is one block of the scales; read a step ahead
        if (k + 1 < k1) {
          next_g = scale_g[k + 1];
          next_u = scale_u[k + 1];
        }
      }
      step_products<T, FP8, NT, STAGES>(acc, ring, stage, count, sg, su, top, fill, [&]() {
        const bool in = 8 + g < count;
        return load_token<FP8>(second + (int64_t)k * (S::kElems * 2), in && k < end0, in && k < end1);
      });
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
          if constexpr (kScaled) {
            const float by = a.token_scale[routed.token[pair]];
            gate *= by;
            up *= by;
          }
          float h = gate / (1.f + expf(-gate)) * up * routed.weight[pair];
          // f16 ends at 65504: the largest value stands for what is beyond (bf16 reaches as far as 32 bits)
          if constexpr (__is_same(IO, __half)) h = h != h ? h : fminf(fmaxf(h, -65504.f), 65504.f);
          const int at = row0 + f;
          if constexpr (kMoved<IO, FP8>) h *= kMovedScale;
          const IO high = IO(h);
          IO *const to = (IO *)a.h + (int64_t)pair * a.d_ff + (kMoved<IO, FP8> ? moved_place(at) : at);
          *to = high;
          if constexpr (kWithRest<NT>)
            if (count <= 4) to[a.h_rest / 2] = IO(fabsf((float)high) < CUDART_INF_F ? h - (float)high : 0.f);
        }
      }
    }
  }
  copy_async_wait<0>();
}

// y for 16 output rows a block: the (expert, step) pairs of all experts in use are dealt to the
// warps in runs of equal work.  At the end of its part of an expert a warp adds the expert's columns to its
// own sums of the tokens in shared memory; the warps' sums are joined at the end, in their order.
// Bound by the weights where the warps are enough to keep them coming: 340 MB (2048 rows, 108 experts
// of 768, 64 tokens) in 68 us, 5.0 TB/s from 128 of the 148 SMs.  e4m3 weights: 25 experts of 7168 x 2048, 16 tokens, 368 MB
// in 130 us, 2.8 TB/s (integer pipe 62%, DRAM 35%): the shifts that make bf16 operands of the codes, and looking out for
// codes that are not a number (3% of a call); 20 with 28 tokens each, 434 us, as the products before.
template <typename T, bool FP8, int NT, int STAGES, int WARPS>
__global__ void __launch_bounds__(WARPS * 32) moe_down_kernel(const __grid_constant__ MoeArgs a) {
  extern __shared__ __align__(128) uint8_t smem[];
  using S = Step<FP8>;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c = lane & 3;
  constexpr bool kOnePart = NT == 1 || kDirect<FP8, NT>;
  const int row0 = blockIdx.x * 16;
  const int steps = (a.d_ff + S::kElems - 1) / S::kElems;
  const int64_t row_bytes = (int64_t)a.d_ff * S::kES;
  const int end0 = (a.d_ff - c * S::kLane + S::kElems - 1) / S::kElems;
  const int end1 = (a.d_ff - c * S::kLane - S::kHalf + S::kElems - 1) / S::kElems;
  float *const sums = (float *)(smem + a.ring_bytes);   // [warp][token][17]
  const int sum_count = (WARPS * a.n_tokens * 17 + 1) / 2 * 2;
  for (int i = threadIdx.x; i < sum_count; i += WARPS * 32) sums[i] = 0.f;
  // The choices were written by the launch before the last, which had ended before that one began its
  // work: they can be read, and weights fetched, while the hidden vectors are still being made.
  Routed routed;
  routed.build(a, (uint8_t *)(sums + sum_count), smem);
  // at most 2048 experts x 16384 steps
  const int s0 = routed.template share<FP8, NT>(steps, warp, WARPS), s1 = routed.template share<FP8, NT>(steps, warp + 1, WARPS);
  const uint8_t *const h_lane = (const uint8_t *)a.h + c * S::kLane * 2;

  Ring<FP8, STAGES> ring(smem);
  struct Cursor {
    int step, expert, k, part, parts, stage;
  } wf = {s0, s0 / steps, s0 % steps, 0, 1, 0}, tf = wf;
  const uint8_t *fill_w = nullptr, *fill_tok = nullptr;
  bool fill_col = false;
  auto enter_weights = [&]() {
    if (wf.expert >= routed.n_active) return;
    wf.parts = stages_of<FP8, NT>(routed.active[wf.expert + 1].y - routed.active[wf.expert].y);
    fill_w = a.down + routed.active[wf.expert].x * a.down_stride + (row0 + g) * row_bytes + c * 16 + wf.k * 128;
  };
  auto enter_tokens = [&]() {
    if (tf.expert >= routed.n_active) return;
    const int first = routed.active[tf.expert].y, count = routed.active[tf.expert + 1].y - first;
    tf.parts = stages_of<FP8, NT>(count);
    const bool rest = kWithRest<NT> && count <= 4 && g >= 4;
    const int column = rest ? g - 4 : g;
    fill_col = column < count;
    fill_tok = h_lane + (fill_col ? (rest ? a.h_rest : 0) + (int64_t)(first + column) * a.d_ff * 2 : 0) + tf.k * (S::kElems * 2);
  };
  auto next = [&](Cursor &cur, auto enter) {   // true: on to the next step
    if (!kOnePart && ++cur.part < cur.parts) return false;
    cur.part = 0;
    ++cur.step;
    if (++cur.k == steps) {
      cur.k = 0;
      ++cur.expert;
      enter();
      return false;   // it has set the pointers itself
    }
    return true;
  };
  auto fill_weights = [&]() {
    if (wf.step < s1) {
      const uint32_t n0 = wf.k < end0 ? 16 : 0, n1 = wf.k < end1 ? 16 : 0;
      if (kOnePart || wf.part == 0) ring.fill_weights(wf.stage, n0 ? fill_w : a.down, n0 ? fill_w + 8 * row_bytes : a.down, n0, n1);
      if (next(wf, enter_weights)) fill_w += 128;
    }
    wf.stage = wf.stage + 1 == STAGES ? 0 : wf.stage + 1;
  };
  auto fill_tokens = [&]() {
    if (tf.step < s1) {
      const uint32_t n0 = tf.k < end0 ? 16 : 0, n1 = tf.k < end1 ? 16 : 0;
      if (kOnePart || tf.part == 0) {
        if (fill_col) ring.fill_token(tf.stage, n0 ? fill_tok : h_lane, n0, n1);
      } else {
        const int first = routed.active[tf.expert].y, end = routed.active[tf.expert + 1].y;
#pragma unroll
        for (int m = 0; m < S::kMore; ++m) {
          const int pair = first + (1 + (tf.part - 1) * S::kMore + m) * 8 + g;
          if (pair < end)
            ring.fill_more(tf.stage, m, h_lane + (n0 ? (int64_t)pair * a.d_ff * 2 + tf.k * (S::kElems * 2) : 0), n0, n1);
        }
      }
      if (next(tf, enter_tokens)) fill_tok += S::kElems * 2;
    }
    copy_async_commit();
    tf.stage = tf.stage + 1 == STAGES ? 0 : tf.stage + 1;
  };
  enter_weights();
  for (int i = 0; i < STAGES - 1; ++i) fill_weights();
  wait_for_previous();
  enter_tokens();
  for (int i = 0; i < STAGES - 1; ++i) fill_tokens();   // the first of these groups holds all those weights too

  int stage = 0, s = s0;
  for (int expert = s0 / steps; s < s1; ++expert) {
    const int2 e = routed.active[expert];
    const int count = routed.active[expert + 1].y - e.y;
    const int first = s - expert * steps, last = min(steps, s1 - expert * steps);
    s += last - first;
    const uint8_t *const second = h_lane + (8 + g < count ? (int64_t)(e.y + 8 + g) * a.d_ff * 2 : 0);
    const float *scale = nullptr;
    float by = 1.f;
    if constexpr (FP8) {
      scale = a.down_scale + (int64_t)e.x * a.scale_stride + (row0 / 128) * ((a.d_ff + 127) / 128);
      by = scale[first];
    }
    float acc[NT][4] = {};
    uint32_t top[2] = {0, 0};
    for (int k = first; k < last; ++k) {
      fill_weights();
      fill_tokens();
      float later = 1.f;
      if constexpr (FP8) {
        if (k + 1 < last) later = scale[k + 1];
      }
      step_products<T, FP8, NT, STAGES>(acc, ring, stage, count, by, by, top, [&]() {
        fill_weights();
        fill_tokens();
      }, [&]() {
        const bool in = 8 + g < count;
        return load_token<FP8>(second + (int64_t)k * (S::kElems * 2), in && k < end0, in && k < end1);
      });
      by = later;
    }
    if constexpr (kMoved<T, FP8>) {   // a weight that is not a number makes its row of sums that
#pragma unroll
      for (int half = 0; half < 2; ++half)
        if (__ballot_sync(0xffffffffu, moved_nan(top[half])) >> (lane & 28) & 15) {
#pragma unroll
          for (int n = 0; n < NT; ++n) acc[n][2 * half] = acc[n][2 * half + 1] = CUDART_NAN_F;
        }
    }
    if constexpr (kWithRest<NT>)
      if (count <= 4) {   // columns 4 to 7 are two lanes further
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[0][i] += __shfl_down_sync(0xffffffffu, acc[0][i], 2);
      }
    float *const mine = sums + warp * a.n_tokens * 17;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (n * 8 >= count) break;
#pragma unroll
      for (int i = 0; i < 2; ++i) {   // columns 2c and 2c + 1: no two lanes have the same token and row
        const int j = n * 8 + 2 * c + i;
        if (j < count) {
          float *const y = mine + routed.token[e.y + j] * 17;
          y[g] += acc[n][i];
          y[g + 8] += acc[n][2 + i];
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
    if constexpr (kMoved<T, FP8>) y *= kMovedScale;
    if (a.out_f32) ((float *)a.out)[t * a.out_stride + row0 + r] = y;
    else ((T *)a.out)[t * a.out_stride + row0 + r] = T(y);
  }
}

template <auto KERNEL>
cudaError_t launch(unsigned grid, int threads, size_t smem, bool early, const MoeArgs &a, cudaStream_t st) {
  const cudaError_t e = allow_shared<KERNEL>();
  if (e != cudaSuccess) return e;
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
  return cudaLaunchKernelEx(&cfg, KERNEL, a);
}

size_t ring_bytes(size_t ring, const MoeArgs &a) {   // the ring's place also serves to group the choices
  const size_t n = ring > scratch_bytes(a) ? ring : scratch_bytes(a);
  return (n + 127) / 128 * 128;
}

template <bool FP8, int STAGES, int WARPS>
size_t down_bytes(const MoeArgs &a) {
  return ring_bytes((size_t)WARPS * STAGES * Step<FP8>::kBytes, a) + (size_t)(WARPS * a.n_tokens * 17 + 1) / 2 * 8 + routed_bytes(a);
}

template <typename T, bool FP8, int NT, int STAGES, int WARPS>
cudaError_t launch_down(MoeArgs a, cudaStream_t st) {
  a.ring_bytes = (int32_t)ring_bytes((size_t)WARPS * STAGES * Step<FP8>::kBytes, a);
  return launch<moe_down_kernel<T, FP8, NT, STAGES, WARPS>>(a.d_model / 16, WARPS * 32, down_bytes<FP8, STAGES, WARPS>(a), true, a, st);
}

template <typename T, bool FP8, int NT>
cudaError_t launch_layer(MoeArgs a, cudaStream_t st) {
  cudaError_t e = a.n_experts <= 256 ? launch<moe_route_kernel<8, kMoved<T, FP8>>>(a.n_tokens, kRouteThreads, 0, false, a, st)
                                     : launch<moe_route_kernel<32, kMoved<T, FP8>>>(a.n_tokens, kRouteThreads, 0, false, a, st);
  if (e != cudaSuccess) return e;
  constexpr int kStages = FP8 ? 3 : 4;   // 96 KB: two blocks an SM
  const int64_t pairs = (int64_t)a.n_tokens * (a.top_k + a.n_shared);
  const int64_t most = (pairs < a.n_slots ? pairs : a.n_slots) * (a.d_ff / 8);
  a.ring_bytes = (int32_t)ring_bytes((size_t)kUpWarps * kStages * Step<FP8>::kBytes, a);
  e = launch<moe_up_kernel<T, FP8, NT, kStages>>((unsigned)(most < 2 * kSms ? most : 2 * kSms), kUpWarps * 32,
             a.ring_bytes + routed_bytes(a), true, a, st);
  if (e != cudaSuccess) return e;
  // A warp's step is a chain of about 100 instructions, so an SM wants 12 to 16 warps, and the blocks have to fit
  // all at once: with up to one block an SM 16 warps each (64 tokens, d_model 2048: 207 us for the layer, 8 warps 221),
  // up to two 8 (16 tokens, d_model 4096, bf16: 73 us, 4 warps 105), up to three 8 with short rings where the
  // registers allow it (d_model 5120, bf16: 100 us, 4 warps 120; e4m3 95 and 87, so not there), beyond that 4
  // (d_model 7168, bf16: 181 us, 8 warps 213, whose 444 places are four too few).
  const int blocks = a.d_model / 16;
  if (blocks <= kSms && down_bytes<FP8, FP8 ? 2 : 3, 16>(a) <= kMaxShared) return launch_down<T, FP8, NT, FP8 ? 2 : 3, 16>(a, st);
  if (blocks <= 2 * kSms) return launch_down<T, FP8, NT, FP8 ? 3 : 4, 8>(a, st);
  if constexpr (NT <= 2 && !FP8)
    if (blocks <= 3 * kSms) return launch_down<T, FP8, NT, 2, 8>(a, st);
  return launch_down<T, FP8, NT, FP8 ? 3 : 4, 4>(a, st);
}

template <typename T, bool FP8>
cudaError_t by_tokens(const MoeArgs &a, cudaStream_t st) {
  if (a.n_tokens <= kMoeWithRest) return launch_layer<T, FP8, 1>(a, st);
  if (a.n_tokens <= 16) return launch_layer<T, FP8, 2>(a, st);
  if (a.n_tokens <= 32) return launch_layer<T, FP8, 4>(a, st);
  return launch_layer<T, FP8, 8>(a, st);
}

}  // namespace

MoeShape moe_shape(int d_model, int d_ff, int n_tokens, int top_k, int n_shared, bool moved) {
  MoeShape s{};
  const int64_t pairs = (int64_t)n_tokens * (top_k + n_shared);
  const auto up = [](int64_t n) { return (n + 255) / 256 * 256; };
  s.token_scale = up(pairs * 8);   // the choices lie at the start
  s.moved_x = s.token_scale + (moved ? up(n_tokens * 4) : 0);
  s.h = s.moved_x + (moved ? up((int64_t)n_tokens * d_model * 2) : 0);
  s.h_rest = up(pairs * d_ff * 2);
  s.bytes = s.h + s.h_rest * (n_tokens <= kMoeWithRest ? 2 : 1);
  return s;
}

cudaError_t launch_moe(const MoeArgs &a, int type, int io, cudaStream_t st) {
  if (type == EMOE_TYPE_E4M3)
    return io == EMOE_TYPE_BF16 ? by_tokens<__nv_bfloat16, true>(a, st) : by_tokens<__half, true>(a, st);
  return io == EMOE_TYPE_BF16 ? by_tokens<__nv_bfloat16, false>(a, st) : by_tokens<__half, false>(a, st);
}

}  // namespace emoe
