// attend_prefix.cu - the shared prefix against the rows of a whole batch on the 5th-generation tensor
// cores.
//
// A batch that shares a prefix has n_seqs * q_len * (query heads per KV head) rows for each KV head: a
// matrix product once there are more than a few.  A block takes a KV head, up to 256 rows and a range of
// the prefix; it holds the rows' queries in shared memory and two accumulator sets ("slots") in tensor memory,
//     S = Q K^T (128 x 64), O += P V (128 x head_dim),   P = 2^(scale S - m) rounded to 16 bits,
// and runs through the tokens in steps of 64 (tiles of 128 are brought in).  S has two buffers a slot, so
// that the next step's scores are there when a step's weights are done; P is written over its S in tensor
// memory and multiplied from there.  With more than 128 rows the slots are two row tiles on the same
// tokens; with fewer they are the same rows on alternating tiles of tokens, so that a single row tile
// also keeps both the tensor cores and the exponentials busy.
//
// Warps: 0-3 and 4-7 the softmax of the two slots (a thread a row, the scores of a step in its
// registers), 8 and 9 issue the slots' products (each keeps the tensor cores fed while the other
// waits), 12-15 bring K and V rows from their pages into the 128-byte-swizzled tiles that the products read (copied
// asynchronously; e4m3 codes are widened on the way).  The maximum in use is only raised when the real one
// passes it by more than 2^8: sums and weights then still fit, and O is rarely rescaled.
//
// Bounds: exponentials (16 a clock and SM: 2048 clocks for 2 x 128 rows x 128 tokens) and products
// (about the same) with many rows, the reads of K and V with few.  Measured: 1024 rows x 4 heads x 65536 tokens, bf16, head_dim
// 128, 140 us = 980 TFLOP/s, 57% of a library product's rate, with the tensor cores and the exponential units
// busy half of the time each: the rest is the chain scores -> maximum -> weights -> product of a step, of which two
// slots run at a time (tensor memory holds no more).  32 rows x 16 heads x 8199 tokens, e4m3: 35 us.
// A start, 18 us for a call of 2000 tokens, is mostly the first tiles and the last products.
#include "attend_item.cuh"
#include "tensor.cuh"

namespace emoe {
namespace {

// Registers a thread of the four warpgroups, out of the 4 x 128 that the block is launched with.
constexpr int kSoftmaxRegs = 152, kMmaRegs = 80, kCopyRegs = 128;
static_assert(2 * kSoftmaxRegs + kMmaRegs + kCopyRegs <= 512, "the block has no more registers than it was launched with");

// Which copying warp has a row of a tile, and which of its lanes finds it in the table.
template <int ROWS> __device__ __forceinline__ constexpr int warp_of_row(int row) { return row / ROWS % kCopyWarps; }
template <int ROWS> __device__ __forceinline__ constexpr int lane_of_row(int row) { return row / (ROWS * kCopyWarps) * ROWS + row % ROWS; }


template <typename IO, int HD, bool FP8>
__global__ void __launch_bounds__(kThreads, 1) attend_prefix_kernel(const __grid_constant__ AttendArgs a) {
  using T = typename Operand<IO, FP8>::type;
  constexpr uint32_t kTileBytes = kTile * HD * 2;
  constexpr float kLift = kWeightLift<T> > 0.f ? kWeightLift<T> - kRaise : 0.f;
  constexpr int kPieces = HD / 8;   // 16-byte pieces of a 16-bit row
  // copying: a row's pieces are taken by kGroup neighbouring lanes, kRows rows at a time by a warp
  constexpr int kGroup = FP8 ? HD / 16 : kPieces, kRows = 32 / kGroup;
  extern __shared__ uint8_t raw_smem[];
  __shared__ __align__(8) uint64_t bars[kBars];
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort;
  __shared__ uint4 s_bad[kKept];   // tokens that nobody sees: a word of 32 rows from each copying warp
  __shared__ __align__(16) float s_scale[2][FP8 ? kKept : 1][FP8 ? kTile : 4];   // of K and V
  uint8_t *const smem = (uint8_t *)(((uintptr_t)raw_smem + 1023) & ~(uintptr_t)1023);
  const uint32_t q_at = shared_address(smem), k_at = q_at + 2 * kTileBytes, v_at = k_at + 2 * kTileBytes;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

  // the item
  const uint32_t heads = a.c.n_heads;
  const int pairs = a.alternate ? 1 : (a.n_seqs * a.seq_rows + 2 * kTile - 1) / (2 * kTile);
  const int split = blockIdx.x / (heads * pairs), unit = blockIdx.x % (heads * pairs);
  const int head = unit % heads, row0 = unit / heads * (2 * kTile);
  const int rows = min(2 * kTile, a.n_seqs * a.seq_rows - row0);
  const int t0 = split * a.prefix_chunk, t1 = min(a.prefix_len, t0 + a.prefix_chunk);
  const int tiles = (t1 - t0 + kTile - 1) / kTile;
  const bool alternate = a.alternate != 0, second = alternate || rows > kTile;
  // steps of the slots: two a tile, unless the last one has no token in its second half
  const int last_halves = t1 - t0 - (tiles - 1) * kTile > kStep ? 2 : 1;
  const int own_tiles[2] = {alternate ? (tiles + 1) / 2 : tiles, alternate ? tiles / 2 : second ? tiles : 0};
  const auto steps_of = [&](int slot) {
    const bool has_last = own_tiles[slot] > 0 && (!alternate || ((tiles - 1) & 1) == slot);
    return 2 * own_tiles[slot] - (has_last ? 2 - last_halves : 0);
  };
  const int steps[2] = {steps_of(0), steps_of(1)};

  const int readers = !alternate && second ? 2 : 1;   // slots that read a tile
  const Bars bar{shared_address(bars)};
  if (threadIdx.x == 0) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      bar_init(bar.k_full(i), kCopyWarps * (FP8 ? 1 : 33));   // copies arrive by the lane; the marks with one arrival more
      bar_init(bar.v_full(i), kCopyWarps * (FP8 ? 1 : 32));
      bar_init(bar.drained(i), 1);
#pragma unroll
      for (int w = 0; w < 4; ++w) bar_init(bar.turn(i, w), 1);
      bar_init(bar.k_empty(i), readers);
      bar_init(bar.v_empty(i), readers);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        bar_init(bar.s_full(i, half), 1);
        bar_init(bar.p_full(i, half), 4);
        bar_init(bar.o_full(i, half), 1);
      }
    }
    bar_init(bar.q_full(), kSoftmaxWarps * 32);
    s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(shared_address(&s_tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  let_next_start();

  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = s_tmem;
  volatile int *const abort = &s_abort;

  if (warp < kSoftmaxWarps) {
    take_registers<kSoftmaxRegs>();
    const int slot = warp >> 2, local = (warp & 3) * 32 + lane;   // this thread's row in the tile
    const int row = alternate ? local : slot * kTile + local;
    const bool busy = (alternate ? 0 : slot * kTile) + (warp & 3) * 32 < rows;   // any real row in the warp
    float x[2][32];   // the row's query, then a step's scores and weights
    // not zero: a masked score, minus infinity, has to stay that (and every other one comes to zero all the same)
    const float c = fmaxf(fabsf(a.scale_log2), 0x1p-149f);
    float query_by = 1.f;   // e4m3: the row's query is this much smaller than the one that is multiplied
    {
      // The row's query (stored by two threads, half each, where both slots have the same rows): rows that do
      // not exist are zero, a negative scale turns the sign.
      uint4 *const w = (uint4 *)x;
      const int r = min(row, rows - 1), token = (row0 + r) / a.group;
      const uint4 *const src = (const uint4 *)((const IO *)a.q + (int64_t)token * a.q_stride + (head * a.group + row0 + r - token * a.group) * HD);
      const uint32_t sign = a.scale_log2 < 0.f ? 0x80008000u : 0;
#pragma unroll
      for (int i = 0; i < kPieces; ++i) w[i] = row < rows ? src[i] : make_uint4(0, 0, 0, 0);
      if constexpr (FP8) {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float2 f = Pair<IO>::unpack(word(w[i], k));
            top = max(top, max(__float_as_uint(f.x) & 0x7fffffffu, __float_as_uint(f.y) & 0x7fffffffu));
          }
        const float by = query_scale(top);
        query_by = 1.f / by;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
          const float2 e0 = Pair<IO>::unpack(w[i].x), e1 = Pair<IO>::unpack(w[i].y), e2 = Pair<IO>::unpack(w[i].z), e3 = Pair<IO>::unpack(w[i].w);
          w[i] = make_uint4(Pair<T>::pack(e0.x * by, e0.y * by), Pair<T>::pack(e1.x * by, e1.y * by), Pair<T>::pack(e2.x * by, e2.y * by),
                            Pair<T>::pack(e3.x * by, e3.y * by));
        }
      }
#pragma unroll
      for (int i = 0; i < kPieces; ++i)
        if (!alternate || i / (kPieces / 2) == slot)
          *(uint4 *)(smem + (alternate ? 0 : slot * kTileBytes) + piece_at(local, i)) =
              make_uint4(w[i].x ^ sign, w[i].y ^ sign, w[i].z ^ sign, w[i].w ^ sign);
      fence_async();
      bar_arrive(bar.q_full());
    }
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;   // lane 32 * (warp % 4) in the address's upper half
    const uint32_t s_base = tmem + lanes + kColS + slot * kTile, o_col = tmem + lanes + kColO + slot * HD;
    float m = -CUDART_INF_F, l = 0.f, v_ref = 0.f;   // v_ref: the largest scale of v so far
    bool ok = true;
    if (steps[slot] > 0) {   // the first step's scores
      ok = bar_wait_warp(bar.s_full(slot, 0), 0, abort, a.wait_ns);
      fence_after();
      if (ok && busy) {
        tmem_load(x[0], s_base);
        tmem_load(x[1], s_base + 32);
      }
    }
    for (int i = 0; i < steps[slot] && ok; ++i) {
      const int half = i & 1, tile = alternate ? 2 * (i >> 1) + slot : i >> 1;
      const uint32_t s_col = s_base + half * kStep;
      // Exponentials of the two slots' warps that share a quarter of the SM take turns, 0 first: while one has
      // them the other fetches its scores and finds their maximum.  Together they would both wait.
      const bool both = steps[1] > 0 && (alternate ? 0 : kTile) + (warp & 3) * 32 < rows;   // the other has rows too
      const bool wait_turn = both && (slot ? i < steps[0] : i > 0 && i - 1 < steps[1]);
      const bool give_turn = both && (slot ? i + 1 < steps[0] : i < steps[1]);
      if (busy) {
        const uint4 bad = s_bad[tile % kKept];
        const bool any_bad = (bad.x | bad.y | bad.z | bad.w) != 0;
        const float *const k_scale = s_scale[0][FP8 ? tile % kKept : 0] + half * kStep;
        const float *const v_scale = s_scale[1][FP8 ? tile % kKept : 0] + half * kStep;
        // the largest score, and of an e4m3 cache the largest scale of v
        float v_top = v_ref, tops[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          tmem_wait(x[j]);
          if constexpr (FP8) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              // the two scales first: either one alone can take a score out of range
              float4 k = *(const float4 *)(k_scale + 32 * j + e);
              mul_pair(k.x, k.y, query_by, query_by);
              mul_pair(k.z, k.w, query_by, query_by);
              mul_pair(x[j][e], x[j][e + 1], k.x, k.y);
              mul_pair(x[j][e + 2], x[j][e + 3], k.z, k.w);
              const float4 v = *(const float4 *)(v_scale + 32 * j + e);
              v_top = max3(max3(v_top, v.x, v.y), v.z, v.w);
            }
          }
          if (__builtin_expect(any_bad, 0)) {
#pragma unroll
            for (int e = 0; e < 32; ++e) {   // both halves' columns of a bit: a row is one lane of one warp
              const int first = 32 * j + e, second = first + kStep;
              if (word(bad, warp_of_row<kRows>(first)) >> (half ? lane_of_row<kRows>(second) : lane_of_row<kRows>(first)) & 1) x[j][e] = -CUDART_INF_F;
            }
          }
          float t0 = x[j][0], t1 = x[j][1];
#pragma unroll
          for (int e = 2; e < 32; e += 4) {
            t0 = max3(t0, x[j][e], x[j][e + 1]);
            if (e + 3 < 32) t1 = max3(t1, x[j][e + 2], x[j][e + 3]);
          }
          tops[j] = fmaxf(t0, t1);
        }
        float top = fmaxf(tops[0], tops[1]);
        top *= c;
        const bool raise = i > 0 && (top > m + kRaise || v_top > v_ref);
        if (i == 0) {
          m = top;
          v_ref = v_top;
        } else if (__any_sync(0xffffffffu, raise)) {   // O may be touched once the last step's product
          // is done (the one before it is: this step's scores came after that)
          ok = bar_wait_warp(bar.o_full(slot, (i - 1) & 1), ((i - 1) >> 1) & 1, abort, a.wait_ns);
          if (!ok) break;
          fence_after();
          const float to = top > m + kRaise ? top : m;
          float by = to == -CUDART_INF_F ? 1.f : exp2_fast(m - to);
          l *= by;
          if constexpr (FP8) by *= v_top > 0.f ? v_ref / v_top : 1.f;
          m = to;
          v_ref = v_top;
#pragma unroll 1
          for (int j = 0; j < HD / 16; ++j) {
            float o[16];
            tmem_load_16(o, o_col + 16 * j);
            uint32_t y[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) y[e] = __float_as_uint(o[e] * by);
            tmem_store_16(o_col + 16 * j, y);
          }
        }
        float safe = m == -CUDART_INF_F ? 0.f : m - kLift;
        const float v_by = FP8 && v_ref > 0.f ? 1.f / v_ref : 0.f;   // powers of two: exact
        if (wait_turn) {
          ok = bar_wait_warp(bar.turn(slot, warp & 3), (slot ? i : i - 1) & 1, abort, a.wait_ns);
          if (!ok) break;
          asm volatile("" : "+f"(safe));   // the exponentials stay behind this
        }
        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          uint32_t p[16];   // rounded once, as the second product's operand
          if (j == 1 && give_turn && lane == 0) bar_arrive(bar.turn(1 - slot, warp & 3));
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            float &u = x[j][e], &v = x[j][e + 1];
            fma_pair(u, v, c, c, -safe);
            u = exp2_fast(u);
            v = exp2_fast(v);
          }
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            add_pair(sum[0], sum[1], x[j][e], x[j][e + 1]);
            add_pair(sum[2], sum[3], x[j][e + 2], x[j][e + 3]);
          }
          if constexpr (FP8) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              const float4 v = *(const float4 *)(v_scale + 32 * j + e);
              x[j][e] *= v.x * v_by;
              x[j][e + 1] *= v.y * v_by;
              x[j][e + 2] *= v.z * v_by;
              x[j][e + 3] *= v.w * v_by;
            }
          }
#pragma unroll
          for (int e = 0; e < 16; ++e) p[e] = Pair<T>::pack(x[j][2 * e], x[j][2 * e + 1]);
          tmem_store_16(s_col + 16 * j, p);   // over columns that have been read
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      }
      // The next step's scores are on their way before this one's weights are waited for and announced.  (They
      // were asked for a step ago; were they not done yet, their product does not need these weights.)
      if (i + 1 < steps[slot]) {
        ok = bar_wait_warp(bar.s_full(slot, half ^ 1), ((i + 1) >> 1) & 1, abort, a.wait_ns);
        if (!ok) break;
        fence_after();
        if (busy) {
          tmem_load(x[0], s_base + (half ^ 1) * kStep);
          tmem_load(x[1], s_base + (half ^ 1) * kStep + 32);
        }
      }
      if (busy) tmem_stored();
      fence_before();
      __syncwarp();
      if (lane == 0) bar_arrive(bar.p_full(slot, half));   // one a warp: arrivals at one barrier go one by one
    }
    if (!ok) tmem_stored();   // what was under way when a wait ran out
    // the part of this range: maximum, sum and unnormalised output of every row
    // The last two products may be under way.  A parity tells one phase from the next only: each half has a
    // barrier of its own, whose phase before is over by then.
    for (int i = max(0, steps[slot] - 2); i < steps[slot] && ok; ++i)
      ok = bar_wait_warp(bar.o_full(slot, i & 1), (i >> 1) & 1, abort, a.wait_ns);
    fence_after();
    const int slots = a.prefix_splits + a.own_splits;
    const int64_t part = row < rows ? output_row(a, 0, head, row0 + row) * slots + (alternate ? 2 * split + slot : split) : 0;
    if (busy && (alternate || slot == 0 || second)) {
      // what a wait that ran out leaves behind is not a number: a part that counts as empty would go unnoticed
      const bool empty = steps[slot] == 0 || !ok;
      if (row < rows) a.part_ml[part] = empty ? make_float2(-CUDART_INF_F, ok ? 0.f : CUDART_NAN_F) : make_float2(m - kLift, l);
      if (!empty) {
        const float by = FP8 ? v_ref : 1.f;
        float x[HD / 32][32];
#pragma unroll
        for (int j = 0; j < HD / 32; ++j) tmem_load(x[j], o_col + 32 * j);
#pragma unroll
        for (int j = 0; j < HD / 32; ++j) {
          tmem_wait(x[j]);
          if (row < rows) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              const float4 y = make_float4(x[j][e] * by, x[j][e + 1] * by, x[j][e + 2] * by, x[j][e + 3] * by);
              *(float4 *)(a.part_o + part * HD + 32 * j + e) = y;
            }
          }
        }
      }
    }
    fence_before();
  } else if (warp < kCopyWarp0) {
    give_registers<kMmaRegs>();
    const int slot = warp - kMmaWarp;
    if (slot < 2 && steps[slot] > 0) {   // the whole warp goes along, one lane issues: addresses stay in uniform registers
      constexpr uint32_t kType = __is_same(T, __half) ? 0 : 1;
      constexpr uint32_t kIdS = instruction(kType, kStep, 0), kIdO = instruction(kType, HD, 1);
      const bool one = elect_one();
      const auto commit = [&](uint32_t b) {
        if (one) mma_commit(b);
      };
      // Operands are made once; a step adds to the address in their lower half only (in units of 16 bytes).
      const uint64_t q_op = operand(q_at, 0), k_op = operand(k_at, 0), v_op = operand(v_at, kTile * 128);
      const uint64_t q = q_op + (alternate ? 0 : slot * (kTileBytes >> 4));
      const uint32_t s_at = tmem + kColS + slot * kTile, o_at = tmem + kColO + slot * HD;
      const auto scores = [&](int stage, int half) {
        if (!one) return;
        const uint64_t k = k_op + stage * (kTileBytes >> 4) + half * (kStep * 128 >> 4);
#pragma unroll
        for (int i = 0; i < HD / 16; ++i) {
          const int off = ((i >> 2) * (kTile * 128) + (i & 3) * 32) >> 4;
          mma_ss(s_at + half * kStep, q + off, k + off, kIdS, i > 0);
        }
      };
      const auto values = [&](int stage, int half, bool add) {
        if (!one) return;
        const uint64_t v = v_op + stage * (kTileBytes >> 4) + half * (kStep * 128 >> 4);
#pragma unroll
        for (int i = 0; i < kStep / 16; ++i) mma_ts(o_at, s_at + half * kStep + i * 8, v + i * (2048 >> 4), kIdO, add || i > 0);
      };
      bool ok = bar_wait_warp(bar.q_full(), 0, abort, a.wait_ns);
      const auto tile_of = [&](int i) { return alternate ? 2 * (i >> 1) + slot : i >> 1; };
      const auto last_of_tile = [&](int i) { return (i & 1) || i + 1 == steps[slot]; };
      const auto start = [&](int i) {   // S of step i
        const int tile = tile_of(i), stage = tile & 1;
        if (!(i & 1)) {
          ok = ok && bar_wait_warp(bar.k_full(stage), (tile >> 1) & 1, abort, a.wait_ns);
          if constexpr (!FP8) fence_async();
        }
        if (!ok) return;
        fence_after();
        scores(stage, i & 1);
        commit(bar.s_full(slot, i & 1));
        if (last_of_tile(i)) commit(bar.k_empty(stage));
      };
      for (int i = 0; i < 2; ++i)
        if (i < steps[slot] && ok) start(i);
      for (int i = 0; i < steps[slot] && ok; ++i) {
        const int tile = tile_of(i), stage = tile & 1;
        if (!(i & 1)) {
          ok = bar_wait_warp(bar.v_full(stage), (tile >> 1) & 1, abort, a.wait_ns);
          if constexpr (!FP8) fence_async();
        }
        ok = ok && bar_wait_warp(bar.p_full(slot, i & 1), (i >> 1) & 1, abort, a.wait_ns);
        if (!ok) break;
        fence_after();
        values(stage, i & 1, i > 0);
        commit(bar.o_full(slot, i & 1));
        if (last_of_tile(i)) commit(bar.v_empty(stage));
        if (i + 2 < steps[slot]) start(i + 2);
      }
      // The products in flight end before the tensor memory is given back, whoever gives up: the slot's softmax may
      // have when this warp has issued its last.
      int undrained = 0;
      commit(bar.drained(slot));
      if (!bar_wait_warp(bar.drained(slot), 0, &undrained, kDrainNs)) *abort = 1;
    }
    __syncwarp();
  } else {
    give_registers<kCopyRegs>();
    const int w = warp - kCopyWarp0;
    // A warp has 32 rows of a tile; each lane finds one of them in the table.
    constexpr int kPasses = kTile / (kCopyWarps * kRows);
    static_assert(kRows * kPasses == 32, "a lane a row");
    const int piece = lane % kGroup;
    const auto row_of = [&](int pass, int r) { return pass * (kCopyWarps * kRows) + w * kRows + r; };
    const int my_row = row_of(lane / kRows, lane % kRows);
    const auto mark = [&](int tile, bool bad) {
      const uint32_t rows_of_warp = __ballot_sync(0xffffffffu, bad);
      if (lane == 0) ((uint32_t *)&s_bad[tile % kKept])[w] = rows_of_warp;
      __syncwarp();
    };
    // this lane's token of a tile, -1 if there is none; its block; its vector index
    const auto token_of = [&](int tile) {
      const int t = t0 + tile * kTile + my_row;
      return tile < tiles && t < t1 ? t : -1;
    };
    const auto block_of = [&](int tile) {
      const int t = token_of(tile);
      return t < 0 ? 0 : a.prefix_table[(uint32_t)t / (uint32_t)a.c.block_tokens];
    };
    const auto vector_of = [&](int tile, int block) {
      const int t = token_of(tile);
      return t < 0 ? (int64_t)-1 : token_vector(a, block, t, head);
    };
    // Order: K of an even tile, K of the next, V of both.  (With one row tile the scores run two tiles
    // ahead: a value buffer that waits for its products must not hold up the keys that those need.)
    bool ok = true;
    if constexpr (!FP8) {
      int block[2] = {block_of(0), block_of(1)};   // the table is read a pair ahead
      for (int first = 0; first < tiles && ok; first += 2) {
        const int64_t vec[2] = {vector_of(first, block[0]), vector_of(first + 1, block[1])};
        block[0] = block_of(first + 2);
        block[1] = block_of(first + 3);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int v = u >> 1, stage = u & 1, tile = first + stage;
          if (tile >= tiles || !ok) continue;
          if (tile >= 2) ok = bar_wait_warp<true>(v ? bar.v_empty(stage) : bar.k_empty(stage), (tile >> 1) + 1 & 1, abort, a.wait_ns);
          if (!ok) continue;
          if (v == 0) {
            mark(tile, vec[stage] < 0);
            if (lane == 0) bar_arrive(bar.k_full(stage));   // the copies' arrivals order the copies only
          }
          const uint8_t *const pool = v ? a.c.v : a.c.k;
          const uint32_t dst = (v ? v_at : k_at) + stage * kTileBytes;
#pragma unroll
          for (int pass = 0; pass < kPasses; ++pass) {
            const int64_t at = __shfl_sync(0xffffffffu, vec[stage], pass * kRows + lane / kGroup);
            const int r = row_of(pass, lane / kGroup);
            copy_async_16(dst + piece_at(r, piece), pool + (at < 0 ? 0 : at * (HD * 2) + piece * 16), at < 0 ? 0 : 16);
          }
          copies_arrive(v ? bar.v_full(stage) : bar.k_full(stage));
        }
      }
      copy_async_wait_all();
      if (!ok) __nanosleep(2000);   // nobody may wait for the arrivals that come behind the copies
    } else {
      // Two buffers of registers, for the even and the odd tiles: while one is widened and stored the
      // other's loads are under way.
      uint4 raw[2][kPasses];
      uint8_t byte[2][2] = {};   // [K, V][tile's parity]: the scale of this lane's row, as it is until it is needed
      const auto load = [&](int v, int parity, int64_t vec) {
        const uint8_t *const pool = v ? a.c.v : a.c.k;
        if (v == 0 && vec >= 0) {
          byte[0][parity] = a.c.k_scale[vec];
          byte[1][parity] = a.c.v_scale[vec];
        }
#pragma unroll
        for (int pass = 0; pass < kPasses; ++pass) {
          const int64_t at = __shfl_sync(0xffffffffu, vec, pass * kRows + lane / kGroup);
          raw[parity][pass] = make_uint4(0, 0, 0, 0);
          if (at >= 0) raw[parity][pass] = *(const uint4 *)(pool + at * HD + piece * 16);
        }
      };
      int block[2] = {block_of(0), block_of(1)};   // the table is read a pair ahead
      int64_t vec[2] = {vector_of(0, block[0]), vector_of(1, block[1])};
      block[0] = block_of(2);
      block[1] = block_of(3);
      load(0, 0, vec[0]);
      load(0, 1, vec[1]);
      for (int first = 0; first < tiles && ok; first += 2) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int v = u >> 1, stage = u & 1, tile = first + stage;
          if (tile >= tiles || !ok) continue;
          if (tile >= 2) ok = bar_wait_warp<true>(v ? bar.v_empty(stage) : bar.k_empty(stage), (tile >> 1) + 1 & 1, abort, a.wait_ns);
          if (!ok) continue;
          if (v == 0) {   // v's scales too: the softmax does not wait for the values
            mark(tile, vec[stage] < 0);
            s_scale[0][tile % kKept][my_row] = vec[stage] < 0 ? 0.f : scale_of(byte[0][stage]);
            s_scale[1][tile % kKept][my_row] = vec[stage] < 0 ? 0.f : scale_of(byte[1][stage]);
          }
          uint8_t *const dst = smem + 2 * kTileBytes + (v ? 2 * kTileBytes : 0) + stage * kTileBytes;
#pragma unroll
          for (int pass = 0; pass < kPasses; ++pass) {
            const int r = row_of(pass, lane / kGroup);
            const uint4 x = raw[stage][pass];
            uint4 lo, hi;
            codes_to_half(lo.x, lo.y, x.x);
            codes_to_half(lo.z, lo.w, x.y);
            codes_to_half(hi.x, hi.y, x.z);
            codes_to_half(hi.z, hi.w, x.w);
            *(uint4 *)(dst + piece_at(r, 2 * piece)) = lo;
            *(uint4 *)(dst + piece_at(r, 2 * piece + 1)) = hi;
          }
          fence_async();
          __syncwarp();
          if (lane == 0) bar_arrive(v ? bar.v_full(stage) : bar.k_full(stage));
          if (v == 0) {
            load(1, stage, vec[stage]);
          } else {
            vec[stage] = vector_of(tile + 2, block[stage]);
            block[stage] = block_of(tile + 4);
            load(0, stage, vec[stage]);
          }
        }
      }
    }
  }

  __syncthreads();
  if (threadIdx.x == 0 && s_abort && a.c.status) *a.c.status = EMOE_ERR_DEVICE_TIMEOUT;
  if (warp == kMmaWarp) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

template <typename IO, int HD, bool FP8>
cudaError_t launch(const AttendArgs &a, cudaStream_t st) {
  // queries, two stages of K and of V, room to align; never two blocks an SM (each takes all tensor memory)
  constexpr size_t need = 6 * (size_t)kTile * HD * 2 + 1024, least = 120 * 1024;
  constexpr size_t smem = need > least ? need : least;
  const cudaError_t e = allow_shared<attend_prefix_kernel<IO, HD, FP8>>();
  if (e != cudaSuccess) return e;
  attend_prefix_kernel<IO, HD, FP8><<<a.prefix_items, kThreads, smem, st>>>(a);
  return cudaGetLastError();
}

template <typename T, bool FP8>
cudaError_t by_head_dim(const AttendArgs &a, cudaStream_t st) {
  return a.c.head_dim == 64 ? launch<T, 64, FP8>(a, st) : launch<T, 128, FP8>(a, st);
}

}  // namespace

cudaError_t launch_attend_prefix(const AttendArgs &a, int type, int io, cudaStream_t st) {
  if (type == EMOE_TYPE_E4M3)
    return io == EMOE_TYPE_BF16 ? by_head_dim<__nv_bfloat16, true>(a, st) : by_head_dim<__half, true>(a, st);
  return io == EMOE_TYPE_BF16 ? by_head_dim<__nv_bfloat16, false>(a, st) : by_head_dim<__half, false>(a, st);
}

}  // namespace emoe
