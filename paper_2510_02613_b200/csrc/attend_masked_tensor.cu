// attend_masked_tensor.cu - attention with masks for many rows a sequence, on the 5th-generation tensor cores.
//
// A tree of drafted tokens or a piece of a prompt has (query tokens) * (query heads per KV head) rows for each KV head of
// its sequence.  A block takes a sequence, a KV head, up to 256 of the rows and a range of the tokens that they
// see; it holds the rows' queries in shared memory and two accumulator sets ("slots") in tensor memory,
//     S = Q K^T (128 x 64), O += P V (128 x head_dim),   P = 2^(scale S - m) rounded to 16 bits,
// and runs through the tokens in steps of 64 (tiles of 128 are brought in), as the prefix kernel does: S has two
// buffers a slot, P is written over its S and multiplied from tensor memory, the maximum in use is only raised when the
// real one passes it by more than 2^8.  With more than 128 rows the slots are two row tiles on the same tokens, each
// without the steps of which its rows see nothing; with fewer they are the same rows on alternating tiles of tokens, joined through
// shared memory at the end.
//
// Masks cost little: a warp whose rows all see a whole step does not look at words of bits.  In a tile that
// some row does not see whole, values that are infinite or not numbers are cleared on their way into shared memory
// (a weight of zero would not silence them); if there was any, the rows that do see them take them from the
// cache at the end.
//
// Warps: 0-3 and 4-7 the softmax of the two slots (a thread a row), 8 and 9 issue the slots' products, 12-15 bring
// K and V rows from their pages into the 128-byte-swizzled tiles that the products read (e4m3 codes widened on the way).
//
// Measured, bf16, head_dim 128, at 1965 MHz: a tile of 128 tokens x 256 rows takes 2.2 us, a unit's start and end 8 us (queries and first
// tiles, 192 KB a block, come for all blocks at once: 3 us; outputs 2.5 us).  8192 tokens of a prompt in a window of 4096, 32 on 4 heads, are
// 1024 units of 33 tiles, 7 rounds on 148 SMs: 572 us by that.  Called for a second the power limit brings the clock down: 637 us at 1762 MHz, 597 at
// 1822, 855 to 920 TFLOP/s, 51 to 55% of a library product's rate.  8 trees of 64 nodes on 16000 tokens: 167 us at 1965 MHz, 182 at 1777.  The same
// prompt on an e4m3 cache: 1060 us at 1965 MHz (codes are widened on their way into shared memory, and each score takes two scales; which of
// the two bounds it was not measured).  Three chains take about as long as one another: of 2.15 us a tile, when it was looked at, 1.88 were
// left without the softmax, 1.94 without the products, 2.15 without the exponentials.  The products of S, 64 columns wide, are bound by
// shared memory (48 clocks for 16 of k, not 32); whole tiles of 128 columns, which are not, leave no scores to work on while the next ones are
// made (2.86 us).
#include "attend_item.cuh"
#include "attend_masked.cuh"
#include "tensor.cuh"

namespace emoe {
namespace {

constexpr int kRows = 2 * kTile;
// Registers a thread of the four warpgroups, out of the 4 x 128 that the block is launched with.
constexpr int kSoftmaxRegs = 160, kMmaRegs = 64, kCopyRegs = 128;
static_assert(2 * kSoftmaxRegs + kMmaRegs + kCopyRegs <= 512, "the block has no more registers than it was launched with");

// The steps of a slot: two runs of 64-token steps, or every second tile.
struct Steps {
  int count, head, skip;   // the first `head` steps are the range's own, the others lie `skip` further on
  bool alternate;
  int slot;
  __device__ __forceinline__ int step(int i) const { return alternate ? ((i >> 1) * 2 + slot) * 2 + (i & 1) : i < head ? i : i + skip; }
};

// Whether the rows first .. last of a tile all see the run's tokens [from, to).
__device__ __forceinline__ bool all_seen(const MaskedArgs &a, const RowTile &t, const Run &r, int last_begin, int first_end, int from, int to) {
  if (a.mask) return to <= t.context;
  return to <= first_end && (from >= last_begin || to <= r.seen || r.seen >= last_begin);
}

// Elements of a 16-byte piece that are infinite or not numbers become zero; whether there were any.
template <typename T, bool FP8>
__device__ __forceinline__ bool clear_odd(uint4 &x) {
  uint32_t *const w = (uint32_t *)&x;
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t odd;
    if constexpr (FP8) odd = __vcmpeq4(w[i] & 0x7f7f7f7fu, 0x7f7f7f7fu);
    else if constexpr (__is_same(T, __half)) odd = __vcmpeq2(w[i] & 0x7c007c00u, 0x7c007c00u);
    else odd = __vcmpeq2(w[i] & 0x7f807f80u, 0x7f807f80u);
    w[i] &= ~odd;
    any |= odd;
  }
  return any != 0;
}

template <typename IO, int HD, bool FP8>
__global__ void __launch_bounds__(kThreads, 1) masked_tensor_kernel(const __grid_constant__ MaskedArgs a) {
  using T = typename Operand<IO, FP8>::type;
  constexpr uint32_t kTileBytes = kTile * HD * 2;
  constexpr float kLift = kWeightLift<T> > 0.f ? kWeightLift<T> - kRaise : 0.f;
  constexpr int kPieces = HD / 8;   // 16-byte pieces of a 16-bit row
  // copying: a row's pieces are taken by kGroup neighbouring lanes, kCopyRows rows at a time by a warp
  constexpr int kGroup = FP8 ? HD / 16 : kPieces, kCopyRows = 32 / kGroup;
  extern __shared__ uint8_t raw_smem[];
  __shared__ __align__(8) uint64_t bars[kBars];
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort, s_odd;
  __shared__ uint32_t s_there[kKept][4];   // tokens that are there: a word of 32 rows from each copying warp
  __shared__ float s_query[FP8 ? kRows : 1];   // e4m3: the queries are this much smaller than those that are multiplied
  __shared__ float2 s_second[kTile];       // the second slot's maximum and sum, where the slots are joined
  __shared__ __align__(16) float s_scale[2][FP8 ? kKept : 1][FP8 ? kTile : 4];   // of K and V
  uint8_t *const smem = (uint8_t *)(((uintptr_t)raw_smem + 1023) & ~(uintptr_t)1023);
  const uint32_t q_at = shared_address(smem), k_at = q_at + 2 * kTileBytes, v_at = k_at + 2 * kTileBytes;
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;

  // the item
  let_next_start();
  const int unit_rank = blockIdx.x / a.tensor_splits, split = blockIdx.x - unit_rank * a.tensor_splits, head = unit_rank % a.c.n_heads;
  const int number = a.tensor_ranked ? ranked_tile(a, a.tensor_tiles_a_seq, unit_rank / a.c.n_heads) : unit_rank / a.c.n_heads;
  const int unit = number * a.c.n_heads + head;
  const RowTile tile = row_tile<kRows>(a, a.tensor_tiles_a_seq, number);
  if (tile.rows == 0 || (a.short_rows && tile.count * a.group <= a.short_rows)) {   // (so few rows may be the other kernel's)
    wait_for_previous();
    return;
  }
  const Run run = run_of(a, tile);
  const int rows = tile.rows;
  const int chunk = ((run.count + a.tensor_splits - 1) / a.tensor_splits + kTile - 1) / kTile * kTile;
  const int u0 = min(run.count, split * chunk), u1 = min(run.count, u0 + chunk);
  const int tiles = (u1 - u0 + kTile - 1) / kTile;
  const bool alternate = rows <= kTile;
  const auto steps_of = [&](int slot) {
    Steps s;
    s.alternate = alternate;
    s.slot = slot;
    const int all = (u1 - u0 + kStep - 1) / kStep;
    if (alternate) {
      const int mine = (tiles + 1 - slot) / 2;
      s.head = s.skip = 0;
      s.count = 2 * mine - (mine > 0 && ((tiles - 1) & 1) == slot ? 2 * tiles - all : 0);
    } else if (a.mask) {
      s.head = s.count = all;
      s.skip = 0;
    } else {
      const Sight first(a, tile, run, slot * kTile), last(a, tile, run, min(slot * kTile + kTile, rows) - 1);
      s.head = max(0, min(all, (run.seen - u0 + kStep - 1) / kStep));
      const int from = max(s.head, max(0, first.begin - u0) / kStep), to = min(all, max(0, last.end - u0 + kStep - 1) / kStep);
      s.skip = from - s.head;
      s.count = s.head + max(0, to - from);
    }
    return s;
  };
  const int readers = alternate ? 1 : 2;   // slots that read a tile
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
    s_abort = s_odd = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(shared_address(&s_tmem)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }

  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = s_tmem;
  volatile int *const abort = &s_abort;

  if (warp < kSoftmaxWarps) {
    take_registers<kSoftmaxRegs>();
    const int slot = warp >> 2, local = (warp & 3) * 32 + lane;   // this thread's row in the slot
    const int row0 = alternate ? 0 : slot * kTile, row = row0 + local;
    const bool busy = row0 + (warp & 3) * 32 < rows;   // any real row in the warp
    const Steps mine = steps_of(slot);
    const int others = steps_of(1 - slot).count, n_steps = mine.count;
    float x[2][32];   // the row's query, then a step's scores and weights
    // not zero: a masked score, minus infinity, has to stay that (and every other one comes to zero all the same)
    const float c = fmaxf(fabsf(a.scale_log2), 0x1p-149f);
    float query_by = 1.f;   // e4m3: the row's query is this much smaller than the one that is multiplied
    {
      // The queries, a row by neighbouring lanes: 32 rows a warp, 16 where the slots have the same ones.  Rows that do not exist are
      // zero.  (Loops here and at the end are short on purpose: a block runs them once, from instructions that are not in its cache yet.)
      constexpr int kRowsAtOnce = 32 / kPieces;
      const bool negative = a.scale_log2 < 0.f;   // scores are multiplied by its magnitude: the queries take the sign
      const int mine = alternate ? 16 : 32, base = warp * mine, piece = lane % kPieces;
      const int64_t from = row_at(a, tile, head, min(base + lane, rows - 1), a.q_stride);
#pragma unroll 2
      for (int i = 0; i < mine; i += kRowsAtOnce) {
        const int r = i + lane / kPieces, row = base + r;
        const IO *const src = (const IO *)a.q + __shfl_sync(0xffffffffu, from, r) + piece * 8;
        const uint32_t at = row / kTile * kTileBytes + piece_at(row % kTile, piece);
        if (!FP8 && !negative) {
          copy_async_16(q_at + at, src, row < rows ? 16 : 0);
        } else if constexpr (!FP8) {
          const uint4 v = row < rows ? *(const uint4 *)src : make_uint4(0, 0, 0, 0);
          *(uint4 *)(smem + at) = make_uint4(v.x ^ 0x80008000u, v.y ^ 0x80008000u, v.z ^ 0x80008000u, v.w ^ 0x80008000u);
        } else {
          const uint4 v = row < rows ? *(const uint4 *)src : make_uint4(0, 0, 0, 0);
          uint32_t top = 0;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float2 f = Pair<IO>::unpack(word(v, k));
            top = max(top, max(__float_as_uint(f.x) & 0x7fffffffu, __float_as_uint(f.y) & 0x7fffffffu));
          }
#pragma unroll
          for (int d = 1; d < kPieces; d *= 2) top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
          float by = query_scale(top);
          if (piece == 0) s_query[row] = 1.f / by;
          by = negative ? -by : by;
          const float2 e0 = Pair<IO>::unpack(v.x), e1 = Pair<IO>::unpack(v.y), e2 = Pair<IO>::unpack(v.z), e3 = Pair<IO>::unpack(v.w);
          *(uint4 *)(smem + at) = make_uint4(Pair<T>::pack(e0.x * by, e0.y * by), Pair<T>::pack(e1.x * by, e1.y * by), Pair<T>::pack(e2.x * by, e2.y * by),
                                             Pair<T>::pack(e3.x * by, e3.y * by));
        }
      }
      if (!FP8 && !negative) {
        copies_arrive(bar.q_full());
      } else {
        fence_async();
        bar_arrive(bar.q_full());
      }
      if constexpr (FP8) {
        asm volatile("bar.sync 1, 256;" ::: "memory");
        query_by = s_query[row0 + local];
      }
    }
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;   // lane 32 * (warp % 4) in the address's upper half
    const uint32_t s_base = tmem + lanes + kColS + slot * kTile, o_col = tmem + lanes + kColO + slot * HD;
    const Sight sight(a, tile, run, min(row, rows - 1));
    const int last_begin = Sight(a, tile, run, min(row0 + (warp & 3) * 32 + 31, rows - 1)).begin;   // of the warp's rows
    const int first_end = Sight(a, tile, run, min(row0 + (warp & 3) * 32, rows - 1)).end;
    float m = -CUDART_INF_F, l = 0.f, v_ref = 0.f;   // v_ref: the largest scale of v so far that the row sees
    bool ok = true;
    if (n_steps > 0) {   // the first step's scores
      ok = bar_wait_warp(bar.s_full(slot, 0), 0, abort, a.wait_ns);
      fence_after();
      if (ok && busy) {
        tmem_load(x[0], s_base);
        tmem_load(x[1], s_base + 32);
      }
    }
    // Exponentials of the two slots' warps that share a quarter of the SM take turns, 0 first: while one has
    // them the other fetches its scores and finds their maximum.  Together they would both wait.
    const bool both = steps_of(1).count > 0 && (alternate ? 0 : kTile) + (warp & 3) * 32 < rows;   // the other has rows too
    for (int i = 0; i < n_steps && ok; ++i) {
      const int half = i & 1, step = mine.step(i), kept = (step >> 1) % kKept, part = step & 1;
      const uint32_t s_col = s_base + half * kStep;
      const bool wait_turn = both && (slot ? i < others : i > 0 && i - 1 < others);
      const bool give_turn = both && (slot ? i + 1 < others : i < others);
      if (busy) {
        const float *const k_scale = s_scale[0][FP8 ? kept : 0] + (FP8 ? part * kStep : 0);
        const float *const v_scale = s_scale[1][FP8 ? kept : 0] + (FP8 ? part * kStep : 0);
        uint32_t seen[2] = {s_there[kept][2 * part], s_there[kept][2 * part + 1]};
        const int at = u0 + step * kStep;
        if (!all_seen(a, tile, run, last_begin, first_end, at, min(at + kStep, u1))) {
          seen[0] &= sight.word(a, tile, run, at);
          seen[1] &= sight.word(a, tile, run, at + 32);
        }
        const bool mixed = !__all_sync(0xffffffffu, (seen[0] & seen[1]) == 0xffffffffu);
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
              if (!mixed) v_top = max3(max3(v_top, v.x, v.y), v.z, v.w);
            }
          }
          if (mixed) {
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              if (!(seen[j] >> e & 1)) x[j][e] = -CUDART_INF_F;
              if constexpr (FP8) v_top = fmaxf(v_top, seen[j] >> e & 1 ? v_scale[32 * j + e] : 0.f);
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
            if (!mixed) {
#pragma unroll
              for (int e = 0; e < 32; e += 4) {
                const float4 v = *(const float4 *)(v_scale + 32 * j + e);
                x[j][e] *= v.x * v_by;
                x[j][e + 1] *= v.y * v_by;
                x[j][e + 2] *= v.z * v_by;
                x[j][e + 3] *= v.w * v_by;
              }
            } else {   // (a scale that the row does not see may be anything)
#pragma unroll
              for (int e = 0; e < 32; ++e) x[j][e] = seen[j] >> e & 1 ? x[j][e] * (v_scale[32 * j + e] * v_by) : 0.f;
            }
          }
#pragma unroll
          for (int e = 0; e < 16; ++e) p[e] = Pair<T>::pack(x[j][2 * e], x[j][2 * e + 1]);
          tmem_store_16(s_col + 16 * j, p);   // over columns that have been read
        }
        l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      }
      // The weights are announced before the next step's scores are waited for: those come behind the last step's product
      // in the tensor cores' queue, and would hold up this one's.
      if (busy) tmem_stored();
      fence_before();
      __syncwarp();
      if (lane == 0) bar_arrive(bar.p_full(slot, half));   // one a warp: arrivals at one barrier go one by one
      if (i + 1 < n_steps) {
        ok = bar_wait_warp(bar.s_full(slot, half ^ 1), ((i + 1) >> 1) & 1, abort, a.wait_ns);
        if (!ok) break;
        fence_after();
        if (busy) {
          tmem_load(x[0], s_base + (half ^ 1) * kStep);
          tmem_load(x[1], s_base + (half ^ 1) * kStep + 32);
        }
      }
    }
    if (!ok) tmem_stored();   // what was under way when a wait ran out
    // The last two products may be under way.  A parity tells one phase from the next only: each half has a
    // barrier of its own, whose phase before is over by then.
    for (int i = max(0, n_steps - 2); i < n_steps && ok; ++i)
      ok = bar_wait_warp(bar.o_full(slot, i & 1), (i >> 1) & 1, abort, a.wait_ns);
    fence_after();

    // 32 columns of this row's unnormalised output.
    const bool odd = *(volatile int *)&s_odd != 0;
    const auto columns = [&](float (&y)[32], int j) {
      __syncwarp();
      if (n_steps == 0 || !ok) {
#pragma unroll
        for (int e = 0; e < 32; ++e) y[e] = 0.f;
        return;
      }
      tmem_load(y, o_col + 32 * j);
      tmem_wait(y);
      if constexpr (FP8) {
#pragma unroll
        for (int e = 0; e < 32; ++e) y[e] *= v_ref;
      }
      if (__builtin_expect(odd, 0)) {   // values that were cleared, for who sees them
        const int tile_begin = Sight(a, tile, run, rows - 1).begin, tile_end = Sight(a, tile, run, 0).end;
        for (int i = 0; i < n_steps; ++i) {
          const int step = mine.step(i), t = step >> 1, from = u0 + t * kTile;
          if (all_seen(a, tile, run, tile_begin, tile_end, from, min(from + kTile, u1))) continue;
          for (int k = 0; k < 2; ++k) {
            uint32_t bits = sight.word(a, tile, run, u0 + step * kStep + 32 * k);
            for (; bits; bits &= bits - 1) {
              const int u = u0 + step * kStep + 32 * k + __ffs(bits) - 1;
              if (u >= u1) break;
              const TokenPlace p = place_of_token(a, run.token(u));
              const int64_t vec = masked_vector(a, a.block_table[(int64_t)tile.seq * a.max_blocks + p.column], p.off, head);
              if (vec < 0) continue;
#pragma unroll
              for (int e = 0; e < 32; ++e) {
                if constexpr (FP8) {
                  if ((a.c.v[vec * HD + 32 * j + e] & 127) == 127) y[e] = CUDART_NAN_F;
                } else {
                  const float v = (float)((const T *)a.c.v)[vec * HD + 32 * j + e];
                  if (!isfinite(v)) y[e] += v;
                }
              }
            }
          }
        }
      }
    };
    // what a wait that ran out leaves behind is not a number
    if (n_steps == 0 || !ok) {
      m = -CUDART_INF_F;
      l = ok ? 0.f : CUDART_NAN_F;
      // No score has waited for the queries, whose place the outputs go through: they are there soon, whoever has given up.
      int late = 0;
      bar_wait_warp(bar.q_full(), 0, &late, kDrainNs);
    } else {
      m -= kLift;
    }
    float to_first = 1.f, to_second = 0.f;   // factors of the two slots' outputs
    bool joined = false;
    float *const other = (float *)(smem + 2 * kTileBytes);   // the second slot's output: in its buffers of K and V, which nobody uses any more
    const auto other_at = [&](int j, int e) {   // 16 bytes of its columns 32 j + e .. + 3
      const int col = 32 * j + e, half = col / (HD / 2), piece = (col % (HD / 2)) / 4;
      return (float4 *)((uint8_t *)other + (half ? 2 * kTileBytes : 0) + kTileBytes + local * (HD * 2) + ((piece ^ (local & (HD / 8 - 1))) << 4));
    };
    if (alternate) {
      if (slot == 1) {
        s_second[local] = make_float2(m, l);
        if (busy && n_steps > 0) {
#pragma unroll 1
          for (int j = 0; j < HD / 32; ++j) {
            float y[32];
            columns(y, j);
#pragma unroll
            for (int e = 0; e < 32; e += 4) *other_at(j, e) = make_float4(y[e], y[e + 1], y[e + 2], y[e + 3]);
          }
        }
      }
      asm volatile("bar.sync 1, 256;" ::: "memory");
      if (slot == 0 && others > 0) {
        const float2 second = s_second[local];
        const float top = fmaxf(m, second.x);
        to_first = top == -CUDART_INF_F ? 0.f : exp2_fast(m - top);
        to_second = top == -CUDART_INF_F ? 0.f : exp2_fast(second.x - top);
        // an empty part does not count; a sum that is not a number shows
        l = (l == 0.f ? 0.f : l * to_first) + (second.y == 0.f ? 0.f : second.y * to_second);
        m = top;
        if (l != l) to_first = CUDART_NAN_F;
        joined = second.y != 0.f;
      }
    }
    wait_for_previous();
    if (busy && (slot == 0 || !alternate)) {
      const bool last = a.tensor_splits == 1;
      const int64_t part = ((int64_t)unit * a.tensor_splits + split) * kRows + row;
      const float by = last ? (l > 0.f || l != l ? 1.f / l : 0.f) : 1.f;
      if (row < rows) {
        if (last) write_lse(a, tile, head, row, m, l);
        else a.tensor_ml[part] = make_float2(m, l);
      }
      // Columns go through shared memory (the queries' place), 128 bytes of a row at a time, from a row a thread to 8 neighbouring
      // lanes a row: a lane's rows are lane / 8 and every fourth one after it.
      constexpr int kBatch = HD / 64;   // 128-byte pieces of a row under way at once: what the place holds
      const int64_t mine = last ? row_at(a, tile, head, min(row, rows - 1), a.out_stride) : part * HD;
      uint8_t *const stage = smem + (alternate ? 0 : slot * kTileBytes) + (warp & 3) * (kBatch * 4096);
      const int lane_row = lane >> 3, piece = lane & 7, left = rows - row0 - (warp & 3) * 32 - lane_row;   // rows from the first one on
      int64_t to[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) to[i] = __shfl_sync(0xffffffffu, mine, 4 * i + lane_row) + piece * 4;
#pragma unroll 1
      for (int j0 = 0; j0 < HD / 32; j0 += kBatch) {
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
          float y[32];
          columns(y, j0 + b);
          if (alternate) {
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
              const float4 z = joined ? *other_at(j0 + b, e) : make_float4(0.f, 0.f, 0.f, 0.f);
              y[e] = y[e] * to_first + z.x * to_second;
              y[e + 1] = y[e + 1] * to_first + z.y * to_second;
              y[e + 2] = y[e + 2] * to_first + z.z * to_second;
              y[e + 3] = y[e + 3] * to_first + z.w * to_second;
            }
          }
#pragma unroll
          for (int e = 0; e < 32; e += 4)
            *(float4 *)(stage + b * 4096 + lane * 128 + ((e / 4 ^ (lane & 7)) << 4)) = make_float4(y[e] * by, y[e + 1] * by, y[e + 2] * by, y[e + 3] * by);
        }
        __syncwarp();
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
          float4 z[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) z[i] = *(const float4 *)(stage + b * 4096 + (4 * i + lane_row) * 128 + ((piece ^ (4 * i + lane_row & 7)) << 4));
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (4 * i < left) {
              if (last) *(uint2 *)((IO *)a.out + to[i] + 32 * (j0 + b)) = make_uint2(Pair<IO>::pack(z[i].x, z[i].y), Pair<IO>::pack(z[i].z, z[i].w));
              else *(float4 *)(a.tensor_o + to[i] + 32 * (j0 + b)) = z[i];
            }
        }
        __syncwarp();
      }
    }
    fence_before();
  } else if (warp < kCopyWarp0) {
    give_registers<kMmaRegs>();
    const int slot = warp - kMmaWarp;
    if (slot < 2) {   // the whole warp goes along, one lane issues: addresses stay in uniform registers
      const Steps mine = steps_of(slot);
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
      const auto scores = [&](int stage, int part, int half) {
        if (!one) return;
        const uint64_t k = k_op + stage * (kTileBytes >> 4) + part * (kStep * 128 >> 4);
#pragma unroll
        for (int i = 0; i < HD / 16; ++i) {
          const int off = ((i >> 2) * (kTile * 128) + (i & 3) * 32) >> 4;
          mma_ss(s_at + half * kStep, q + off, k + off, kIdS, i > 0);
        }
      };
      const auto values = [&](int stage, int part, int half, bool add) {
        if (!one) return;
        const uint64_t v = v_op + stage * (kTileBytes >> 4) + part * (kStep * 128 >> 4);
#pragma unroll
        for (int i = 0; i < kStep / 16; ++i) mma_ts(o_at, s_at + half * kStep + i * 8, v + i * (2048 >> 4), kIdO, add || i > 0);
      };
      bool ok = bar_wait_warp(bar.q_full(), 0, abort, a.wait_ns);
      if constexpr (!FP8) fence_async();   // (copied as ordinary writes)
      const auto tile_of = [&](int i) { return mine.step(i) >> 1; };
      const auto last_of_tile = [&](int i) { return i + 1 == mine.count || tile_of(i + 1) != tile_of(i); };
      // A slot that leaves out a tile of both still gives its buffers back, once they have been filled: the
      // phases of a barrier are told apart by their parity only.
      int k_next = alternate ? slot : 0, v_next = k_next;   // tiles not yet taken or left out
      const auto pass = [&](int &next, int to, bool v) {
        for (; next < to && ok; next += alternate ? 2 : 1) {
          const int stage = next & 1;
          ok = bar_wait_warp(v ? bar.v_full(stage) : bar.k_full(stage), (next >> 1) & 1, abort, a.wait_ns);
          if (ok && lane == 0) bar_arrive(v ? bar.v_empty(stage) : bar.k_empty(stage));
        }
      };
      const auto start = [&](int i) {   // S of step i
        const int step = mine.step(i), tile = step >> 1, stage = tile & 1;
        if (i == 0 || tile_of(i - 1) != tile) {
          pass(k_next, tile, false);
          k_next = tile + (alternate ? 2 : 1);
          ok = ok && bar_wait_warp(bar.k_full(stage), (tile >> 1) & 1, abort, a.wait_ns);
          if constexpr (!FP8) fence_async();
        }
        if (!ok) return;
        fence_after();
        scores(stage, step & 1, i & 1);
        commit(bar.s_full(slot, i & 1));
        if (last_of_tile(i)) commit(bar.k_empty(stage));
      };
      for (int i = 0; i < 2; ++i)
        if (i < mine.count && ok) start(i);
      for (int i = 0; i < mine.count && ok; ++i) {
        const int step = mine.step(i), tile = step >> 1, stage = tile & 1;
        if (i == 0 || tile_of(i - 1) != tile) {
          pass(v_next, tile, true);
          v_next = tile + (alternate ? 2 : 1);
          ok = ok && bar_wait_warp(bar.v_full(stage), (tile >> 1) & 1, abort, a.wait_ns);
          fence_async();
        }
        ok = ok && bar_wait_warp(bar.p_full(slot, i & 1), (i >> 1) & 1, abort, a.wait_ns);
        if (!ok) break;
        fence_after();
        values(stage, step & 1, i & 1, i > 0);
        commit(bar.o_full(slot, i & 1));
        if (last_of_tile(i)) commit(bar.v_empty(stage));
        if (i + 2 < mine.count) start(i + 2);
      }
      while (ok && (k_next < tiles || v_next < tiles)) {   // what the other slot still reads
        pass(k_next, min(tiles, k_next + 1), false);
        pass(v_next, min(tiles, min(k_next, v_next + 1)), true);
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
    // A warp has 32 neighbouring rows of a tile; each lane finds one of them in the table.
    constexpr int kPasses = 32 / kCopyRows;
    const int piece = lane % kGroup, my_row = w * 32 + lane;
    const auto row_of = [&](int pass) { return w * 32 + pass * kCopyRows + lane / kGroup; };
    const int32_t *const table = a.block_table + (int64_t)tile.seq * a.max_blocks;
    const int tile_begin = Sight(a, tile, run, rows - 1).begin, tile_end = Sight(a, tile, run, 0).end;
    const auto whole = [&](int t) {   // all rows see the whole tile
      const int from = u0 + t * kTile;
      return all_seen(a, tile, run, tile_begin, tile_end, from, min(from + kTile, u1));
    };
    const auto mark = [&](int t, bool there) {
      const uint32_t word = __ballot_sync(0xffffffffu, there);
      if (lane == 0) s_there[t % kKept][w] = word;
      __syncwarp();
    };
    // What the table says of this lane's token of a tile: the block, and the place there (beyond any block: there is no token).
    constexpr uint32_t kNone = 0xffffffffu;
    struct Found { int block; uint32_t off; };
    const auto find = [&](int t) {
      const int u = u0 + t * kTile + my_row;
      if (t >= tiles || u >= u1) return Found{0, kNone};
      const TokenPlace p = place_of_token(a, run.token(u));
      return Found{table[p.column], p.off};
    };
    const auto vector_of = [&](const Found &f) { return f.off == kNone ? (int64_t)-1 : masked_vector(a, f.block, f.off, head); };
    // Order: K of an even tile, K of the next, V of both.  (With one row tile the scores run two tiles
    // ahead: a value buffer that waits for its products must not hold up the keys that those need.)
    bool ok = true;
    if constexpr (!FP8) {
      Found next[2] = {find(0), find(1)};   // the table is read a pair ahead
      for (int first = 0; first < tiles && ok; first += 2) {
        int64_t vec[2];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int v = u >> 1, stage = u & 1, t = first + stage;
          if (v == 0) {
            vec[stage] = vector_of(next[stage]);
            next[stage] = find(t + 2);
          }
          if (t >= tiles || !ok) continue;
          if (t >= 2) ok = bar_wait_warp<true>(v ? bar.v_empty(stage) : bar.k_empty(stage), (t >> 1) + 1 & 1, abort, a.wait_ns);
          if (!ok) continue;
          if (v == 0) {
            mark(t, vec[stage] >= 0);
            if (lane == 0) bar_arrive(bar.k_full(stage));   // the copies' arrivals order the copies only
          }
          const uint8_t *const pool = v ? a.c.v : a.c.k;
          if (v == 0 || whole(t)) {
            const uint32_t dst = (v ? v_at : k_at) + stage * kTileBytes;
#pragma unroll
            for (int pass = 0; pass < kPasses; ++pass) {
              const int64_t at = __shfl_sync(0xffffffffu, vec[stage], pass * kCopyRows + lane / kGroup);
              copy_async_16(dst + piece_at(row_of(pass), piece), pool + (at < 0 ? 0 : at * (HD * 2) + piece * 16), at < 0 ? 0 : 16);
            }
            copies_arrive(v ? bar.v_full(stage) : bar.k_full(stage));
          } else {   // through registers, in groups
            constexpr int kAtOnce = 8 < kPasses ? 8 : kPasses;
            uint8_t *const dst = smem + 4 * kTileBytes + stage * kTileBytes;
            bool any = false;
#pragma unroll 1
            for (int p0 = 0; p0 < kPasses; p0 += kAtOnce) {
              uint4 raw[kAtOnce];
#pragma unroll
              for (int p = 0; p < kAtOnce; ++p) {
                const int64_t at = __shfl_sync(0xffffffffu, vec[stage], (p0 + p) * kCopyRows + lane / kGroup);
                raw[p] = make_uint4(0, 0, 0, 0);
                if (at >= 0) raw[p] = *(const uint4 *)(pool + at * (HD * 2) + piece * 16);
              }
#pragma unroll
              for (int p = 0; p < kAtOnce; ++p) {
                any |= clear_odd<T, false>(raw[p]);
                *(uint4 *)(dst + piece_at(row_of(p0 + p), piece)) = raw[p];
              }
            }
            if (any) s_odd = 1;
            fence_async();
            bar_arrive(bar.v_full(stage));
          }
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
          const int64_t at = __shfl_sync(0xffffffffu, vec, pass * kCopyRows + lane / kGroup);
          raw[parity][pass] = make_uint4(0, 0, 0, 0);
          if (at >= 0) raw[parity][pass] = *(const uint4 *)(pool + at * HD + piece * 16);
        }
      };
      Found next[2] = {find(0), find(1)};   // the table is read a pair ahead
      int64_t vec[2] = {vector_of(next[0]), vector_of(next[1])};
      load(0, 0, vec[0]);
      load(0, 1, vec[1]);
      next[0] = find(2);
      next[1] = find(3);
      for (int first = 0; first < tiles && ok; first += 2) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int v = u >> 1, stage = u & 1, t = first + stage;
          if (t >= tiles || !ok) continue;
          if (t >= 2) ok = bar_wait_warp<true>(v ? bar.v_empty(stage) : bar.k_empty(stage), (t >> 1) + 1 & 1, abort, a.wait_ns);
          if (!ok) continue;
          if (v == 0) {   // v's scales too: the softmax does not wait for the values
            mark(t, vec[stage] >= 0);
            s_scale[0][t % kKept][my_row] = vec[stage] < 0 ? 0.f : scale_of(byte[0][stage]);
            s_scale[1][t % kKept][my_row] = vec[stage] < 0 ? 0.f : scale_of(byte[1][stage]);
          }
          uint8_t *const dst = smem + 2 * kTileBytes + (v ? 2 * kTileBytes : 0) + stage * kTileBytes;
          const bool look = v && !whole(t);
          bool any = false;
#pragma unroll
          for (int pass = 0; pass < kPasses; ++pass) {
            const int r = row_of(pass);
            uint4 x = raw[stage][pass];
            if (look) any |= clear_odd<T, true>(x);
            uint4 lo, hi;
            codes_to_half(lo.x, lo.y, x.x);
            codes_to_half(lo.z, lo.w, x.y);
            codes_to_half(hi.x, hi.y, x.z);
            codes_to_half(hi.z, hi.w, x.w);
            *(uint4 *)(dst + piece_at(r, 2 * piece)) = lo;
            *(uint4 *)(dst + piece_at(r, 2 * piece + 1)) = hi;
          }
          if (any) s_odd = 1;
          fence_async();
          __syncwarp();
          if (lane == 0) bar_arrive(v ? bar.v_full(stage) : bar.k_full(stage));
          if (v == 0) {
            load(1, stage, vec[stage]);
          } else {
            vec[stage] = vector_of(next[stage]);
            next[stage] = find(t + 4);
            load(0, stage, vec[stage]);
          }
        }
      }
    }
    wait_for_previous();
  }

  __syncthreads();
  if (threadIdx.x == 0 && s_abort && a.c.status) *a.c.status = EMOE_ERR_DEVICE_TIMEOUT;
  if (warp == kMmaWarp) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
  }
}

template <typename IO, int HD, bool FP8>
cudaError_t launch(const MaskedArgs &a, bool early, cudaStream_t st) {
  // queries, two stages of K and of V, room to align; never two blocks an SM (each takes all tensor memory)
  constexpr size_t need = 6 * (size_t)kTile * HD * 2 + 1024, least = 120 * 1024;
  constexpr size_t smem = need > least ? need : least;
  const cudaError_t e = allow_shared<masked_tensor_kernel<IO, HD, FP8>>();
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)a.tensor_tiles * a.c.n_heads * a.tensor_splits);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = early ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, masked_tensor_kernel<IO, HD, FP8>, a);
}

template <typename T, bool FP8>
cudaError_t by_head_dim(const MaskedArgs &a, bool early, cudaStream_t st) {
  return a.c.head_dim == 64 ? launch<T, 64, FP8>(a, early, st) : launch<T, 128, FP8>(a, early, st);
}

}  // namespace

cudaError_t launch_masked_tensor(const MaskedArgs &a, int type, int io, bool early, cudaStream_t st) {
  if (type == EMOE_TYPE_E4M3)
    return io == EMOE_TYPE_BF16 ? by_head_dim<__nv_bfloat16, true>(a, early, st) : by_head_dim<__half, true>(a, early, st);
  return io == EMOE_TYPE_BF16 ? by_head_dim<__nv_bfloat16, false>(a, early, st) : by_head_dim<__half, false>(a, early, st);
}

}  // namespace emoe
