// kv_extend.cu - blocks for the next tokens of a batch (tables, lengths, slots), and the move of an accepted path.
#include <cooperative_groups.h>

#include "serve.h"

namespace emoe {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int32_t kNoBlock = -1;   // an entry of the table whose block is not the sequence's any more

struct Sums {
  int64_t tokens;        // new ones
  int32_t back, wanted;  // blocks
};
__device__ __forceinline__ Sums operator+(const Sums &a, const Sums &b) { return {a.tokens + b.tokens, a.back + b.back, a.wanted + b.wanted}; }
__device__ __forceinline__ Sums shifted_up(const Sums &a, int d) {
  return {__shfl_up_sync(0xffffffffu, a.tokens, d), __shfl_up_sync(0xffffffffu, a.back, d), __shfl_up_sync(0xffffffffu, a.wanted, d)};
}
__device__ __forceinline__ Sums running(Sums x, int lane) {   // sums of the lanes up to this one
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const Sums y = shifted_up(x, d);
    if (lane >= d) x = x + y;
  }
  return x;
}

// n / block_tokens and what is left, n below 2^32: the quotient by the floor of (2^32 - 1) / block_tokens is one too small at most for n
// below 2^31, two beyond.
__device__ __forceinline__ uint32_t block_of(const ExtendArgs &a, uint32_t n, uint32_t &rest) {
  uint32_t q = __umulhi(n, a.per_token);
  rest = n - q * (uint32_t)a.block_tokens;
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (rest >= (uint32_t)a.block_tokens) ++q, rest -= (uint32_t)a.block_tokens;
  return q;
}

// One sequence's change.  (Lengths and block sizes are below 2^31, a length after below 2^32.)
struct Change {
  uint32_t after;              // length
  int32_t had, back, wanted;   // blocks
  int32_t tokens;
  bool fits;                   // its row of the table
};
__device__ __forceinline__ Change change_of(const ExtendArgs &a, int32_t before, int32_t add) {
  Change c;
  c.after = (uint32_t)max((int64_t)0, (int64_t)before + add);
  c.tokens = max(0, add);
  const auto blocks_of = [&](uint32_t n) {
    uint32_t rest;
    const uint32_t q = block_of(a, n, rest);
    return q + (rest != 0);
  };
  const uint32_t has = blocks_of(c.after), most = (uint32_t)a.max_blocks;
  c.had = (int32_t)min(blocks_of((uint32_t)before), most);   // a length beyond the row has no more blocks than that
  c.fits = add <= 0 || has <= most;
  c.back = add < 0 ? max(0, c.had - (int32_t)min(has, most)) : 0;
  c.wanted = add > 0 && c.fits ? (int32_t)has - c.had : 0;
  return c;
}

// Every block of the cluster sums up the whole batch for itself, from lengths that it keeps in shared memory: nothing
// is handed from one to another, and with the one cluster barrier behind the loads the results may go over the
// inputs.  (A second barrier only where blocks are given back, which may be taken again at once.)  What is written is then
// shared out: new and returned blocks by groups of 32 sequences, flattened over a warp's lanes, slots by runs of 128
// tokens a warp, whose sequences are found among the starts in shared memory: those of the run's ends by the warp, those between
// by each lane.  A slot of a new token does not wait for the table: a block that is not in it yet is read from the list.
//
// Bound by latency: loads, a scan, a barrier, loads that depend on it, stores.  Measured: 64 sequences with a new token each 9.8 us on the
// stream (the call on the host; the kernel 8.3), 1021 with up to 127 and a slot map of 129672 18.5 us (16.9 without the count of what does
// not go back).
__global__ void __launch_bounds__(kThreads, 1) kv_extend_kernel(const __grid_constant__ ExtendArgs a) {
  extern __shared__ int32_t s_seq[];   // [5][n_seqs]
  __shared__ Sums s_warp[kWarps];
  __shared__ int32_t s_taken;
  int32_t *const s_before = s_seq, *const s_add = s_seq + a.n_seqs, *const s_first = s_seq + 2 * a.n_seqs, *const s_at = s_seq + 3 * a.n_seqs, *const s_had = s_seq + 4 * a.n_seqs;
  cg::cluster_group cluster = cg::this_cluster();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = (int)cluster.block_rank(), blocks = (int)cluster.num_blocks();
  const auto report = [&](int code) {
    if (a.status) *a.status = code;
  };

  bool some_back = false;
  for (int i = threadIdx.x; i < a.n_seqs; i += kThreads) {
    s_before[i] = max(0, a.lens[i]);
    s_add[i] = a.add[i];
    s_at[i] = 0;   // entries that do not go back
    some_back |= s_add[i] < 0;
  }
  const int32_t n_free = max(0, min(*a.n_free, a.free_capacity));
  if (threadIdx.x == 0) s_taken = 0;
  some_back = __syncthreads_or(some_back);

  const auto check_id = [&](int32_t id) {
    if (id < 0 || id >= a.num_blocks) report(EMOE_ERR_BLOCK_TABLE);
  };
  // Entries that do not go back - blocks that the sequence has given back before, ids beyond the pool - leave no hole in the list: each
  // block of the cluster counts all of them, a lane the first entries of a sequence, the warp what is behind them.
  const auto goes_back = [&](int32_t id) { return id != kNoBlock && id < a.num_blocks; };
  const auto returned_row = [&](int i, const Change &c) { return a.block_table + (int64_t)i * a.max_blocks + (c.had - c.back); };
  if (some_back) {
    for (int i0 = warp * 32; i0 < a.n_seqs; i0 += kThreads) {
      constexpr int kFirst = 8;
      const int i = i0 + lane;
      const int32_t *row = nullptr;
      int32_t n = 0, none = 0, id[kFirst];
      if (i < a.n_seqs) {
        const Change c = change_of(a, s_before[i], s_add[i]);
        n = c.back;
        row = returned_row(i, c);
      }
#pragma unroll
      for (int j = 0; j < kFirst; ++j) id[j] = j < n ? row[j] : 0;
#pragma unroll
      for (int j = 0; j < kFirst; ++j) {
        if (id[j] != kNoBlock) check_id(id[j]);
        none += !goes_back(id[j]);
      }
      for (uint32_t more = __ballot_sync(0xffffffffu, n > kFirst); more; more &= more - 1) {
        const int owner = __ffs(more) - 1;
        const int32_t end = __shfl_sync(0xffffffffu, n, owner);
        const int32_t *const of = (const int32_t *)__shfl_sync(0xffffffffu, (unsigned long long)row, owner);
        int32_t mine = 0;
#pragma unroll 4
        for (int32_t j = kFirst + lane; j < end; j += 32) {
          const int32_t x = of[j];
          if (x != kNoBlock) check_id(x);
          mine += !goes_back(x);
        }
        mine = __reduce_add_sync(0xffffffffu, mine);
        if (lane == owner) none += mine;
      }
      if (i < a.n_seqs) s_at[i] = none;
    }
    __syncthreads();
  }
  // this thread's sequences, one after the other in the batch
  const int per = (a.n_seqs + kThreads - 1) / kThreads, first = min(a.n_seqs, (int)threadIdx.x * per), last = min(a.n_seqs, first + per);
  Sums mine{0, 0, 0};
  for (int i = first; i < last; ++i) {
    const Change c = change_of(a, s_before[i], s_add[i]);
    mine = mine + Sums{(int64_t)c.tokens, c.back - s_at[i], c.wanted};
  }
  const Sums upto = running(mine, lane);
  if (lane == 31) s_warp[warp] = upto;
  __syncthreads();
  if (warp == 0) s_warp[lane] = running(s_warp[lane], lane);
  __syncthreads();
  Sums before = upto;
  before.tokens -= mine.tokens;
  before.back -= mine.back;
  before.wanted -= mine.wanted;
  if (warp > 0) before = before + s_warp[warp - 1];
  const Sums all = s_warp[kWarps - 1];
  const int32_t room = a.free_capacity - n_free, back = min(all.back, room), top = n_free + back;

  // what each sequence gets: its start, and where its blocks lie in the order of those given back or taken (-1: refused)
  for (int i = first; i < last; ++i) {
    const Change c = change_of(a, s_before[i], s_add[i]);
    const int32_t given = c.back - s_at[i];
    s_first[i] = (int32_t)min(before.tokens, (int64_t)a.n_slots);
    s_had[i] = c.had;
    const bool granted = c.fits && (c.tokens == 0 || before.tokens + c.tokens <= a.n_slots) && (c.wanted == 0 || before.wanted + c.wanted <= top);
    if (!granted) report(EMOE_ERR_TOO_LARGE);
    s_at[i] = !granted ? -1 : c.back ? before.back : before.wanted;
    if (granted && c.wanted) atomicMax(&s_taken, before.wanted + c.wanted);
    before = before + Sums{(int64_t)c.tokens, given, c.wanted};
  }
  if (all.back > room && threadIdx.x == 0) report(EMOE_ERR_TOO_LARGE);
  const int32_t tokens = (int32_t)min(all.tokens, (int64_t)a.n_slots);
  cluster.sync();   // all blocks have read what the results may go over

  // Blocks of the 32 sequences of a group, four a lane at a time: read(sequence, which of its blocks) gives an id, and
  // once four of them are under way use(sequence, which, id) takes them on, by all lanes of the warp in the blocks' order (which < 0: this
  // lane has none).  start(sequence): the first one of a group that has any.
  const auto for_blocks = [&](bool returned, auto start, auto read, auto use) {
    for (int group = warp * blocks + rank; group * 32 < a.n_seqs; group += kWarps * blocks) {
      const int i = group * 32 + lane;
      int32_t n = 0;
      if (i < a.n_seqs && s_at[i] >= 0) {
        const Change c = change_of(a, s_before[i], s_add[i]);
        n = returned ? c.back : c.wanted;
      }
      const uint32_t have = __ballot_sync(0xffffffffu, n > 0);
      if (have == 0) continue;
      start(group * 32 + __ffs(have) - 1);
      int32_t end = n;
#pragma unroll
      for (int d = 1; d < 32; d *= 2) {
        const int32_t y = __shfl_up_sync(0xffffffffu, end, d);
        if (lane >= d) end += y;
      }
      const int32_t count = __shfl_sync(0xffffffffu, end, 31);
      for (int32_t base = 0; base < count; base += 4 * 32) {
        int seq[4];
        int32_t which[4], id[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int32_t j = base + 32 * k + lane;
          int owner = 0;   // the first lane whose sum is above j
#pragma unroll
          for (int d = 16; d; d /= 2)
            if (__shfl_sync(0xffffffffu, end, owner + d - 1) <= j) owner += d;
          owner = min(owner, 31);
          seq[k] = group * 32 + owner;
          const int32_t first = __shfl_sync(0xffffffffu, end - n, owner);
          which[k] = j < count ? j - first : -1;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) id[k] = which[k] < 0 ? 0 : read(seq[k], which[k]);
#pragma unroll
        for (int k = 0; k < 4; ++k) use(seq[k], which[k], id[k]);
      }
    }
  };
  const auto row_of = [&](int i) { return a.block_table + (int64_t)i * a.max_blocks + s_had[i]; };   // behind the blocks that the sequence had
  if (all.back > 0) {
    int32_t listed = 0;   // where the group's next id goes
    for_blocks(
        true, [&](int i) { listed = n_free + s_at[i]; },
        [&](int i, int32_t j) { return returned_row(i, change_of(a, s_before[i], s_add[i]))[j]; },
        [&](int, int32_t j, int32_t id) {
          const bool goes = j >= 0 && goes_back(id);
          const uint32_t those = __ballot_sync(0xffffffffu, goes);
          if (goes) {
            const int32_t at = listed + __popc(those & ((1u << lane) - 1));
            if (at < a.free_capacity) a.free_blocks[at] = id;
          }
          listed += __popc(those);
        });
    __threadfence();
    cluster.sync();
  }
  const auto taken_block = [&](int i, int32_t j) { return a.free_blocks[top - 1 - (s_at[i] + j)]; };
  for_blocks(
      false, [](int) {}, taken_block,
      [&](int i, int32_t j, int32_t id) {
        if (j < 0) return;
        check_id(id);
        row_of(i)[j] = id;
      });
  if (rank == 0) {
    for (int i = threadIdx.x; i < a.n_seqs; i += kThreads) {
      const Change c = change_of(a, s_before[i], s_add[i]);
      a.lens_out[i] = s_at[i] < 0 ? s_before[i] : (int32_t)c.after;
      a.q_start[i] = s_first[i];
    }
    if (threadIdx.x == 0) {
      a.q_start[a.n_seqs] = tokens;
      *a.n_free_out = top - s_taken;
    }
  }
  constexpr int kAtOnce = 4, kRun = 32 * kAtOnce;   // tokens of a thread whose table entries are read without waiting for one another
  const auto sequence_of = [&](int i) {   // the last one that starts at token i or before: 32 probes at a time
    int lo = 0;
    for (int hi = a.n_seqs; hi - lo > 1;) {
      const int step = (hi - lo + 31) / 32, at = lo + lane * step;
      const int found = __popc(__ballot_sync(0xffffffffu, at < hi && s_first[at] <= i));
      lo += max(0, found - 1) * step;
      hi = min(hi, lo + step);
    }
    return lo;
  };
  for (int run = rank + blocks * warp; run < (a.n_slots + kRun - 1) / kRun; run += blocks * kWarps) {
    const int base = run * kRun + lane, first_seq = sequence_of(run * kRun), last_seq = sequence_of(run * kRun + kRun - 1);
    int seq[kAtOnce], hi[kAtOnce];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) seq[j] = first_seq, hi[j] = last_seq + 1;
    for (int left = last_seq + 1 - first_seq; left > 1; left = (left + 1) >> 1)
#pragma unroll
      for (int j = 0; j < kAtOnce; ++j) {
        const int mid = (seq[j] + hi[j]) >> 1;
        if (hi[j] - seq[j] > 1) {
          if (s_first[mid] <= base + j * 32) seq[j] = mid;
          else hi[j] = mid;
        }
      }
    int32_t id[kAtOnce];
    uint32_t off[kAtOnce];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      const int i = base + j * 32, s = seq[j];
      id[j] = -1;
      off[j] = 0;
      if (i < tokens && s_at[s] >= 0) {
        const uint32_t column = block_of(a, (uint32_t)(s_before[s] + (i - s_first[s])), off[j]);
        id[j] = (int32_t)column < s_had[s] ? a.block_table[(int64_t)s * a.max_blocks + column] : taken_block(s, (int32_t)column - s_had[s]);
        if (id[j] < 0 || id[j] >= a.num_blocks) {
          report(EMOE_ERR_BLOCK_TABLE);
          id[j] = -1;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j)
      if (base + j * 32 < a.n_slots)
        a.slots[base + j * 32] = id[j] < 0 ? -1 : (int64_t)id[j] * a.block_tokens + off[j];
  }
}

// A thread takes one piece of the head vectors of a path, in one layer's keys or values, and moves it along
// the whole path: sources are read in groups, in rising order, before they are written.  A place that is
// written lies before all sources that are still to be read (the i-th node is at place i or behind it, and
// nodes rise), so a path may overlap its own new places.
// Bound by three loads one after the other (path, table, data).  Measured: 16 paths in 4 layers 8.8 us on the stream (the call on
// the host; the kernel 6), 128 in 24 layers, 22 MB read and written, 10.5 to 12 us.
constexpr int kMoveThreads = 256, kAhead = 8;
template <typename V>   // a piece: 8 or 16 bytes
__global__ void __launch_bounds__(kMoveThreads) kv_keep_kernel(const __grid_constant__ KeepArgs a) {
  extern __shared__ int2 s_move[];   // slots of a node and of its new place, -1 if there is no move
  __shared__ int32_t s_end;
  const int seq = blockIdx.y;
  const int32_t q0 = a.q_start[seq], nodes = max(0, a.q_start[seq + 1] - q0), want = a.n_accepted[seq];
  const int32_t most = max(0, min(want, a.max_accepted));
  const int32_t *const path = a.accepted + (int64_t)seq * a.max_accepted;
  const int64_t start = (int64_t)a.lens[seq] - nodes;
  const auto report = [&]() {
    if (a.c.status) *a.c.status = EMOE_ERR_BLOCK_TABLE;
  };
  if (a.slots) {   // a sequence without a slot for any of its nodes has none of them: it was refused
    bool some = nodes == 0;
    for (int64_t i = (int64_t)q0 + threadIdx.x; i < (int64_t)q0 + nodes; i += kMoveThreads) some |= i >= 0 && i < a.n_slots && a.slots[i] >= 0;
    if (!__syncthreads_or(some)) {
      if (blockIdx.x == 0 && threadIdx.x == 0) a.change[seq] = 0;
      return;
    }
  }
  if (threadIdx.x == 0) s_end = most;
  __syncthreads();
  for (int i = threadIdx.x; i < most; i += kMoveThreads)
    if (path[i] < 0 || path[i] >= nodes || (i > 0 && path[i] <= path[i - 1])) atomicMin(&s_end, i);
  __syncthreads();
  const int32_t count = s_end;
  if (threadIdx.x == 0 && count < want) report();
  const auto slot_of = [&](int64_t place) {
    if (place < 0 || place >= (int64_t)a.max_blocks * a.c.block_tokens) return -1;
    const int32_t column = (int32_t)(place / a.c.block_tokens), id = a.block_table[(int64_t)seq * a.max_blocks + column];
    return id < 0 || id >= a.num_blocks ? -1 : (int32_t)(id * (int64_t)a.c.block_tokens + (place - (int64_t)column * a.c.block_tokens));
  };
  for (int i = threadIdx.x; i < count; i += kMoveThreads) {
    int2 m = make_int2(-1, -1);
    if (path[i] != i) {
      m = make_int2(slot_of(start + path[i]), slot_of(start + i));
      if (m.x < 0 || m.y < 0) {
        m.x = -1;
        report();
      }
    }
    s_move[i] = m;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) a.change[seq] = count - nodes;
  __syncthreads();

  const uint32_t piece_of_head = a.pieces, of_pool = a.c.n_heads * piece_of_head;
  const uint32_t item = blockIdx.x * kMoveThreads + threadIdx.x;
  if (item < a.pools * of_pool) {
    const uint32_t pool = item / of_pool, rest = item - pool * of_pool, head = rest / piece_of_head, piece = rest - head * piece_of_head;
    V *const base = (V *)(a.c.k + pool * a.pool_bytes) + piece;
    uint8_t *const scale = a.c.k_scale && piece == 0 ? a.c.k_scale + pool * a.pool_vectors : nullptr;
    for (int i = 0; i < count; i += kAhead) {
      V x[kAhead];
      uint8_t y[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (i + j < count && s_move[i + j].x >= 0) {
          const int64_t at = kv_vector(a.c, s_move[i + j].x, head);
          x[j] = base[at * piece_of_head];
          if (scale) y[j] = scale[at];
        }
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (i + j < count && s_move[i + j].x >= 0) {
          const int64_t at = kv_vector(a.c, s_move[i + j].y, head);
          base[at * piece_of_head] = x[j];
          if (scale) scale[at] = y[j];
        }
    }
  }
}

}  // namespace

cudaError_t launch_kv_extend(const ExtendArgs &a, cudaStream_t st) {
  const cudaError_t e = allow_shared<kv_extend_kernel>();
  if (e != cudaSuccess) return e;
  // A block writes a slot in 2 ns: more blocks, up to the 8 that a cluster always may have, for long slot maps.
  int blocks = 1;
  while (blocks < 8 && a.n_slots > 2048 * blocks) blocks *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = 20 * (size_t)a.n_seqs;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim = {(unsigned)blocks, 1, 1};
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kv_extend_kernel, a);
}

cudaError_t launch_kv_keep(const KeepArgs &a, bool wide, cudaStream_t st) {
  const dim3 grid((unsigned)(((uint64_t)a.pools * a.c.n_heads * a.pieces + kMoveThreads - 1) / kMoveThreads), a.n_seqs);
  const size_t smem = sizeof(int2) * (size_t)a.max_accepted;
  if (wide) kv_keep_kernel<uint4><<<grid, kMoveThreads, smem, st>>>(a);
  else kv_keep_kernel<uint2><<<grid, kMoveThreads, smem, st>>>(a);
  return cudaGetLastError();
}

}  // namespace emoe
