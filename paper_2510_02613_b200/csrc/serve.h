// serve.h - operators that serve from one rank's arenas: geometry shared by host and device,
// device helpers, launchers.  The entry points are in serve.cpp.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "../../include/emoe.h"

namespace emoe {

// One layer of a paged KV cache.  Vector indices count head vectors inside one pool (K or V).
struct KvLayer {
  uint8_t *k, *v;            // first byte of the layer's pools
  uint8_t *k_scale, *v_scale;  // first scale byte (e4m3), else null
  int32_t *status;
  int64_t n_slots;           // num_blocks * block_tokens
  int32_t block_tokens, n_heads, head_dim;
  int32_t head_major;
};

// Vector index of (slot, head) inside a pool; slot must be in [0, n_slots).
__host__ __device__ __forceinline__ int64_t kv_vector(const KvLayer &c, int64_t slot, int32_t head) {
  if (!c.head_major) return slot * c.n_heads + head;
  const uint32_t s = (uint32_t)slot, b = (uint32_t)c.block_tokens;  // n_slots < 2^31
  const uint32_t block = s / b, off = s - block * b;
  return ((int64_t)block * c.n_heads + head) * b + off;
}

__host__ __device__ __forceinline__ bool kv_slot_ok(const KvLayer &c, int64_t slot) {
  return slot >= 0 && slot < c.n_slots;
}

cudaError_t launch_kv_append(const KvLayer &c, int type, const void *k, const void *v, int64_t ks, int64_t vs,
                             int in_type, const int64_t *slots, int n, cudaStream_t st);
cudaError_t launch_kv_gather(const KvLayer &c, int type, const int64_t *slots, int n, void *k, void *v,
                             int64_t ks, int64_t vs, int out_type, cudaStream_t st);

struct ExtendArgs {
  const int32_t *lens, *add;
  int32_t *block_table, *free_blocks;
  const int32_t *n_free;
  int32_t *q_start;
  int64_t *slots;
  int32_t *lens_out, *n_free_out, *status;
  int32_t n_seqs, max_blocks, free_capacity, n_slots, num_blocks, block_tokens;
  uint32_t per_token;                   // (2^32 - 1) / block_tokens
};
cudaError_t launch_kv_extend(const ExtendArgs &a, cudaStream_t st);

struct KeepArgs {
  KvLayer c;                 // of layer 0: the others follow, K and V in turn
  uint64_t pool_bytes, pool_vectors;
  const int32_t *block_table, *lens, *q_start, *accepted, *n_accepted;
  const int64_t *slots;      // null: every sequence has its nodes
  int32_t *change;
  uint32_t pools, pieces;    // 2 * layers; pieces of a head vector
  int32_t n_seqs, max_blocks, max_accepted, num_blocks, n_slots;
};
cudaError_t launch_kv_keep(const KeepArgs &a, bool wide, cudaStream_t st);   // wide: pieces of 16 bytes, else of 8

// How attention is cut: a function of what the caller knows on the host.
struct AttendShape {
  int32_t seq_rows;                     // rows of one sequence and KV head: q_len * query heads per KV head
  int32_t prefix_splits, prefix_chunk;  // token ranges of the prefix, tokens of each
  int32_t own_splits, own_chunk;
  int64_t prefix_items, own_items;
  int32_t tensor;                       // the prefix goes through its own kernel on the 5th-generation tensor cores
  int32_t alternate;                    // ... whose two slots take the same rows on alternating tiles of tokens
  int64_t parts;                        // (row, split) pairs that go through the workspace; 0: none
};
AttendShape attend_shape(int n_heads, int n_seqs, int q_len, int n_q_heads, int head_dim, bool e4m3, int64_t own_max, int prefix_len);
// The most `parts` of a call of up to these sizes: grows with each of them (n_heads and head_dim are the cache's).
int64_t attend_parts(int n_heads, int n_seqs, int q_len, int n_q_heads, int head_dim, bool e4m3, int64_t own_max, int prefix_len);

struct AttendArgs {
  KvLayer c;
  int32_t num_blocks;
  const void *q;
  void *out;
  float *lse;
  int64_t q_stride, out_stride;         // elements from one query token to the next
  const int32_t *block_table, *own_lens, *prefix_table;
  float2 *part_ml;                      // [row][split]: maximum (log2) and sum
  float *part_o;                        // [row][split][head_dim]
  int32_t n_seqs, q_len, n_q_heads, group, max_blocks, prefix_len;
  float scale_log2;
  int32_t seq_rows, prefix_splits, prefix_chunk, own_splits, own_chunk;
  int32_t tensor, alternate;
  uint32_t prefix_items, own_items;
  unsigned long long wait_ns;           // bound of a wait inside a kernel, 0: for nothing
};
cudaError_t launch_attend_prefix(const AttendArgs &a, int type, int io, cudaStream_t st);
cudaError_t launch_attend(const AttendArgs &a, int type, int io, cudaStream_t st);

// Attention of packed query tokens over their own sequences, with masks: how it is cut.
constexpr int kMaskedFewRows = 8, kMaskedRows = 16, kMaskedTensorRows = 256;   // rows of a tile
struct MaskedShape {
  int32_t tiles, tiles_a_seq;      // row tiles: in all; of each sequence, 0: as many as its tokens make
  int32_t splits;                  // token ranges a tile
  int64_t parts;                   // rows that go through the workspace
};
struct MaskedShapes {
  MaskedShape rows, tensor;        // tiles 0: the kernel has nothing to do
  int32_t few;                     // rows: tiles of kMaskedFewRows
  int32_t ranked, tensor_ranked;   // sequences in the order of their lengths, the longest first
};
struct MaskedSizes {
  int32_t n_heads, n_seqs, n_tokens, max_q, n_q_heads, head_dim;
  bool e4m3;
  int64_t most_tokens;             // that a tile of rows runs through
  bool by_length;                  // ... which goes by the sequence's length, not by the window
};
MaskedShapes masked_shapes(const MaskedSizes &n);
// The most `parts` of a call of up to these sizes, of either kernel.
void masked_parts(const MaskedSizes &n, int64_t &rows, int64_t &tensor);

struct MaskedArgs {
  KvLayer c;
  int32_t num_blocks;
  const void *q;
  void *out;
  float *lse;
  int64_t q_stride, out_stride;         // elements from one query token to the next
  const int32_t *block_table, *own_lens, *q_start;
  const uint32_t *mask;                 // null: the window
  float2 *part_ml, *tensor_ml;          // [tile][head][part][row]: maximum (log2) and sum
  float *part_o, *tensor_o;             // the same, [head_dim]
  int32_t n_seqs, n_tokens, max_q, n_q_heads, group, max_blocks, mask_words, window, sinks;
  float scale_log2;
  int32_t tiles, tiles_a_seq, splits, few, ranked, tensor_ranked;
  int32_t tensor_tiles, tensor_tiles_a_seq, tensor_splits;
  uint32_t per_token;                   // (2^32 - 1) / block_tokens
  int32_t short_rows;                   // both kernels run: sequences of up to so many rows a head go to the row kernel; 0: one runs
  unsigned long long wait_ns;
};
cudaError_t launch_masked_few(const MaskedArgs &a, int type, int io, cudaStream_t st);
cudaError_t launch_masked_tensor(const MaskedArgs &a, int type, int io, bool early, cudaStream_t st);
cudaError_t launch_attend_masked(const MaskedArgs &a, int type, int io, cudaStream_t st);

// Calls of up to so many tokens keep what rounding takes from the hidden vectors.
constexpr int kMoeWithRest = 8;
// Byte offsets of a layer call's workspace.  moved: e4m3 weights, whose bf16 tokens are kept in f16 by a power
// of two each.
struct MoeShape {
  int64_t token_scale, moved_x, h, h_rest, bytes;         // h_rest: from h to what its rounding took, up to 8 tokens
};
MoeShape moe_shape(int d_model, int d_ff, int n_tokens, int top_k, int n_shared, bool moved);

struct MoeArgs {
  const uint8_t *gate, *up, *down;                        // slot 0 of the layer
  int64_t gate_stride, down_stride;                       // bytes from slot to slot
  const float *gate_scale, *up_scale, *down_scale;        // e4m3: slot 0's block scales
  int64_t scale_stride;                                   // floats from slot to slot
  const void *x;
  const float *logits;
  const int32_t *slot_of_expert;
  void *out;
  int32_t *ids_out;
  float *weights_out;
  int32_t *status;
  int64_t x_stride, logits_stride, out_stride;            // elements
  int2 *choice;                                           // workspace: [token][chosen] slot (-1: none) and weight
  float *token_scale;
  void *moved_x;                                          // [token][d_model]
  void *h;                                                // [pair][d_ff]
  int64_t h_rest;                                         // bytes
  int32_t n_slots, d_model, d_ff, n_tokens, n_experts, n_shared, top_k, renormalize, out_f32;
  int32_t ring_bytes;                                     // shared memory in front of a kernel's tables
  float routed_scale;
};
cudaError_t launch_moe(const MoeArgs &a, int type, int io, cudaStream_t st);

// Lets a kernel ask for all the dynamic shared memory there is; done once a device.
template <auto KERNEL>
cudaError_t allow_shared() {
  static std::atomic<uint64_t> done{0};
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (dev < 64 && (done.load(std::memory_order_acquire) & bit)) return cudaSuccess;
  cudaFuncAttributes at;
  e = cudaFuncGetAttributes(&at, KERNEL);
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024 - (int)at.sharedSizeBytes);
  if (e == cudaSuccess && dev < 64) done.fetch_or(bit, std::memory_order_release);
  return e;
}

constexpr int kSms = 148;  // streaming multiprocessors of a B200: launch shapes are made for it

}  // namespace emoe
