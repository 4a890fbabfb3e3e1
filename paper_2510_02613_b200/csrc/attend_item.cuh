// attend_item.cuh - what the attention kernels share: rows and their outputs.
#pragma once

#include <math_constants.h>

#include "convert.cuh"
#include "serve.h"

namespace emoe {

__device__ __forceinline__ int own_length(const AttendArgs &a, int seq) {
  return a.max_blocks ? max(0, min(a.own_lens[seq], a.max_blocks * a.c.block_tokens)) : 0;
}

// Output row (sequence, query token, query head) of a tile row.
__device__ __forceinline__ int64_t output_row(const AttendArgs &a, int seq, int head, int row) {
  const int token = row / a.group;   // over the batch for the prefix: seq * q_len + t
  return ((int64_t)seq * a.q_len + token) * a.n_q_heads + head * a.group + row - token * a.group;
}

// Vector index of token t, which lies on `block`; -1 (and the status word) if that is outside the pool.
// (The table is read apart from this and well before: a branch on what it says waits for it.)
__device__ __forceinline__ int64_t token_vector(const AttendArgs &a, int block, int t, int head) {
  const uint32_t off = (uint32_t)t % (uint32_t)a.c.block_tokens;
  if (block < 0 || block >= a.num_blocks) {
    if (a.c.status) *a.c.status = EMOE_ERR_BLOCK_TABLE;
    return -1;
  }
  return a.c.head_major ? ((int64_t)block * a.c.n_heads + head) * a.c.block_tokens + off
                        : ((int64_t)block * a.c.block_tokens + off) * a.c.n_heads + head;
}

// A scale byte as the number it stands for.
__device__ __forceinline__ float scale_of(uint32_t byte) {
  return byte == 255 ? CUDART_NAN_F : __uint_as_float(byte ? byte << 23 : 0x400000u);
}

}  // namespace emoe
