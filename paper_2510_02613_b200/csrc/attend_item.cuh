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

// e4m3 caches are computed with f16 operands whatever the type of q: cvt widens codes to f16 exactly, two an
// instruction (to bf16 it takes seven for four, on a pipe half as wide).  A query row is brought to f16 by
// the power of two that puts its largest element below 2^15: exact but for elements 2^29 times smaller, whose
// error (2^-40 of the largest) is far below that of a 32-bit sum.  Weights carry the scale of v relative to the
// largest met so far, the output the rest.
template <typename IO, bool FP8> struct Operand { using type = IO; };
template <typename IO> struct Operand<IO, true> { using type = __half; };
// f16 weights are kept 2^14 above their natural size where their largest is 1 (2^6 where it is 2^8), so that they
// become denormal below 2^-28 of the largest only: the maximum that goes with a sum is lower by as much.
template <typename T> constexpr float kWeightLift = __is_same(T, __half) ? 14.f : 0.f;

// The power of two for a row whose largest magnitude has these bits (1 where that is not finite, or zero).
__device__ __forceinline__ float query_scale(uint32_t top) {
  if (top == 0 || top >= 0x7f800000u) return 1.f;
  return __uint_as_float((uint32_t)min(254, 127 + 14 + 127 - max(1, (int)(top >> 23))) << 23);
}

// A scale byte as the number it stands for.
__device__ __forceinline__ float scale_of(uint32_t byte) {
  return byte == 255 ? CUDART_NAN_F : __uint_as_float(byte ? byte << 23 : 0x400000u);
}

// The scale of byte v relative to that of byte `largest`, which is not below it (but for 255: not a number).
__device__ __forceinline__ float v_relative(uint32_t v, uint32_t largest) {
  return v == 255 ? CUDART_NAN_F : largest - v < 127 ? __uint_as_float((127 - (largest - v)) << 23) : 0.f;
}

}  // namespace emoe
