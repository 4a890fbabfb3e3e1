// serve.h - operators that serve from one rank's arenas: geometry shared by host and device,
// device helpers, launchers.  The entry points are in serve.cpp.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

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

constexpr int kSms = 148;  // streaming multiprocessors of a B200: launch shapes are made for it

}  // namespace emoe
