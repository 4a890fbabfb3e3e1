// serve.cpp - entry points of the serving operators: argument checks, then one launcher call.
#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>

#include "serve.h"

using namespace emoe;

namespace {

struct TraceRange {   // a named range for timelines, as around the other entry points
  explicit TraceRange(const char *name) { nvtxRangePushA(name); }
  ~TraceRange() { nvtxRangePop(); }
  TraceRange(const TraceRange &) = delete;
  TraceRange &operator=(const TraceRange &) = delete;
};

int type_bytes(int type) {
  switch (type) {
    case EMOE_TYPE_BF16: case EMOE_TYPE_F16: return 2;
    case EMOE_TYPE_F32: return 4;
    case EMOE_TYPE_E4M3: return 1;
  }
  return 0;
}

bool aligned(const void *p, uintptr_t n) { return (uintptr_t)p % n == 0; }

emoe_status_t cuda_status(cudaError_t e) {
  if (e == cudaSuccess) return EMOE_OK;
  return e == cudaErrorMemoryAllocation ? EMOE_ERR_OOM : EMOE_ERR_CUDA;
}

// The arena has to be memory of the current device: a launch there with another device's
// pointers would fault or go over the interconnect unasked.
emoe_status_t on_current_device(const void *p) {
  int dev = -1;
  cudaPointerAttributes at;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaPointerGetAttributes(&at, p) != cudaSuccess) {
    cudaGetLastError();
    return EMOE_ERR_CUDA;
  }
  if ((at.type != cudaMemoryTypeDevice && at.type != cudaMemoryTypeManaged) || at.device != dev) return EMOE_ERR_CUDA;
  return EMOE_OK;
}

// Sizes and types of a cache; pointers apart.
emoe_status_t check_cache(const emoe_kv_cache_t *c) {
  if (!c || c->reserved || (c->layout & ~EMOE_LAYOUT_KV_HEAD_MAJOR)) return EMOE_ERR_INVALID_ARG;
  if (c->type != EMOE_TYPE_BF16 && c->type != EMOE_TYPE_F16 && c->type != EMOE_TYPE_E4M3) return EMOE_ERR_INVALID_ARG;
  if (c->n_layers <= 0 || c->num_blocks <= 0 || c->block_tokens <= 0 || c->n_heads <= 0 || c->head_dim <= 0)
    return EMOE_ERR_SHAPE;
  if ((int64_t)c->num_blocks * c->block_tokens >= (int64_t)1 << 31) return EMOE_ERR_SHAPE;
  // every byte offset has to fit 63 bits
  const unsigned __int128 total = (unsigned __int128)c->n_layers * 2 * c->num_blocks * c->block_tokens * c->n_heads *
                                  ((unsigned __int128)c->head_dim * type_bytes(c->type));
  return total >> 62 ? EMOE_ERR_SHAPE : EMOE_OK;
}

emoe_status_t check_cache_memory(const emoe_kv_cache_t *c, int32_t layer) {
  const emoe_status_t st = check_cache(c);
  if (st != EMOE_OK) return st;
  if (!c->arena || layer < 0 || layer >= c->n_layers || (c->type == EMOE_TYPE_E4M3) != (c->scales != nullptr))
    return EMOE_ERR_INVALID_ARG;
  if (!aligned(c->arena, 16) || !aligned(c->status, 4)) return EMOE_ERR_ALIGNMENT;
  return EMOE_OK;
}

int64_t pool_vectors(const emoe_kv_cache_t *c) {
  return (int64_t)c->num_blocks * c->block_tokens * c->n_heads;
}

KvLayer layer_of(const emoe_kv_cache_t *c, int32_t layer) {
  KvLayer l{};
  const int64_t vecs = pool_vectors(c), bytes = vecs * c->head_dim * type_bytes(c->type);
  l.k = (uint8_t *)c->arena + 2 * (int64_t)layer * bytes;
  l.v = l.k + bytes;
  if (c->scales) {
    l.k_scale = (uint8_t *)c->scales + 2 * (int64_t)layer * vecs;
    l.v_scale = l.k_scale + vecs;
  }
  l.status = c->status;
  l.n_slots = (int64_t)c->num_blocks * c->block_tokens;
  l.block_tokens = c->block_tokens;
  l.n_heads = c->n_heads;
  l.head_dim = c->head_dim;
  l.head_major = (c->layout & EMOE_LAYOUT_KV_HEAD_MAJOR) != 0;
  return l;
}

// The dense side of emoe_kv_append / _gather.
emoe_status_t check_copy(const emoe_kv_cache_t *c, int32_t layer, const void *k, const void *v, int64_t ks, int64_t vs,
                         int32_t io, const int64_t *slots, int32_t n) {
  const emoe_status_t st = check_cache_memory(c, layer);
  if (st != EMOE_OK) return st;
  if (n < 0 || io < EMOE_TYPE_BF16 || io > EMOE_TYPE_F32) return EMOE_ERR_INVALID_ARG;
  if (c->type != EMOE_TYPE_E4M3 && io != c->type && io != EMOE_TYPE_F32) return EMOE_ERR_UNSUPPORTED;
  if (c->head_dim % 8 || c->head_dim > 256) return EMOE_ERR_UNSUPPORTED;
  if ((int64_t)n * c->n_heads >= (int64_t)1 << 31) return EMOE_ERR_TOO_LARGE;
  if (n == 0) return EMOE_OK;
  if (!k || !v || !slots) return EMOE_ERR_INVALID_ARG;
  const int64_t row = (int64_t)c->n_heads * c->head_dim;
  if (n > 1 && (ks < row || vs < row)) return EMOE_ERR_SHAPE;
  const int size = type_bytes(io);
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 8)) return EMOE_ERR_ALIGNMENT;
  if (n > 1 && (ks * size % 16 || vs * size % 16)) return EMOE_ERR_ALIGNMENT;
  return on_current_device(c->arena);
}

}  // namespace

extern "C" {

emoe_status_t emoe_kv_cache_bytes(const emoe_kv_cache_t *c, uint64_t *arena_bytes, uint64_t *scale_bytes) {
  const emoe_status_t st = check_cache(c);
  if (st != EMOE_OK) return st;
  const uint64_t vecs = 2ull * c->n_layers * pool_vectors(c);
  if (arena_bytes) *arena_bytes = vecs * c->head_dim * type_bytes(c->type);
  if (scale_bytes) *scale_bytes = c->type == EMOE_TYPE_E4M3 ? vecs : 0;
  return EMOE_OK;
}

int64_t emoe_kv_vector_index(const emoe_kv_cache_t *c, int32_t layer, int32_t kv, int64_t slot, int32_t head) {
  if (check_cache(c) != EMOE_OK || layer < 0 || layer >= c->n_layers || kv < 0 || kv > 1 || head < 0 || head >= c->n_heads)
    return -1;
  const KvLayer l = layer_of(c, 0);
  if (!kv_slot_ok(l, slot)) return -1;
  return (2 * (int64_t)layer + kv) * pool_vectors(c) + kv_vector(l, slot, head);
}

emoe_status_t emoe_kv_append(const emoe_kv_cache_t *c, int32_t layer, const void *k, const void *v, int64_t ks,
                             int64_t vs, int32_t in_type, const int64_t *slots, int32_t n, void *stream) {
  TraceRange trace("emoe_kv_append");
  const emoe_status_t st = check_copy(c, layer, k, v, ks, vs, in_type, slots, n);
  if (st != EMOE_OK || n == 0) return st;
  return cuda_status(launch_kv_append(layer_of(c, layer), c->type, k, v, ks, vs, in_type, slots, n, (cudaStream_t)stream));
}

emoe_status_t emoe_kv_gather(const emoe_kv_cache_t *c, int32_t layer, const int64_t *slots, int32_t n, void *k, void *v,
                             int64_t ks, int64_t vs, int32_t out_type, void *stream) {
  TraceRange trace("emoe_kv_gather");
  const emoe_status_t st = check_copy(c, layer, k, v, ks, vs, out_type, slots, n);
  if (st != EMOE_OK || n == 0) return st;
  return cuda_status(launch_kv_gather(layer_of(c, layer), c->type, slots, n, k, v, ks, vs, out_type, (cudaStream_t)stream));
}

}  // extern "C"
