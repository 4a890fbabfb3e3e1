// serve.cpp - entry points of the serving operators: argument checks, then one launcher call.
#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>

#include <algorithm>
#include <cmath>

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
  const int size = type_bytes(io);
  if (row * size >= (int64_t)1 << 32) return EMOE_ERR_TOO_LARGE;   // places inside a token are kept in 32 bits
  if (n > 1 && (ks < row || vs < row)) return EMOE_ERR_SHAPE;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(slots, 8)) return EMOE_ERR_ALIGNMENT;
  if (n > 1 && (ks * size % 16 || vs * size % 16)) return EMOE_ERR_ALIGNMENT;
  return on_current_device(c->arena);
}

constexpr double kLog2e = 1.4426950408889634;
constexpr unsigned long long kDefaultWaitNs = 4000000000ull;

emoe_status_t check_attend_sizes(const emoe_kv_cache_t *c, int64_t n_seqs, int64_t q_len, int64_t hq, int64_t max_blocks,
                                 int64_t prefix_len) {
  if (n_seqs < 0 || q_len <= 0 || hq <= 0 || max_blocks < 0 || prefix_len < 0 || hq % c->n_heads) return EMOE_ERR_SHAPE;
  if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return EMOE_ERR_UNSUPPORTED;
  // row and token numbers are kept in 32 bits
  if (q_len > 1 << 20 || hq > 1 << 20 || n_seqs > 1 << 24 || n_seqs * q_len >= 1 << 24 || n_seqs * q_len * hq >= 1 << 28 ||
      max_blocks * c->block_tokens >= 1 << 30 || prefix_len >= 1 << 30)
    return EMOE_ERR_TOO_LARGE;
  return EMOE_OK;
}

// Sizes of a call of emoe_kv_attend_tree or _window; window 0: a tree.
emoe_status_t check_rows_sizes(const emoe_kv_cache_t *c, int64_t n_seqs, int64_t n_tokens, int64_t max_q, int64_t hq, int64_t max_blocks,
                               bool tree, int64_t window, int64_t sinks) {
  if (n_seqs < 0 || n_tokens < 0 || max_q <= 0 || hq <= 0 || max_blocks < 0 || hq % c->n_heads) return EMOE_ERR_SHAPE;
  if (tree ? window != 0 || sinks != 0 : window <= 0 || sinks < 0) return EMOE_ERR_SHAPE;
  if (c->head_dim != 32 && c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return EMOE_ERR_UNSUPPORTED;
  // row and token numbers are kept in 32 bits
  if (max_q > 1 << 24 || hq > 1 << 20 || n_seqs > 1 << 20 || n_tokens > 1 << 24 || n_tokens * hq >= 1 << 28 ||
      max_blocks * c->block_tokens >= 1 << 30)
    return EMOE_ERR_TOO_LARGE;
  return EMOE_OK;
}

// Tokens that a tile of rows runs through at most.
int64_t most_tokens(const emoe_kv_cache_t *c, int64_t max_blocks, bool tree, int64_t window, int64_t sinks) {
  const int64_t all = max_blocks * c->block_tokens;
  return tree ? all : std::min(all, sinks + window + kMaskedRows - 1);
}

constexpr int32_t kNoLimit = 1 << 30;   // of a window, or of the first tokens

uint64_t up_256(uint64_t n) { return (n + 255) / 256 * 256; }

// Sizes, type and layout of an expert arena; pointers apart.
emoe_status_t check_experts(const emoe_expert_arena_t *e) {
  if (!e || e->reserved || (e->layout & ~EMOE_LAYOUT_FUSED_W13)) return EMOE_ERR_INVALID_ARG;
  if (e->type != EMOE_TYPE_BF16 && e->type != EMOE_TYPE_F16 && e->type != EMOE_TYPE_E4M3) return EMOE_ERR_INVALID_ARG;
  if (e->n_layers <= 0 || e->n_slots <= 0 || e->d_model <= 0 || e->d_ff <= 0) return EMOE_ERR_SHAPE;
  if (e->d_model % 16 || e->d_ff % 16) return EMOE_ERR_UNSUPPORTED;
  if (e->n_slots > EMOE_MOE_MAX_SLOTS || e->d_model > 1 << 20 || e->d_ff > 1 << 20) return EMOE_ERR_TOO_LARGE;
  const int64_t m = (int64_t)e->d_model * e->d_ff * type_bytes(e->type);
  if (e->matrix_stride) {
    if (e->layout || e->type == EMOE_TYPE_E4M3) return EMOE_ERR_UNSUPPORTED;
    if (e->matrix_stride < (uint64_t)m || e->matrix_stride > (uint64_t)1 << 42) return EMOE_ERR_SHAPE;
    if (e->matrix_stride % 16) return EMOE_ERR_ALIGNMENT;
  }
  const unsigned __int128 total = (unsigned __int128)e->n_layers * 3 * e->n_slots * (e->matrix_stride ? e->matrix_stride : m);
  return total >> 61 ? EMOE_ERR_SHAPE : EMOE_OK;
}

int64_t scale_floats(const emoe_expert_arena_t *e) {
  return (int64_t)((e->d_model + 127) / 128) * ((e->d_ff + 127) / 128);
}

emoe_status_t check_moe_sizes(const emoe_expert_arena_t *e, int64_t n_tokens, int64_t top_k, int64_t n_experts, int64_t n_shared) {
  if (n_tokens < 0 || top_k <= 0 || n_experts <= 0 || n_shared < 0 || top_k > n_experts) return EMOE_ERR_SHAPE;
  if (n_tokens > EMOE_MOE_MAX_TOKENS || n_experts > EMOE_MOE_MAX_EXPERTS || top_k + n_shared > EMOE_MOE_MAX_CHOSEN)
    return EMOE_ERR_TOO_LARGE;
  return EMOE_OK;
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

emoe_status_t emoe_kv_attend_workspace(const emoe_kv_cache_t *c, int32_t n_seqs, int32_t q_len, int32_t n_q_heads,
                                       int32_t max_blocks, int32_t prefix_len, uint64_t *bytes) {
  emoe_status_t st = check_cache(c);
  if (st == EMOE_OK && !bytes) st = EMOE_ERR_INVALID_ARG;
  if (st == EMOE_OK) st = check_attend_sizes(c, n_seqs, q_len, n_q_heads, max_blocks, prefix_len);
  if (st != EMOE_OK) return st;
  *bytes = 0;
  if (n_seqs == 0) return EMOE_OK;
  const int64_t parts = attend_parts(c->n_heads, n_seqs, q_len, n_q_heads, c->head_dim, c->type == EMOE_TYPE_E4M3,
                                     (int64_t)max_blocks * c->block_tokens, prefix_len);
  *bytes = up_256(parts * sizeof(float2)) + up_256(parts * c->head_dim * sizeof(float));
  return EMOE_OK;
}

emoe_status_t emoe_kv_attend(const emoe_kv_cache_t *c, int32_t layer, const emoe_attend_t *p, void *stream) {
  TraceRange trace("emoe_kv_attend");
  emoe_status_t st = check_cache_memory(c, layer);
  if (st != EMOE_OK) return st;
  if (!p || p->reserved || p->reserved2 || p->wait_limit_us < -1) return EMOE_ERR_INVALID_ARG;
  if (p->io_type != EMOE_TYPE_BF16 && p->io_type != EMOE_TYPE_F16) return EMOE_ERR_INVALID_ARG;
  const float scale_log2 = (float)(p->scale * kLog2e);
  if (!std::isfinite(scale_log2)) return EMOE_ERR_INVALID_ARG;
  if (c->type != EMOE_TYPE_E4M3 && c->type != p->io_type) return EMOE_ERR_UNSUPPORTED;
  st = check_attend_sizes(c, p->n_seqs, p->q_len, p->n_q_heads, p->max_blocks, p->prefix_len);
  if (st != EMOE_OK || p->n_seqs == 0) return st;
  if (!p->q || !p->out || (p->max_blocks && (!p->block_table || !p->own_lens)) || (p->prefix_len && !p->prefix_table))
    return EMOE_ERR_INVALID_ARG;
  const int64_t row = (int64_t)p->n_q_heads * c->head_dim, tokens = (int64_t)p->n_seqs * p->q_len;
  if (tokens > 1 && (p->q_stride < row || p->out_stride < row)) return EMOE_ERR_SHAPE;
  if (!aligned(p->q, 16) || !aligned(p->out, 16) || !aligned(p->lse, 4) || !aligned(p->block_table, 4) ||
      !aligned(p->own_lens, 4) || !aligned(p->prefix_table, 4) || !aligned(p->workspace, 256))
    return EMOE_ERR_ALIGNMENT;
  if (tokens > 1 && (p->q_stride % 8 || p->out_stride % 8)) return EMOE_ERR_ALIGNMENT;
  const AttendShape s = attend_shape(c->n_heads, p->n_seqs, p->q_len, p->n_q_heads, c->head_dim, c->type == EMOE_TYPE_E4M3,
                                     (int64_t)p->max_blocks * c->block_tokens, p->prefix_len);
  const uint64_t ml = up_256(s.parts * sizeof(float2)), need = ml + up_256(s.parts * c->head_dim * sizeof(float));
  if (need && (!p->workspace || p->workspace_bytes < need)) return EMOE_ERR_INVALID_ARG;
  if (s.prefix_items + s.own_items >= (int64_t)1 << 31) return EMOE_ERR_TOO_LARGE;
  st = on_current_device(c->arena);
  if (st != EMOE_OK) return st;
  AttendArgs a{};
  a.c = layer_of(c, layer);
  a.num_blocks = c->num_blocks;
  a.q = p->q;
  a.out = p->out;
  a.lse = p->lse;
  a.q_stride = tokens > 1 ? p->q_stride : row;
  a.out_stride = tokens > 1 ? p->out_stride : row;
  a.block_table = p->block_table;
  a.own_lens = p->own_lens;
  a.prefix_table = p->prefix_table;
  a.part_ml = (float2 *)p->workspace;
  a.part_o = (float *)((uint8_t *)p->workspace + ml);
  a.n_seqs = p->n_seqs;
  a.q_len = p->q_len;
  a.n_q_heads = p->n_q_heads;
  a.group = p->n_q_heads / c->n_heads;
  a.max_blocks = p->max_blocks;
  a.prefix_len = p->prefix_len;
  a.scale_log2 = scale_log2;
  a.seq_rows = s.seq_rows;
  a.prefix_splits = s.prefix_splits;
  a.prefix_chunk = s.prefix_chunk;
  a.own_splits = s.own_splits;
  a.own_chunk = s.own_chunk;
  a.tensor = s.tensor;
  a.alternate = s.alternate;
  a.prefix_items = (uint32_t)s.prefix_items;
  a.own_items = (uint32_t)s.own_items;
  a.wait_ns = p->wait_limit_us < 0 ? 0 : p->wait_limit_us ? p->wait_limit_us * 1000ull : kDefaultWaitNs;
  return cuda_status(launch_attend(a, c->type, p->io_type, (cudaStream_t)stream));
}

}  // extern "C"

namespace {

MaskedSizes masked_sizes(const emoe_kv_cache_t *c, int32_t n_seqs, int32_t n_tokens, int32_t max_q, int32_t n_q_heads, int32_t max_blocks,
                         bool tree, int32_t window, int32_t sinks) {
  return {c->n_heads, n_seqs, n_tokens, std::min(max_q, n_tokens), n_q_heads, c->head_dim, c->type == EMOE_TYPE_E4M3,
          most_tokens(c, max_blocks, tree, window, sinks), tree || sinks + (int64_t)window >= (int64_t)max_blocks * c->block_tokens};
}

uint64_t part_bytes(const emoe_kv_cache_t *c, int64_t parts) {   // maxima and sums, then outputs
  return up_256(parts * sizeof(float2)) + up_256(parts * c->head_dim * sizeof(float));
}

emoe_status_t rows_workspace(const emoe_kv_cache_t *c, int32_t n_seqs, int32_t n_tokens, int32_t max_q, int32_t n_q_heads,
                             int32_t max_blocks, bool tree, int32_t window, int32_t sinks, uint64_t *bytes) {
  emoe_status_t st = check_cache(c);
  if (st == EMOE_OK && !bytes) st = EMOE_ERR_INVALID_ARG;
  if (st == EMOE_OK) st = check_rows_sizes(c, n_seqs, n_tokens, max_q, n_q_heads, max_blocks, tree, window, sinks);
  if (st != EMOE_OK) return st;
  *bytes = 0;
  if (n_seqs == 0 || n_tokens == 0) return EMOE_OK;
  int64_t rows, tensor;
  masked_parts(masked_sizes(c, n_seqs, n_tokens, max_q, n_q_heads, max_blocks, tree, window, sinks), rows, tensor);
  *bytes = part_bytes(c, rows) + part_bytes(c, tensor);
  return EMOE_OK;
}

emoe_status_t attend_rows(const emoe_kv_cache_t *c, int32_t layer, const emoe_attend_rows_t *p, bool tree, void *stream) {
  emoe_status_t st = check_cache_memory(c, layer);
  if (st != EMOE_OK) return st;
  if (!p || p->reserved || p->wait_limit_us < -1 || (!tree && (p->mask || p->mask_words))) return EMOE_ERR_INVALID_ARG;
  if (p->io_type != EMOE_TYPE_BF16 && p->io_type != EMOE_TYPE_F16) return EMOE_ERR_INVALID_ARG;
  const float scale_log2 = (float)(p->scale * kLog2e);
  if (!std::isfinite(scale_log2)) return EMOE_ERR_INVALID_ARG;
  if (c->type != EMOE_TYPE_E4M3 && c->type != p->io_type) return EMOE_ERR_UNSUPPORTED;
  st = check_rows_sizes(c, p->n_seqs, p->n_tokens, p->max_q, p->n_q_heads, p->max_blocks, tree, p->window, p->sinks);
  if (st != EMOE_OK) return st;
  const int32_t max_q = std::min(p->max_q, p->n_tokens);
  if (tree && (int64_t)p->mask_words * 32 < max_q) return EMOE_ERR_SHAPE;
  if (p->n_seqs == 0 || p->n_tokens == 0) return EMOE_OK;
  if (!p->q || !p->out || !p->own_lens || !p->q_start || (p->max_blocks && !p->block_table) || (tree && !p->mask)) return EMOE_ERR_INVALID_ARG;
  const int64_t row = (int64_t)p->n_q_heads * c->head_dim;
  if (p->n_tokens > 1 && (p->q_stride < row || p->out_stride < row)) return EMOE_ERR_SHAPE;
  if (!aligned(p->q, 16) || !aligned(p->out, 16) || !aligned(p->lse, 4) || !aligned(p->block_table, 4) || !aligned(p->own_lens, 4) ||
      !aligned(p->q_start, 4) || !aligned(p->mask, 4) || !aligned(p->workspace, 256))
    return EMOE_ERR_ALIGNMENT;
  if (p->n_tokens > 1 && (p->q_stride % 8 || p->out_stride % 8)) return EMOE_ERR_ALIGNMENT;
  const MaskedShapes s = masked_shapes(masked_sizes(c, p->n_seqs, p->n_tokens, max_q, p->n_q_heads, p->max_blocks, tree, p->window, p->sinks));
  const uint64_t of_rows = part_bytes(c, s.rows.parts), need = of_rows + part_bytes(c, s.tensor.parts);
  if (need && (!p->workspace || p->workspace_bytes < need)) return EMOE_ERR_INVALID_ARG;
  if ((int64_t)s.rows.tiles * c->n_heads * std::max(s.rows.splits, 1) >= (int64_t)1 << 31) return EMOE_ERR_TOO_LARGE;   // a grid's blocks
  st = on_current_device(c->arena);
  if (st != EMOE_OK) return st;
  MaskedArgs a{};
  a.c = layer_of(c, layer);
  a.num_blocks = c->num_blocks;
  a.q = p->q;
  a.out = p->out;
  a.lse = p->lse;
  a.q_stride = p->n_tokens > 1 ? p->q_stride : row;
  a.out_stride = p->n_tokens > 1 ? p->out_stride : row;
  a.block_table = p->block_table;
  a.own_lens = p->own_lens;
  a.q_start = p->q_start;
  a.mask = p->mask;
  uint8_t *const work = (uint8_t *)p->workspace;
  a.part_ml = (float2 *)work;
  a.part_o = (float *)(work + up_256(s.rows.parts * sizeof(float2)));
  a.tensor_ml = (float2 *)(work + of_rows);
  a.tensor_o = (float *)(work + of_rows + up_256(s.tensor.parts * sizeof(float2)));
  a.n_seqs = p->n_seqs;
  a.n_tokens = p->n_tokens;
  a.max_q = max_q;
  a.n_q_heads = p->n_q_heads;
  a.group = p->n_q_heads / c->n_heads;
  a.max_blocks = p->max_blocks;
  a.mask_words = p->mask_words;
  a.window = std::min(p->window, kNoLimit);
  a.sinks = std::min(p->sinks, kNoLimit);
  a.scale_log2 = scale_log2;
  a.tiles = s.rows.tiles;
  a.tiles_a_seq = s.rows.tiles_a_seq;
  a.splits = s.rows.splits;
  a.tensor_tiles = s.tensor.tiles;
  a.tensor_tiles_a_seq = s.tensor.tiles_a_seq;
  a.tensor_splits = s.tensor.splits;
  a.few = s.few;
  a.ranked = s.ranked;
  a.tensor_ranked = s.tensor_ranked;
  a.per_token = 0xffffffffu / (uint32_t)c->block_tokens;
  a.short_rows = !s.rows.tiles || !s.tensor.tiles ? 0 : s.few ? kMaskedFewRows : kMaskedRows;
  a.wait_ns = p->wait_limit_us < 0 ? 0 : p->wait_limit_us ? p->wait_limit_us * 1000ull : kDefaultWaitNs;
  return cuda_status(launch_attend_masked(a, c->type, p->io_type, (cudaStream_t)stream));
}

}  // namespace

extern "C" {

emoe_status_t emoe_kv_attend_tree_workspace(const emoe_kv_cache_t *c, int32_t n_seqs, int32_t n_tokens, int32_t max_q,
                                            int32_t n_q_heads, int32_t max_blocks, uint64_t *bytes) {
  return rows_workspace(c, n_seqs, n_tokens, max_q, n_q_heads, max_blocks, true, 0, 0, bytes);
}

emoe_status_t emoe_kv_attend_window_workspace(const emoe_kv_cache_t *c, int32_t n_seqs, int32_t n_tokens, int32_t max_q,
                                              int32_t n_q_heads, int32_t max_blocks, int32_t window, int32_t sinks, uint64_t *bytes) {
  return rows_workspace(c, n_seqs, n_tokens, max_q, n_q_heads, max_blocks, false, window, sinks, bytes);
}

emoe_status_t emoe_kv_attend_tree(const emoe_kv_cache_t *c, int32_t layer, const emoe_attend_rows_t *p, void *stream) {
  TraceRange trace("emoe_kv_attend_tree");
  return attend_rows(c, layer, p, true, stream);
}

emoe_status_t emoe_kv_attend_window(const emoe_kv_cache_t *c, int32_t layer, const emoe_attend_rows_t *p, void *stream) {
  TraceRange trace("emoe_kv_attend_window");
  return attend_rows(c, layer, p, false, stream);
}

emoe_status_t emoe_kv_extend(const emoe_kv_cache_t *c, const emoe_extend_t *p, void *stream) {
  TraceRange trace("emoe_kv_extend");
  emoe_status_t st = check_cache(c);
  if (st != EMOE_OK) return st;
  if (!p || p->reserved || p->reserved2) return EMOE_ERR_INVALID_ARG;
  if (p->n_seqs < 0 || p->max_blocks < 0 || p->free_capacity < 0 || p->n_slots < 0) return EMOE_ERR_SHAPE;
  if (p->n_seqs > EMOE_KV_MAX_SEQS || (int64_t)p->n_seqs * p->max_blocks >= (int64_t)1 << 31 ||
      (int64_t)p->max_blocks * c->block_tokens >= (int64_t)1 << 30 || p->n_slots > 1 << 30 || p->free_capacity > 1 << 30)
    return EMOE_ERR_TOO_LARGE;
  if (!p->n_free || !p->n_free_out || !p->q_start || (p->n_seqs && (!p->lens || !p->add || !p->lens_out)) ||
      (p->n_seqs && p->max_blocks && !p->block_table) || (p->free_capacity && !p->free_blocks) || (p->n_slots && !p->slots))
    return EMOE_ERR_INVALID_ARG;
  if (!aligned(c->status, 4) || !aligned(p->lens, 4) || !aligned(p->add, 4) || !aligned(p->block_table, 4) || !aligned(p->free_blocks, 4) ||
      !aligned(p->n_free, 4) || !aligned(p->q_start, 4) || !aligned(p->slots, 8) || !aligned(p->lens_out, 4) || !aligned(p->n_free_out, 4))
    return EMOE_ERR_ALIGNMENT;
  st = on_current_device(p->q_start);
  if (st != EMOE_OK) return st;
  ExtendArgs a{};
  a.lens = p->lens;
  a.add = p->add;
  a.block_table = p->block_table;
  a.free_blocks = p->free_blocks;
  a.n_free = p->n_free;
  a.q_start = p->q_start;
  a.slots = p->slots;
  a.lens_out = p->lens_out;
  a.n_free_out = p->n_free_out;
  a.status = c->status;
  a.n_seqs = p->n_seqs;
  a.max_blocks = p->max_blocks;
  a.free_capacity = p->free_capacity;
  a.n_slots = p->n_slots;
  a.num_blocks = c->num_blocks;
  a.block_tokens = c->block_tokens;
  a.per_token = 0xffffffffu / (uint32_t)c->block_tokens;
  return cuda_status(launch_kv_extend(a, (cudaStream_t)stream));
}

emoe_status_t emoe_kv_keep(const emoe_kv_cache_t *c, const emoe_keep_t *p, void *stream) {
  TraceRange trace("emoe_kv_keep");
  emoe_status_t st = check_cache_memory(c, 0);
  if (st != EMOE_OK) return st;
  if (!p || p->reserved || p->reserved2) return EMOE_ERR_INVALID_ARG;
  if (p->n_seqs < 0 || p->max_blocks < 0 || p->max_accepted < 0 || p->n_slots < 0) return EMOE_ERR_SHAPE;
  if (c->head_dim % 8) return EMOE_ERR_UNSUPPORTED;
  const uint64_t vector = (uint64_t)c->head_dim * type_bytes(c->type), pieces = vector % 16 ? vector / 8 : vector / 16;
  if (p->n_seqs > 65535 || p->max_accepted > EMOE_KV_MAX_ACCEPTED || (int64_t)p->max_blocks * c->block_tokens >= (int64_t)1 << 30 ||
      (unsigned __int128)2 * c->n_layers * c->n_heads * pieces >= 1u << 31)
    return EMOE_ERR_TOO_LARGE;
  if (p->n_seqs == 0) return EMOE_OK;
  if (!p->lens || !p->q_start || !p->n_accepted || !p->change || (p->max_accepted && !p->accepted) || (p->max_blocks && !p->block_table) ||
      (p->n_slots && !p->slots))
    return EMOE_ERR_INVALID_ARG;
  if (!aligned(p->block_table, 4) || !aligned(p->lens, 4) || !aligned(p->q_start, 4) || !aligned(p->accepted, 4) ||
      !aligned(p->n_accepted, 4) || !aligned(p->change, 4) || !aligned(p->slots, 8))
    return EMOE_ERR_ALIGNMENT;
  st = on_current_device(c->arena);
  if (st != EMOE_OK) return st;
  KeepArgs a{};
  a.c = layer_of(c, 0);
  a.pool_vectors = pool_vectors(c);
  a.pool_bytes = a.pool_vectors * vector;
  a.block_table = p->block_table;
  a.lens = p->lens;
  a.q_start = p->q_start;
  a.accepted = p->accepted;
  a.n_accepted = p->n_accepted;
  a.slots = p->slots;
  a.change = p->change;
  a.pools = 2 * c->n_layers;
  a.pieces = (uint32_t)pieces;
  a.n_seqs = p->n_seqs;
  a.max_blocks = p->max_blocks;
  a.max_accepted = p->max_accepted;
  a.num_blocks = c->num_blocks;
  a.n_slots = p->n_slots;
  return cuda_status(launch_kv_keep(a, vector % 16 == 0, (cudaStream_t)stream));
}

emoe_status_t emoe_expert_arena_bytes(const emoe_expert_arena_t *e, uint64_t *bytes) {
  const emoe_status_t st = check_experts(e);
  if (st != EMOE_OK) return st;
  if (!bytes) return EMOE_ERR_INVALID_ARG;
  const uint64_t matrices = 3ull * e->n_layers * e->n_slots;
  const uint64_t m = (uint64_t)e->d_model * e->d_ff * type_bytes(e->type);
  *bytes = matrices * (e->matrix_stride ? e->matrix_stride : m);
  if (e->type == EMOE_TYPE_E4M3) *bytes = up_256(*bytes) + matrices * scale_floats(e) * 4;
  return EMOE_OK;
}

emoe_status_t emoe_moe_decode_workspace(const emoe_expert_arena_t *e, int32_t n_tokens, int32_t top_k, int32_t n_experts,
                                        int32_t n_shared, uint64_t *bytes) {
  emoe_status_t st = check_experts(e);
  if (st == EMOE_OK && !bytes) st = EMOE_ERR_INVALID_ARG;
  if (st == EMOE_OK) st = check_moe_sizes(e, n_tokens, top_k, n_experts, n_shared);
  if (st != EMOE_OK) return st;
  // Calls of up to kMoeWithRest tokens keep more for each: the most that this many or fewer need.
  *bytes = 0;
  for (int n : {n_tokens, n_tokens < kMoeWithRest ? n_tokens : kMoeWithRest})
    if (n) {
      const uint64_t need = moe_shape(e->d_model, e->d_ff, n, top_k, n_shared, e->type == EMOE_TYPE_E4M3).bytes;
      if (need > *bytes) *bytes = need;
    }
  return EMOE_OK;
}

emoe_status_t emoe_moe_decode(const emoe_expert_arena_t *e, int32_t layer, const emoe_moe_t *p, void *stream) {
  TraceRange trace("emoe_moe_decode");
  emoe_status_t st = check_experts(e);
  if (st != EMOE_OK) return st;
  if (!p || p->reserved || (p->flags & ~EMOE_MOE_RENORMALIZE) || layer < 0 || layer >= e->n_layers || !e->arena)
    return EMOE_ERR_INVALID_ARG;
  if (p->io_type != EMOE_TYPE_BF16 && p->io_type != EMOE_TYPE_F16) return EMOE_ERR_INVALID_ARG;
  if (p->out_type != p->io_type && p->out_type != EMOE_TYPE_F32) return EMOE_ERR_INVALID_ARG;
  if (e->type != EMOE_TYPE_E4M3 && e->type != p->io_type) return EMOE_ERR_UNSUPPORTED;
  st = check_moe_sizes(e, p->n_tokens, p->top_k, p->n_experts, p->n_shared);
  if (st != EMOE_OK || p->n_tokens == 0) return st;
  if (!p->x || !p->logits || !p->slot_of_expert || !p->out || !p->workspace) return EMOE_ERR_INVALID_ARG;
  const MoeShape s = moe_shape(e->d_model, e->d_ff, p->n_tokens, p->top_k, p->n_shared, e->type == EMOE_TYPE_E4M3);
  if (p->workspace_bytes < (uint64_t)s.bytes) return EMOE_ERR_INVALID_ARG;
  const bool many = p->n_tokens > 1;
  if (many && (p->x_stride < e->d_model || p->out_stride < e->d_model || p->logits_stride < p->n_experts)) return EMOE_ERR_SHAPE;
  if (!aligned(e->arena, 16) || !aligned(e->status, 4) || !aligned(p->x, 16) || !aligned(p->logits, 4) ||
      !aligned(p->slot_of_expert, 4) || !aligned(p->out, type_bytes(p->out_type)) || !aligned(p->ids_out, 4) ||
      !aligned(p->weights_out, 4) || !aligned(p->workspace, 256) || (many && p->x_stride % 8))
    return EMOE_ERR_ALIGNMENT;
  st = on_current_device(e->arena);
  if (st != EMOE_OK) return st;

  MoeArgs a{};
  const int64_t m = (int64_t)e->d_model * e->d_ff * type_bytes(e->type), stride = e->matrix_stride ? (int64_t)e->matrix_stride : m;
  const uint8_t *base = (const uint8_t *)e->arena + (int64_t)layer * 3 * e->n_slots * stride;
  if (e->layout & EMOE_LAYOUT_FUSED_W13) {
    a.gate = base;
    a.up = base + m;
    a.down = base + 2 * e->n_slots * m;
    a.gate_stride = 2 * m;
    a.down_stride = m;
  } else {
    a.gate = base;
    a.up = base + e->n_slots * stride;
    a.down = base + 2 * e->n_slots * stride;
    a.gate_stride = a.down_stride = stride;
  }
  if (e->type == EMOE_TYPE_E4M3) {
    const int64_t per = scale_floats(e);
    const float *scales = (const float *)((const uint8_t *)e->arena + up_256(3ull * e->n_layers * e->n_slots * m));
    a.gate_scale = scales + (int64_t)layer * 3 * e->n_slots * per;
    a.up_scale = a.gate_scale + e->n_slots * per;
    a.down_scale = a.up_scale + e->n_slots * per;
    a.scale_stride = per;
  }
  uint8_t *const work = (uint8_t *)p->workspace;
  a.x = p->x;
  a.logits = p->logits;
  a.slot_of_expert = p->slot_of_expert;
  a.out = p->out;
  a.ids_out = p->ids_out;
  a.weights_out = p->weights_out;
  a.status = e->status;
  a.x_stride = many ? p->x_stride : e->d_model;
  a.logits_stride = many ? p->logits_stride : p->n_experts;
  a.out_stride = many ? p->out_stride : e->d_model;
  a.choice = (int2 *)work;
  a.token_scale = (float *)(work + s.token_scale);
  a.moved_x = work + s.moved_x;
  a.h = work + s.h;
  a.h_rest = s.h_rest;
  a.n_slots = e->n_slots;
  a.d_model = e->d_model;
  a.d_ff = e->d_ff;
  a.n_tokens = p->n_tokens;
  a.n_experts = p->n_experts;
  a.n_shared = p->n_shared;
  a.top_k = p->top_k;
  a.renormalize = (p->flags & EMOE_MOE_RENORMALIZE) != 0;
  a.out_f32 = p->out_type == EMOE_TYPE_F32;
  a.routed_scale = p->routed_scale;
  return cuda_status(launch_moe(a, e->type, p->io_type, (cudaStream_t)stream));
}

}  // extern "C"
