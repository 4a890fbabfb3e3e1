// kv_cache.cu - tokens into a paged KV cache and out of it.
//
// Both kernels only move and convert: bound by memory (the smallest calls by the launch: 64 tokens 8.5 us on the
// stream).  Measured at 16 heads of 128, e4m3: 8191 tokens in 24.6 us (4.1 TB/s of 101 MB), 65536 tokens out in
// 152 us (5.3 TB/s of 808 MB, 83% of a copy's rate).  A
// head vector is taken by a group of lanes, 8 elements (16 bytes of a 16-bit type) a lane, so a
// vector is read once, its largest magnitude is found by shuffles and its codes are written
// from registers.  The scale is a power of two: no division, scaling exact, and a value read
// back is exact in bf16.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "serve.h"

namespace emoe {
namespace {

// 8 elements of a lane as they lie in memory
template <int TYPE> struct Raw;
template <> struct Raw<EMOE_TYPE_BF16> { uint4 x; };
template <> struct Raw<EMOE_TYPE_F16> { uint4 x; };
template <> struct Raw<EMOE_TYPE_F32> { uint4 x, y; };
template <> struct Raw<EMOE_TYPE_E4M3> { uint2 x; };

template <int TYPE>
__device__ __forceinline__ void unpack(const Raw<TYPE> &r, float (&f)[8]) {
  if constexpr (TYPE == EMOE_TYPE_F32) {
    const uint32_t w[8] = {r.x.x, r.x.y, r.x.z, r.x.w, r.y.x, r.y.y, r.y.z, r.y.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i]);
  } else if constexpr (TYPE == EMOE_TYPE_E4M3) {
    const uint32_t w[2] = {r.x.x, r.x.y};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i >> 1] >> (16 * (i & 1))), __NV_E4M3);
      const float2 g = __half22float2(__half2(h));
      f[2 * i] = g.x;
      f[2 * i + 1] = g.y;
    }
  } else {
    const uint32_t w[4] = {r.x.x, r.x.y, r.x.z, r.x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (TYPE == EMOE_TYPE_BF16) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      } else {
        const float2 g = __half22float2(*(const __half2 *)&w[i]);
        f[2 * i] = g.x;
        f[2 * i + 1] = g.y;
      }
    }
  }
}

template <int TYPE>
__device__ __forceinline__ Raw<TYPE> pack(const float (&f)[8]) {
  Raw<TYPE> r;
  if constexpr (TYPE == EMOE_TYPE_F32) {
    r.x = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    r.y = make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7]));
  } else if constexpr (TYPE == EMOE_TYPE_E4M3) {
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i >> 1] |= (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(f[2 * i], f[2 * i + 1]), __NV_SATFINITE, __NV_E4M3)
                   << (16 * (i & 1));
    r.x = make_uint2(w[0], w[1]);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (TYPE == EMOE_TYPE_BF16) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *(const uint32_t *)&h;
      } else {
        const __half2 h = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *(const uint32_t *)&h;
      }
    }
    r.x = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return r;
}

__host__ __device__ constexpr int bytes_of(int type) { return type == EMOE_TYPE_F32 ? 4 : type == EMOE_TYPE_E4M3 ? 1 : 2; }

// Scale byte of a vector whose largest magnitude has the bits `top` (0 .. infinity, NaN): the
// smallest k with value <= 448 * 2^k = 1.75 * 2^(8 + k) is the exponent less 8, one more when
// the mantissa is above 1.75.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  if (top >= 0x7f800000u) return 255;
  if (top == 0) return 127;
  const int byte = (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  return byte < 1 ? 1 : (uint32_t)byte;
}

struct Args {
  KvLayer c;
  uint8_t *k, *v;            // the dense side
  int64_t k_stride, v_stride;  // bytes
  const int64_t *slots;
  uint32_t n_vec;            // n_tokens * n_heads
  uint32_t n_tokens;
  uint32_t step_tokens, step_heads;  // from one vector of a thread to its next
  uint32_t lanes;            // lanes per vector, a power of two >= head_dim / 8
};

// U vectors a group of lanes: all loads are issued before the first is used.  blockIdx.y: K or V.
template <int IN, int CACHE, int U, bool APPEND>
__global__ void __launch_bounds__(256, 6) kv_copy_kernel(const __grid_constant__ Args a) {
  const uint32_t group = 256 / a.lanes, lane = threadIdx.x & (a.lanes - 1);
  const uint32_t first = blockIdx.x * (group * U) + threadIdx.x / a.lanes;
  const bool mine = lane * 8 < (uint32_t)a.c.head_dim;  // head_dim / 8 need not be a power of two
  uint8_t *const dense = blockIdx.y ? a.v : a.k;
  const int64_t stride = blockIdx.y ? a.v_stride : a.k_stride;
  uint8_t *const pool = blockIdx.y ? a.c.v : a.c.k;
  uint8_t *const scale = blockIdx.y ? a.c.v_scale : a.c.k_scale;
  constexpr int kIn = bytes_of(IN), kCache = bytes_of(CACHE);

  // Slots first, and in an append the rows, which do not wait for them: a branch on a slot would.  One division a
  // thread: from one of its vectors to the next it is a fixed number of tokens and heads.
  int64_t slot[U], at[U];   // at: vector index in the pool; -1: nothing to do
  uint32_t head[U];
  uint8_t *row[U];
  Raw<APPEND ? IN : CACHE> raw[U];
  uint32_t sb[U];
  uint32_t token = first / (uint32_t)a.c.n_heads, h = first - token * a.c.n_heads;
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const bool there = first + u * group < a.n_vec;   // else the last vector once more, which nobody writes
    const uint32_t t = there ? token : a.n_tokens - 1;
    head[u] = there ? h : 0;
    slot[u] = a.slots[t];
    row[u] = dense + t * stride + (head[u] * a.c.head_dim + lane * 8) * kIn;
    token += a.step_tokens;
    h += a.step_heads;
    if (h >= (uint32_t)a.c.n_heads) {
      h -= a.c.n_heads;
      ++token;
    }
    raw[u] = {};
    if constexpr (APPEND) {
      if (mine) raw[u] = *(const Raw<IN> *)row[u];
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    at[u] = -1;
    sb[u] = 127;
    if (first + u * group >= a.n_vec) continue;
    if (kv_slot_ok(a.c, slot[u]))
      at[u] = kv_vector(a.c, slot[u], head[u]);
    else if (slot[u] >= 0 && a.c.status)
      *a.c.status = EMOE_ERR_BLOCK_TABLE;
    if constexpr (!APPEND) {
      if (at[u] < 0) continue;
      if (mine) raw[u] = *(const Raw<CACHE> *)(pool + (at[u] * a.c.head_dim + lane * 8) * kCache);
      if constexpr (CACHE == EMOE_TYPE_E4M3) sb[u] = scale[at[u]];
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if constexpr (APPEND) {
      if constexpr (IN == CACHE) {
        if (at[u] >= 0 && mine) *(Raw<CACHE> *)(pool + (at[u] * a.c.head_dim + lane * 8) * kCache) = raw[u];
      } else {
        float f[8];
        unpack<IN>(raw[u], f);
        if constexpr (CACHE == EMOE_TYPE_E4M3) {
          uint32_t top = 0;   // magnitudes compare as their bits do, NaN above infinity
          if constexpr (IN == EMOE_TYPE_F32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(f[i]) & 0x7fffffffu);
          } else {   // so do those of 16 bits, two at a time
            const uint4 w = raw[u].x;
            const uint32_t two = __vmaxu2(__vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu), __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu));
            top = max(two >> 16, two & 0xffffu);
          }
          for (uint32_t m = a.lanes >> 1; m; m >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, m));
          if constexpr (IN == EMOE_TYPE_BF16) top <<= 16;
          if constexpr (IN == EMOE_TYPE_F16) top = __float_as_uint(__half2float(__ushort_as_half((unsigned short)top)));
          const uint32_t byte = scale_byte(top);
          const float by = __uint_as_float((254u - byte) << 23);  // 2^-k: byte is 1 .. 247 here, or 255
          Raw<CACHE> codes;
#pragma unroll
          for (int i = 0; i < 8; ++i) f[i] *= by;
          codes = pack<CACHE>(f);
          if (byte == 255) codes = {};
          if (at[u] >= 0 && mine) *(Raw<CACHE> *)(pool + (at[u] * a.c.head_dim + lane * 8) * kCache) = codes;
          if (at[u] >= 0 && lane == 0) scale[at[u]] = (uint8_t)byte;
        }
        if constexpr (CACHE != EMOE_TYPE_E4M3)
          if (at[u] >= 0 && mine) *(Raw<CACHE> *)(pool + (at[u] * a.c.head_dim + lane * 8) * kCache) = pack<CACHE>(f);
      }
    } else {
      if (at[u] < 0 || !mine) continue;
      if constexpr (IN == CACHE) {
        *(Raw<IN> *)row[u] = raw[u];
      } else {
        float f[8];
        unpack<CACHE>(raw[u], f);
        if constexpr (CACHE == EMOE_TYPE_E4M3) {
          const float by = sb[u] == 255 ? __uint_as_float(0x7fc00000u)
                                        : sb[u] ? __uint_as_float(sb[u] << 23) : __uint_as_float(0x400000u);
#pragma unroll
          for (int i = 0; i < 8; ++i) f[i] *= by;
        }
        *(Raw<IN> *)row[u] = pack<IN>(f);
      }
    }
  }
}

template <int IN, int CACHE, bool APPEND>
cudaError_t launch(Args a, cudaStream_t st) {
  const uint32_t group = 256 / a.lanes;
  const uint32_t ctas = (a.n_vec + group - 1) / group;
  // Four vectors a thread from about three waves of blocks on (8191 tokens: 24.7 us, one a thread 31.4; 65536: 152 and
  // 214); below that they would leave SMs idle, and with one the loads of a small call start at once.
  if (ctas >= 16 * kSms) {
    kv_copy_kernel<IN, CACHE, 4, APPEND><<<dim3((ctas + 3) / 4, 2), 256, 0, st>>>(a);
  } else {
    kv_copy_kernel<IN, CACHE, 1, APPEND><<<dim3(ctas, 2), 256, 0, st>>>(a);
  }
  return cudaGetLastError();
}

template <bool APPEND>
cudaError_t dispatch(const Args &a, int io, int type, cudaStream_t st) {
  if (type == EMOE_TYPE_E4M3) {
    if (io == EMOE_TYPE_BF16) return launch<EMOE_TYPE_BF16, EMOE_TYPE_E4M3, APPEND>(a, st);
    if (io == EMOE_TYPE_F16) return launch<EMOE_TYPE_F16, EMOE_TYPE_E4M3, APPEND>(a, st);
    return launch<EMOE_TYPE_F32, EMOE_TYPE_E4M3, APPEND>(a, st);
  }
  if (type == EMOE_TYPE_BF16) {
    if (io == EMOE_TYPE_F32) return launch<EMOE_TYPE_F32, EMOE_TYPE_BF16, APPEND>(a, st);
    return launch<EMOE_TYPE_BF16, EMOE_TYPE_BF16, APPEND>(a, st);
  }
  if (io == EMOE_TYPE_F32) return launch<EMOE_TYPE_F32, EMOE_TYPE_F16, APPEND>(a, st);
  return launch<EMOE_TYPE_F16, EMOE_TYPE_F16, APPEND>(a, st);
}

Args make(const KvLayer &c, void *k, void *v, int64_t ks, int64_t vs, int io, const int64_t *slots, int n) {
  Args a{};
  a.c = c;
  a.k = (uint8_t *)k;
  a.v = (uint8_t *)v;
  a.k_stride = ks * bytes_of(io);
  a.v_stride = vs * bytes_of(io);
  a.slots = slots;
  a.n_vec = (uint32_t)n * (uint32_t)c.n_heads;
  a.lanes = 1;
  while (a.lanes * 8 < (uint32_t)c.head_dim) a.lanes *= 2;
  a.n_tokens = (uint32_t)n;
  a.step_tokens = 256 / a.lanes / c.n_heads;
  a.step_heads = 256 / a.lanes % c.n_heads;
  return a;
}

}  // namespace

cudaError_t launch_kv_append(const KvLayer &c, int type, const void *k, const void *v, int64_t ks, int64_t vs,
                             int in_type, const int64_t *slots, int n, cudaStream_t st) {
  return dispatch<true>(make(c, (void *)k, (void *)v, ks, vs, in_type, slots, n), in_type, type, st);
}

cudaError_t launch_kv_gather(const KvLayer &c, int type, const int64_t *slots, int n, void *k, void *v,
                             int64_t ks, int64_t vs, int out_type, cudaStream_t st) {
  return dispatch<false>(make(c, k, v, ks, vs, out_type, slots, n), out_type, type, st);
}

}  // namespace emoe
