// convert.cuh - 16-bit pairs and e4m3 codes as tensor-core operands.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace emoe {

template <typename T> struct Pair;
template <> struct Pair<__nv_bfloat16> {
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *(const uint32_t *)&h;
  }
  static __device__ __forceinline__ float2 unpack(uint32_t x) {
    return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
  }
};
template <> struct Pair<__half> {
  static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *(const uint32_t *)&h;
  }
  static __device__ __forceinline__ float2 unpack(uint32_t x) { return __half22float2(*(const __half2 *)&x); }
};

// e4m3 as bf16 operands without a product: a code's magnitude bits, moved to their place, are a bf16 2^120
// too small (denormal where the code is), which the tensor cores take as it is.  The other operand
// carries 2^60 of that and the sums the rest, so that neither side leaves its range.  A word's
// codes come out as (0, 2) and (1, 3), so the other operand is kept in that order ("moved").  f16 operands are
// what cvt gives: in order and at their own size.  (Codes 0x7f and 0xff, not a number, would become 480: see moved_top.)
template <typename T, bool FP8> constexpr bool kMoved = FP8 && !__is_same(T, __half);
constexpr float kMovedScale = 0x1p60f;   // of the other operand, and of the sums
// Two pairs of operands from a word of four codes.
template <typename T>
__device__ __forceinline__ void word_of_codes(uint32_t &first, uint32_t &second, uint32_t w) {
  if constexpr (__is_same(T, __half)) {
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\tcvt.rn.f16x2.e4m3x2 %1, hi;\n\t}"
        : "=r"(first), "=r"(second) : "r"(w));
  } else {
    first = ((w << 4) & 0x07f007f0u) | ((w << 8) & 0x80008000u);
    second = ((w >> 4) & 0x07f007f0u) | (w & 0x80008000u);
  }
}

// The largest magnitudes of moved codes so far, and whether a code that is not a number, the largest there is, was
// among them.
__device__ __forceinline__ uint32_t moved_top(uint32_t top, uint32_t w) {
  return __vimax3_u16x2(top, (w << 4) & 0x07f007f0u, (w >> 4) & 0x07f007f0u);
}
__device__ __forceinline__ bool moved_nan(uint32_t top) { return (top & 0xffffu) == 0x07f0u || top >> 16 == 0x07f0u; }

// Four codes as f16 pairs (0, 1) and (2, 3).
__device__ __forceinline__ void codes_to_half(uint32_t &lo, uint32_t &hi, uint32_t w) {
  asm("{\n\t.reg .b16 x, y;\n\tmov.b32 {x, y}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, x;\n\tcvt.rn.f16x2.e4m3x2 %1, y;\n\t}"
      : "=r"(lo), "=r"(hi) : "r"(w));
}

// d += a b: a 16 x 16 (rows), b 16 x 8 (columns), 32-bit sums.
template <typename T>
__device__ __forceinline__ void mma_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (sizeof(T) == 2 && __is_same(T, __half)) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  } else {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  }
}

__device__ __forceinline__ float exp2_fast(float x) {  // 2 units in the last place; -inf gives 0
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ uint32_t shared_address(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
// 16 bytes global -> shared; `bytes` of them are read (0 or 16), the rest is zero.
__device__ __forceinline__ void copy_async_16(uint32_t dst, const void *src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global.L2::128B [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}

// Programmatic dependent launch: let the next kernel of the stream start its own prologue; wait
// until the kernels before have finished and their results can be read.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

}  // namespace emoe
