// tensor.cuh - 5th-generation tensor cores as the attention kernels use them: the roles of a block's warps and their
// barriers, bounded waits, operands in 128-byte-swizzled shared memory, products, tensor memory, and pairs of 32-bit operations.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace emoe {

constexpr int kTile = 128, kStep = 64;     // rows of a slot and tokens that are brought in at once; tokens of a step
constexpr int kSoftmaxWarps = 8, kMmaWarp = 8, kCopyWarp0 = 12, kCopyWarps = 4, kThreads = 512;
constexpr int kKept = 4;                   // tiles whose marks and scales are kept
constexpr unsigned long long kDrainNs = 1000000000ull;
constexpr float kRaise = 8.f;              // log2 of how far the real maximum may pass the one in use
constexpr uint32_t kColS = 0, kColO = 256; // tensor memory columns: S (and P) of the slots, then O

// Barriers of a block: two stages of K and of V tiles, two slots with two buffers of scores each.
struct Bars {
  uint32_t base;
  __device__ __forceinline__ uint32_t k_full(int stage) const { return base + 8 * stage; }
  __device__ __forceinline__ uint32_t k_empty(int stage) const { return base + 16 + 8 * stage; }
  __device__ __forceinline__ uint32_t v_full(int stage) const { return base + 32 + 8 * stage; }
  __device__ __forceinline__ uint32_t v_empty(int stage) const { return base + 48 + 8 * stage; }
  __device__ __forceinline__ uint32_t s_full(int slot, int half) const { return base + 64 + 16 * slot + 8 * half; }
  __device__ __forceinline__ uint32_t p_full(int slot, int half) const { return base + 96 + 16 * slot + 8 * half; }
  __device__ __forceinline__ uint32_t o_full(int slot, int half) const { return base + 128 + 16 * slot + 8 * half; }
  __device__ __forceinline__ uint32_t q_full() const { return base + 160; }
  __device__ __forceinline__ uint32_t drained(int slot) const { return base + 168 + 8 * slot; }
  // a warp of a slot may make its exponentials: warps w of both slots share a quarter of the SM
  __device__ __forceinline__ uint32_t turn(int slot, int w) const { return base + 184 + 32 * slot + 8 * w; }
};
constexpr int kBars = 31;

__device__ __forceinline__ unsigned long long now_ns() {
  unsigned long long t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
__device__ __forceinline__ bool bar_test(uint32_t bar, uint32_t parity) {   // without bar_try's own wait
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// For whole warps: false, in every lane, if the phase does not complete within `limit` nanoseconds (0: is not
// over already) or another role has given up.  The lanes agree on each try, so that a wait that is over already
// costs one try and no divergence.  A try waits by itself, 4 us where nothing comes: the timer, which takes long to answer, is read
// from the first one on that failed, and a wait runs out up to two tries after its limit.
// PATIENT: who has time sleeps between tries and leaves the issue slots to the others.
template <bool PATIENT = false>
__device__ __forceinline__ bool bar_wait_warp(uint32_t bar, uint32_t parity, volatile int *abort, unsigned long long limit) {
  if (__all_sync(0xffffffffu, bar_test(bar, parity))) return true;
  if (limit == 0) {
    *abort = 1;
    return false;
  }
  unsigned long long t0 = 0;
  for (;;) {
    if constexpr (PATIENT) __nanosleep(100);
    if (__all_sync(0xffffffffu, bar_try(bar, parity))) return true;
    const unsigned long long now = now_ns();
    if (t0 == 0) t0 = now;
    if (__any_sync(0xffffffffu, *abort != 0 || now - t0 > limit)) {
      *abort = 1;
      return false;
    }
  }
}

// This thread's arrival once all its copies so far have landed.  (They are ordinary writes: who waits for
// the barrier orders them before the tensor cores' reads with fence_async.)
__device__ __forceinline__ void copies_arrive(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void copy_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Shared memory operand, 128-byte swizzle: rows of 128 bytes, 8 rows (1024 bytes) an atom.  Queries and keys
// have the k axis along the row (chunks of 64 elements, `chunk` bytes apart, are addressed by the
// caller); values have it across the rows, and their 64-element chunks follow one another at `chunk`.
__device__ __forceinline__ uint64_t operand(uint32_t at, uint32_t chunk) {
  return (uint64_t)(at >> 4) | (uint64_t)(chunk >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// 32-bit sums, 16-bit operands (0 f16, 1 bf16), 128 rows, n columns; b_across: b's k axis across its rows.
__host__ __device__ constexpr uint32_t instruction(uint32_t type, uint32_t n, uint32_t b_across) {
  return 1u << 4 | type << 7 | type << 10 | b_across << 16 | (n >> 3) << 17 | (128u >> 4) << 24;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
               "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t word(const uint4 &v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(p));
  return p != 0;
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// 32 and 16 columns of this thread's row.  The values are there after tmem_wait on them.
__device__ __forceinline__ void tmem_load(float (&x)[32], uint32_t at) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
      "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]), "=f"(x[8]),
        "=f"(x[9]), "=f"(x[10]), "=f"(x[11]), "=f"(x[12]), "=f"(x[13]), "=f"(x[14]), "=f"(x[15]), "=f"(x[16]), "=f"(x[17]),
        "=f"(x[18]), "=f"(x[19]), "=f"(x[20]), "=f"(x[21]), "=f"(x[22]), "=f"(x[23]), "=f"(x[24]), "=f"(x[25]), "=f"(x[26]),
        "=f"(x[27]), "=f"(x[28]), "=f"(x[29]), "=f"(x[30]), "=f"(x[31])
      : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_wait(float (&x)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+f"(x[0]), "+f"(x[1]), "+f"(x[2]), "+f"(x[3]), "+f"(x[4]), "+f"(x[5]), "+f"(x[6]), "+f"(x[7]), "+f"(x[8]),
                 "+f"(x[9]), "+f"(x[10]), "+f"(x[11]), "+f"(x[12]), "+f"(x[13]), "+f"(x[14]), "+f"(x[15]), "+f"(x[16]),
                 "+f"(x[17]), "+f"(x[18]), "+f"(x[19]), "+f"(x[20]), "+f"(x[21]), "+f"(x[22]), "+f"(x[23]), "+f"(x[24]),
                 "+f"(x[25]), "+f"(x[26]), "+f"(x[27]), "+f"(x[28]), "+f"(x[29]), "+f"(x[30]), "+f"(x[31])
               :: "memory");
}
__device__ __forceinline__ void tmem_load_16(float (&x)[16], uint32_t at) {   // waits
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]), "=f"(x[4]), "=f"(x[5]), "=f"(x[6]), "=f"(x[7]), "=f"(x[8]),
        "=f"(x[9]), "=f"(x[10]), "=f"(x[11]), "=f"(x[12]), "=f"(x[13]), "=f"(x[14]), "=f"(x[15])
      : "r"(at) : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// Two 32-bit operations in one instruction.
__device__ __forceinline__ void fma_pair(float &x, float &y, float ax, float ay, float b) {
  asm("{\n\t.reg .b64 v, k, s;\n\tmov.b64 v, {%0, %1};\n\tmov.b64 k, {%2, %3};\n\tmov.b64 s, {%4, %4};\n\t"
      "fma.rn.f32x2 v, v, k, s;\n\tmov.b64 {%0, %1}, v;\n\t}"
      : "+f"(x), "+f"(y) : "f"(ax), "f"(ay), "f"(b));
}
__device__ __forceinline__ void add_pair(float &x, float &y, float ax, float ay) {
  asm("{\n\t.reg .b64 v, k;\n\tmov.b64 v, {%0, %1};\n\tmov.b64 k, {%2, %3};\n\tadd.rn.f32x2 v, v, k;\n\tmov.b64 {%0, %1}, v;\n\t}"
      : "+f"(x), "+f"(y) : "f"(ax), "f"(ay));
}
__device__ __forceinline__ void mul_pair(float &x, float &y, float ax, float ay) {
  asm("{\n\t.reg .b64 v, k;\n\tmov.b64 v, {%0, %1};\n\tmov.b64 k, {%2, %3};\n\tmul.rn.f32x2 v, v, k;\n\tmov.b64 {%0, %1}, v;\n\t}"
      : "+f"(x), "+f"(y) : "f"(ax), "f"(ay));
}
template <int N> __device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void give_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

__device__ __forceinline__ void tmem_store_16(uint32_t at, const uint32_t (&x)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(at),
      "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]), "r"(x[8]), "r"(x[9]), "r"(x[10]),
      "r"(x[11]), "r"(x[12]), "r"(x[13]), "r"(x[14]), "r"(x[15]) : "memory");
}
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 16-byte piece `piece` of row r in a tile of 128-byte rows, tiles of 64 elements one after the other.
__device__ __forceinline__ uint32_t piece_at(int r, int piece) {
  return (piece >> 3) * (kTile * 128) + r * 128 + (((piece & 7) ^ (r & 7)) << 4);
}

}  // namespace emoe
