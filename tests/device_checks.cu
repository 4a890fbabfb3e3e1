// device_checks.cu - parts of the attention kernels by themselves: the order of a batch's sequences, waits that run out.
#include "../paper_2510_02613_b200/csrc/attend_masked.cuh"
#include "../paper_2510_02613_b200/csrc/tensor.cuh"

using namespace emoe;

namespace {

__global__ void __launch_bounds__(128) order_kernel(const __grid_constant__ MaskedArgs a, int32_t *out) {
  const int seq = ranked_tile(a, 1, blockIdx.x);
  if (threadIdx.x == 0) out[blockIdx.x] = seq;
}

// A warp waits for a barrier that nobody arrives at; another one, if asked to, gives up after a while.
template <bool PATIENT>
__global__ void __launch_bounds__(64) wait_kernel(unsigned long long limit, unsigned long long give_up, unsigned long long *took, int32_t *result) {
  __shared__ uint64_t bar;
  __shared__ int s_abort;
  if (threadIdx.x == 0) {
    bar_init(shared_address(&bar), 1);
    s_abort = 0;
  }
  __syncthreads();
  const unsigned long long t0 = now_ns();
  if (threadIdx.x >= 32) {
    while (give_up && now_ns() - t0 < give_up) __nanosleep(100);
    if (give_up) *(volatile int *)&s_abort = 1;
    return;
  }
  const bool ok = bar_wait_warp<PATIENT>(shared_address(&bar), 0, &s_abort, limit);
  if (threadIdx.x == 0) {
    *took = now_ns() - t0;
    *result = ok ? 1 : s_abort ? 2 : 0;
  }
}

}  // namespace

// out[rank]: the sequence of that rank; pointers are device memory.
extern "C" int check_order(const int32_t *own_lens, int32_t n_seqs, int32_t max_blocks, int32_t block_tokens, int32_t window, int32_t sinks, int32_t *out) {
  if (n_seqs <= 0 || n_seqs > kMostRanked) return -1;
  MaskedArgs a{};
  a.own_lens = own_lens;
  a.n_seqs = n_seqs;
  a.max_blocks = max_blocks;
  a.c.block_tokens = block_tokens;
  a.window = window;
  a.sinks = sinks;
  order_kernel<<<n_seqs, 128>>>(a, out);
  return (int)cudaDeviceSynchronize();
}

extern "C" int check_wait(int32_t patient, unsigned long long limit_ns, unsigned long long give_up_ns, unsigned long long *took, int32_t *result) {
  if (patient) wait_kernel<true><<<1, 64>>>(limit_ns, give_up_ns, took, result);
  else wait_kernel<false><<<1, 64>>>(limit_ns, give_up_ns, took, result);
  return (int)cudaDeviceSynchronize();
}
