// One block whose threads wait, with a short limit, on a barrier that nothing
// arrives on, through the waits of the attention kernels.
#include "../../paper_2504_13850_gb300/csrc/fo_scored_tc.cuh"

namespace fo {
namespace {

__device__ GaveUp g_err;

// out[0..2]: nanoseconds of a wait by one thread, of the same thread's next
// wait, and of a whole warp's; out[3]: how many of the three gave up.
__global__ void wait_k(uint64_t limit, int code, unsigned long long* out) {
  __shared__ uint64_t bar;
  if (threadIdx.x == 0) {
    mbar_init(&bar, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    Waits wait(&g_err, limit);
    const uint64_t t0 = global_ns();
    wait.on(&bar, 0, code);
    const uint64_t t1 = global_ns();
    const bool gave_up = wait.dead;
    wait.on(&bar, 0, code + 1);
    out[0] = t1 - t0;
    out[1] = global_ns() - t1;
    out[3] = gave_up + wait.dead;
  }
  __syncthreads();
  Waits wait(&g_err, limit);
  const uint64_t t0 = global_ns();
  wait.on_warp(&bar, 0, code + 2);
  if (threadIdx.x == 0) {
    out[2] = global_ns() - t0;
    out[3] += wait.dead;
  }
}

}  // namespace
}  // namespace fo

extern "C" __attribute__((visibility("default"))) int probe_wait(uint64_t limit, int code, unsigned long long* host) {
  unsigned long long* out = nullptr;
  cudaError_t e = cudaMalloc(&out, 4 * sizeof(*out));
  if (e != cudaSuccess) return int(e);
  fo::wait_k<<<1, 32>>>(limit, code, out);
  e = cudaGetLastError();
  if (e == cudaSuccess) e = cudaMemcpy(host, out, 4 * sizeof(*out), cudaMemcpyDeviceToHost);
  cudaFree(out);
  return int(e);
}
extern "C" __attribute__((visibility("default"))) int probe_told(unsigned* told, int* code) {
  return int(fo::gave_up_since(fo::g_err, told, code));
}
