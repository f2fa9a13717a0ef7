// Self-test of the bounded device-side wait (diagnostic; not on the decode path).
//
// Every wait inside the decode kernels gives up, records kStatusTimeout in the status word and lets the kernel return, so that a lost
// signal shows up as AMLA_ERR_DEVICE_TIMEOUT instead of a hung GPU: after a time limit (mbar_wait), or in the kernel for a 4-bit
// cache after a number of tries (mbar_wait_spend).  These kernels make that observable without disturbing a real decode: one warp initialises
// an mbarrier that nothing ever arrives on, waits on it through the same routine that the kernels use, with a caller-chosen (short) limit
// or number of tries, and records the outcome.  No TMA, no tensor memory, no second CTA: then the kernel simply ends.
#include "amla_common.cuh"
#include "amla_sm100.cuh"

namespace amla {

__global__ void __launch_bounds__(32, 1) wait_selftest_kernel(int* status, unsigned long long limit_ns) {
  __shared__ __align__(8) unsigned long long bar_storage;
  const uint32_t bar = sm100::smem_u32(&bar_storage);
  if (threadIdx.x == 0) {
    *status = kStatusOk;
    sm100::mbar_init(bar, 1);
  }
  __syncwarp();
  // phase 0 never completes: there is no arrival
  const bool ok = __all_sync(0xffffffffu, sm100::mbar_wait(bar, 0, limit_ns));
  if (!ok && threadIdx.x == 0) atomicExch(status, kStatusTimeout);
}

cudaError_t launch_wait_selftest(int* status, unsigned long long limit_ns, cudaStream_t stream) {
  wait_selftest_kernel<<<1, 32, 0, stream>>>(status, limit_ns);
  return cudaGetLastError();
}

// report: the tries that are left behind a wait for what never comes, behind a second one with none left, and behind a wait for what has come; the
// nanoseconds that the first two took.
__global__ void __launch_bounds__(32, 1) tries_selftest_kernel(int* status, int tries, int* report) {
  __shared__ __align__(8) unsigned long long bar_storage[2];
  const uint32_t never = sm100::smem_u32(bar_storage), done = never + 8;
  if (threadIdx.x == 0) {
    *status = kStatusOk;
    sm100::mbar_init(never, 1);
    sm100::mbar_init(done, 1);
    sm100::mbar_arrive(done);
  }
  __syncwarp();
  int left = tries, still = tries;
  const uint64_t t0 = sm100::global_timer_ns();
  sm100::mbar_wait_spend(never, 0, left);
  const uint64_t t1 = sm100::global_timer_ns();
  const int after = left;
  sm100::mbar_wait_spend(never, 0, left);
  const uint64_t t2 = sm100::global_timer_ns();
  sm100::mbar_wait_spend(done, 0, still);
  if (!__all_sync(0xffffffffu, after > 0) && threadIdx.x == 0) atomicExch(status, kStatusTimeout);
  if (threadIdx.x == 0) {
    report[0] = after;
    report[1] = left;
    report[2] = still;
    report[3] = static_cast<int>(t1 - t0);
    report[4] = static_cast<int>(t2 - t1);
  }
}

cudaError_t launch_tries_selftest(int* status, int tries, int* report, cudaStream_t stream) {
  tries_selftest_kernel<<<1, 32, 0, stream>>>(status, tries, report);
  return cudaGetLastError();
}

}  // namespace amla
