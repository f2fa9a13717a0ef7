// Host-side helpers of the decode kernels: tensor maps and launches.
#pragma once

#include <atomic>

#include <cuda.h>
#include <cuda_runtime.h>

#include "amla_common.cuh"

namespace amla {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn get_encode_fn() {
  static std::atomic<EncodeTiledFn> fn{nullptr};
  EncodeTiledFn f = fn.load(std::memory_order_acquire);
  if (!f) {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult qres;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &qres) == cudaSuccess &&
        qres == cudaDriverEntryPointSuccess) {
      f = reinterpret_cast<EncodeTiledFn>(p);
      fn.store(f, std::memory_order_release);
    }
  }
  return f;
}

// Rows of 576 bf16 seen as (64 columns, rows, 9 column blocks); a box is box_rows x box_blocks, laid out in shared
// memory as [block][row][128 B] with the 128-byte swizzle.
inline bool encode_rows(EncodeTiledFn encode, CUtensorMap* map, const void* base, cuuint64_t rows, cuuint32_t box_rows, cuuint32_t box_blocks) {
  const cuuint64_t dims[3] = {64, rows, static_cast<cuuint64_t>(kDqk / 64)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(kDqk) * 2, 128};
  const cuuint32_t box[3] = {64, box_rows, box_blocks};
  const cuuint32_t estr[3] = {1, 1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The opt-in to large dynamic shared memory is per device and per kernel: `done` remembers the devices that have it.
template <typename Kernel>
cudaError_t allow_shared(Kernel kern, std::atomic<uint64_t>& done, uint32_t smem_bytes) {
  int device = 0;
  cudaError_t err = cudaGetDevice(&device);
  if (err != cudaSuccess) return err;
  const uint64_t bit = 1ull << (device & 63);
  if (!(done.load(std::memory_order_acquire) & bit)) {
    err = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem_bytes));
    if (err != cudaSuccess) return err;
    done.fetch_or(bit, std::memory_order_release);
  }
  return cudaSuccess;
}

// Launches `kern` on `stream` with programmatic stream serialization.
template <typename... Params, typename... Args>
cudaError_t launch_in_order(void (*kern)(Params...), dim3 grid, int threads, uint32_t smem_bytes, cudaStream_t stream, const Args&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem_bytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, Params(args)...);
}

// The same with `smem_bytes` of dynamic shared memory that the kernel always has.
template <typename Kernel, typename... Args>
cudaError_t launch_serialized(Kernel kern, std::atomic<uint64_t>& done, int grid, int threads, uint32_t smem_bytes, cudaStream_t stream, const Args&... args) {
  const cudaError_t err = allow_shared(kern, done, smem_bytes);
  return err != cudaSuccess ? err : launch_in_order(kern, dim3(grid), threads, smem_bytes, stream, args...);
}

}  // namespace amla
