// Host side of the tensor copies: maps of row-major matrices in the 128-byte swizzle.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

namespace stq {

// `elem` 1: bytes, 2: bf16.  The box is box_cols x box_rows elements, box_cols * elem <= 128 bytes; base and pitch are
// multiples of 16 bytes; elements outside rows x cols read as zero.
cudaError_t make_tensor_map(CUtensorMap* map, const void* p, int elem, uint64_t rows, uint64_t cols, uint64_t pitch,
                            uint32_t box_rows, uint32_t box_cols, bool swizzle);

// Largest of 32, 16, 1 bytes that every row of a matrix with this pitch in bytes is aligned to.
inline int row_alignment(const void* p, size_t pitch) {
  const uintptr_t b = reinterpret_cast<uintptr_t>(p) | pitch;
  return (b & 31) == 0 ? 32 : (b & 15) == 0 ? 16 : 1;
}

// Lets a kernel take `bytes` of dynamic shared memory; `seen` has a bit for each device where that is settled.
template <class K>
cudaError_t allow_smem(K kernel, size_t bytes, int device, std::atomic<uint64_t>& seen) {
  const uint64_t bit = device < 64 ? 1ull << device : 0;
  if (bit && (seen.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == cudaSuccess) seen.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

template <class K, class... A>
cudaError_t launch_cluster(K kernel, unsigned grid, unsigned threads, size_t smem, unsigned cluster, cudaStream_t stream,
                           const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = threads;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = cluster;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = cluster > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace stq
