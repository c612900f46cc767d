// Host side of the tensor copies (maps of row-major matrices in the 128-byte swizzle) and of launches with attributes.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

namespace stq {

// `elem` 1: bytes, 2: bf16, 4: fp32.  The box is box_cols x box_rows elements, box_cols * elem <= 128 bytes; base and pitch are
// multiples of 16 bytes; elements outside rows x cols read as zero.
cudaError_t make_tensor_map(CUtensorMap* map, const void* p, int elem, uint64_t rows, uint64_t cols, uint64_t pitch,
                            uint32_t box_rows, uint32_t box_cols, bool swizzle);

// Whether every row of a matrix with this pitch in bytes is aligned to 16 bytes.
inline bool rows_aligned(const void* p, size_t pitch) { return ((reinterpret_cast<uintptr_t>(p) | pitch) & 15) == 0; }

// Whether tensor copies can write a matrix: rows on 16 bytes, and whole numbers of 16 bytes (at a row's end a copy to memory
// is cut off by pieces of 16 bytes, not by elements, and would write into what lies between the rows).
inline bool copy_fits(const void* p, size_t row, size_t pitch) { return rows_aligned(p, row | pitch); }

// Lets a kernel take `bytes` of dynamic shared memory; `seen` has a bit for each device where that is settled.
template <class K>
cudaError_t allow_smem(K kernel, size_t bytes, int device, std::atomic<uint64_t>& seen) {
  const uint64_t bit = device < 64 ? 1ull << device : 0;
  if (bit && (seen.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
  if (e == cudaSuccess) seen.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

// early: the kernel may start while the one before it in the stream still runs (it waits for that one's results itself).
template <class... P, class... A>
cudaError_t launch_with(void (*kernel)(P...), dim3 grid, dim3 threads, size_t smem, unsigned cluster, bool early, cudaStream_t stream,
                        const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = threads;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute at[2];
  unsigned n = 0;
  if (cluster > 1) {
    at[n].id = cudaLaunchAttributeClusterDimension;
    at[n].val.clusterDim.x = cluster;
    at[n].val.clusterDim.y = at[n].val.clusterDim.z = 1;
    ++n;
  }
  if (early) {
    at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[n].val.programmaticStreamSerializationAllowed = 1;
    ++n;
  }
  cfg.attrs = at;
  cfg.numAttrs = n;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace stq
