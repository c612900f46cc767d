// Products of the 8-bit operators, one 64 x 64 tile of the result to a CTA, on the CUDA cores.
#include <cuda_bf16.h>

#include "../../include/stq.h"
#include "stq_internal.h"
#include "stq_q8.h"

namespace stq {
namespace {

constexpr int kT = 64, kD = 32;   // tile of the result, depth of a step

template <class O>
__device__ __forceinline__ void put(void* out, size_t at, float v) {
  static_cast<O*>(out)[at] = static_cast<O>(v);
}

// out[i][j] = sum_c A(i, c) * B(c, j), 256 threads, 4 x 4 results each
template <class Acc, class FA, class FB, class FO>
__device__ __forceinline__ void tile_product(uint64_t m, uint32_t n, uint64_t depth, FA fa, FB fb, FO fo) {
  __shared__ Acc sa[kD][kT + 1], sb[kD][kT + 1];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const uint64_t i0 = (uint64_t)blockIdx.y * kT;
  const uint32_t j0 = blockIdx.x * kT;
  Acc acc[4][4] = {};
  for (uint64_t c0 = 0; c0 < depth; c0 += kD) {
    for (int e = threadIdx.x; e < kT * kD; e += 256) {
      const int c = e % kD, i = e / kD;
      sa[c][i] = (i0 + i < m && c0 + c < depth) ? fa(i0 + i, c0 + c) : Acc(0);
      const int j = e % kT, d = e / kT;
      sb[d][j] = (j0 + j < n && c0 + d < depth) ? fb(c0 + d, j0 + j) : Acc(0);
    }
    __syncthreads();
#pragma unroll 4
    for (int c = 0; c < kD; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] += sa[c][ty * 4 + i] * sb[c][tx + 16 * j];
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i0 + ty * 4 + i < m && j0 + tx + 16 * j < n) fo(i0 + ty * 4 + i, j0 + tx + 16 * j, acc[i][j]);
}

template <class O>
__global__ void __launch_bounds__(256) q8_linear_dx_kernel(const GemmArgs a) {
  const __nv_bfloat16* dy = static_cast<const __nv_bfloat16*>(a.dy);
  tile_product<float>(
      a.t, a.k, a.n, [&](uint64_t i, uint64_t c) { return (float)dy[i * a.lddy + c]; },
      [&](uint64_t c, uint32_t j) { return (float)a.wq[c * a.ldw + j] * a.ws[c]; },
      [&](uint64_t i, uint32_t j, float v) { put<O>(a.out, i * a.ldo + j, v); });
}

template <class O>
__global__ void __launch_bounds__(256) q8_linear_dw_kernel(const GemmArgs a) {
  const __nv_bfloat16* dy = static_cast<const __nv_bfloat16*>(a.dy);
  tile_product<float>(
      a.n, a.k, a.t, [&](uint64_t i, uint64_t c) { return (float)dy[c * a.lddy + i]; },
      [&](uint64_t c, uint32_t j) { return (float)a.xq[c * a.ldx + j] * a.xs[c]; },
      [&](uint64_t i, uint32_t j, float v) { put<O>(a.out, i * a.ldo + j, v); });
}

dim3 tiles(uint64_t m, uint32_t n) { return dim3((n + kT - 1) / kT, (unsigned)((m + kT - 1) / kT)); }

}  // namespace

cudaError_t launch_q8_linear_dx(const GemmArgs& a, cudaStream_t stream) {
  if (a.out_dtype == STQ_GRAD_F32)
    q8_linear_dx_kernel<float><<<tiles(a.t, a.k), 256, 0, stream>>>(a);
  else
    q8_linear_dx_kernel<__nv_bfloat16><<<tiles(a.t, a.k), 256, 0, stream>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_q8_linear_dw(const GemmArgs& a, cudaStream_t stream) {
  if (a.out_dtype == STQ_GRAD_F32)
    q8_linear_dw_kernel<float><<<tiles(a.n, a.k), 256, 0, stream>>>(a);
  else
    q8_linear_dw_kernel<__nv_bfloat16><<<tiles(a.n, a.k), 256, 0, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace stq
