// The handle behind the C ABI and what every entry point needs of it.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include <string>
#include <vector>

#include "../../include/stq.h"
#include "stq_internal.h"
#include "stq_q8.h"

namespace stq {
struct KeptBuffer {
  void* p;
  KeptBuffer* next;
};
}  // namespace stq

struct stq_handle {
  int device = 0;
  int sm_count = 0;
  int grid = 0;
  uint64_t launches = 0;
  std::string cuda_err;

  // cached caller table (to skip re-uploads) and its device image
  std::vector<stq_tensor> cached;
  int cached_kind = -1;          // which entry point built the device table
  std::vector<uint64_t> cached_sig;   // numel | wide<<63 per tensor: decides the tile map
  stq::TensorDesc* d_table = nullptr;
  size_t d_table_cap = 0;
  // tile -> tensor index; order: fast tiles, then the remaining narrow tiles, then wide ones
  uint32_t* d_tile_map = nullptr;
  size_t d_tile_cap = 0;
  uint32_t n_tiles = 0, n_fast = 0, n_narrow = 0;   // n_narrow counts fast + remaining narrow
  uint32_t n_main = 0, n_var_end = 0;               // fast tiles: [0, n_main) fused bodies, [n_main, n_var_end) fused bodies
                                                    // of the "sr" / "ts" codes, [n_var_end, n_fast) change width
  int fast_grid = 0;
  bool any_lp = false;              // some tensor of the current table wants a low-precision copy
  bool any_variant = false;         // some tensor's second moment uses a code only the generic kernel serves
  // Raised by a kernel whose bounded wait ran out.  It lies in host memory that the device writes to, so that later calls
  // see it without waiting for anything.
  int* h_err = nullptr;         // as the host sees it
  int* d_err = nullptr;         // as the device does
  int* d_valid = nullptr;       // non-zero if the last call that carried statistics really produced them (a skipped step does not)
  float* d_scalars = nullptr;   // {step_size, rsqrt_bc2, lr} when the step count lives on the device
  stq::FastSched* d_sched = nullptr;   // two work lists of the main step kernel (fused bodies, width changes)

  // pinned staging for uploads
  void* h_stage = nullptr;
  size_t h_stage_cap = 0;
  cudaEvent_t stage_ev = nullptr;
  // the generic kernel's share of a step (ragged tails, 32-bit states) runs beside the main kernel:
  cudaStream_t side = nullptr;
  cudaEvent_t ev_fork = nullptr, ev_join = nullptr;
  bool stage_busy = false;

  // statistics
  double* d_partials = nullptr;
  size_t d_partials_cap = 0;
  double* d_stats = nullptr;
  size_t d_stats_cap = 0;
  uint32_t* d_seg_map = nullptr;   // statistics segment -> tensor
  size_t d_seg_map_cap = 0;
  double* d_seg_sums = nullptr;
  size_t d_seg_sums_cap = 0;
  uint32_t n_seg = 0;
  double* h_stats = nullptr;
  size_t h_stats_cap = 0;
  int stats_L = 0;            // > 0: partials of a table with this many tensors are pending

  // device arena, streams and events of stq_step_host
  uint8_t* d_arena = nullptr;
  size_t d_arena_cap = 0;
  cudaStream_t host_streams[3] = {nullptr, nullptr, nullptr};
  std::vector<cudaEvent_t> host_events;

  // workspace of the 8-bit operators: partial sums of split products and column sums, a pitched copy of a gradient
  uint8_t* d_q8 = nullptr;
  size_t d_q8_cap = 0;
  bool q8_in_graph = false;            // a captured graph uses d_q8: when it is replaced it stays until the handle goes,
  stq::KeptBuffer* q8_kept = nullptr;  // in this list
  uint32_t* d_q8_counters = nullptr;   // kQ8Counters of them, zero between launches
};

namespace stq {

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Whether a bounded wait of an earlier launch is known to have run out.
inline bool gave_up(const stq_handle* h) { return *static_cast<const volatile int*>(h->h_err) != 0; }

inline int fail_cuda(stq_handle* h, cudaError_t e) {
  h->cuda_err = cudaGetErrorString(e);
  return STQ_E_CUDA;
}
#define STQ_CUDA(h, call)                                   \
  do {                                                      \
    cudaError_t e__ = (call);                               \
    if (e__ != cudaSuccess) return fail_cuda((h), e__);     \
  } while (0)

template <class T>
inline int grow(stq_handle* h, T*& p, size_t& cap, size_t need) {
  if (need <= cap) return STQ_OK;
  if (p) cudaFree(p);
  p = nullptr;
  cap = 0;
  size_t want = need + need / 4 + 256;
  cudaError_t e = cudaMalloc(reinterpret_cast<void**>(&p), want * sizeof(T));
  if (e != cudaSuccess) {
    h->cuda_err = cudaGetErrorString(e);
    (void)cudaGetLastError();      // (or the next launch that is asked for its error would report this one)
    p = nullptr;
    return STQ_E_WORKSPACE;
  }
  cap = want;
  return STQ_OK;
}

}  // namespace stq
