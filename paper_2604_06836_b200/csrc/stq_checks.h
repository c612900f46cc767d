// Checks of arguments, and the workspace, that the entry points of the operators share.
#pragma once
#include <new>

#include "stq_handle.h"

namespace stq {

constexpr uint64_t kMaxRows = 0x7fffffffull;   // (one CTA per row in some kernels)

inline size_t elem(int dtype) { return dtype == STQ_GRAD_F32 ? 4 : 2; }

// A range of memory that a call reads or writes.
struct Span {
  const void* p;
  size_t bytes;
};
inline Span mat(const void* p, uint64_t ld, uint64_t rows, uint64_t cols, size_t e) {
  return {p, p && rows ? (size_t)(((rows - 1) * ld + cols) * e) : 0};
}
template <size_t N, size_t M>
bool clash(const Span (&out)[N], const Span (&in)[M]) {
  auto hit = [](const Span& a, const Span& b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    return a.p && b.p && a.bytes && b.bytes && x < y + b.bytes && y < x + a.bytes;
  };
  for (size_t i = 0; i < N; ++i) {
    for (const Span& s : in)
      if (hit(out[i], s)) return true;
    for (size_t j = 0; j < i; ++j)
      if (hit(out[i], out[j])) return true;
  }
  return false;
}

// (results of a launch that gave up are invalid, and so is what is computed from them: the handle's later calls say so)
inline int check_handle(const stq_handle* h) { return !h ? STQ_E_NULL : gave_up(h) ? STQ_E_TIMEOUT : STQ_OK; }
inline int check_dtype(int dtype) { return dtype == STQ_GRAD_F32 || dtype == STQ_GRAD_BF16 ? STQ_OK : STQ_E_ARG; }
inline int check_size(uint64_t rows, uint64_t cols) {
  if (cols == 0) return STQ_E_NUMEL;
  return rows > kMaxRows || cols > kQ8MaxCols ? STQ_E_TOO_LARGE : STQ_OK;
}
inline int check_mat(const void* p, uint64_t ld, uint64_t cols, size_t e) {
  if (!p) return STQ_E_NULL;
  if (!aligned(p, e)) return STQ_E_ALIGN;
  return ld < cols || ld > (1ull << 40) ? STQ_E_ARG : STQ_OK;
}
inline int check_codes(const void* q, uint64_t ldq, uint64_t cols, const void* scale) {
  if (!q || !scale) return STQ_E_NULL;
  if (!aligned(q, 16) || !aligned(scale, 4) || (ldq & 15)) return STQ_E_ALIGN;
  return ldq < cols || ldq > (1ull << 40) ? STQ_E_ARG : STQ_OK;
}
#define STQ_TRY(call)                \
  do {                               \
    const int rc__ = (call);         \
    if (rc__ != STQ_OK) return rc__; \
  } while (0)

// Lets this thread allocate while one of its streams is captured.
struct AllocInCapture {
  cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
  AllocInCapture() { cudaThreadExchangeStreamCaptureMode(&mode); }
  ~AllocInCapture() { cudaThreadExchangeStreamCaptureMode(&mode); }
};

// The workspace of a call on `stream`.  It grows by being replaced.  A graph that was captured with the old buffer goes on
// using it whenever it is replayed, so such a buffer is not freed; nor is any during a capture, where freeing would wait.
template <class T>
int workspace(stq_handle* h, size_t count, cudaStream_t stream, T** out) {
  const size_t need = count * sizeof(T);
  cudaStreamCaptureStatus status = cudaStreamCaptureStatusNone;
  STQ_CUDA(h, cudaStreamIsCapturing(stream, &status));
  const bool capturing = status != cudaStreamCaptureStatusNone;
  if (need > h->d_q8_cap) {
    if (h->d_q8 && (h->q8_in_graph || capturing)) {
      auto* kept = new (std::nothrow) KeptBuffer{h->d_q8, h->q8_kept};
      if (!kept) return STQ_E_WORKSPACE;
      h->q8_kept = kept;
      h->d_q8 = nullptr;
      h->d_q8_cap = 0;
      h->q8_in_graph = false;
    }
    AllocInCapture relaxed;
    STQ_TRY(grow(h, h->d_q8, h->d_q8_cap, need));
  }
  h->q8_in_graph |= capturing;
  *out = reinterpret_cast<T*>(h->d_q8);
  return STQ_OK;
}

inline int zero(stq_handle* h, void* p, uint64_t ld, uint64_t rows, uint64_t cols, size_t e, cudaStream_t s) {
  STQ_CUDA(h, cudaMemset2DAsync(p, ld * e, 0, cols * e, rows, s));
  return STQ_OK;
}

}  // namespace stq
