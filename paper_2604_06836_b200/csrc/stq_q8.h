// Internal interface between the host layer of the 8-bit operators (stq_q8_api.cu) and their kernels.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace stq {

constexpr int kQ8Block = 128;             // columns that share a scale in an activation checkpoint
constexpr uint64_t kQ8MaxCols = 1u << 24; // widest row any operator takes

// A dense row-major matrix as the row kernels see it (pitch in elements; p may be null where that is allowed).
struct Mat {
  void* p;
  size_t ld;
};

enum Q8Kind { kQ8Copy = 0, kQ8SiluGated = 1, kQ8Gelu = 2 };

struct RowArgs {
  Mat x;                 // input of the activation / x of the norm
  Mat res;               // norm: residual that is added, or null
  const float* weight;   // norm: fp32 weight
  Mat h;                 // norm: x + res, written if res is there
  float* rstd;           // norm
  float eps;
  uint64_t rows;
  uint32_t cols;         // columns of the 8-bit result
  int8_t* q;             // 8-bit rows, pitch ldq bytes
  size_t ldq;
  float* scale;
  Mat values;            // bf16 values of the codes, or null
  int8_t* ckq;           // checkpoint [rows][parts][ldck], or null
  size_t ldck;
  float* cks;            // its scales [rows][parts][ceil(cols/128)]
};

cudaError_t launch_q8_act(int dtype, Q8Kind kind, const RowArgs& a, int sms, cudaStream_t stream);
cudaError_t launch_q8_norm(int dtype, const RowArgs& a, int sms, cudaStream_t stream);

struct NormBwdArgs {
  Mat dy, h, dres, dx;   // dres may be null
  const float* weight;
  const float* rstd;
  float* dweight;
  float* partial;        // q8_norm_bwd_partial() floats
  size_t ldp;            // columns, rounded up to a multiple of 8
  uint32_t* counters;
  uint64_t rows;
  uint32_t cols;
};
// Counters in the handle, zero between launches, at which CTAs arrive whose partial sums are added up.
constexpr uint32_t kQ8Counters = 4096;
constexpr uint32_t kNormBwdMaxCols = 49152;   // widest row: the sums of the widest variant stay in shared memory
size_t q8_norm_bwd_partial(int dtype, const NormBwdArgs& a, int sms);
cudaError_t launch_q8_norm_bwd(int dtype, const NormBwdArgs& a, int sms, cudaStream_t stream, int* launches);

struct ActBwdArgs {
  Mat da, dz;
  const int8_t* ckq;
  size_t ldck;
  const float* cks;
  uint64_t rows;
  uint32_t cols;
};
cudaError_t launch_q8_act_bwd(int dtype, Q8Kind kind, const ActBwdArgs& a, cudaStream_t stream);

// out[c] = sum over rows of x[r][c], in fp32, through q8_colsum_partial() floats of partial sums.
uint32_t q8_colsum_splits(uint64_t rows, uint32_t cols, int sms);
size_t q8_colsum_partial(uint32_t cols, uint32_t splits);
cudaError_t launch_q8_colsum(int dtype, Mat x, uint64_t rows, uint32_t cols, uint32_t splits, float* partial, uint32_t* counters,
                             float* out, cudaStream_t stream);

struct GemmArgs {
  const int8_t* xq;      // 8-bit operand whose row scales lie along the rows of the result (or along the sum)
  size_t ldx;
  const float* xs;
  const int8_t* wq;
  size_t ldw;
  const float* ws;
  const float* bias;
  const void* dy;        // bf16 gradient
  size_t lddy;
  void* out;
  size_t ldo;
  int out_dtype;
  uint64_t t;            // tokens
  uint32_t n, k;         // output and input channels
  int device;
};
// (err: the handle's flag, raised by a wait that ran out)
cudaError_t launch_q8_linear(const GemmArgs& a, int sms, int* err, cudaStream_t stream);
// Bytes of workspace (aligned to 256) that a gradient needs; launches: how many kernels went out.
size_t q8_grad_workspace(const GemmArgs& a, bool dw, int sms);
cudaError_t launch_q8_linear_dx(const GemmArgs& a, void* ws, int sms, int* err, cudaStream_t stream, int* launches);
cudaError_t launch_q8_linear_dw(const GemmArgs& a, void* ws, int sms, int* err, cudaStream_t stream, int* launches);

}  // namespace stq
