// C-ABI host layer of the 8-bit operators: argument checks, workspace, launches.
#include "stq_checks.h"
#include "stq_handle.h"
#include "stq_q8.h"

using namespace stq;

static_assert(STQ_CKPT_BLOCK == stq::kQ8Block, "the checkpoint's block promised in the header");
static_assert(STQ_NORM_BWD_MAX_COLS == stq::kNormBwdMaxCols, "the widest row promised in the header");

extern "C" {

int stq_q8_rows(stq_handle* h, const void* x, uint64_t ldx, int dtype, uint64_t rows, uint32_t cols, int8_t* q,
                uint64_t ldq, float* scale, void* stream) {
  STQ_TRY(check_handle(h));
  STQ_TRY(check_dtype(dtype));
  STQ_TRY(check_size(rows, cols));
  if (rows == 0) return STQ_OK;
  STQ_TRY(check_mat(x, ldx, cols, elem(dtype)));
  STQ_TRY(check_codes(q, ldq, cols, scale));
  const Span out[] = {mat(q, ldq, rows, cols, 1), {scale, rows * 4}}, in[] = {mat(x, ldx, rows, cols, elem(dtype))};
  if (clash(out, in)) return STQ_E_ALIAS;
  stq::RowArgs a = {};
  a.x = {const_cast<void*>(x), ldx};
  a.rows = rows; a.cols = cols;
  a.q = q; a.ldq = ldq; a.scale = scale;
  STQ_CUDA(h, cudaSetDevice(h->device));
  STQ_CUDA(h, stq::launch_q8_act(dtype, stq::kQ8Copy, a, h->sm_count, static_cast<cudaStream_t>(stream)));
  h->launches++;
  return STQ_OK;
}

int stq_q8_norm(stq_handle* h, const void* x, uint64_t ldx, const void* res, uint64_t ldres, const float* weight,
                float eps, int dtype, uint64_t rows, uint32_t cols, void* hsum, uint64_t ldh, float* rstd, int8_t* q,
                uint64_t ldq, float* scale, void* values, uint64_t ldv, void* stream) {
  STQ_TRY(check_handle(h));
  STQ_TRY(check_dtype(dtype));
  STQ_TRY(check_size(rows, cols));
  if (!(eps > 0.f)) return STQ_E_ARG;
  if (rows == 0) return STQ_OK;
  const size_t e = elem(dtype);
  STQ_TRY(check_mat(x, ldx, cols, e));
  if (!weight || !rstd || (res == nullptr) != (hsum == nullptr)) return STQ_E_NULL;
  if (!aligned(weight, 4) || !aligned(rstd, 4)) return STQ_E_ALIGN;
  if (res) {
    STQ_TRY(check_mat(res, ldres, cols, e));
    STQ_TRY(check_mat(hsum, ldh, cols, e));
  }
  STQ_TRY(check_codes(q, ldq, cols, scale));
  if (values) STQ_TRY(check_mat(values, ldv, cols, 2));
  const Span out[] = {mat(hsum, ldh, rows, cols, e), {rstd, rows * 4}, mat(q, ldq, rows, cols, 1), {scale, rows * 4},
                      mat(values, ldv, rows, cols, 2)};
  const Span in[] = {mat(x, ldx, rows, cols, e), mat(res, ldres, rows, cols, e), {weight, cols * 4ull}};
  if (clash(out, in)) return STQ_E_ALIAS;
  stq::RowArgs a = {};
  a.x = {const_cast<void*>(x), ldx};
  a.res = {const_cast<void*>(res), ldres};
  a.weight = weight; a.eps = eps;
  a.h = {hsum, ldh};
  a.rstd = rstd;
  a.rows = rows; a.cols = cols;
  a.q = q; a.ldq = ldq; a.scale = scale;
  a.values = {values, ldv};
  STQ_CUDA(h, cudaSetDevice(h->device));
  STQ_CUDA(h, stq::launch_q8_norm(dtype, a, h->sm_count, static_cast<cudaStream_t>(stream)));
  h->launches++;
  return STQ_OK;
}

int stq_q8_norm_backward(stq_handle* h, const void* dy, uint64_t lddy, const void* hsum, uint64_t ldh,
                         const float* weight, const float* rstd, const void* dres, uint64_t lddres, int dtype,
                         uint64_t rows, uint32_t cols, void* dx, uint64_t lddx, float* dweight, void* stream) {
  STQ_TRY(check_handle(h));
  STQ_TRY(check_dtype(dtype));
  STQ_TRY(check_size(rows, cols));
  if (cols > STQ_NORM_BWD_MAX_COLS) return STQ_E_TOO_LARGE;
  if (!dweight) return STQ_E_NULL;
  if (!aligned(dweight, 4)) return STQ_E_ALIGN;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  STQ_CUDA(h, cudaSetDevice(h->device));
  if (rows == 0) return zero(h, dweight, cols, 1, cols, 4, s);
  const size_t e = elem(dtype);
  STQ_TRY(check_mat(dy, lddy, cols, e));
  STQ_TRY(check_mat(hsum, ldh, cols, e));
  STQ_TRY(check_mat(dx, lddx, cols, e));
  if (dres) STQ_TRY(check_mat(dres, lddres, cols, e));
  if (!weight || !rstd) return STQ_E_NULL;
  if (!aligned(weight, 4) || !aligned(rstd, 4)) return STQ_E_ALIGN;
  const Span out[] = {mat(dx, lddx, rows, cols, e), {dweight, cols * 4ull}};
  const Span in[] = {mat(dy, lddy, rows, cols, e), mat(hsum, ldh, rows, cols, e), mat(dres, lddres, rows, cols, e),
                     {weight, cols * 4ull}, {rstd, rows * 4}};
  if (clash(out, in)) return STQ_E_ALIAS;
  stq::NormBwdArgs a = {};
  a.dy = {const_cast<void*>(dy), lddy};
  a.h = {const_cast<void*>(hsum), ldh};
  a.dres = {const_cast<void*>(dres), lddres};
  a.dx = {dx, lddx};
  a.weight = weight; a.rstd = rstd; a.dweight = dweight;
  a.rows = rows; a.cols = cols;
  a.ldp = ((size_t)cols + 7) / 8 * 8;
  a.counters = h->d_q8_counters;
  STQ_TRY(workspace(h, stq::q8_norm_bwd_partial(dtype, a, h->sm_count), s, &a.partial));
  int launches = 0;
  STQ_CUDA(h, stq::launch_q8_norm_bwd(dtype, a, h->sm_count, s, &launches));
  h->launches += launches;
  return STQ_OK;
}

int stq_q8_act(stq_handle* h, const void* z, uint64_t ldz, int kind, int dtype, uint64_t rows, uint32_t cols, int8_t* q,
               uint64_t ldq, float* scale, void* values, uint64_t ldv, int8_t* ckq, uint64_t ldck, float* ckscale,
               void* stream) {
  STQ_TRY(check_handle(h));
  if (kind != STQ_ACT_SILU_GATED && kind != STQ_ACT_GELU) return STQ_E_ARG;
  STQ_TRY(check_dtype(dtype));
  STQ_TRY(check_size(rows, cols));
  if (rows == 0) return STQ_OK;
  const uint64_t parts = kind == STQ_ACT_SILU_GATED ? 2 : 1, blocks = (cols + stq::kQ8Block - 1) / stq::kQ8Block;
  STQ_TRY(check_mat(z, ldz, parts * cols, elem(dtype)));
  STQ_TRY(check_codes(q, ldq, cols, scale));
  if (values) STQ_TRY(check_mat(values, ldv, cols, 2));
  if (ckq) STQ_TRY(check_codes(ckq, ldck, cols, ckscale));
  const Span out[] = {mat(q, ldq, rows, cols, 1), {scale, rows * 4}, mat(values, ldv, rows, cols, 2),
                      mat(ckq, ldck, rows * parts, cols, 1), {ckq ? ckscale : nullptr, rows * parts * blocks * 4}};
  const Span in[] = {mat(z, ldz, rows, parts * cols, elem(dtype))};
  if (clash(out, in)) return STQ_E_ALIAS;
  stq::RowArgs a = {};
  a.x = {const_cast<void*>(z), ldz};
  a.rows = rows; a.cols = cols;
  a.q = q; a.ldq = ldq; a.scale = scale;
  a.values = {values, ldv};
  a.ckq = ckq; a.ldck = ldck; a.cks = ckscale;
  STQ_CUDA(h, cudaSetDevice(h->device));
  STQ_CUDA(h, stq::launch_q8_act(dtype, kind == STQ_ACT_SILU_GATED ? stq::kQ8SiluGated : stq::kQ8Gelu, a,
                                 h->sm_count, static_cast<cudaStream_t>(stream)));
  h->launches++;
  return STQ_OK;
}

int stq_q8_act_backward(stq_handle* h, const void* da, uint64_t ldda, int kind, int dtype, uint64_t rows, uint32_t cols,
                        const int8_t* ckq, uint64_t ldck, const float* ckscale, void* dz, uint64_t lddz, void* stream) {
  STQ_TRY(check_handle(h));
  if (kind != STQ_ACT_SILU_GATED && kind != STQ_ACT_GELU) return STQ_E_ARG;
  STQ_TRY(check_dtype(dtype));
  STQ_TRY(check_size(rows, cols));
  if (rows == 0) return STQ_OK;
  const uint64_t parts = kind == STQ_ACT_SILU_GATED ? 2 : 1, blocks = (cols + stq::kQ8Block - 1) / stq::kQ8Block;
  const size_t e = elem(dtype);
  STQ_TRY(check_mat(da, ldda, cols, e));
  STQ_TRY(check_mat(dz, lddz, parts * cols, e));
  STQ_TRY(check_codes(ckq, ldck, cols, ckscale));
  const Span out[] = {mat(dz, lddz, rows, parts * cols, e)};
  const Span in[] = {mat(da, ldda, rows, cols, e), mat(ckq, ldck, rows * parts, cols, 1), {ckscale, rows * parts * blocks * 4}};
  if (clash(out, in)) return STQ_E_ALIAS;
  stq::ActBwdArgs a = {};
  a.da = {const_cast<void*>(da), ldda};
  a.dz = {dz, lddz};
  a.ckq = ckq; a.ldck = ldck; a.cks = ckscale;
  a.rows = rows; a.cols = cols;
  STQ_CUDA(h, cudaSetDevice(h->device));
  STQ_CUDA(h, stq::launch_q8_act_bwd(dtype, kind == STQ_ACT_SILU_GATED ? stq::kQ8SiluGated : stq::kQ8Gelu, a,
                                     static_cast<cudaStream_t>(stream)));
  h->launches++;
  return STQ_OK;
}

int stq_q8_linear(stq_handle* h, const int8_t* xq, uint64_t ldx, const float* xscale, const int8_t* wq, uint64_t ldw,
                  const float* wscale, const float* bias, uint64_t t, uint32_t n, uint32_t k, void* out, uint64_t ldo,
                  int out_dtype, void* stream) {
  STQ_TRY(check_handle(h));
  STQ_TRY(check_dtype(out_dtype));
  STQ_TRY(check_size(t, n));
  STQ_TRY(check_size(t, k));
  if (k > STQ_LINEAR_MAX_K) return STQ_E_TOO_LARGE;
  if (t == 0) return STQ_OK;
  STQ_TRY(check_codes(xq, ldx, k, xscale));
  STQ_TRY(check_codes(wq, ldw, k, wscale));
  STQ_TRY(check_mat(out, ldo, n, elem(out_dtype)));
  if (!aligned(bias, 4)) return STQ_E_ALIGN;
  const Span o[] = {mat(out, ldo, t, n, elem(out_dtype))};
  const Span in[] = {mat(xq, ldx, t, k, 1), {xscale, t * 4}, mat(wq, ldw, n, k, 1), {wscale, n * 4ull}, {bias, n * 4ull}};
  if (clash(o, in)) return STQ_E_ALIAS;
  stq::GemmArgs a = {};
  a.xq = xq; a.ldx = ldx; a.xs = xscale;
  a.wq = wq; a.ldw = ldw; a.ws = wscale;
  a.bias = bias;
  a.out = out; a.ldo = ldo; a.out_dtype = out_dtype;
  a.t = t; a.n = n; a.k = k;
  a.device = h->device;
  STQ_CUDA(h, cudaSetDevice(h->device));
  STQ_CUDA(h, stq::launch_q8_linear(a, h->sm_count, h->d_err, static_cast<cudaStream_t>(stream)));
  h->launches++;
  return STQ_OK;
}

int stq_q8_linear_dx(stq_handle* h, const void* dy, uint64_t lddy, const int8_t* wq, uint64_t ldw, const float* wscale,
                     uint64_t t, uint32_t n, uint32_t k, void* dx, uint64_t lddx, int out_dtype, void* stream) {
  STQ_TRY(check_handle(h));
  STQ_TRY(check_dtype(out_dtype));
  STQ_TRY(check_size(t, n));
  STQ_TRY(check_size(t, k));
  if (t == 0) return STQ_OK;
  STQ_TRY(check_mat(dy, lddy, n, 2));
  STQ_TRY(check_codes(wq, ldw, k, wscale));
  STQ_TRY(check_mat(dx, lddx, k, elem(out_dtype)));
  const Span o[] = {mat(dx, lddx, t, k, elem(out_dtype))};
  const Span in[] = {mat(dy, lddy, t, n, 2), mat(wq, ldw, n, k, 1), {wscale, n * 4ull}};
  if (clash(o, in)) return STQ_E_ALIAS;
  stq::GemmArgs a = {};
  a.dy = dy; a.lddy = lddy;
  a.wq = wq; a.ldw = ldw; a.ws = wscale;
  a.out = dx; a.ldo = lddx; a.out_dtype = out_dtype;
  a.t = t; a.n = n; a.k = k;
  a.device = h->device;
  STQ_CUDA(h, cudaSetDevice(h->device));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  uint8_t* ws = nullptr;
  int launches = 0;
  if (const size_t need = stq::q8_grad_workspace(a, false, h->sm_count)) STQ_TRY(workspace(h, need, s, &ws));
  STQ_CUDA(h, stq::launch_q8_linear_dx(a, ws, h->sm_count, h->d_err, s, &launches));
  h->launches += launches;
  return STQ_OK;
}

int stq_q8_linear_dw(stq_handle* h, const void* dy, uint64_t lddy, const int8_t* xq, uint64_t ldx, const float* xscale,
                     uint64_t t, uint32_t n, uint32_t k, void* dw, uint64_t lddw, int out_dtype, void* stream) {
  STQ_TRY(check_handle(h));
  STQ_TRY(check_dtype(out_dtype));
  STQ_TRY(check_size(t, n));
  STQ_TRY(check_size(t, k));
  STQ_TRY(check_mat(dw, lddw, k, elem(out_dtype)));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  STQ_CUDA(h, cudaSetDevice(h->device));
  if (t == 0) return zero(h, dw, lddw, n, k, elem(out_dtype), s);
  STQ_TRY(check_mat(dy, lddy, n, 2));
  STQ_TRY(check_codes(xq, ldx, k, xscale));
  const Span o[] = {mat(dw, lddw, n, k, elem(out_dtype))};
  const Span in[] = {mat(dy, lddy, t, n, 2), mat(xq, ldx, t, k, 1), {xscale, t * 4}};
  if (clash(o, in)) return STQ_E_ALIAS;
  stq::GemmArgs a = {};
  a.dy = dy; a.lddy = lddy;
  a.xq = xq; a.ldx = ldx; a.xs = xscale;
  a.out = dw; a.ldo = lddw; a.out_dtype = out_dtype;
  a.t = t; a.n = n; a.k = k;
  a.device = h->device;
  uint8_t* ws = nullptr;
  int launches = 0;
  if (const size_t need = stq::q8_grad_workspace(a, true, h->sm_count)) STQ_TRY(workspace(h, need, s, &ws));
  STQ_CUDA(h, stq::launch_q8_linear_dw(a, ws, h->sm_count, h->d_err, s, &launches));
  h->launches += launches;
  return STQ_OK;
}

int stq_q8_bias_grad(stq_handle* h, const void* dy, uint64_t lddy, int dtype, uint64_t t, uint32_t n, float* db,
                     void* stream) {
  STQ_TRY(check_handle(h));
  if (!db) return STQ_E_NULL;
  STQ_TRY(check_dtype(dtype));
  STQ_TRY(check_size(t, n));
  if (!aligned(db, 4)) return STQ_E_ALIGN;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  STQ_CUDA(h, cudaSetDevice(h->device));
  if (t == 0) return zero(h, db, n, 1, n, 4, s);
  STQ_TRY(check_mat(dy, lddy, n, elem(dtype)));
  const Span o[] = {{db, n * 4ull}}, in[] = {mat(dy, lddy, t, n, elem(dtype))};
  if (clash(o, in)) return STQ_E_ALIAS;
  const uint32_t splits = stq::q8_colsum_splits(t, n, h->sm_count);
  float* partial = nullptr;
  if (const size_t need = stq::q8_colsum_partial(n, splits)) STQ_TRY(workspace(h, need, s, &partial));
  STQ_CUDA(h, stq::launch_q8_colsum(dtype, {const_cast<void*>(dy), lddy}, t, n, splits, partial, h->d_q8_counters, db, s));
  h->launches++;
  return STQ_OK;
}

}  // extern "C"
