// The 2-norm of all gradients together and the factor that clips them, and gradients times that factor.
//   norm = inv * sqrt(sum over all tensors of g^2),  factor = inv * min(1, max_norm / (norm + eps)),  out = g * factor
// with inv = 1 / loss scale (or 1).  Norm and factor stay on the device: the optimizer's step takes the factor from there.
//
// One launch serves up to kMost tensors; their addresses and lengths are launch parameters, so nothing is uploaded, nothing is kept
// between calls, and a captured graph holds what it needs.
//
// Bound by memory: the norm reads every gradient once, 256 threads with eight 16-byte loads in flight each, four CTAs to an SM.
// A thread squares up to 64 numbers in fp32 and adds that to a double; where the fp32 sum may have left fp32's range (or have
// lost small squares) it is formed again in double from the registers, so that the norm is right for all finite gradients.
// The sums of CTAs are added in a fixed order by the CTA that comes last: the same result from run to run.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include <algorithm>
#include <type_traits>
#include <vector>

#include "stq_checks.h"
#include "stq_q8_tma.h"

namespace stq {
namespace {

constexpr int kThreads = 256, kPerSm = 4;
constexpr int kNormPieces = 8, kScalePieces = 4;      // 16-byte pieces that a thread has in flight
constexpr int kMost = 1024;                           // tensors to a launch (28 KB of launch parameters)

// Tensors as 16-byte pieces of memory: the first and the last may be partly outside.
template <int N, bool OUT>
struct List {
  uint64_t in[N], out[OUT ? N : 1];
  uint64_t numel[N];      // types of in and out above bit 56
  uint32_t first[N];      // number of the tensor's first chunk
  uint32_t n, chunks;
};

__device__ __forceinline__ uint32_t elem_log(uint32_t dtype) { return dtype == STQ_GRAD_F32 ? 2 : 1; }

// What chunk c is: the tensor, and its pieces from `piece` on.  `first`: the list's, in parameters or in shared memory.
struct Chunk {
  uint64_t in, out, numel;
  uint32_t type, out_type;
  uint64_t piece;
  bool whole;             // no piece of it reaches outside the tensor
};
template <int N, bool OUT>
__device__ __forceinline__ Chunk chunk_of(const List<N, OUT>& l, const uint32_t* first, uint32_t c, uint32_t per_chunk) {
  uint32_t lo = 0, hi = l.n;
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) / 2;
    if (first[mid] <= c) lo = mid; else hi = mid;
  }
  const uint64_t w = l.numel[lo], n = w & ((1ull << 56) - 1), at = l.in[lo], piece = (uint64_t)(c - first[lo]) * per_chunk;
  const uint32_t type = (uint32_t)(w >> 56) & 3;
  const bool whole = (piece > 0 || (at & 15) == 0) && 16 * (piece + per_chunk) <= (at & 15) + (n << elem_log(type));
  return {at, l.out[OUT ? lo : 0], n, type, (uint32_t)(w >> 58) & 3, piece, whole};
}

// Piece q of a tensor: numbers [from, from + 16 / size) of it, some of them outside at its ends.
__device__ __forceinline__ bool piece_at(const Chunk& c, uint64_t q, int64_t& from, uint64_t& at) {
  at = (c.in & ~15ull) + 16 * q;
  from = ((int64_t)at - (int64_t)c.in) >> elem_log(c.type);
  return from < (int64_t)c.numel;
}
__device__ __forceinline__ uint4 load_piece(const Chunk& c, int64_t from, uint64_t at) {
  const int per = 16 >> elem_log(c.type);
  if (from >= 0 && from + per <= (int64_t)c.numel) return __ldcs(reinterpret_cast<const uint4*>(at));
  uint32_t w[4] = {0, 0, 0, 0};      // numbers outside read as zero
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (i >= per || from + i < 0 || from + i >= (int64_t)c.numel) continue;
    if (c.type == STQ_GRAD_F32)
      w[i & 3] = reinterpret_cast<const uint32_t*>(at)[i];
    else
      w[i / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(at)[i] << (16 * (i & 1));
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// Number i of a piece (a constant after unrolling).
template <int TYPE>
__device__ __forceinline__ float number(const uint4& v, int i) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  if constexpr (TYPE == STQ_GRAD_F32) return __uint_as_float(w[i]);
  const uint32_t x = w[i / 2];
  if constexpr (TYPE == STQ_GRAD_BF16) return __uint_as_float(i & 1 ? x & 0xffff0000u : x << 16);
  return __half2float(__ushort_as_half((unsigned short)(i & 1 ? x >> 16 : x & 0xffffu)));
}

template <int TYPE>
__device__ __forceinline__ double squares(const uint4 (&v)[kNormPieces]) {
  constexpr int kPer = TYPE == STQ_GRAD_F32 ? 4 : 8;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int p = 0; p < kNormPieces; ++p)
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const float g = number<TYPE>(v[p], i);
      s[i & 3] = __fmaf_rn(g, g, s[i & 3]);
    }
  const float sum = (s[0] + s[1]) + (s[2] + s[3]);
  if (sum > 1e-20f && sum < 1e37f) return (double)sum;      // what underflowed next to 1e-20 does not count
  if (sum == 0.f) {
    uint32_t any = 0;
#pragma unroll
    for (int p = 0; p < kNormPieces; ++p) any |= v[p].x | v[p].y | v[p].z | v[p].w;
    if (any == 0) return 0.0;
  }
  double d = 0.0;
#pragma unroll 1
  for (int p = 0; p < kNormPieces; ++p) {
    uint4 w = v[0];
#pragma unroll
    for (int q = 1; q < kNormPieces; ++q) w = q == p ? v[q] : w;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const double g = (double)number<TYPE>(w, i);
      d = fma(g, g, d);
    }
  }
  return d;
}

// Sum over the CTA (in every thread of its first warp).
__device__ __forceinline__ double cta_sum(double v, double* shared) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) shared[threadIdx.x >> 5] = v;
  __syncthreads();
  v = threadIdx.x < kThreads / 32 ? shared[threadIdx.x] : 0.0;
  if (threadIdx.x < 32)
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

struct NormOut {
  double* part;            // a sum per CTA, of earlier launches of the call too
  uint32_t at, total;      // of this launch's first CTA, and of all
  uint32_t* counter;       // zero between launches
  int last;                // this launch finishes
  const float* inv;
  float max_norm, eps;
  float *norm, *factor, *found_inf;
};

template <int N>
__global__ void __launch_bounds__(kThreads, kPerSm) norm_kernel(const __grid_constant__ List<N, false> l, const NormOut o) {
  __shared__ double shared[kThreads / 32];
  __shared__ bool is_last;
  __shared__ uint32_t first[N];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  // (ten steps of a search, each of which waits for the one before: not in the parameters' cache, which the list is too long for, and
  // while the numbers are on their way; 580 tensors, 3.1 GB: 515 -> 458 us)
  for (uint32_t i = threadIdx.x; i < l.n; i += kThreads) first[i] = l.first[i];
  __syncthreads();
  double sum = 0.0;
  uint32_t c = blockIdx.x;
  Chunk k;
  if (c < l.chunks) k = chunk_of(l, first, c, kThreads * kNormPieces);
  while (c < l.chunks) {
    uint4 v[kNormPieces];
    if (k.whole) {
      const uint4* p = reinterpret_cast<const uint4*>((k.in & ~15ull) + 16 * k.piece) + threadIdx.x;
#pragma unroll
      for (int i = 0; i < kNormPieces; ++i) v[i] = __ldcs(p + i * kThreads);
    } else {
#pragma unroll
      for (int p = 0; p < kNormPieces; ++p) {
        int64_t from;
        uint64_t at;
        v[p] = make_uint4(0, 0, 0, 0);
        if (piece_at(k, k.piece + p * kThreads + threadIdx.x, from, at)) v[p] = load_piece(k, from, at);
      }
    }
    const uint32_t type = k.type;
    c += gridDim.x;
    if (c < l.chunks) k = chunk_of(l, first, c, kThreads * kNormPieces);
    sum += type == STQ_GRAD_F32 ? squares<STQ_GRAD_F32>(v) : type == STQ_GRAD_BF16 ? squares<STQ_GRAD_BF16>(v) : squares<STQ_GRAD_F16>(v);
  }
  sum = cta_sum(sum, shared);
  if (threadIdx.x == 0) {
    o.part[o.at + blockIdx.x] = sum;
    __threadfence();
    is_last = o.last && atomicAdd(o.counter, 1u) == gridDim.x - 1;
  }
  __syncthreads();
  if (!is_last) return;
  __threadfence();
  sum = 0.0;
  for (uint32_t i = threadIdx.x; i < o.total; i += kThreads) sum += __ldcg(o.part + i);
  __syncthreads();
  sum = cta_sum(sum, shared);
  if (threadIdx.x == 0) {
    *o.counter = 0;
    const float inv = o.inv ? *o.inv : 1.f, norm = (float)(sqrt(sum) * (double)inv);
    float f = 1.f;
    if (o.max_norm < INFINITY) {
      f = __fdiv_rn(o.max_norm, __fadd_rn(norm, o.eps));
      f = f > 1.f ? 1.f : f;      // (NaN stays)
    }
    *o.norm = norm;
    *o.factor = __fmul_rn(f, inv);
    if (o.found_inf && !(fabsf(norm) < INFINITY)) *o.found_inf = 1.f;
  }
}

template <int TYPE, int OUT>
__device__ __forceinline__ void scale_piece(const Chunk& c, int64_t from, const uint4& v, float f) {
  constexpr int kPer = TYPE == STQ_GRAD_F32 ? 4 : 8, kSize = OUT == STQ_GRAD_F32 ? 4 : 2;
  float x[kPer];
#pragma unroll
  for (int i = 0; i < kPer; ++i) x[i] = __fmul_rn(number<TYPE>(v, i), f);
  const uint64_t to = c.out + from * kSize;
  if (from >= 0 && from + kPer <= (int64_t)c.numel && (to & 15) == 0) {
    if constexpr (OUT == STQ_GRAD_F32 && kPer == 8) {      // (32 bytes at once: halves of sectors cost as much as whole ones)
      if ((to & 31) == 0) {
        asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(to), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]),
                     "f"(x[5]), "f"(x[6]), "f"(x[7])
                     : "memory");
        return;
      }
    }
    if constexpr (OUT == STQ_GRAD_F32) {
#pragma unroll
      for (int i = 0; i < kPer; i += 4)
        __stcs(reinterpret_cast<float4*>(to + 4 * i), make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]));
    } else {
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (OUT == STQ_GRAD_BF16) {
          const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
          w[i] = *reinterpret_cast<const uint32_t*>(&h);
        } else {
          const __half2 h = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
          w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
      }
      __stcs(reinterpret_cast<uint4*>(to), make_uint4(w[0], w[1], w[2], w[3]));
    }
    return;
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    if (from + i < 0 || from + i >= (int64_t)c.numel) continue;
    if constexpr (OUT == STQ_GRAD_F32) reinterpret_cast<float*>(to)[i] = x[i];
    else if constexpr (OUT == STQ_GRAD_BF16) reinterpret_cast<__nv_bfloat16*>(to)[i] = __float2bfloat16_rn(x[i]);
    else reinterpret_cast<__half*>(to)[i] = __float2half_rn(x[i]);
  }
}

template <int TYPE, int OUT>
__device__ __forceinline__ void scale_chunk(const Chunk& k, const uint4 (&v)[kScalePieces], float f) {
#pragma unroll
  for (int p = 0; p < kScalePieces; ++p) {
    int64_t from;
    uint64_t at;
    if (piece_at(k, k.piece + p * kThreads + threadIdx.x, from, at)) scale_piece<TYPE, OUT>(k, from, v[p], f);
  }
}

// From the last chunk to the first: what the norm read last is still in the cache.  A CTA to each chunk: CTAs that stay and walk
// through the chunks, as above, took longer (774 M fp32: 1525 instead of 1355 us with the norm), since loads and stores of a CTA
// then wait for one another.
template <int N>
__global__ void __launch_bounds__(kThreads) scale_kernel(const __grid_constant__ List<N, true> l, const float* factor, int in_place) {
  const Chunk k = chunk_of(l, l.first, l.chunks - 1 - blockIdx.x, kThreads * kScalePieces);
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const float f = *factor;
  if (in_place && f == 1.f) return;      // (nothing would change)
  uint4 v[kScalePieces];
  if (k.whole) {
    const uint4* p = reinterpret_cast<const uint4*>((k.in & ~15ull) + 16 * k.piece) + threadIdx.x;
#pragma unroll
    for (int i = 0; i < kScalePieces; ++i) v[i] = __ldcs(p + i * kThreads);
  } else {
#pragma unroll
    for (int p = 0; p < kScalePieces; ++p) {
      int64_t from;
      uint64_t at;
      if (piece_at(k, k.piece + p * kThreads + threadIdx.x, from, at)) v[p] = load_piece(k, from, at);
    }
  }
  if (k.type == STQ_GRAD_F32) scale_chunk<STQ_GRAD_F32, STQ_GRAD_F32>(k, v, f);
  else if (k.type == STQ_GRAD_BF16 && k.out_type == STQ_GRAD_BF16) scale_chunk<STQ_GRAD_BF16, STQ_GRAD_BF16>(k, v, f);
  else if (k.type == STQ_GRAD_BF16) scale_chunk<STQ_GRAD_BF16, STQ_GRAD_F32>(k, v, f);
  else if (k.out_type == STQ_GRAD_F16) scale_chunk<STQ_GRAD_F16, STQ_GRAD_F16>(k, v, f);
  else scale_chunk<STQ_GRAD_F16, STQ_GRAD_F32>(k, v, f);
}

size_t size_of(int dtype) { return dtype == STQ_GRAD_F32 ? 4 : 2; }

// Tensors [at, at + N) or what is left of them, in chunks of `pieces` pieces; `at` moves on.
template <int N, bool OUT>
List<N, OUT> list_of(const stq_grad* g, int n, int& at, uint32_t pieces) {
  List<N, OUT> l;
  l.n = l.chunks = 0;
  for (; at < n && l.n < N; ++at) {
    if (g[at].numel == 0) continue;
    const uint64_t p = reinterpret_cast<uintptr_t>(g[at].grad), bytes = (p & 15) + g[at].numel * size_of(g[at].dtype);
    const uint64_t chunks = (bytes + 16ull * pieces - 1) / (16ull * pieces);
    if (l.chunks + chunks > 0x7fffffffull) break;
    l.in[l.n] = p;
    if (OUT) l.out[l.n] = reinterpret_cast<uintptr_t>(g[at].out);
    l.numel[l.n] = g[at].numel | (uint64_t)g[at].dtype << 56 | (uint64_t)g[at].out_dtype << 58;
    l.first[l.n++] = l.chunks;
    l.chunks += (uint32_t)chunks;
  }
  return l;
}

// scalars: what the call writes next to the results, 4 bytes each (or null)
int check_list(const stq_grad* g, int n, bool write, const float* const (&scalars)[3], bool* in_place) try {
  if (n < 0) return STQ_E_ARG;
  if (n > 0 && !g) return STQ_E_NULL;
  *in_place = true;
  std::vector<std::pair<uintptr_t, uintptr_t>> written;
  std::vector<std::pair<uintptr_t, uintptr_t>> read;
  if (write) {
    written.reserve(n);
    read.reserve(n);
  }
  for (int i = 0; i < n; ++i) {
    const int dt = g[i].dtype;
    if (dt != STQ_GRAD_F32 && dt != STQ_GRAD_BF16 && dt != STQ_GRAD_F16) return STQ_E_ARG;
    if (write && g[i].out_dtype != dt && g[i].out_dtype != STQ_GRAD_F32) return STQ_E_ARG;
    if (g[i].numel == 0) continue;
    if (g[i].numel >> 40) return STQ_E_TOO_LARGE;
    if (!g[i].grad || (write && !g[i].out)) return STQ_E_NULL;
    if (!aligned(g[i].grad, size_of(dt)) || (write && !aligned(g[i].out, size_of(g[i].out_dtype)))) return STQ_E_ALIGN;
    if (!write) continue;
    const uintptr_t a = reinterpret_cast<uintptr_t>(g[i].grad), b = reinterpret_cast<uintptr_t>(g[i].out);
    written.push_back({b, b + g[i].numel * size_of(g[i].out_dtype)});
    if (a != b || dt != g[i].out_dtype) {
      *in_place = false;
      read.push_back({a, a + g[i].numel * size_of(dt)});
    }
  }
  // a result may lie where its own gradient does, and nowhere else that is read or written
  if (!std::is_sorted(written.begin(), written.end())) std::sort(written.begin(), written.end());
  for (size_t i = 1; i < written.size(); ++i)
    if (written[i].first < written[i - 1].second) return STQ_E_ALIAS;
  for (const auto& r : read) {
    if (r.second <= written.front().first || r.first >= written.back().second) continue;
    const auto w = std::lower_bound(written.begin(), written.end(), std::make_pair(r.second, (uintptr_t)0));
    if (w != written.begin() && (w - 1)->second > r.first) return STQ_E_ALIAS;
  }
  // nor may a scalar lie where a result or another scalar does, or in a gradient that is read again after it has been written
  for (int i = 0; i < 3; ++i) {
    const uintptr_t s = reinterpret_cast<uintptr_t>(scalars[i]);
    if (!s) continue;
    for (int j = 0; j < i; ++j)
      if (scalars[j] == scalars[i]) return STQ_E_ALIAS;
    const auto w = std::lower_bound(written.begin(), written.end(), std::make_pair(s + 4, (uintptr_t)0));
    if (w != written.begin() && (w - 1)->second > s) return STQ_E_ALIAS;
    for (const auto& r : read)
      if (r.first < s + 4 && s < r.second) return STQ_E_ALIAS;
  }
  return STQ_OK;
} catch (const std::bad_alloc&) {
  return STQ_E_WORKSPACE;
}

int check_scalars(const float* inv, float max_norm, float eps, const float* norm, const float* factor, const float* found_inf) {
  if (!norm || !factor) return STQ_E_NULL;
  if (!(max_norm > 0.f) || !(eps >= 0.f) || !(eps < INFINITY)) return STQ_E_ARG;
  return aligned(inv, 4) && aligned(norm, 4) && aligned(factor, 4) && aligned(found_inf, 4) ? STQ_OK : STQ_E_ALIGN;
}

template <int N>
cudaError_t launch_norm(const stq_grad* g, int n, NormOut o, int sms, cudaStream_t s, int* launches) {
  int at = 0;
  do {
    const List<N, false> l = list_of<N, false>(g, n, at, kThreads * kNormPieces);
    const uint32_t most = sms * kPerSm, grid = l.chunks < 1 ? 1 : l.chunks < most ? l.chunks : most;
    o.last = at >= n;
    o.total = o.at + grid;
    const cudaError_t e = launch_with(norm_kernel<N>, dim3(grid), dim3(kThreads), 0, 1, true, s, l, o);
    if (e != cudaSuccess) return e;
    o.at += grid;
    ++*launches;
  } while (at < n);
  return cudaSuccess;
}

template <int N>
cudaError_t launch_scale(const stq_grad* g, int n, const float* factor, bool in_place, cudaStream_t s, int* launches) {
  for (int at = 0; at < n;) {
    const List<N, true> l = list_of<N, true>(g, n, at, kThreads * kScalePieces);
    if (l.chunks == 0) continue;
    const cudaError_t e = launch_with(scale_kernel<N>, dim3(l.chunks), dim3(kThreads), 0, 1, true, s, l, factor, (int)in_place);
    if (e != cudaSuccess) return e;
    ++*launches;
  }
  return cudaSuccess;
}

// A call's sums, one to each CTA of each launch.  (A launch ends early only where its chunks run out, after 2^31 of them.)
size_t sums_of(const stq_grad* g, int n, int sms) {
  uint64_t bytes = 0;
  for (int i = 0; i < n; ++i) bytes += g[i].numel * size_of(g[i].dtype);
  return (size_t)(n / kMost + 2 + (bytes >> 45)) * sms * kPerSm;
}

// The launch parameters that a list needs: passing them costs about a microsecond a KB, before the kernel starts.
template <class F>
cudaError_t by_length(int n, F&& f) {
  if (n <= 64) return f(std::integral_constant<int, 64>());
  if (n <= 160) return f(std::integral_constant<int, 160>());
  if (n <= 256) return f(std::integral_constant<int, 256>());
  if (n <= 384) return f(std::integral_constant<int, 384>());
  if (n <= 512) return f(std::integral_constant<int, 512>());
  if (n <= 640) return f(std::integral_constant<int, 640>());
  return f(std::integral_constant<int, kMost>());
}

int norm_of(stq_handle* h, const stq_grad* g, int n, const float* inv, float max_norm, float eps, float* norm, float* factor, float* found_inf,
            cudaStream_t s) {
  NormOut o = {};
  STQ_TRY(workspace(h, sums_of(g, n, h->sm_count), s, &o.part));
  o.counter = h->d_q8_counters;
  o.inv = inv;
  o.max_norm = max_norm;
  o.eps = eps;
  o.norm = norm;
  o.factor = factor;
  o.found_inf = found_inf;
  int launches = 0;
  STQ_CUDA(h, by_length(n, [&](auto most) { return launch_norm<most.value>(g, n, o, h->sm_count, s, &launches); }));
  h->launches += launches;
  return STQ_OK;
}

}  // namespace
}  // namespace stq

using namespace stq;

extern "C" {

int stq_grad_norm(stq_handle* h, const stq_grad* grads, int n, const float* inv_scale, float max_norm, float eps, float* norm, float* factor,
                  float* found_inf, void* stream) {
  STQ_TRY(check_handle(h));
  bool in_place;
  STQ_TRY(check_list(grads, n, false, {norm, factor, found_inf}, &in_place));
  STQ_TRY(check_scalars(inv_scale, max_norm, eps, norm, factor, found_inf));
  STQ_CUDA(h, cudaSetDevice(h->device));
  return norm_of(h, grads, n, inv_scale, max_norm, eps, norm, factor, found_inf, static_cast<cudaStream_t>(stream));
}

int stq_grad_clip(stq_handle* h, const stq_grad* grads, int n, const float* inv_scale, float max_norm, float eps, float* norm, float* factor,
                  float* found_inf, void* stream) {
  STQ_TRY(check_handle(h));
  bool in_place;
  STQ_TRY(check_list(grads, n, true, {norm, factor, found_inf}, &in_place));
  STQ_TRY(check_scalars(inv_scale, max_norm, eps, norm, factor, found_inf));
  STQ_CUDA(h, cudaSetDevice(h->device));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  STQ_TRY(norm_of(h, grads, n, inv_scale, max_norm, eps, norm, factor, found_inf, s));
  int launches = 0;
  STQ_CUDA(h, by_length(n, [&](auto most) { return launch_scale<most.value>(grads, n, factor, in_place, s, &launches); }));
  h->launches += launches;
  return STQ_OK;
}

}  // extern "C"
