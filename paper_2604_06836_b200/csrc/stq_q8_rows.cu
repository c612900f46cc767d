// Row kernels of the 8-bit operators: quantising rows, the norm with the residual's addition, the activations
// with their 8-bit checkpoints, and the backward passes of both.  All of them are bound by memory: every kernel
// reads its inputs once, keeps a row in registers while the row's maximum and sum are formed, and writes each
// result once.
//
// A row is cut into units of 256 columns; a unit belongs to one warp, 8 columns to a lane.  With VEC = 8 these
// are 8 neighbours (one 16-byte load of bf16); with VEC = 2 or 1 (odd widths and pitches) a lane takes every
// 32nd pair or single, so that a warp's loads stay contiguous.  In all three the first 128 columns of a unit and
// the last 128 can be told apart by lane or by register, which is what a checkpoint's block of 128 needs.
#include <cuda_bf16.h>

#include <type_traits>

#include "../../include/stq.h"
#include "stq_internal.h"
#include "stq_q8.h"

namespace stq {
namespace {

constexpr uint32_t kFullMask = 0xffffffffu;
constexpr float kTinyScale = 7.8886090522101181e-31f;   // 2^-100: rows and blocks below it are stored as zeros
constexpr uint32_t kUnit = 256;

// column of element e (0..7) of `lane` in the unit that begins at `base`
template <int VEC>
__device__ __forceinline__ uint32_t col_of(uint32_t base, int lane, int e) {
  if (VEC == 8) return base + lane * 8 + e;
  return base + (e / VEC) * 32 * VEC + lane * VEC + e % VEC;
}

__device__ __forceinline__ void unpack2(uint32_t w, float& lo, float& hi) {
  lo = __uint_as_float(w << 16);
  hi = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// the 8 elements of a lane in one unit of a row; columns from `cols` on read as zero and are not touched
template <class T, int VEC>
__device__ __forceinline__ void load_unit(const T* row, uint32_t base, int lane, uint32_t cols, float (&v)[8]) {
  if constexpr (VEC == 8) {
    const uint32_t c = base + lane * 8;
    if (c < cols) {
      if constexpr (sizeof(T) == 2) {
        const uint4 w = *reinterpret_cast<const uint4*>(row + c);
        unpack2(w.x, v[0], v[1]); unpack2(w.y, v[2], v[3]); unpack2(w.z, v[4], v[5]); unpack2(w.w, v[6], v[7]);
      } else {
        const float4 a = *reinterpret_cast<const float4*>(row + c), b = *reinterpret_cast<const float4*>(row + c + 4);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 0.f;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; e += VEC) {
      const uint32_t c = col_of<VEC>(base, lane, e);
      if (c < cols) {
        if constexpr (VEC == 2) {
          if constexpr (sizeof(T) == 2) {
            unpack2(*reinterpret_cast<const uint32_t*>(row + c), v[e], v[e + 1]);
          } else {
            const float2 a = *reinterpret_cast<const float2*>(row + c);
            v[e] = a.x; v[e + 1] = a.y;
          }
        } else {
          v[e] = static_cast<float>(row[c]);
        }
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) v[e + i] = 0.f;
      }
    }
  }
}

template <class T, int VEC>
__device__ __forceinline__ void store_unit(T* row, uint32_t base, int lane, uint32_t cols, const float (&v)[8]) {
  if constexpr (VEC == 8) {
    const uint32_t c = base + lane * 8;
    if (c >= cols) return;
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<uint4*>(row + c) = make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
    } else {
      *reinterpret_cast<float4*>(row + c) = make_float4(v[0], v[1], v[2], v[3]);
      *reinterpret_cast<float4*>(row + c + 4) = make_float4(v[4], v[5], v[6], v[7]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; e += VEC) {
      const uint32_t c = col_of<VEC>(base, lane, e);
      if (c >= cols) continue;
      if constexpr (VEC == 2) {
        if constexpr (sizeof(T) == 2)
          *reinterpret_cast<uint32_t*>(row + c) = pack2(v[e], v[e + 1]);
        else
          *reinterpret_cast<float2*>(row + c) = make_float2(v[e], v[e + 1]);
      } else {
        row[c] = static_cast<T>(v[e]);
      }
    }
  }
}

// the codes of a lane's 8 elements, each the low byte of a word
template <int VEC>
__device__ __forceinline__ void store_codes(int8_t* row, uint32_t base, int lane, uint32_t cols, const uint32_t (&k)[8]) {
  if constexpr (VEC == 8) {
    const uint32_t c = base + lane * 8;
    if (c >= cols) return;
    uint2 w;
    w.x = __byte_perm(__byte_perm(k[0], k[1], 0x0040), __byte_perm(k[2], k[3], 0x0040), 0x5410);
    w.y = __byte_perm(__byte_perm(k[4], k[5], 0x0040), __byte_perm(k[6], k[7], 0x0040), 0x5410);
    *reinterpret_cast<uint2*>(row + c) = w;
  } else {
#pragma unroll
    for (int e = 0; e < 8; e += VEC) {
      const uint32_t c = col_of<VEC>(base, lane, e);
      if (c >= cols) continue;
      if constexpr (VEC == 2)
        *reinterpret_cast<uint16_t*>(row + c) = (uint16_t)__byte_perm(k[e], k[e + 1], 0x0040);
      else
        row[c] = (int8_t)k[e];
    }
  }
}

// the 8 codes of a lane as numbers
template <int VEC>
__device__ __forceinline__ void load_codes(const int8_t* row, uint32_t base, int lane, uint32_t cols, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = 0.f;
  if constexpr (VEC == 8) {
    const uint32_t c = base + lane * 8;
    if (c >= cols) return;
    const uint2 w = *reinterpret_cast<const uint2*>(row + c);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)(int8_t)((e < 4 ? w.x : w.y) >> (8 * (e & 3)));
  } else {
#pragma unroll
    for (int e = 0; e < 8; e += VEC) {
      const uint32_t c = col_of<VEC>(base, lane, e);
      if (c >= cols) continue;
      if constexpr (VEC == 2) {
        const uint16_t w = *reinterpret_cast<const uint16_t*>(row + c);
        v[e] = (float)(int8_t)w;
        v[e + 1] = (float)(int8_t)(w >> 8);
      } else {
        v[e] = (float)row[c];
      }
    }
  }
}

// Largest magnitudes travel as the bit patterns of |x|: they order like the numbers, infinity is above every
// number and NaN above infinity, so one unsigned maximum also finds what must not be stored as a code.
__device__ __forceinline__ uint32_t mag(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// How a row or block with largest magnitude `top` is coded: q = rne(x * inv) & mask, value q * scale.  (inv is
// formed like that of the first moment's codes: 127 * fl(1/top).)
struct Coding {
  float inv, scale;
  uint32_t mask;
};
__device__ __forceinline__ Coding coding_of(uint32_t top) {
  const float a = __uint_as_float(top);
  Coding c;
  c.mask = 0xffffffffu;
  c.inv = 127.f * (1.f / a);
  c.scale = a / 127.f;
  if (a < kTinyScale) { c.inv = 0.f; c.scale = 0.f; }
  // something in the row is not finite: no code can say so, the scale does
  if (top >= 0x7f800000u) { c.inv = 0.f; c.scale = __uint_as_float(0x7fc00000u); c.mask = 0u; }
  return c;
}
// Round to nearest even by the addition of 1.5 * 2^23: the low byte of the sum is the two's complement code
// (|x * inv| <= 127 up to a rounding).
__device__ __forceinline__ uint32_t code_of(float x, const Coding& c) {
  return __float_as_uint(__fadd_rn(__fmul_rn(x, c.inv), 12582912.f)) & c.mask;
}
__device__ __forceinline__ float value_of(uint32_t code, const Coding& c) { return (float)(int8_t)code * c.scale; }

__device__ __forceinline__ float sigmoid(float x) { return __fdividef(1.f, 1.f + __expf(-x)); }
constexpr float kGeluA = 1.5957691216057308f;             // 2 sqrt(2/pi): gelu(x) = x sigmoid(kGeluA (x + 0.044715 x^3))
constexpr float kGeluB = 0.044715f;

// ---- activation (or plain rows) -> 8-bit rows, and the input into a checkpoint ----------------------------------
// One row per CTA of `warps` warps, or, with one warp per row, four rows per CTA.  A lane keeps NS units' results
// in registers between the row's maximum and the writing; rows of more than NS * warps units are read a second
// time (the checkpoint is written in the first pass).
template <class T, int VEC, int NS, int KIND>
__global__ void __launch_bounds__(1024) q8_act_kernel(const RowArgs a, int warps) {
  __shared__ uint32_t sh[32];
  const int lane = threadIdx.x & 31;
  const int warp = warps == 1 ? 0 : threadIdx.x >> 5;
  const uint64_t row = warps == 1 ? (uint64_t)blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x;
  if (warps == 1 && row >= a.rows) return;
  const uint32_t cols = a.cols, step = kUnit * warps;
  const T* x = static_cast<const T*>(a.x.p) + row * a.x.ld;
  constexpr int kParts = KIND == kQ8SiluGated ? 2 : 1;
  const uint32_t blocks = (cols + kQ8Block - 1) / kQ8Block;

  // NS units from `base` on: the results, and on the first pass the checkpoint of what they came from
  auto produce = [&](uint32_t base, float (&r)[NS][8], bool keep) {
    float in[kParts][NS][8];
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int p = 0; p < kParts; ++p) load_unit<T, VEC>(x + (size_t)p * cols, base + s * step, lane, cols, in[p][s]);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float g = in[0][s][e];
        if constexpr (KIND == kQ8Copy) r[s][e] = g;
        if constexpr (KIND == kQ8SiluGated) r[s][e] = g * sigmoid(g) * in[1][s][e];
        if constexpr (KIND == kQ8Gelu) r[s][e] = g * sigmoid(kGeluA * (g + kGeluB * g * g * g));
      }
      if (KIND != kQ8Copy && keep) {
        const uint32_t b = base + s * step;
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
          // VEC 8: lanes 0-15 and 16-31 hold a block each; otherwise registers 0-3 and 4-7 do
          uint32_t t0 = 0, t1 = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            t0 = max(t0, mag(in[p][s][e]));
            t1 = max(t1, mag(in[p][s][e + 4]));
          }
          if constexpr (VEC == 8) {
            t0 = max(t0, t1);
#pragma unroll
            for (int m = 8; m; m >>= 1) t0 = max(t0, __shfl_xor_sync(kFullMask, t0, m));
            t1 = t0;
          } else {
            t0 = __reduce_max_sync(kFullMask, t0);
            t1 = __reduce_max_sync(kFullMask, t1);
          }
          const Coding c0 = coding_of(t0), c1 = VEC == 8 ? c0 : coding_of(t1);
          uint32_t k[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) k[e] = code_of(in[p][s][e], e < 4 ? c0 : c1);
          const size_t at = row * kParts + p;
          store_codes<VEC>(a.ckq + at * a.ldck, b, lane, cols, k);
          const uint32_t blk = b / kQ8Block;
          if constexpr (VEC == 8) {
            if ((lane & 15) == 0 && blk + (lane >> 4) < blocks) a.cks[at * blocks + blk + (lane >> 4)] = c0.scale;
          } else {
            if (lane == 0 && blk < blocks) a.cks[at * blocks + blk] = c0.scale;
            if (lane == 1 && blk + 1 < blocks) a.cks[at * blocks + blk + 1] = c1.scale;
          }
        }
      }
    }
  };

  float r[NS][8];
  uint32_t top = 0;
  const uint32_t first = warp * kUnit, span = step * NS;
  const bool once = cols <= span;
  for (uint32_t at = 0; at < cols; at += span) {
    produce(at + first, r, a.ckq != nullptr);
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, mag(r[s][e]));
  }
  top = __reduce_max_sync(kFullMask, top);
  if (warps > 1) {
    if (lane == 0) sh[warp] = top;
    __syncthreads();
    top = __reduce_max_sync(kFullMask, lane < warps ? sh[lane] : 0u);
  }
  const Coding c = coding_of(top);
  if (warp == 0 && lane == 0) a.scale[row] = c.scale;
  for (uint32_t at = 0; at < cols; at += span) {
    if (!once) produce(at + first, r, false);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const uint32_t b = at + first + s * step;
      uint32_t k[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) k[e] = code_of(r[s][e], c);
      store_codes<VEC>(a.q + row * a.ldq, b, lane, cols, k);
      if (a.values.p) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = value_of(k[e], c);
        store_unit<__nv_bfloat16, VEC>(static_cast<__nv_bfloat16*>(a.values.p) + row * a.values.ld, b, lane, cols, v);
      }
    }
  }
}

// ---- residual + root-mean-square norm -> 8-bit rows --------------------------------------------------------------
// y = h * rstd * w with one rstd per row, so the codes of y are the codes of h * w (rstd cancels in x / max|x|) and
// the row needs ONE reduction for both the sum of squares and the maximum.
template <class T, int VEC, int NS>
__global__ void __launch_bounds__(1024) q8_norm_kernel(const RowArgs a, int warps) {
  __shared__ uint32_t sh_top[32];
  __shared__ float sh_sum[32];
  const int lane = threadIdx.x & 31;
  const int warp = warps == 1 ? 0 : threadIdx.x >> 5;
  const uint64_t row = warps == 1 ? (uint64_t)blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x;
  if (warps == 1 && row >= a.rows) return;
  const uint32_t cols = a.cols, step = kUnit * warps;
  const T* x = static_cast<const T*>(a.x.p) + row * a.x.ld;
  const T* res = a.res.p ? static_cast<const T*>(a.res.p) + row * a.res.ld : nullptr;

  // h * w of NS units; on the first pass h is written and its squares are added to `sum`
  auto produce = [&](uint32_t base, float (&r)[NS][8], float& sum, bool keep) {
    float w[NS][8];
#pragma unroll
    for (int s = 0; s < NS; ++s) load_unit<T, VEC>(x, base + s * step, lane, cols, r[s]);
    if (res) {
      float o[NS][8];
#pragma unroll
      for (int s = 0; s < NS; ++s) load_unit<T, VEC>(res, base + s * step, lane, cols, o[s]);
#pragma unroll
      for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int e = 0; e < 8; ++e) r[s][e] += o[s][e];
    }
#pragma unroll
    for (int s = 0; s < NS; ++s) load_unit<float, VEC>(a.weight, base + s * step, lane, cols, w[s]);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      if (keep && res)
        store_unit<T, VEC>(static_cast<T*>(a.h.p) + row * a.h.ld, base + s * step, lane, cols, r[s]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        sum = fmaf(r[s][e], r[s][e], sum);
        r[s][e] *= w[s][e];
      }
    }
  };

  float r[NS][8], sum = 0.f, unused = 0.f;
  uint32_t top = 0;
  const uint32_t first = warp * kUnit, span = step * NS;
  const bool once = cols <= span;
  for (uint32_t at = 0; at < cols; at += span) {
    produce(at + first, r, sum, true);
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) top = max(top, mag(r[s][e]));
  }
  top = __reduce_max_sync(kFullMask, top);
#pragma unroll
  for (int m = 16; m; m >>= 1) sum += __shfl_xor_sync(kFullMask, sum, m);
  if (warps > 1) {
    if (lane == 0) { sh_top[warp] = top; sh_sum[warp] = sum; }
    __syncthreads();
    top = __reduce_max_sync(kFullMask, lane < warps ? sh_top[lane] : 0u);
    sum = lane < warps ? sh_sum[lane] : 0.f;
#pragma unroll
    for (int m = 16; m; m >>= 1) sum += __shfl_xor_sync(kFullMask, sum, m);
  }
  const float rstd = 1.f / sqrtf(sum / (float)cols + a.eps);
  Coding c = coding_of(top);
  c.scale *= rstd;                                       // the scale of y; c.inv codes h * w
  if (!(__uint_as_float(top) * rstd >= kTinyScale) && c.mask) { c.inv = 0.f; c.scale = 0.f; }
  if (rstd != rstd) { c.mask = 0u; c.scale = rstd; }
  if (warp == 0 && lane == 0) {
    a.scale[row] = c.scale;
    a.rstd[row] = rstd;
  }
  for (uint32_t at = 0; at < cols; at += span) {
    if (!once) produce(at + first, r, unused, false);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const uint32_t b = at + first + s * step;
      uint32_t k[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) k[e] = code_of(r[s][e], c);
      store_codes<VEC>(a.q + row * a.ldq, b, lane, cols, k);
      if (a.values.p) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = value_of(k[e], c);
        store_unit<__nv_bfloat16, VEC>(static_cast<__nv_bfloat16*>(a.values.p) + row * a.values.ld, b, lane, cols, v);
      }
    }
  }
}

// ---- backward of the norm -----------------------------------------------------------------------------------------
// dx = rstd (w dy - xh mean(w dy xh)) + dres with xh = h rstd; dweight = sum over rows of dy xh.  A group of `warps`
// warps walks rows group, group + groups, ...; a lane's columns stay the same, so its share of dweight stays in
// registers until the end.  The groups' shares are added in a fixed order by q8_colsum_finish_kernel.
template <class T, int VEC, int NS>
__global__ void __launch_bounds__(1024) q8_norm_bwd_kernel(const NormBwdArgs a, int warps, uint32_t groups) {
  __shared__ float sh[2][32];
  const int lane = threadIdx.x & 31;
  const int warp = warps == 1 ? 0 : threadIdx.x >> 5;
  const uint32_t group = warps == 1 ? blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x;
  if (group >= groups) return;
  const uint32_t cols = a.cols, step = kUnit * warps, first = warp * kUnit;
  float w[NS][8], dw[NS][8];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    load_unit<float, VEC>(a.weight, first + s * step, lane, cols, w[s]);
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[s][e] = 0.f;
  }
  const float inv_n = 1.f / (float)cols;
  int flip = 0;
  for (uint64_t row = group; row < a.rows; row += groups, flip ^= 1) {
    const T* dy = static_cast<const T*>(a.dy.p) + row * a.dy.ld;
    const T* h = static_cast<const T*>(a.h.p) + row * a.h.ld;
    const float rstd = a.rstd[row];
    float g[NS][8], xh[NS][8], o[NS][8], dot = 0.f;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      load_unit<T, VEC>(dy, first + s * step, lane, cols, g[s]);
      load_unit<T, VEC>(h, first + s * step, lane, cols, xh[s]);
      if (a.dres.p)
        load_unit<T, VEC>(static_cast<const T*>(a.dres.p) + row * a.dres.ld, first + s * step, lane, cols, o[s]);
    }
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        xh[s][e] *= rstd;
        dw[s][e] = fmaf(g[s][e], xh[s][e], dw[s][e]);
        g[s][e] *= w[s][e];
        dot = fmaf(g[s][e], xh[s][e], dot);
      }
#pragma unroll
    for (int m = 16; m; m >>= 1) dot += __shfl_xor_sync(kFullMask, dot, m);
    if (warps > 1) {   // two buffers: a warp reaches the next row's store only after all have passed this row's barrier
      if (lane == 0) sh[flip][warp] = dot;
      __syncthreads();
      dot = lane < warps ? sh[flip][lane] : 0.f;
#pragma unroll
      for (int m = 16; m; m >>= 1) dot += __shfl_xor_sync(kFullMask, dot, m);
    }
    const float c = dot * inv_n;
    T* dx = static_cast<T*>(a.dx.p) + row * a.dx.ld;
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] = rstd * fmaf(-xh[s][e], c, g[s][e]);
        if (a.dres.p) v[e] += o[s][e];
      }
      store_unit<T, VEC>(dx, first + s * step, lane, cols, v);
    }
  }
#pragma unroll
  for (int s = 0; s < NS; ++s)
    store_unit<float, VEC>(a.partial + (size_t)group * cols, first + s * step, lane, cols, dw[s]);
}

// The same for rows that do not fit in registers: a row is read twice (the second time from L2) and the sums of
// dweight lie in shared memory, each column touched by one lane only.
template <class T, int VEC>
__global__ void __launch_bounds__(1024) q8_norm_bwd_wide_kernel(const NormBwdArgs a, uint32_t groups) {
  extern __shared__ float dwsum[];
  __shared__ float sh[2][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const uint32_t cols = a.cols, step = kUnit * warps;
  for (uint32_t c = threadIdx.x; c < cols; c += blockDim.x) dwsum[c] = 0.f;
  __syncthreads();
  int flip = 0;
  for (uint64_t row = blockIdx.x; row < a.rows; row += groups, flip ^= 1) {
    const T* dy = static_cast<const T*>(a.dy.p) + row * a.dy.ld;
    const T* h = static_cast<const T*>(a.h.p) + row * a.h.ld;
    const float rstd = a.rstd[row];
    float dot = 0.f;
    for (uint32_t b = warp * kUnit; b < cols; b += step) {
      float g[8], xh[8], w[8];
      load_unit<T, VEC>(dy, b, lane, cols, g);
      load_unit<T, VEC>(h, b, lane, cols, xh);
      load_unit<float, VEC>(a.weight, b, lane, cols, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t c = col_of<VEC>(b, lane, e);
        const float p = g[e] * (xh[e] * rstd);
        if (c < cols) dwsum[c] += p;
        dot = fmaf(p, w[e], dot);
      }
    }
#pragma unroll
    for (int m = 16; m; m >>= 1) dot += __shfl_xor_sync(kFullMask, dot, m);
    if (lane == 0) sh[flip][warp] = dot;
    __syncthreads();
    dot = lane < warps ? sh[flip][lane] : 0.f;
#pragma unroll
    for (int m = 16; m; m >>= 1) dot += __shfl_xor_sync(kFullMask, dot, m);
    const float c = dot / (float)cols;
    T* dx = static_cast<T*>(a.dx.p) + row * a.dx.ld;
    for (uint32_t b = warp * kUnit; b < cols; b += step) {
      float g[8], xh[8], w[8], o[8], v[8];
      load_unit<T, VEC>(dy, b, lane, cols, g);
      load_unit<T, VEC>(h, b, lane, cols, xh);
      load_unit<float, VEC>(a.weight, b, lane, cols, w);
      if (a.dres.p) load_unit<T, VEC>(static_cast<const T*>(a.dres.p) + row * a.dres.ld, b, lane, cols, o);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] = rstd * fmaf(-(xh[e] * rstd), c, g[e] * w[e]);
        if (a.dres.p) v[e] += o[e];
      }
      store_unit<T, VEC>(dx, b, lane, cols, v);
    }
  }
  __syncthreads();
  for (uint32_t c = threadIdx.x; c < cols; c += blockDim.x) a.partial[(size_t)blockIdx.x * cols + c] = dwsum[c];
}

// ---- column sums ---------------------------------------------------------------------------------------------------
// partial[split][c] = sum over the split's rows; 8 warps share the rows of a split, 256 columns to a CTA.
template <class T, int VEC>
__global__ void __launch_bounds__(256) q8_colsum_kernel(Mat x, uint64_t rows, uint32_t cols, uint32_t splits, float* partial) {
  __shared__ float sh[8][kUnit];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t base = blockIdx.x * kUnit, split = blockIdx.y;
  const uint64_t per = (rows + splits - 1) / splits, r0 = split * per, r1 = min(r0 + per, rows);
  float s[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (uint64_t r = r0 + warp; r < r1; r += 8) {
    float v[8];
    load_unit<T, VEC>(static_cast<const T*>(x.p) + r * x.ld, base, lane, cols, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] += v[e];
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) sh[warp][col_of<VEC>(0, lane, e)] = s[e];
  __syncthreads();
  const uint32_t c = base + threadIdx.x;
  float sum = 0.f;
#pragma unroll
  for (int w = 0; w < 8; ++w) sum += sh[w][threadIdx.x];
  if (c < cols) partial[(size_t)split * cols + c] = sum;
}

// out[c] = sum of partial[g][c] over g, in a fixed order: 32 columns to a CTA, 32 shares of the groups added up
// in shared memory.
__global__ void __launch_bounds__(1024) q8_colsum_finish_kernel(const float* partial, uint32_t groups, uint32_t cols, float* out) {
  __shared__ float sh[32][33];
  const uint32_t c = blockIdx.x * 32 + threadIdx.x;
  float s = 0.f;
  if (c < cols) {
#pragma unroll 4
    for (uint32_t g = threadIdx.y; g < groups; g += 32) s += partial[(size_t)g * cols + c];
  }
  sh[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  s = sh[threadIdx.x][threadIdx.y];     // warp y adds the 32 shares of column y
#pragma unroll
  for (int m = 16; m; m >>= 1) s += __shfl_xor_sync(kFullMask, s, m);
  if (threadIdx.x == 0 && blockIdx.x * 32 + threadIdx.y < cols) out[blockIdx.x * 32 + threadIdx.y] = s;
}

// ---- backward of the activations, from the checkpoint -------------------------------------------------------------
// One warp per unit of a row: 8-bit codes, their scales and da in, dz out.
template <class T, int VEC, int KIND>
__global__ void __launch_bounds__(256) q8_act_bwd_kernel(const ActBwdArgs a, uint32_t units, uint64_t total) {
  const int lane = threadIdx.x & 31;
  const uint64_t id = (uint64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (id >= total) return;
  const uint64_t row = id / units;
  const uint32_t base = (uint32_t)(id - row * units) * kUnit, cols = a.cols, blk = base / kQ8Block;
  const uint32_t blocks = (cols + kQ8Block - 1) / kQ8Block;
  constexpr int kParts = KIND == kQ8SiluGated ? 2 : 1;
  float da[8], in[kParts][8];
  load_unit<T, VEC>(static_cast<const T*>(a.da.p) + row * a.da.ld, base, lane, cols, da);
#pragma unroll
  for (int p = 0; p < kParts; ++p) {
    const size_t at = row * kParts + p;
    load_codes<VEC>(a.ckq + at * a.ldck, base, lane, cols, in[p]);
    const float* sc = a.cks + at * blocks + blk;
    const float s0 = sc[0], s1 = blk + 1 < blocks ? sc[1] : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) in[p][e] *= (VEC == 8 ? lane < 16 : e < 4) ? s0 : s1;
  }
  float d0[8], d1[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float g = in[0][e];
    if constexpr (KIND == kQ8SiluGated) {
      const float sg = sigmoid(g);
      d0[e] = da[e] * in[kParts - 1][e] * (sg * fmaf(g, 1.f - sg, 1.f));
      d1[e] = da[e] * (g * sg);
    } else {
      const float g2 = g * g;
      const float sg = sigmoid(kGeluA * fmaf(kGeluB * g2, g, g));
      d0[e] = da[e] * sg * fmaf(g * (1.f - sg), kGeluA * fmaf(3.f * kGeluB, g2, 1.f), 1.f);
    }
  }
  T* dz = static_cast<T*>(a.dz.p) + row * a.dz.ld;
  store_unit<T, VEC>(dz, base, lane, cols, d0);
  if constexpr (kParts == 2) store_unit<T, VEC>(dz + cols, base, lane, cols, d1);
}

// ---- launches ------------------------------------------------------------------------------------------------------
// Widest access that every row of every matrix allows: 8 elements (16 bytes of bf16), 2, or 1.
struct Width {
  uint64_t bits = 0;
  void add(const Mat& m, size_t elem) {
    if (!m.p) return;
    const uint64_t p = reinterpret_cast<uint64_t>(m.p);
    // a pointer on 16 bytes allows 8 elements, one on two elements allows 2
    bits |= m.ld | ((p & 15) == 0 ? 0 : (p & (2 * elem - 1)) == 0 ? 2 : 1);
  }
  int vec(uint32_t cols) const {
    const uint64_t b = bits | cols;
    return (b & 7) == 0 ? 8 : (b & 1) == 0 ? 2 : 1;
  }
};

// Warps per row and units per warp of the row kernels (rows of more than 64 units are read twice).
struct Shape {
  int warps, ns;
};
Shape shape_of(uint32_t cols) {
  const uint32_t units = (cols + kUnit - 1) / kUnit;
  const int ns = units <= 32 ? 1 : 2;
  const uint32_t w = (units + ns - 1) / ns;
  return {(int)(w < 32 ? w : 32), ns};
}

template <class F>
cudaError_t by_ns(int ns, F f) {
  if (ns == 1) return f(std::integral_constant<int, 1>());
  return f(std::integral_constant<int, 2>());
}
template <class F>
cudaError_t by_vec(int vec, F f) {
  if (vec == 8) return f(std::integral_constant<int, 8>());
  if (vec == 2) return f(std::integral_constant<int, 2>());
  return f(std::integral_constant<int, 1>());
}
template <class F>
cudaError_t by_type(int dtype, F f) {
  if (dtype == STQ_GRAD_F32) return f(0.f);
  return f(__nv_bfloat16());
}

size_t elem_bytes(int dtype) { return dtype == STQ_GRAD_F32 ? 4 : 2; }

}  // namespace

cudaError_t launch_q8_act(int dtype, Q8Kind kind, const RowArgs& a, cudaStream_t stream) {
  Width w;
  w.add(a.x, elem_bytes(dtype));
  w.add(a.values, 2);
  const Shape sh = shape_of(a.cols);
  const unsigned grid = (unsigned)(sh.warps == 1 ? (a.rows + 3) / 4 : a.rows);
  const int threads = sh.warps == 1 ? 128 : sh.warps * 32;
  return by_type(dtype, [&](auto tv) {
    using T = decltype(tv);
    return by_vec(w.vec(a.cols), [&](auto vec) {
      return by_ns(sh.ns, [&](auto ns) {
        if (kind == kQ8Copy) q8_act_kernel<T, vec(), ns(), kQ8Copy><<<grid, threads, 0, stream>>>(a, sh.warps);
        if (kind == kQ8SiluGated) q8_act_kernel<T, vec(), ns(), kQ8SiluGated><<<grid, threads, 0, stream>>>(a, sh.warps);
        if (kind == kQ8Gelu) q8_act_kernel<T, vec(), ns(), kQ8Gelu><<<grid, threads, 0, stream>>>(a, sh.warps);
        return cudaGetLastError();
      });
    });
  });
}

cudaError_t launch_q8_norm(int dtype, const RowArgs& a, cudaStream_t stream) {
  Width w;
  w.add(a.x, elem_bytes(dtype));
  w.add(a.res, elem_bytes(dtype));
  if (a.res.p) w.add(a.h, elem_bytes(dtype));
  w.add(a.values, 2);
  w.add(Mat{const_cast<float*>(a.weight), 0}, 4);
  const Shape sh = shape_of(a.cols);
  const unsigned grid = (unsigned)(sh.warps == 1 ? (a.rows + 3) / 4 : a.rows);
  const int threads = sh.warps == 1 ? 128 : sh.warps * 32;
  return by_type(dtype, [&](auto tv) {
    using T = decltype(tv);
    return by_vec(w.vec(a.cols), [&](auto vec) {
      return by_ns(sh.ns, [&](auto ns) {
        q8_norm_kernel<T, vec(), ns()><<<grid, threads, 0, stream>>>(a, sh.warps);
        return cudaGetLastError();
      });
    });
  });
}

namespace {
constexpr uint32_t kBwdRegCols = 32 * 2 * kUnit;   // widest row whose sums stay in registers (32 warps, 2 units each)
Shape bwd_shape(uint32_t cols) {
  const uint32_t units = (cols + kUnit - 1) / kUnit;
  const int ns = units <= 8 ? 1 : 2;
  return {(int)((units + ns - 1) / ns), ns};
}
}  // namespace

uint32_t q8_norm_bwd_groups(uint64_t rows, uint32_t cols, int sms) {
  uint32_t most;
  if (cols > kBwdRegCols) {
    most = sms;
  } else {
    const Shape sh = bwd_shape(cols);
    most = (uint32_t)sms * (sh.warps >= 32 ? 1 : 32 / sh.warps);
  }
  return (uint32_t)(rows < most ? rows : most);
}

cudaError_t launch_q8_norm_bwd(int dtype, const NormBwdArgs& a, uint32_t groups, cudaStream_t stream) {
  Width w;
  w.add(a.dy, elem_bytes(dtype));
  w.add(a.h, elem_bytes(dtype));
  w.add(a.dres, elem_bytes(dtype));
  w.add(a.dx, elem_bytes(dtype));
  w.add(Mat{const_cast<float*>(a.weight), 0}, 4);
  cudaError_t e = by_type(dtype, [&](auto tv) {
    using T = decltype(tv);
    return by_vec(w.vec(a.cols), [&](auto vec) {
      if (a.cols > kBwdRegCols) {
        const int bytes = (int)(a.cols * sizeof(float));
        cudaError_t e2 = cudaFuncSetAttribute(q8_norm_bwd_wide_kernel<T, vec()>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e2 != cudaSuccess) return e2;
        q8_norm_bwd_wide_kernel<T, vec()><<<groups, 1024, bytes, stream>>>(a, groups);
        return cudaGetLastError();
      }
      const Shape sh = bwd_shape(a.cols);
      const unsigned grid = sh.warps == 1 ? (groups + 3) / 4 : groups;
      const int threads = sh.warps == 1 ? 128 : sh.warps * 32;
      if (sh.ns == 1)
        q8_norm_bwd_kernel<T, vec(), 1><<<grid, threads, 0, stream>>>(a, sh.warps, groups);
      else
        q8_norm_bwd_kernel<T, vec(), 2><<<grid, threads, 0, stream>>>(a, sh.warps, groups);
      return cudaGetLastError();
    });
  });
  if (e != cudaSuccess) return e;
  q8_colsum_finish_kernel<<<(a.cols + 31) / 32, dim3(32, 32), 0, stream>>>(a.partial, groups, a.cols, a.dweight);
  return cudaGetLastError();
}

uint32_t q8_colsum_splits(uint64_t rows, uint32_t cols, int sms) {
  // about four CTAs of 8 warps per SM, at least 32 rows to a split
  const uint32_t tiles = (cols + kUnit - 1) / kUnit, want = (uint32_t)(4 * sms + tiles - 1) / tiles;
  const uint64_t most = (rows + 31) / 32;
  return (uint32_t)(want < most ? want : most);
}

cudaError_t launch_q8_colsum(int dtype, Mat x, uint64_t rows, uint32_t cols, uint32_t splits, float* partial, float* out,
                             cudaStream_t stream) {
  Width w;
  w.add(x, elem_bytes(dtype));
  const dim3 grid((cols + kUnit - 1) / kUnit, splits);
  float* to = splits == 1 ? out : partial;
  cudaError_t e = by_type(dtype, [&](auto tv) {
    using T = decltype(tv);
    return by_vec(w.vec(cols), [&](auto vec) {
      q8_colsum_kernel<T, vec()><<<grid, 256, 0, stream>>>(x, rows, cols, splits, to);
      return cudaGetLastError();
    });
  });
  if (e != cudaSuccess || splits == 1) return e;
  q8_colsum_finish_kernel<<<(cols + 31) / 32, dim3(32, 32), 0, stream>>>(partial, splits, cols, out);
  return cudaGetLastError();
}

cudaError_t launch_q8_act_bwd(int dtype, Q8Kind kind, const ActBwdArgs& a, cudaStream_t stream) {
  Width w;
  w.add(a.da, elem_bytes(dtype));
  w.add(a.dz, elem_bytes(dtype));
  const uint32_t units = (a.cols + kUnit - 1) / kUnit;
  const uint64_t total = a.rows * units;
  const unsigned grid = (unsigned)((total + 7) / 8);
  return by_type(dtype, [&](auto tv) {
    using T = decltype(tv);
    return by_vec(w.vec(a.cols), [&](auto vec) {
      if (kind == kQ8SiluGated)
        q8_act_bwd_kernel<T, vec(), kQ8SiluGated><<<grid, 256, 0, stream>>>(a, units, total);
      else
        q8_act_bwd_kernel<T, vec(), kQ8Gelu><<<grid, 256, 0, stream>>>(a, units, total);
      return cudaGetLastError();
    });
  });
}

}  // namespace stq
