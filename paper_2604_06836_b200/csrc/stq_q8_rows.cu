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

#include <atomic>
#include <type_traits>

#include "../../include/stq.h"
#include "stq_internal.h"
#include "stq_q8.h"
#include "stq_q8_tma.h"

namespace stq {
namespace {

constexpr uint32_t kFullMask = 0xffffffffu;
constexpr float kTinyScale = 7.8886090522101181e-31f;   // 2^-100: rows and blocks below it are stored as zeros
constexpr float kTinyProduct = 7.5231638452626401e-37f; // 2^-120: the least h * w that the norm codes
constexpr uint32_t kUnit = 256;

// column of element e (0..7) of `lane` in the unit that begins at `base`
template <int VEC>
__device__ __forceinline__ uint32_t col_of(uint32_t base, int lane, int e) {
  if (VEC == 8) return base + lane * 8 + e;
  return base + (e / VEC) * 32 * VEC + lane * VEC + e % VEC;
}

__device__ __forceinline__ uint32_t pack2(float2 x) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(x.x, x.y);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// Pairs of fp32 operations in one instruction.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("mul.rn.f32x2 %0, %1, %2;"
      : "=l"(*reinterpret_cast<uint64_t*>(&r))
      : "l"(*reinterpret_cast<const uint64_t*>(&a)), "l"(*reinterpret_cast<const uint64_t*>(&b)));
  return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(*reinterpret_cast<uint64_t*>(&r))
      : "l"(*reinterpret_cast<const uint64_t*>(&a)), "l"(*reinterpret_cast<const uint64_t*>(&b)));
  return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(*reinterpret_cast<uint64_t*>(&r))
      : "l"(*reinterpret_cast<const uint64_t*>(&a)), "l"(*reinterpret_cast<const uint64_t*>(&b)),
        "l"(*reinterpret_cast<const uint64_t*>(&c)));
  return r;
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// The 8 elements of a lane in one unit of a row as they lie in memory, so that the loads of many units can be in flight
// in few registers; columns from `cols` on read as zero and are not touched.
template <class T, int VEC>
struct Raw {
  static constexpr int kWords = VEC == 1 ? 8 : 2 * (int)sizeof(T);   // (single elements take a register each)
  uint32_t w[kWords];
  // ONCE: nothing reads this again, so it may leave the caches first (the norm's backward pass on 8192 x 1600: 23.8 -> 20.8
  // us; the norm and the activations are no faster for it)
  template <bool ONCE = false>
  __device__ __forceinline__ void load(const T* row, uint32_t base, int lane, uint32_t cols) {
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = 0u;
    if constexpr (VEC == 8) {
      const uint32_t c = base + lane * 8;
      if (c < cols) {
#pragma unroll
        for (int i = 0; i < kWords; i += 4) {
          const uint4* at = reinterpret_cast<const uint4*>(row + c) + i / 4;
          const uint4 v = ONCE ? __ldcs(at) : *at;
          w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
        }
      }
    } else if (base + kUnit <= cols) {       // a whole unit: loads at fixed distances, nothing to ask
      const T* from = row + base + lane * VEC;
#pragma unroll
      for (int i = 0; i < 8 / VEC; ++i) one(from + i * 32 * VEC, i);
    } else {
#pragma unroll
      for (int i = 0; i < 8 / VEC; ++i)
        if (base + i * 32 * VEC + lane * VEC < cols) one(row + base + i * 32 * VEC + lane * VEC, i);
    }
  }
  __device__ __forceinline__ void one(const T* from, int i) {      // access i of VEC = 2 or 1
    if constexpr (VEC == 2 && sizeof(T) == 2) {
      w[i] = *reinterpret_cast<const uint32_t*>(from);
    } else if constexpr (VEC == 2) {
      const uint2 v = *reinterpret_cast<const uint2*>(from);
      w[2 * i] = v.x; w[2 * i + 1] = v.y;
    } else if constexpr (VEC == 1) {
      w[i] = sizeof(T) == 2 ? (uint32_t)*reinterpret_cast<const uint16_t*>(from) << 16 : *reinterpret_cast<const uint32_t*>(from);
    }
  }
  __device__ __forceinline__ float2 pair(int p) const {      // elements 2p, 2p + 1
    if constexpr (sizeof(T) == 2 && VEC != 1) return make_float2(__uint_as_float(w[p] << 16), __uint_as_float(w[p] & 0xffff0000u));
    return make_float2(__uint_as_float(w[2 * p % kWords]), __uint_as_float(w[(2 * p + 1) % kWords]));
  }
};

template <class T, int VEC>
__device__ __forceinline__ void load_unit(const T* row, uint32_t base, int lane, uint32_t cols, float2 (&v)[4]) {
  Raw<T, VEC> r;
  r.load(row, base, lane, cols);
#pragma unroll
  for (int p = 0; p < 4; ++p) v[p] = r.pair(p);
}

template <class T, int VEC, bool ONCE = false>
__device__ __forceinline__ void store_unit(T* row, uint32_t base, int lane, uint32_t cols, const float2 (&v)[4]) {
  if constexpr (VEC == 8) {
    const uint32_t c = base + lane * 8;
    if (c >= cols) return;
    if constexpr (sizeof(T) == 2) {
      const uint4 w = make_uint4(pack2(v[0]), pack2(v[1]), pack2(v[2]), pack2(v[3]));
      if constexpr (ONCE)
        __stcs(reinterpret_cast<uint4*>(row + c), w);
      else
        *reinterpret_cast<uint4*>(row + c) = w;
    } else {
      *reinterpret_cast<float4*>(row + c) = make_float4(v[0].x, v[0].y, v[1].x, v[1].y);
      *reinterpret_cast<float4*>(row + c + 4) = make_float4(v[2].x, v[2].y, v[3].x, v[3].y);
    }
  } else {
    T* to = row + base + lane * VEC;
    auto one = [&](int i) {
      T* at = to + i * 32 * VEC;
      if constexpr (VEC == 2 && sizeof(T) == 2)
        *reinterpret_cast<uint32_t*>(at) = pack2(v[i % 4]);
      else if constexpr (VEC == 2)
        *reinterpret_cast<float2*>(at) = v[i % 4];
      else
        *at = static_cast<T>(i & 1 ? v[i / 2].y : v[i / 2].x);
    };
    if (base + kUnit <= cols) {
#pragma unroll
      for (int i = 0; i < 8 / VEC; ++i) one(i);
    } else {
#pragma unroll
      for (int i = 0; i < 8 / VEC; ++i)
        if (base + i * 32 * VEC + lane * VEC < cols) one(i);
    }
  }
}

// the codes of a lane's 8 elements, four to a word
template <int VEC>
__device__ __forceinline__ void store_codes(int8_t* row, uint32_t base, int lane, uint32_t cols, const uint32_t (&k)[2]) {
  if constexpr (VEC == 8) {
    const uint32_t c = base + lane * 8;
    if (c < cols) *reinterpret_cast<uint2*>(row + c) = make_uint2(k[0], k[1]);
  } else {
    int8_t* to = row + base + lane * VEC;
    auto one = [&](int i) {
      const uint32_t w = k[i * VEC / 4] >> (8 * (i * VEC & 3));
      if constexpr (VEC == 2)
        *reinterpret_cast<uint16_t*>(to + i * 64) = (uint16_t)w;
      else
        to[i * 32] = (int8_t)w;
    };
    if (base + kUnit <= cols) {
#pragma unroll
      for (int i = 0; i < 8 / VEC; ++i) one(i);
    } else {
#pragma unroll
      for (int i = 0; i < 8 / VEC; ++i)
        if (base + i * 32 * VEC + lane * VEC < cols) one(i);
    }
  }
}

// the codes of a lane's 8 elements, four to a word, 128 added to each
template <int VEC>
__device__ __forceinline__ void load_codes(const int8_t* row, uint32_t base, int lane, uint32_t cols, uint32_t (&k)[2]) {
  k[0] = k[1] = 0u;
  if constexpr (VEC == 8) {
    const uint32_t c = base + lane * 8;
    if (c < cols) {
      const uint2 w = *reinterpret_cast<const uint2*>(row + c);
      k[0] = w.x; k[1] = w.y;
    }
  } else {
    const int8_t* from = row + base + lane * VEC;
    auto one = [&](int i) {
      const uint32_t w = VEC == 2 ? (uint32_t)*reinterpret_cast<const uint16_t*>(from + i * 64) : (uint32_t)(uint8_t)from[i * 32];
      k[i * VEC / 4] |= w << (8 * (i * VEC & 3));
    };
    if (base + kUnit <= cols) {
#pragma unroll
      for (int i = 0; i < 8 / VEC; ++i) one(i);
    } else {
#pragma unroll
      for (int i = 0; i < 8 / VEC; ++i)
        if (base + i * 32 * VEC + lane * VEC < cols) one(i);
    }
  }
  k[0] ^= 0x80808080u;
  k[1] ^= 0x80808080u;
}
// elements 2p, 2p + 1 of such codes as numbers: a byte under the exponent of 2^23 is 2^23 + byte
__device__ __forceinline__ float2 code_pair(const uint32_t (&k)[2], int p) {
  const uint32_t w = k[p / 2];
  const int i = (p & 1) * 2;
  return add2(make_float2(__uint_as_float(__byte_perm(w, 0x4b000000u, 0x7650 + i)),
                          __uint_as_float(__byte_perm(w, 0x4b000000u, 0x7651 + i))),
              both(-8388736.f));
}

// Largest magnitudes travel as the bit patterns of |x|: they order like the numbers, infinity is above every
// number and NaN above infinity, so one unsigned maximum also finds what must not be stored as a code.
__device__ __forceinline__ float max_abs(float m, float2 x) {      // max(m, |x.x|, |x.y|), NaN if one is
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(m), "f"(x.x), "f"(x.y));
  return r;
}
__device__ __forceinline__ uint32_t bits_of(float m) { return __float_as_uint(m) & 0x7fffffffu; }

// How a row or block with largest magnitude `top` is coded: q = rne(x * inv) & mask, value q * scale.  (inv is
// formed like that of the first moment's codes: 127 * fl(1/top).)
struct Coding {
  float inv, scale;
  uint32_t mask;
};
__device__ __forceinline__ Coding coding_of(uint32_t top, float tiny = kTinyScale) {
  const float a = __uint_as_float(top);
  Coding c;
  c.mask = 0xffffffffu;
  c.inv = 127.f * (1.f / a);
  c.scale = a * (1.f / 127.f);
  if (a < tiny) { c.inv = 0.f; c.scale = 0.f; }
  // something in the row is not finite: no code can say so, the scale does
  if (top >= 0x7f800000u) { c.inv = 0.f; c.scale = __uint_as_float(0x7fc00000u); c.mask = 0u; }
  return c;
}
// Round to nearest even by the addition of 1.5 * 2^23: the low byte of the sum is the two's complement code
// (|x * inv| <= 127 up to a rounding), and the sum less 1.5 * 2^23 is the code as a number.
// The product is rounded before the addition: single multiplications, since a packed pair of the two is contracted to a
// fused one by the assembler (codes then differ where the exact product lies next to a tie).
constexpr float kRound = 12582912.f;
__device__ __forceinline__ float2 rounded(float2 x, float inv) {
  return add2(make_float2(__fmul_rn(x.x, inv), __fmul_rn(x.y, inv)), both(kRound));
}
__device__ __forceinline__ uint32_t codes4(float2 a, float2 b, uint32_t mask) {
  return __byte_perm(__byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x0040),
                     __byte_perm(__float_as_uint(b.x), __float_as_uint(b.y), 0x0040), 0x5410) & mask;
}
// A unit of a row as codes and, if asked for, as the bf16 values that these stand for.
template <int VEC>
__device__ __forceinline__ void write_unit(const RowArgs& a, uint64_t row, uint32_t base, int lane, const float2 (&x)[4],
                                           const Coding& c) {
  float2 t[4];
#pragma unroll
  for (int p = 0; p < 4; ++p) t[p] = rounded(x[p], c.inv);
  const uint32_t k[2] = {codes4(t[0], t[1], c.mask), codes4(t[2], t[3], c.mask)};
  store_codes<VEC>(a.q + row * a.ldq, base, lane, a.cols, k);
  if (a.values.p) {
#pragma unroll
    for (int p = 0; p < 4; ++p) t[p] = mul2(add2(t[p], both(-kRound)), both(c.scale));
    store_unit<__nv_bfloat16, VEC>(static_cast<__nv_bfloat16*>(a.values.p) + row * a.values.ld, base, lane, a.cols, t);
  }
}

// 1 / (1 + exp(-x)): the special-function unit's exponential and reciprocal, 2^-22 each, and the rounding of the exponential's
// argument, |x| 2^-24 of the result where that is small; an exponential that overflows gives 0.
__device__ __forceinline__ float2 sigmoid2(float2 x) {
  float2 t = mul2(x, both(-1.4426950408889634f)), r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(t.x) : "f"(t.x));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(t.y) : "f"(t.y));
  t = add2(t, both(1.f));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(t.x));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(t.y));
  return r;
}
// x held to [-most, most], NaN kept
__device__ __forceinline__ float2 held(float2 x, float most) {
  asm("min.NaN.f32 %0, %0, %1;" : "+f"(x.x) : "f"(most));
  asm("min.NaN.f32 %0, %0, %1;" : "+f"(x.y) : "f"(most));
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(x.x) : "f"(-most));
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(x.y) : "f"(-most));
  return x;
}
constexpr float kGeluA = 1.5957691216057308f;             // 2 sqrt(2/pi): gelu(x) = x sigmoid(kGeluA (x + 0.044715 x^3))
constexpr float kGeluB = 0.044715f;

// Most warps that share a row, by the units that each of them keeps.
__host__ __device__ constexpr int most_warps(int ns) { return ns == 1 ? 32 : 16; }

// ---- activation (or plain rows) -> 8-bit rows, and the input into a checkpoint ----------------------------------
// One row per CTA of `warps` warps, or, with one warp per row, four rows per CTA.  A lane keeps NS units' results
// in registers between the row's maximum and the writing; rows of more than NS * warps units are read a second
// time (the checkpoint is written in the first pass).
template <class T, int VEC, int NS, int KIND>
__global__ void __launch_bounds__(most_warps(NS) * 32) q8_act_kernel(const RowArgs a, int warps) {
  __shared__ uint32_t sh[32];
  const int lane = threadIdx.x & 31;
  const int warp = warps == 1 ? 0 : threadIdx.x >> 5;
  const uint64_t row = warps == 1 ? (uint64_t)blockIdx.x * 4 + (threadIdx.x >> 5) : blockIdx.x;
  if (warps == 1 && row >= a.rows) return;
  const uint32_t cols = a.cols, step = kUnit * warps;
  const T* x = static_cast<const T*>(a.x.p) + row * a.x.ld;
  constexpr int kParts = KIND == kQ8SiluGated ? 2 : 1;
  const uint32_t blocks = (cols + kQ8Block - 1) / kQ8Block;
  int8_t* ckq = a.ckq + row * kParts * a.ldck;
  float* cks = a.cks + row * kParts * blocks;

  // NS units from `base` on: the results, and on the first pass the checkpoint of what they came from
  auto produce = [&](uint32_t base, float2 (&r)[NS][4], bool keep) {
    Raw<T, VEC> raw[NS][kParts];
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int p = 0; p < kParts; ++p) raw[s][p].load(x + (size_t)p * cols, base + s * step, lane, cols);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      const uint32_t b = base + s * step;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 g = raw[s][0].pair(i);
        if constexpr (KIND == kQ8Copy) r[s][i] = g;
        if constexpr (KIND == kQ8SiluGated) r[s][i] = mul2(mul2(g, sigmoid2(g)), raw[s][kParts - 1].pair(i));
        if constexpr (KIND == kQ8Gelu) {
          const float2 u = mul2(both(kGeluA), mul2(g, fma2(mul2(both(kGeluB), g), g, both(1.f))));
          r[s][i] = mul2(g, sigmoid2(u));
        }
      }
      if (KIND != kQ8Copy && keep) {
        // VEC 8: lanes 0-15 and 16-31 hold a block each (per part); otherwise pairs 0-1 and 2-3 do
        uint32_t t0[kParts], t1[kParts];
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
          t0[p] = bits_of(max_abs(max_abs(0.f, raw[s][p].pair(0)), raw[s][p].pair(1)));
          t1[p] = bits_of(max_abs(max_abs(0.f, raw[s][p].pair(2)), raw[s][p].pair(3)));
          if constexpr (VEC == 8) {
            t0[p] = max(t0[p], t1[p]);
#pragma unroll
            for (int m = 8; m; m >>= 1) t0[p] = max(t0[p], __shfl_xor_sync(kFullMask, t0[p], m));
          } else {
            t0[p] = __reduce_max_sync(kFullMask, t0[p]);
            t1[p] = __reduce_max_sync(kFullMask, t1[p]);
          }
        }
        // The maxima are turned into codings side by side, one to a lane: lane 0 (VEC 8: of each half) that of the
        // first part, lane 1 of the second; without VEC 8 lanes 2 and 3 the second block's.
        const int role = lane & (VEC == 8 ? 1 : 3);
        uint32_t mine = t0[0];
        if (kParts == 2 && (role & 1)) mine = t0[kParts - 1];
        if (VEC != 8 && (role & 2)) mine = kParts == 2 && (role & 1) ? t1[kParts - 1] : t1[0];
        const Coding own = coding_of(mine);
        const uint32_t blk = b / kQ8Block + (VEC == 8 ? lane >> 4 : lane >> 1);
        if ((VEC == 8 ? (lane & 15) < kParts : lane < 4 && (lane & 1) < kParts) && blk < blocks) cks[(lane & 1) * blocks + blk] = own.scale;
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
          const int from = VEC == 8 ? (lane & 16) + p : p;
          const float inv0 = __shfl_sync(kFullMask, own.inv, from);
          const float inv1 = VEC == 8 ? inv0 : __shfl_sync(kFullMask, own.inv, from + 2);
          const uint32_t m0 = t0[p] < 0x7f800000u ? 0xffffffffu : 0u, m1 = VEC == 8 || t1[p] < 0x7f800000u ? 0xffffffffu : 0u;
          const uint32_t k[2] = {codes4(rounded(raw[s][p].pair(0), inv0), rounded(raw[s][p].pair(1), inv0), m0),
                                 codes4(rounded(raw[s][p].pair(2), inv1), rounded(raw[s][p].pair(3), inv1), VEC == 8 ? m0 : m1)};
          store_codes<VEC>(ckq + p * a.ldck, b, lane, cols, k);
        }
      }
    }
  };

  float2 r[NS][4];
  float most = 0.f;
  const uint32_t first = warp * kUnit, span = step * NS;
  const bool once = cols <= span;
  for (uint32_t at = 0; at < cols; at += span) {
    produce(at + first, r, a.ckq != nullptr);
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i) most = max_abs(most, r[s][i]);
  }
  uint32_t top = __reduce_max_sync(kFullMask, bits_of(most));
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
    for (int s = 0; s < NS; ++s) write_unit<VEC>(a, row, at + first + s * step, lane, r[s], c);
  }
}

// ---- residual + root-mean-square norm -> 8-bit rows --------------------------------------------------------------
// y = h * rstd * w with one rstd per row, so the codes of y are the codes of h * w (rstd cancels in x / max|x|) and
// the row needs ONE reduction for both the sum of squares and the maximum.
template <class T, int VEC, int NS>
__global__ void __launch_bounds__(most_warps(NS) * 32) q8_norm_kernel(const RowArgs a, int warps) {
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
  auto produce = [&](uint32_t base, float2 (&r)[NS][4], float2& sum, bool keep) {
    Raw<T, VEC> in[NS], other[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) in[s].load(x, base + s * step, lane, cols);
    if (res) {
#pragma unroll
      for (int s = 0; s < NS; ++s) other[s].load(res, base + s * step, lane, cols);
    }
#pragma unroll
    for (int s = 0; s < NS; ++s) {
#pragma unroll
      for (int i = 0; i < 4; ++i) r[s][i] = res ? add2(in[s].pair(i), other[s].pair(i)) : in[s].pair(i);
      if (keep && res)
        store_unit<T, VEC>(static_cast<T*>(a.h.p) + row * a.h.ld, base + s * step, lane, cols, r[s]);
      float2 w[4];
      load_unit<float, VEC>(a.weight, base + s * step, lane, cols, w);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sum = fma2(r[s][i], r[s][i], sum);
        r[s][i] = mul2(r[s][i], w[i]);
      }
    }
  };

  float2 r[NS][4], sums = both(0.f), unused = both(0.f);
  float most = 0.f;
  const uint32_t first = warp * kUnit, span = step * NS;
  const bool once = cols <= span;
  for (uint32_t at = 0; at < cols; at += span) {
    produce(at + first, r, sums, true);
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
      for (int i = 0; i < 4; ++i) most = max_abs(most, r[s][i]);
  }
  uint32_t top = __reduce_max_sync(kFullMask, bits_of(most));
  float sum = sums.x + sums.y;
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
  // Whether the row is stored as zeros goes by y, which eps can lift far above h * w.  127 / max|h * w| is in range from 2^-120
  // on; what lies below has a y below 2^-100 unless eps is below 2^-40.
  Coding c = coding_of(top, kTinyProduct);
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
    for (int s = 0; s < NS; ++s) write_unit<VEC>(a, row, at + first + s * step, lane, r[s], c);
  }
}

// ---- sums over CTAs -------------------------------------------------------------------------------------------------
// out[c] = sum over rows of rows[r][c] (pitch ld, a multiple of 4 floats), by all threads of a CTA, in order.
__device__ __forceinline__ void sum_rows(const float* rows, uint32_t n, size_t ld, uint32_t cols, float* out, bool aligned) {
  for (uint32_t c = threadIdx.x * 4; c < cols; c += blockDim.x * 4) {
    float2 lo = both(0.f), hi = both(0.f);
#pragma unroll 8
    for (uint32_t r = 0; r < n; ++r) {
      const float4 v = __ldcg(reinterpret_cast<const float4*>(rows + r * ld + c));
      lo = add2(lo, make_float2(v.x, v.y));
      hi = add2(hi, make_float2(v.z, v.w));
    }
    if (aligned && c + 4 <= cols) {
      *reinterpret_cast<float4*>(out + c) = make_float4(lo.x, lo.y, hi.x, hi.y);
    } else {
      const float v[4] = {lo.x, lo.y, hi.x, hi.y};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (c + i < cols) out[c + i] = v[i];
    }
  }
}
// True for the CTA that arrives last of `n` at a counter, which it sets back to zero; what the others wrote before they
// arrived is visible to it.
__device__ __forceinline__ bool arrived_last(uint32_t* counter, uint32_t n) {
  __shared__ bool last;
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    last = atomicAdd(counter, 1u) == n - 1;
    if (last) *counter = 0;
  }
  __syncthreads();
  if (last) __threadfence();
  return last;
}
// Every CTA has written row blockIdx.x of `partial` (pitch ld).  Up to kJoin rows are added up by the CTA that comes last;
// more of them by q8_join_rows_kernel, which spreads the columns over the device: on 8192 x 4096 the two take 47 us, with
// everything joined inside one launch (in two levels) 59.
constexpr uint32_t kJoin = 16;
__device__ __forceinline__ void join_rows(float* partial, size_t ld, uint32_t cols, float* out, uint32_t* counter) {
  const uint32_t n = gridDim.x;
  if (n > kJoin) {
    asm volatile("griddepcontrol.launch_dependents;");
    return;
  }
  if (n == 1)
    __syncthreads();
  else if (!arrived_last(counter, n))
    return;
  sum_rows(partial, n, ld, cols, out, (reinterpret_cast<uintptr_t>(out) & 15) == 0);
}
// 32 columns to a CTA, 32 shares of the rows added up in shared memory: a fixed order.
__global__ void __launch_bounds__(1024) q8_join_rows_kernel(const float* partial, size_t ld, uint32_t n, uint32_t cols, float* out) {
  __shared__ float sh[32][33];
  const uint32_t c = blockIdx.x * 32 + threadIdx.x;
  asm volatile("griddepcontrol.wait;" ::: "memory");      // (launched while the kernel before it still runs)
  float s = 0.f;
  if (c < cols) {
#pragma unroll 4
    for (uint32_t r = threadIdx.y; r < n; r += 32) s += __ldcg(partial + r * ld + c);
  }
  sh[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  s = sh[threadIdx.x][threadIdx.y];     // warp y adds the 32 shares of column y
#pragma unroll
  for (int m = 16; m; m >>= 1) s += __shfl_xor_sync(kFullMask, s, m);
  if (threadIdx.x == 0 && blockIdx.x * 32 + threadIdx.y < cols) out[blockIdx.x * 32 + threadIdx.y] = s;
}

constexpr int kBwdWarps = 16;                             // most warps to a row (two rows' operands live in registers)

// ---- backward of the norm -----------------------------------------------------------------------------------------
// dx = rstd (w dy - xh mean(w dy xh)) + dres with xh = h rstd; dweight = sum over rows of dy xh.  A CTA holds `gangs`
// groups of `warps` warps; a group walks rows group, group + groups, ..., with the next row's loads in flight while a row
// is summed and written.  A lane's columns stay the same, so its share of dweight stays in registers until the end; then
// the CTA's groups add theirs up in shared memory, and the CTAs' are joined, both in a fixed order.
template <class T, int VEC, int NS>
__global__ void __launch_bounds__(kBwdWarps * 32) q8_norm_bwd_kernel(const NormBwdArgs a, int warps, int gangs) {
  extern __shared__ float dwsum[];
  __shared__ float sh[2][kBwdWarps];
  const int lane = threadIdx.x & 31, gang = (threadIdx.x >> 5) / warps, warp = (threadIdx.x >> 5) - gang * warps;
  const uint32_t group = blockIdx.x * gangs + gang, groups = gridDim.x * gangs;
  const uint32_t cols = a.cols, step = kUnit * warps, first = warp * kUnit;
  float2 w[NS][4], dw[NS][4];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    load_unit<float, VEC>(a.weight, first + s * step, lane, cols, w[s]);
#pragma unroll
    for (int i = 0; i < 4; ++i) dw[s][i] = both(0.f);
  }
  const float inv_n = 1.f / (float)cols;
  const T* dy = static_cast<const T*>(a.dy.p) + group * a.dy.ld;
  const T* h = static_cast<const T*>(a.h.p) + group * a.h.ld;
  const T* dres = a.dres.p ? static_cast<const T*>(a.dres.p) + group * a.dres.ld : nullptr;
  T* dx = static_cast<T*>(a.dx.p) + group * a.dx.ld;
  Raw<T, VEC> rg[NS], rh[NS], ro[NS];
  float rstd = 0.f;
  auto fetch = [&](uint64_t row) {
    rstd = a.rstd[row];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      rg[s].template load<true>(dy, first + s * step, lane, cols);
      rh[s].template load<true>(h, first + s * step, lane, cols);
      if (dres) ro[s].template load<true>(dres, first + s * step, lane, cols);
    }
    dy += (size_t)groups * a.dy.ld;
    h += (size_t)groups * a.h.ld;
    if (dres) dres += (size_t)groups * a.dres.ld;
  };
  if (group < a.rows) fetch(group);
  int flip = 0;
  for (uint64_t row = group; row < a.rows; row += groups, flip ^= 1, dx += (size_t)groups * a.dx.ld) {
    const float rs = rstd;
    float2 g[NS][4], xh[NS][4], dots = both(0.f);
    Raw<T, VEC> o[NS];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      if (a.dres.p) o[s] = ro[s];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 y = rg[s].pair(i);
        xh[s][i] = mul2(rh[s].pair(i), both(rs));
        dw[s][i] = fma2(y, xh[s][i], dw[s][i]);
        g[s][i] = mul2(y, w[s][i]);
        dots = fma2(g[s][i], xh[s][i], dots);
      }
    }
    if (row + groups < a.rows) fetch(row + groups);      // (in flight while this row is summed and written)
    float dot = dots.x + dots.y;
#pragma unroll
    for (int m = 16; m; m >>= 1) dot += __shfl_xor_sync(kFullMask, dot, m);
    if (warps > 1) {   // two buffers: a warp reaches the next row's store only after all have passed this row's barrier
      if (lane == 0) sh[flip][gang * warps + warp] = dot;
      asm volatile("bar.sync %0, %1;" ::"r"(1 + gang), "r"(warps * 32) : "memory");
      dot = lane < warps ? sh[flip][gang * warps + lane] : 0.f;
#pragma unroll
      for (int m = 16; m; m >>= 1) dot += __shfl_xor_sync(kFullMask, dot, m);
    }
    const float2 c = both(-dot * inv_n);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      float2 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = mul2(both(rs), fma2(xh[s][i], c, g[s][i]));
        if (a.dres.p) v[i] = add2(v[i], o[s].pair(i));
      }
      store_unit<T, VEC, true>(dx, first + s * step, lane, cols, v);
    }
  }
  for (int g = 0; g < gangs - 1; ++g) {
    if (gang == g) {
#pragma unroll
      for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t at = ((s * warps + warp) * 32 + lane) * 2 + i * 64 * NS * warps;
          if (g > 0) dw[s][i] = add2(dw[s][i], make_float2(dwsum[at], dwsum[at + 1]));
          dwsum[at] = dw[s][i].x;
          dwsum[at + 1] = dw[s][i].y;
        }
    }
    __syncthreads();
  }
  if (gang == gangs - 1) {
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      if (gangs > 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t at = ((s * warps + warp) * 32 + lane) * 2 + i * 64 * NS * warps;
          dw[s][i] = add2(dw[s][i], make_float2(dwsum[at], dwsum[at + 1]));
        }
      }
      store_unit<float, VEC>(a.partial + blockIdx.x * a.ldp, first + s * step, lane, cols, dw[s]);
    }
  }
  join_rows(a.partial, a.ldp, cols, a.dweight, a.counters);
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
    float2 dots = both(0.f);
    for (uint32_t b = warp * kUnit; b < cols; b += step) {
      float2 g[4], xh[4], w[4];
      load_unit<T, VEC>(dy, b, lane, cols, g);
      load_unit<T, VEC>(h, b, lane, cols, xh);
      load_unit<float, VEC>(a.weight, b, lane, cols, w);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t c = col_of<VEC>(b, lane, 2 * i), d = col_of<VEC>(b, lane, 2 * i + 1);
        const float2 p = mul2(g[i], mul2(xh[i], both(rstd)));
        if (c < cols) dwsum[c] += p.x;
        if (d < cols) dwsum[d] += p.y;
        dots = fma2(p, w[i], dots);
      }
    }
    float dot = dots.x + dots.y;
#pragma unroll
    for (int m = 16; m; m >>= 1) dot += __shfl_xor_sync(kFullMask, dot, m);
    if (lane == 0) sh[flip][warp] = dot;
    __syncthreads();
    dot = lane < warps ? sh[flip][lane] : 0.f;
#pragma unroll
    for (int m = 16; m; m >>= 1) dot += __shfl_xor_sync(kFullMask, dot, m);
    const float2 c = both(-dot / (float)cols);
    T* dx = static_cast<T*>(a.dx.p) + row * a.dx.ld;
    for (uint32_t b = warp * kUnit; b < cols; b += step) {
      float2 g[4], xh[4], w[4], o[4], v[4];
      load_unit<T, VEC>(dy, b, lane, cols, g);
      load_unit<T, VEC>(h, b, lane, cols, xh);
      load_unit<float, VEC>(a.weight, b, lane, cols, w);
      if (a.dres.p) load_unit<T, VEC>(static_cast<const T*>(a.dres.p) + row * a.dres.ld, b, lane, cols, o);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = mul2(both(rstd), fma2(mul2(xh[i], both(rstd)), c, mul2(g[i], w[i])));
        if (a.dres.p) v[i] = add2(v[i], o[i]);
      }
      store_unit<T, VEC>(dx, b, lane, cols, v);
    }
  }
  __syncthreads();
  for (uint32_t c = threadIdx.x; c < cols; c += blockDim.x) a.partial[blockIdx.x * a.ldp + c] = dwsum[c];
  join_rows(a.partial, a.ldp, cols, a.dweight, a.counters);
}

// ---- column sums ---------------------------------------------------------------------------------------------------
// A CTA sums 256 columns of one split of the rows, 8 warps sharing the rows; the last of the splits' CTAs adds their sums
// up, in order.
template <class T, int VEC>
__global__ void __launch_bounds__(256) q8_colsum_kernel(Mat x, uint64_t rows, uint32_t cols, float* partial, float* out,
                                                        uint32_t* counters) {
  __shared__ __align__(16) float sh[8][kUnit];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const uint32_t base = blockIdx.x * kUnit, split = blockIdx.y, splits = gridDim.y;
  const uint64_t per = (rows + splits - 1) / splits, r0 = split * per, r1 = min(r0 + per, rows);
  float2 s[4] = {both(0.f), both(0.f), both(0.f), both(0.f)};
#pragma unroll 8
  for (uint64_t r = r0 + warp; r < r1; r += 8) {
    float2 v[4];
    load_unit<T, VEC>(static_cast<const T*>(x.p) + r * x.ld, base, lane, cols, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = add2(s[i], v[i]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    sh[warp][col_of<VEC>(0, lane, 2 * i)] = s[i].x;
    sh[warp][col_of<VEC>(0, lane, 2 * i + 1)] = s[i].y;
  }
  __syncthreads();
  const uint32_t c = base + threadIdx.x;
  float sum = 0.f;
#pragma unroll
  for (int w = 0; w < 8; ++w) sum += sh[w][threadIdx.x];
  if (splits == 1) {
    if (c < cols) out[c] = sum;
    return;
  }
  float* mine = partial + (size_t)blockIdx.x * splits * kUnit;
  mine[split * kUnit + threadIdx.x] = sum;
  if (!arrived_last(counters + blockIdx.x, splits)) return;
  // four columns and every fourth split to a thread, then the four shares of a column
  const uint32_t quarter = threadIdx.x >> 6, at = (threadIdx.x & 63) * 4;
  float2 lo = both(0.f), hi = both(0.f);
#pragma unroll 8
  for (uint32_t i = quarter; i < splits; i += 4) {
    const float4 v = __ldcg(reinterpret_cast<const float4*>(mine + i * kUnit + at));
    lo = add2(lo, make_float2(v.x, v.y));
    hi = add2(hi, make_float2(v.z, v.w));
  }
  *reinterpret_cast<float4*>(&sh[quarter][at]) = make_float4(lo.x, lo.y, hi.x, hi.y);
  __syncthreads();
  if (c < cols) out[c] = (sh[0][threadIdx.x] + sh[1][threadIdx.x]) + (sh[2][threadIdx.x] + sh[3][threadIdx.x]);
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
  Raw<T, VEC> da;
  da.load(static_cast<const T*>(a.da.p) + row * a.da.ld, base, lane, cols);
  uint32_t k[kParts][2];
  float s0[kParts], s1[kParts];
#pragma unroll
  for (int p = 0; p < kParts; ++p) {
    const size_t at = row * kParts + p;
    load_codes<VEC>(a.ckq + at * a.ldck, base, lane, cols, k[p]);
    const float* sc = a.cks + at * blocks + blk;
    s0[p] = VEC != 8 || lane < 16 ? sc[0] : blk + 1 < blocks ? sc[1] : 0.f;      // (VEC 8: one block to a lane)
    s1[p] = VEC == 8 ? s0[p] : blk + 1 < blocks ? sc[1] : 0.f;
  }
  float2 d0[4], d1[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 g = mul2(code_pair(k[0], i), both(i < 2 ? s0[0] : s1[0])), y = da.pair(i);
    if constexpr (KIND == kQ8SiluGated) {
      const float2 u = mul2(code_pair(k[kParts - 1], i), both(i < 2 ? s0[kParts - 1] : s1[kParts - 1]));
      const float2 sg = sigmoid2(g);
      const float2 t = mul2(y, sg);
      d1[i] = mul2(t, g);
      // y u sg (1 + g (1 - sg))
      d0[i] = mul2(mul2(t, u), fma2(g, fma2(sg, both(-1.f), both(1.f)), both(1.f)));
    } else {
      // y sg (1 + x (1 - sg) kGeluA (1 + 3 kGeluB x^2)).  From |x| = 14 on the derivative is 0 or 1 in fp32, so x is held
      // at 20: its cube would overflow and meet the 0.
      const float2 x = held(g, 20.f), x2 = mul2(x, x), v = mul2(both(kGeluA), mul2(x, fma2(both(kGeluB), x2, both(1.f))));
      const float2 sg = sigmoid2(v);
      const float2 in = mul2(both(kGeluA), fma2(both(3.f * kGeluB), x2, both(1.f)));
      d0[i] = mul2(mul2(y, sg), fma2(mul2(x, fma2(sg, both(-1.f), both(1.f))), in, both(1.f)));
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

// Warps per row and units per warp.  One unit to a warp, so many warps to a row, is fastest as long as all rows run at once;
// beyond that fewer warps, with several units each, wait for one another.  Rows of more units than 16 warps keep are read
// twice: with 4 units to a warp, which only the norm of bf16 in 16-byte accesses has, those are the rows of more than 64
// units, and for them 2 are faster again.  (Just past a whole number of rounds each choice loses up to 15 % to one whose
// rounds fit: norm, bf16, 512 x 6400 9.0 us with one unit, 10.3 with the four that are taken.)  In us with 1, 2 (and 4) units
// to a warp, * what is taken:
//   rows x columns        585 x 1600       857 x 1600       1342 x 1600      512 x 4096       750 x 4096      8192 x 4096
//   norm, bf16            3.30* 3.55 4.31  4.82* 5.00 5.79  7.18 7.69 6.78*  6.03* 5.80 6.73  8.44 8.65 7.70*  57.0 53.2 43.3*
//   norm, fp32            4.90* 5.33       6.20* 6.15       8.74 9.44*       8.75 7.91*       10.7 11.2*       86.2 68.9*
//   rows x columns        4096 x 512       64 x 10240       256 x 16384      4096 x 16384     4096 x 20480
//   norm, bf16            6.31* 5.52 7.39  - 5.01 3.81*     - 10.4 10.9*     - 109 102*       - 138* 188
//   rows x columns        585 x 1600       671 x 1600       96 x 6400        163 x 6400       8192 x 6400
//   gated, checkpoint     3.31* 3.64       4.49 4.02*       3.30* 3.47       5.30 4.52*       131 89.8*
//   rows x columns        512 x 1600       1600 x 1600      128 x 6400       512 x 6400       6400 x 6400
//   plain rows, fp32      2.29* 2.30       4.78 4.52*       2.43* 2.42       6.02 5.34*       43.5 35.1*
struct Shape {
  int warps, ns;
  unsigned grid;
  int threads;
};
// CTAs of a kernel that an SM holds at once, asked for once per number of warps (the same on every device of this kind).
template <auto* KERNEL>
int resident(int warps) {
  static std::atomic<int> known[33];
  int n = known[warps].load(std::memory_order_relaxed);
  if (n == 0) {
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, KERNEL, warps * 32, 0) != cudaSuccess || n < 1) n = 1;
    known[warps].store(n, std::memory_order_relaxed);
  }
  return n;
}
// ONE: the kernel with one unit to a warp; most: the most units that a warp keeps.
template <auto* ONE>
Shape shape_of(uint64_t rows, uint32_t cols, int most, int sms) {
  const uint32_t units = (cols + kUnit - 1) / kUnit;
  const bool at_once = units <= 32 && (rows <= (uint64_t)sms || rows <= (uint64_t)sms * resident<ONE>((int)units));
  const int ns = units == 1 || at_once ? 1 : units == 2 || units > 64 ? 2 : most;
  const int w = (int)((units + ns - 1) / ns), warps = w < most_warps(ns) ? w : most_warps(ns);
  return {warps, ns, (unsigned)(warps == 1 ? (rows + 3) / 4 : rows), warps == 1 ? 128 : warps * 32};
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

cudaError_t launch_q8_act(int dtype, Q8Kind kind, const RowArgs& a, int sms, cudaStream_t stream) {
  Width w;
  w.add(a.x, elem_bytes(dtype));
  w.add(a.values, 2);
  return by_type(dtype, [&](auto tv) {
    using T = decltype(tv);
    return by_vec(w.vec(a.cols), [&](auto vec) {
      auto launch = [&](auto k) {
        const Shape sh = shape_of<q8_act_kernel<T, vec(), 1, k()>>(a.rows, a.cols, 2, sms);
        return by_ns(sh.ns, [&](auto ns) {
          q8_act_kernel<T, vec(), ns(), k()><<<sh.grid, sh.threads, 0, stream>>>(a, sh.warps);
          return cudaGetLastError();
        });
      };
      if (kind == kQ8SiluGated) return launch(std::integral_constant<int, kQ8SiluGated>());
      if (kind == kQ8Gelu) return launch(std::integral_constant<int, kQ8Gelu>());
      return launch(std::integral_constant<int, kQ8Copy>());
    });
  });
}

cudaError_t launch_q8_norm(int dtype, const RowArgs& a, int sms, cudaStream_t stream) {
  Width w;
  w.add(a.x, elem_bytes(dtype));
  w.add(a.res, elem_bytes(dtype));
  if (a.res.p) w.add(a.h, elem_bytes(dtype));
  w.add(a.values, 2);
  w.add(Mat{const_cast<float*>(a.weight), 0}, 4);
  return by_type(dtype, [&](auto tv) {
    using T = decltype(tv);
    return by_vec(w.vec(a.cols), [&](auto vec) {
      constexpr int kMost = sizeof(T) == 2 && vec() == 8 ? 4 : 2;
      const Shape sh = shape_of<q8_norm_kernel<T, vec(), 1>>(a.rows, a.cols, kMost, sms);
      if constexpr (kMost == 4) {
        if (sh.ns == 4) {
          q8_norm_kernel<T, vec(), 4><<<sh.grid, sh.threads, 0, stream>>>(a, sh.warps);
          return cudaGetLastError();
        }
      }
      return by_ns(sh.ns, [&](auto ns) {
        q8_norm_kernel<T, vec(), ns()><<<sh.grid, sh.threads, 0, stream>>>(a, sh.warps);
        return cudaGetLastError();
      });
    });
  });
}

namespace {
struct BwdShape {
  int warps, ns, gangs;      // (0 warps: the wide kernel)
  size_t smem;
  uint32_t ctas;             // rows of partial sums
};
// Whether there is a variant with two units to a warp, for rows of 17 to 32 units (with one they end at 16; without the
// variant the wide kernel takes over).  Next to the wide kernel, in us on 4096 rows of 5120 to 5122 and of 8190 to 8192
// columns:       16-byte accesses          pairs                 single elements
//   bf16         33.5 (84), 42.6 (117)     - , 47.4 (75)         113 (82), 144 (114)
//   fp32         86.7 (111), 113 (159)     89.0 (74), 108 (108)  78.0 (79), 99.3 (112)
// (bf16 in 16-byte accesses and pairs spill at most 16 bytes, the others 200 to 324).
constexpr bool two_units(size_t elem, int vec) { return elem == 2 ? vec != 1 : vec != 2; }
bool bwd_wide(uint32_t cols, int dtype, int vec) { return cols > kBwdWarps * (two_units(elem_bytes(dtype), vec) ? 2 : 1) * kUnit; }

template <class T, int VEC, class F>
cudaError_t by_units(int ns, F f) {
  if constexpr (two_units(sizeof(T), VEC))
    if (ns == 2) return f(std::integral_constant<int, 2>());
  return f(std::integral_constant<int, 1>());
}
// CTAs of a kernel that an SM holds at once, asked for once per number of warps to a row, which decides the rest (the same
// on every device of this kind).
template <class T, int VEC, int NS>
int bwd_resident(int warps, int gangs, size_t smem) {
  static std::atomic<int> known[kBwdWarps + 1];
  int n = known[warps].load(std::memory_order_relaxed);
  if (n == 0) {
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, q8_norm_bwd_kernel<T, VEC, NS>, warps * gangs * 32, smem) != cudaSuccess || n < 1) n = 1;
    known[warps].store(n, std::memory_order_relaxed);
  }
  return n;
}

// CTAs of at least 8 warps, as many as are resident at once (with more, some would start when the others are done).
// Where one unit to a warp is enough, two are faster with bf16 in 16-byte accesses or pairs (8192 x 4096: 59 -> 47 us,
// 8192 x 1600: 36 -> 24 us) and slower with fp32 (4096 x 4096: 46 -> 78 us) and single elements.
BwdShape bwd_shape(uint64_t rows, uint32_t cols, int dtype, int vec, int sms) {
  if (bwd_wide(cols, dtype, vec)) return {0, 0, 0, 0, (uint32_t)(rows < (uint64_t)sms ? rows : sms)};
  const uint32_t units = (cols + kUnit - 1) / kUnit;
  const int ns = units > kBwdWarps || (units > 1 && dtype == STQ_GRAD_BF16 && vec > 1) ? 2 : 1;
  const int warps = (int)((units + ns - 1) / ns), most_of = ns == 2 ? kBwdWarps : 8;
  const int gangs = warps >= most_of ? 1 : most_of / warps;
  const size_t smem = gangs > 1 ? (size_t)warps * ns * kUnit * 4 : 0;      // (at most 8 warps then: 16 KB)
  int per_sm = 1;
  by_type(dtype, [&](auto tv) {
    using T = decltype(tv);
    return by_vec(vec, [&](auto v) {
      return by_units<T, v()>(ns, [&](auto n) {
        per_sm = bwd_resident<T, v(), n()>(warps, gangs, smem);
        return cudaSuccess;
      });
    });
  });
  const uint64_t want = (rows + gangs - 1) / gangs, most = (uint64_t)sms * per_sm;
  return {warps, ns, gangs, smem, (uint32_t)(want < most ? want : most)};
}

int bwd_vec(int dtype, const NormBwdArgs& a) {
  Width w;
  w.add(a.dy, elem_bytes(dtype));
  w.add(a.h, elem_bytes(dtype));
  w.add(a.dres, elem_bytes(dtype));
  w.add(a.dx, elem_bytes(dtype));
  w.add(Mat{const_cast<float*>(a.weight), 0}, 4);
  return w.vec(a.cols);
}
}  // namespace

size_t q8_norm_bwd_partial(int dtype, const NormBwdArgs& a, int sms) {
  const uint32_t n = bwd_shape(a.rows, a.cols, dtype, bwd_vec(dtype, a), sms).ctas;
  return (size_t)n * a.ldp;
}

cudaError_t launch_q8_norm_bwd(int dtype, const NormBwdArgs& a, int sms, cudaStream_t stream, int* launches) {
  const int width = bwd_vec(dtype, a);
  const BwdShape sh = bwd_shape(a.rows, a.cols, dtype, width, sms);
  *launches = sh.ctas > kJoin ? 2 : 1;
  const cudaError_t e = by_type(dtype, [&](auto tv) {
    using T = decltype(tv);
    return by_vec(width, [&](auto vec) {
      if (sh.warps == 0) {
        const int bytes = (int)(a.cols * sizeof(float));
        cudaError_t e2 = cudaFuncSetAttribute(q8_norm_bwd_wide_kernel<T, vec()>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e2 != cudaSuccess) return e2;
        q8_norm_bwd_wide_kernel<T, vec()><<<sh.ctas, 1024, bytes, stream>>>(a, sh.ctas);
        return cudaGetLastError();
      }
      const int threads = sh.warps * sh.gangs * 32;
      return by_units<T, vec()>(sh.ns, [&](auto n) {
        q8_norm_bwd_kernel<T, vec(), n()><<<sh.ctas, threads, sh.smem, stream>>>(a, sh.warps, sh.gangs);
        return cudaGetLastError();
      });
    });
  });
  if (e != cudaSuccess || sh.ctas <= kJoin) return e;
  return launch_with(q8_join_rows_kernel, dim3((a.cols + 31) / 32), dim3(32, 32), 0, 1, true, stream, (const float*)a.partial, a.ldp, sh.ctas,
                     a.cols, a.dweight);
}

uint32_t q8_colsum_splits(uint64_t rows, uint32_t cols, int sms) {
  // about four CTAs of 8 warps per SM, at least 32 rows to a split; so many columns that there is no counter for each
  // tile of them fill the device by themselves
  const uint32_t tiles = (cols + kUnit - 1) / kUnit, want = (uint32_t)(4 * sms + tiles - 1) / tiles;
  const uint64_t most = (rows + 31) / 32;
  return tiles > kQ8Counters ? 1 : (uint32_t)(want < most ? want : most);
}
size_t q8_colsum_partial(uint32_t cols, uint32_t splits) { return splits == 1 ? 0 : (size_t)((cols + kUnit - 1) / kUnit) * kUnit * splits; }

cudaError_t launch_q8_colsum(int dtype, Mat x, uint64_t rows, uint32_t cols, uint32_t splits, float* partial, uint32_t* counters,
                             float* out, cudaStream_t stream) {
  Width w;
  w.add(x, elem_bytes(dtype));
  const dim3 grid((cols + kUnit - 1) / kUnit, splits);
  return by_type(dtype, [&](auto tv) {
    using T = decltype(tv);
    return by_vec(w.vec(cols), [&](auto vec) {
      q8_colsum_kernel<T, vec()><<<grid, 256, 0, stream>>>(x, rows, cols, partial, out, counters);
      return cudaGetLastError();
    });
  });
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
