// Gradients of the 8-bit product on the tensor cores:
//   dx[t][k] = sum_n dy[t][n] * ws[n] * wq[n][k]          (rows of the result: tokens, sum over output channels)
//   dw[n][k] = sum_t dy[t][n] * xs[t] * xq[t][k]          (rows of the result: output channels, sum over tokens)
// Both are D[m][j] = sum_c G(m, c) * s[c] * q[c][j] with the bf16 gradient G as it lies in memory (K-major for dx,
// MN-major for dw) and an 8-bit operand q with j contiguous and a scale that varies along the sum.
//
// The matrix unit takes two bf16 operands, so the codes are turned into bf16 on the way.  For a bf16 result the operand
// is bf16(s * q), one rounding to 8 significant bits (relative error 2^-8 a term, random in sign), which is of the order
// of the rounding of the result itself.  For an fp32 result (PARTS = 3) the fp32 product s * q is cut into three bf16
// numbers whose sum is exactly that product, and three products are added up: the error is that of fp32 arithmetic.
// Folding s into G instead would round as much and touch the larger operand.
//
// The matrix unit cuts its fp32 sums off instead of rounding them (measured: 2e-8 of the sum a step, always towards zero),
// which adds up to 5e-6 over a sum of 1300.  For a bf16 result that is nothing; for an fp32 result the small parts go in
// first, and every kChunk stages the sum is taken out and added, rounded to nearest, to a running sum that the writing
// warps keep in tensor memory.
//
// Two forms.  CONV: the codes are converted inside the product kernel, once per row of tiles of the result.  Otherwise a
// small kernel writes the converted operand to the workspace first and the product kernel only copies and multiplies;
// that pays once the result has many rows (plan_of), and only for the single operand: in three parts the products take
// longer than the conversion anyway.  Both form the same operand.
//
// Per CTA: warp 0 copies tiles of G and q into a ring of stages, two groups of four warps convert q in alternate stages,
// one warp issues the products, four warps write results; accumulators are doubled in tensor memory as in the forward
// product.  (Without conversion there are the copying, the issuing and the four writing warps.)
#include "../../include/stq.h"
#include "stq_internal.h"
#include "stq_q8.h"
#include "stq_q8_mma.cuh"
#include "stq_q8_ring.h"
#include "stq_q8_tma.h"

namespace stq {
namespace {

constexpr int kDepth = 64;             // length of the sum per stage
constexpr int kStepK = 16;             // and per product instruction
constexpr int kGroups = 2, kGroupWarps = 4;        // conversion: groups of warps, a stage to a group

struct GradArgs {
  const float* scale;                  // s[c]
  void* out;
  size_t ldo;                          // elements
  float* part;                         // partial results of the tiles whose sum is shared, a tile to each
  uint64_t m;
  uint32_t n, depth, ksteps;           // columns, length of the sum, its stages
  uint32_t tiles_m, tiles;
  uint32_t full, splits;               // tiles from `full` on are shared by `splits` work items each
  int aligned;                         // tensor copies can write `out`: map_o describes it
  int* err;
};

template <int CG, int BN, int PARTS, bool CONV>
struct GradShape {
  static constexpr int kThreads = 32 * (2 + 4 + (CONV ? kGroups * kGroupWarps : 0));
  static constexpr int kNB = BN / CG;                             // columns of the 8-bit operand in this CTA
  static constexpr int kA = 128 * kDepth * 2, kQ = CONV ? kDepth * kNB : 0, kB = kDepth * kNB * 2;
  static constexpr int kStage = kA + kQ + kB * PARTS;
  static constexpr int kFit = (204 * 1024) / kStage;
  static constexpr int kStages = kFit < 6 ? kFit : 6;
  static constexpr int kChunk = PARTS == 3 ? 2 : 1 << 30;         // stages to one accumulator
  static constexpr int kCols = (PARTS == 3 ? 4 : 2) * BN;         // two accumulators (and the running sum)
  static constexpr int kSmem = kStages * kStage + 4 * kStageBytes + 1024;
};

__device__ __forceinline__ uint32_t bf2_add(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t bf2_mul(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t bf2_fma(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}

// A row's scale for two columns at a time: s = hi + lo up to 2^-17.
struct Scale2 {
  float s;
  uint32_t hi, lo;
};
__device__ __forceinline__ Scale2 scale2_of(float s) {
  Scale2 r;
  r.s = s;
  const __nv_bfloat16 h = __float2bfloat16_rn(s), l = __float2bfloat16_rn(s - __bfloat162float(h));
  r.hi = (uint32_t)__bfloat16_as_ushort(h) * 0x10001u;
  r.lo = (uint32_t)__bfloat16_as_ushort(l) * 0x10001u;
  return r;
}

// Codes i, i + 1 (i = 0 or 2) of four codes as a pair of bf16(s * q), without a conversion instruction (those run at
// an eighth of the rate of the arithmetic here).  The 7 low bits of a code under the exponent of 128 are the number
// 128 + bits, its sign bit under that of -128 is -128 or -256; their sum is the code, exactly.
__device__ __forceinline__ uint32_t decode_pair(uint32_t w, int i, const Scale2& s) {
  const uint32_t t = __byte_perm(w, 0u, i == 0 ? 0x4140 : 0x4342);
  const uint32_t q = bf2_add((t & 0x007f007fu) | 0x43004300u, (t & 0x00800080u) | 0xc300c300u);
  return bf2_fma(q, s.hi, bf2_mul(q, s.lo));
}

__device__ __forceinline__ uint64_t f2_pair(uint32_t lo, uint32_t hi) { return (uint64_t)hi << 32 | lo; }
__device__ __forceinline__ uint64_t f2_add(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t f2_mul(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// The same as three pairs whose sum is fl32(s * q): 8 bits of the product to each, cut off, the rest exact.
__device__ __forceinline__ void decode_pair3(uint32_t w, int i, const Scale2& s, uint32_t (&out)[3]) {
  const uint32_t u = w ^ 0x80808080u, sb = __float_as_uint(s.s);      // a byte under the exponent of 2^23 is 2^23 + byte
  constexpr uint32_t kMinus = 0xcb000080u;                            // -(2^23 + 128)
  uint64_t v = f2_mul(f2_add(f2_pair(__byte_perm(u, 0x4b000000u, 0x7650 + i), __byte_perm(u, 0x4b000000u, 0x7651 + i)), f2_pair(kMinus, kMinus)),
                      f2_pair(sb, sb));
#pragma unroll
  for (int p = 0; p < 3; ++p) {
    const uint32_t lo = (uint32_t)v, hi = (uint32_t)(v >> 32);
    out[p] = __byte_perm(lo, hi, 0x7632);
    if (p < 2) v = f2_add(v, f2_pair((lo & 0xffff0000u) ^ 0x80000000u, (hi & 0xffff0000u) ^ 0x80000000u));
  }
}

template <int CG, int BN, int PARTS, bool CONV, bool DW, class O>
__global__ void __launch_bounds__((GradShape<CG, BN, PARTS, CONV>::kThreads), 1)
q8_grad_kernel(const __grid_constant__ CUtensorMap map_g, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_o,
               const GradArgs a) {
  using S = GradShape<CG, BN, PARTS, CONV>;
  constexpr int kStages = S::kStages, kNB = S::kNB;
  using Codes = ArrivalRing<kStages, kGroups>;
  extern __shared__ uint8_t raw[];
  __shared__ uint64_t bars[Codes::kBars + 3 * kStages + 4];
  __shared__ uint32_t tmem_slot;
  const uint32_t ring = (smem_addr(raw) + 1023u) & ~1023u, stages = ring + kStages * S::kStage;
  // codes have landed (this CTA, see ArrivalRing); per stage: gradient has landed and codes are converted (both CTAs, at the
  // leader), stage is free; per accumulator: done, read (both CTAs, at the leader)
  const uint32_t full_q = smem_addr(bars), full_g = full_q + 8 * Codes::kBars, ready = full_g + 8 * kStages;
  const uint32_t empty = ready + 8 * kStages, done = empty + 8 * kStages, freed = done + 16;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CG == 2 ? cluster_rank() : 0;
  const bool leader = rank == 0;
  const uint32_t unit = blockIdx.x / CG, units = gridDim.x / CG, work = a.full + (a.tiles - a.full) * a.splits;

  if (threadIdx.x == 0) {
    for (int i = 0; i < Codes::kBars; ++i) bar_init(full_q + 8 * i, 1);
    for (int i = 0; i < kStages; ++i) {
      bar_init(full_g + 8 * i, 1);
      bar_init(ready + 8 * i, CG * kGroupWarps);
      bar_init(empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      bar_init(done + 8 * i, 1);
      bar_init(freed + 8 * i, 4 * CG);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc<CG>(smem_addr(&tmem_slot), S::kCols);
  mma_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync_all();
  asm volatile("griddepcontrol.wait;" ::: "memory");      // (launched while a copy or conversion kernel before it still runs)
  mma_fence_after();
  const uint32_t tmem = tmem_slot;

  // work item -> tile and its share [k0, k1) of the stages of the sum
  auto share = [&](uint32_t w, uint32_t& tile, uint32_t& k0, uint32_t& k1) {
    tile = w;
    k0 = 0;
    k1 = a.ksteps;
    if (w >= a.full) {
      const uint32_t i = w - a.full, sp = i % a.splits;
      tile = a.full + i / a.splits;
      k0 = (uint32_t)((uint64_t)a.ksteps * sp / a.splits);
      k1 = (uint32_t)((uint64_t)a.ksteps * (sp + 1) / a.splits);
    }
  };

  bool ok = true;
  if (warp == 0) {
    if (elect_one()) {
      uint32_t it = 0, tile, k0, k1;
      const uint32_t full_g0 = CG == 2 ? peer_addr(full_g, 0) : full_g;
      for (uint32_t w = unit; ok && w < work; w += units) {
        share(w, tile, k0, k1);
        const int row = (int)(tile % a.tiles_m) * 128 * CG + 128 * rank, col = (int)(tile / a.tiles_m) * BN + kNB * rank;
        for (uint32_t k = k0; k < k1; ++k, ++it) {
          const uint32_t s = it % kStages, ph = (it / kStages) & 1;
          if (!(ok = bar_wait(empty + 8 * s, ph ^ 1))) break;
          const uint32_t at = ring + s * S::kStage, c = k * kDepth;
          if (leader) bar_expect(full_g + 8 * s, CG * (S::kA + (CONV ? 0 : S::kB)));
          if constexpr (CONV) {
            const uint32_t landed = full_q + 8 * Codes::bar(it);
            bar_expect(landed, S::kQ);
            tensor_load<1>(at + S::kA, &map_q, col, (int)c, landed);
          } else {
#pragma unroll
            for (int i = 0; i < kNB / 64; ++i)
              tensor_load<CG>(at + S::kA + i * (kDepth * 128), &map_q, col + 64 * i, (int)c, full_g0 + 8 * s);
          }
          if constexpr (DW) {
            tensor_load<CG>(at, &map_g, row, (int)c, full_g0 + 8 * s);
            tensor_load<CG>(at + S::kA / 2, &map_g, row + 64, (int)c, full_g0 + 8 * s);
          } else {
            tensor_load<CG>(at, &map_g, (int)c, row, full_g0 + 8 * s);
          }
        }
      }
      if (!ok)      // leave no copy in flight
        for (uint32_t i = it > kStages ? it - kStages : 0; i < it; ++i) {
          if (CONV) bar_wait(full_q + 8 * Codes::bar(i), Codes::parity(i));
          if (leader) bar_wait(full_g + 8 * (i % kStages), (i / kStages) & 1);
        }
    }
  } else if (warp == 1) {
    if (leader && elect_one()) {
      constexpr uint32_t id = idesc(kIdescBf16, 128 * CG, BN, DW, true);
      uint32_t it = 0, n = 0, tile, k0, k1;
      for (uint32_t w = unit; ok && w < work; w += units) {
        share(w, tile, k0, k1);
        for (uint32_t k = k0; k < k1; ++k, ++it) {
          const uint32_t s = it % kStages, ph = (it / kStages) & 1, acc = n & 1, place = (k - k0) % S::kChunk;
          if (place == 0) {
            if (!(ok = bar_wait<CG == 2>(freed + 8 * acc, ((n >> 1) & 1) ^ 1))) break;
            mma_fence_after();
          }
          if (!(ok = bar_wait<CG == 2>(full_g + 8 * s, ph) && (!CONV || bar_wait<CG == 2>(ready + 8 * s, ph)))) break;
          mma_fence_after();
          const uint32_t at = ring + s * S::kStage;
          const uint64_t da = DW ? operand_desc(at, S::kA / 2, 1024) : operand_desc(at, 16, 1024);
          const uint64_t db = operand_desc(at + S::kA + S::kQ, kDepth * 128, 1024);
          constexpr uint32_t kStepA = DW ? (kStepK * 128) >> 4 : (kStepK * 2) >> 4, kStepB = (kStepK * 128) >> 4;
#pragma unroll
          for (int p = PARTS - 1; p >= 0; --p)                  // the smallest part first
#pragma unroll
            for (int j = 0; j < kDepth / kStepK; ++j)
              mma<CG, false>(tmem + acc * BN, da + j * kStepA, db + p * (S::kB >> 4) + j * kStepB, id,
                             place != 0 || p < PARTS - 1 || j != 0);
          mma_commit<CG>(empty + 8 * s);
          if (place == S::kChunk - 1 || k + 1 == k1) {
            mma_commit<CG>(done + 8 * acc);
            ++n;
          }
        }
      }
    }
  } else if (CONV && warp < 2 + kGroups * kGroupWarps) {
    if constexpr (CONV) {
    // A row of the stage has kNB codes: kNB / 16 lanes take 16 bytes each.
    constexpr int kLanes = kNB / 16, kRowsAtOnce = kGroupWarps * 32 / kLanes, kPasses = kDepth / kRowsAtOnce;
    const int group = (warp - 2) / kGroupWarps, thread = (threadIdx.x - 64) % (kGroupWarps * 32);
    const uint32_t sub = thread % kLanes, row0 = thread / kLanes;
    // 16 columns are two 16-byte pieces of the row's 128 bytes in its atom of 64 columns; the lanes of the second atom
    // write theirs in the other order, so that eight lanes reach eight different pieces
    const uint32_t atom = sub / 4, piece = (sub % 4) * 2, odd = atom & 1;
    const uint32_t ready0 = CG == 2 ? peer_addr(ready, 0) : ready;
    uint32_t it = 0, tile, k0, k1;             // it: stages before this work item
    for (uint32_t w = unit; ok && w < work; w += units) {
      share(w, tile, k0, k1);
      float sc[kPasses];
      auto scales = [&](uint32_t k) {
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
          const uint32_t c = k * kDepth + p * kRowsAtOnce + row0;
          sc[p] = k < k1 && c < a.depth ? __ldg(a.scale + c) : 0.f;
        }
      };
      const uint32_t mine = (group + kGroups - it % kGroups) % kGroups;      // the group's first stage of this item
      scales(k0 + mine);
      for (uint32_t k = k0 + mine; k < k1; k += kGroups) {
        const uint32_t i = it + k - k0, s = i % kStages;
        if (!(ok = bar_wait(full_q + 8 * Codes::bar(i), Codes::parity(i)))) break;
        Scale2 now[kPasses];
#pragma unroll
        for (int p = 0; p < kPasses; ++p) now[p] = scale2_of(sc[p]);
        scales(k + kGroups);                   // (for the group's next stage, so that their latency is hidden)
        const uint32_t from = ring + s * S::kStage + S::kA, to = from + S::kQ;
        uint32_t q[kPasses][4];
#pragma unroll
        for (int p = 0; p < kPasses; ++p)
          asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];"
                       : "=r"(q[p][0]), "=r"(q[p][1]), "=r"(q[p][2]), "=r"(q[p][3])
                       : "r"(from + (p * kRowsAtOnce + row0) * kNB + sub * 16));
#pragma unroll
        for (int p = 0; p < kPasses; ++p) {
          const uint32_t row = p * kRowsAtOnce + row0, base = to + atom * (kDepth * 128) + row * 128;
          uint32_t v[PARTS][8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            // the order of the two halves follows that of the writes
            const uint32_t word = odd ? q[p][(j >> 1) ^ 2] : q[p][j >> 1];
            if constexpr (PARTS == 1) {
              v[0][j] = decode_pair(word, (j & 1) * 2, now[p]);
            } else {
              uint32_t o[3];
              decode_pair3(word, (j & 1) * 2, now[p], o);
#pragma unroll
              for (int x = 0; x < PARTS; ++x) v[x][j] = o[x];
            }
          }
          const uint32_t x7 = row & 7, p0 = base + (((piece + odd) ^ x7) << 4), p1 = base + (((piece + 1 - odd) ^ x7) << 4);
#pragma unroll
          for (int x = 0; x < PARTS; ++x) {
            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(p0 + x * S::kB), "r"(v[x][0]), "r"(v[x][1]), "r"(v[x][2]),
                         "r"(v[x][3])
                         : "memory");
            asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(p1 + x * S::kB), "r"(v[x][4]), "r"(v[x][5]), "r"(v[x][6]),
                         "r"(v[x][7])
                         : "memory");
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the products read shared memory by another path
        __syncwarp();
        if (lane == 0) bar_arrive_leader<CG>(ready + 8 * s, ready0 + 8 * s, leader);
      }
      it += k1 - k0;
    }
    }
  } else {
    const int quad = warp & 3;
    const uint32_t freed0 = CG == 2 ? peer_addr(freed, 0) : freed;
    uint32_t n = 0, tile, k0, k1;
    for (uint32_t w = unit; ok && w < work; w += units) {
      share(w, tile, k0, k1);
      const uint32_t lanes = (uint32_t)(quad * 32) << 16, running = tmem + lanes + 2 * BN;
      const uint64_t row = (uint64_t)(tile % a.tiles_m) * 128 * CG + 128 * rank + quad * 32;
      const uint32_t col = tile / a.tiles_m * BN;
      O* out = static_cast<O*>(a.out) + row * a.ldo + col;
      float* part = w >= a.full && a.splits > 1 ? a.part + ((size_t)(w - a.full) * CG * 128 + 128 * rank + quad * 32) * BN : nullptr;
      const int rows = row >= a.m ? 0 : (int)min((uint64_t)32, a.m - row);
      constexpr int kC = 128 / sizeof(O);
      uint32_t k = k0;
      do {
        const uint32_t acc = n & 1, from = tmem + lanes + acc * BN;
        const bool first = k == k0, last = k1 - k <= (uint32_t)S::kChunk;
        ok = bar_wait(done + 8 * acc, (n >> 1) & 1);
        if (!(ok = all_of<128>(ok))) break;       // (the four warps leave together)
        mma_fence_after();
#pragma unroll 1
        for (int c = 0; c < BN; c += kC) {
          if (col + c >= a.n) break;
          float v[kC];
          load_block(from + c, v);
          if constexpr (PARTS == 3) {
            static_assert(PARTS == 1 || kC == 32, "one block of columns to a load");
            if (!first) {
              float old[32];
              load_block(running + c, old);
#pragma unroll
              for (int i = 0; i < 32; ++i) v[i] = __fadd_rn(v[i], old[i]);
            }
            if (!last) {
              uint32_t r[32];
#pragma unroll
              for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(v[i]);
              tmem_store(running + c, r);
              continue;
            }
          }
          if (part) {
#pragma unroll
            for (int i = 0; i < kC; i += 32) store_part(part + c + i, BN, v + i, lane);
          } else if (!a.aligned) {
            store_ragged(out + c, a.ldo, v, rows, (int)min((uint32_t)kC, a.n - col - c), lane, raw + (stages - smem_addr(raw)) + quad * kStageBytes);
          } else if (rows > 0) {
            store_block<O>(&map_o, (int)(col + c), (int)row, v, lane, stages + quad * kStageBytes);
          }
        }
        if (PARTS == 3) tmem_store_wait();
        mma_fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive_leader<CG>(freed + 8 * acc, freed0 + 8 * acc, leader);
        ++n;
        k += S::kChunk;
        if (last) break;
      } while (true);
    }
    store_blocks_done(lane);
  }
  asm volatile("griddepcontrol.launch_dependents;");
  if (!ok) *a.err = 1;
  __syncwarp();
  mma_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync_all();
  if (warp == 1) {
    mma_fence_after();
    tmem_free<CG>(tmem, S::kCols);
  }
}

// The operand converted beforehand: `plane` rows of ld bf16 numbers; rows from `rows` on and columns from `cols` on are
// zero.  16 columns to a thread.
__global__ void __launch_bounds__(256) q8_convert_kernel(const int8_t* q, size_t ldq, const float* scale, uint32_t rows,
                                                         uint32_t cols, uint32_t plane, __nv_bfloat16* out, size_t ld) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  const uint32_t per_row = (uint32_t)((ld + 15) / 16);
  const uint64_t id = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  const uint64_t row = id / per_row;
  if (row >= plane) return;
  const uint32_t c = (uint32_t)(id - row * per_row) * 16;
  uint32_t w[4] = {0, 0, 0, 0}, v[8];
  float sc = 0.f;
  if (row < rows) {
    const uint4 x = *reinterpret_cast<const uint4*>(q + row * ldq + c);      // (a row's pitch is a multiple of 16)
    w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
    sc = scale[row];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int left = (int)cols - (int)c - 4 * i;
      if (left < 4) w[i] &= left <= 0 ? 0u : (1u << (8 * left)) - 1;
    }
  }
  const Scale2 s = scale2_of(sc);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = decode_pair(w[j >> 1], (j & 1) * 2, s);
  __nv_bfloat16* to = out + row * ld + c;
  *reinterpret_cast<uint4*>(to) = make_uint4(v[0], v[1], v[2], v[3]);
  if (c + 8 < ld) *reinterpret_cast<uint4*>(to + 8) = make_uint4(v[4], v[5], v[6], v[7]);
}

// The shared tiles from their partial results, added in order: 4 columns to a thread.
template <class O>
__global__ void __launch_bounds__(256) q8_join_kernel(const float* part, uint32_t splits, uint32_t tile_m, uint32_t tile_n, uint32_t first,
                                                      uint32_t count, uint32_t tiles_m, uint64_t m, uint32_t n, O* out, size_t ldo, bool aligned) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const uint32_t per_row = tile_n / 4, per_tile = per_row * tile_m;
  const uint64_t id = (uint64_t)blockIdx.x * 256 + threadIdx.x;
  const uint32_t t = (uint32_t)(id / per_tile), in = (uint32_t)(id - (uint64_t)t * per_tile);
  if (t >= count) return;
  const uint64_t row = (uint64_t)((first + t) % tiles_m) * tile_m + in / per_row;
  const uint32_t col = (first + t) / tiles_m * tile_n + in % per_row * 4;
  if (row >= m || col >= n) return;
  const float4* p = reinterpret_cast<const float4*>(part) + (size_t)t * splits * per_tile + in;
  float4 s = __ldcg(p);
#pragma unroll 4
  for (uint32_t i = 1; i < splits; ++i) {
    const float4 v = __ldcg(p + (size_t)i * per_tile);
    s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
  }
  O* o = out + row * ldo + col;
  if (aligned && col + 4 <= n) {
    if constexpr (sizeof(O) == 4)
      *reinterpret_cast<float4*>(o) = s;
    else
      *reinterpret_cast<uint2*>(o) = make_uint2(bf16_pair(s.x, s.y), bf16_pair(s.z, s.w));
  } else {
    const float v[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (col + i < n) o[i] = static_cast<O>(v[i]);
  }
}

// A gradient whose rows are not aligned to 16 bytes, copied to rows that are.  A warp moves 256 columns: its lanes load the
// 16-byte pieces that hold them (the first and last may reach outside the row, never outside the piece of an element of
// it), take the next piece from the next lane and shift the two into place.
__global__ void __launch_bounds__(256) q8_pitch_kernel(const __nv_bfloat16* in, size_t ldi, uint64_t rows, uint32_t cols,
                                                       __nv_bfloat16* out, size_t ldo) {
  asm volatile("griddepcontrol.launch_dependents;");
  const uint32_t per_row = (cols + 255) / 256;
  const uint64_t id = (uint64_t)blockIdx.x * 8 + (threadIdx.x >> 5), row = id / per_row;
  if (row >= rows) return;
  const int lane = threadIdx.x & 31;
  const uint32_t base = (uint32_t)(id - row * per_row) * 256;
  const uintptr_t from = reinterpret_cast<uintptr_t>(in + row * ldi + base), end = reinterpret_cast<uintptr_t>(in + row * ldi + cols);
  const uint32_t off = from & 15;
  const uintptr_t piece = from - off + 16 * lane;
  uint4 v = make_uint4(0, 0, 0, 0), next = v;
  if (piece < end) v = *reinterpret_cast<const uint4*>(piece);
  if (lane == 31 && off && piece + 16 < end) next = *reinterpret_cast<const uint4*>(piece + 16);
  uint32_t w[8] = {v.x, v.y, v.z, v.w, __shfl_down_sync(0xffffffffu, v.x, 1), __shfl_down_sync(0xffffffffu, v.y, 1),
                   __shfl_down_sync(0xffffffffu, v.z, 1), __shfl_down_sync(0xffffffffu, v.w, 1)};
  if (lane == 31) { w[4] = next.x; w[5] = next.y; w[6] = next.z; w[7] = next.w; }
  if (off & 8) {
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  }
  if (off & 4) {
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  }
  if (off & 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
  }
  const uint32_t c = base + lane * 8;
  if (c < cols) *reinterpret_cast<uint4*>(out + row * ldo + c) = make_uint4(w[0], w[1], w[2], w[3]);
}

// ---- launches ------------------------------------------------------------------------------------------------------
struct Plan {
  int cg, bn;                // CTAs and columns of a tile
  bool conv;                 // convert inside the product
  uint32_t tiles, full, splits;      // the tiles that do not fill a round are shared by `splits` work items each
};

// Time of a plan in clock cycles.  A stage takes 4096 multiply-adds a cycle and SM (three times as many for an operand in
// three parts) or, where that is longer, the copies and the conversion; a tile costs a fixed beginning and end; partial
// results and an operand converted beforehand cost their way through memory (3000 bytes a cycle) and one more launch.
Plan plan_of(uint64_t m, uint32_t n, uint32_t depth, int parts, size_t out_elem, int sms) {
  static const int shapes[2][3][2] = {{{2, 256}, {1, 128}, {1, 64}}, {{2, 128}, {1, 64}, {1, 64}}};
  const uint32_t ksteps = (depth + kDepth - 1) / kDepth;
  Plan best = {};
  double least = 1e300;
  auto weigh = [&](int cg, int bn, bool conv, double stage, double fixed) {
    const uint64_t tiles = ((m + 128 * cg - 1) / (128 * cg)) * ((n + bn - 1) / bn), units = sms / cg, rounds = tiles / units;
    const uint64_t full = rounds * units, rest = tiles - full;
    for (uint32_t sp = 1; sp <= 32 && sp * 4 <= (ksteps < 4 ? 4 : ksteps); ++sp) {
      const double part = sp > 1 ? (double)rest * sp * cg * 128 * bn : 0.0;
      if (part * 4 > 256e6) break;      // (a quarter of a gigabyte of partial results at most)
      double c = fixed + rounds * (ksteps * stage + 2500.0);
      if (rest) c += (double)((rest * sp + units - 1) / units) * ((ksteps + sp - 1) / sp * stage + 2500.0);
      if (sp > 1) c += (part * 8 + (double)rest * cg * 128 * bn * out_elem) / 3000.0 + 4000.0;
      if (c < least) { least = c; best = {cg, bn, conv, (uint32_t)tiles, (uint32_t)(sp > 1 ? full : tiles), sp}; }
      if (!rest) break;
    }
  };
  for (const auto& sh : shapes[parts == 3]) {
    const int cg = sh[0], bn = sh[1];
    const double product = 2.0 * bn * parts, other = 200.0 + 2.5 * bn / cg * (parts == 3 ? 2 : 1) + (cg == 2 ? 150.0 : 0.0);
    weigh(cg, bn, true, product > other ? product : other, 0.0);
  }
  if (parts == 1 && (double)n * depth * 2 < 1e9) weigh(2, 256, false, 520.0, (double)n * depth * 5.0 / 3000.0 + 4000.0);
  return best;
}

struct Work {
  Plan plan;
  bool pitch;                // dy has to be copied
  size_t lddy, ldb;          // pitches of dy and of the converted operand
  uint32_t plane;
  size_t pitch_bytes, part_bytes, conv_bytes;
};
Work work_of(const GemmArgs& g, bool dw, int sms) {
  Work w;
  const uint64_t m = dw ? g.n : g.t, depth = dw ? g.t : g.n;
  const size_t e = g.out_dtype == STQ_GRAD_F32 ? 4 : 2;
  const int parts = e == 4 ? 3 : 1;
  auto up = [](size_t v, size_t to) { return (v + to - 1) / to * to; };
  w.plan = plan_of(m, g.k, (uint32_t)depth, parts, e, sms);
  w.pitch = ((g.lddy & 7) != 0 && g.t > 1) || (reinterpret_cast<uintptr_t>(g.dy) & 15) != 0;
  w.lddy = w.pitch || g.t == 1 ? up(g.n, 8) : g.lddy;
  w.pitch_bytes = w.pitch ? up(g.t * w.lddy * 2, 256) : 0;
  w.part_bytes = (size_t)(w.plan.splits > 1 ? w.plan.tiles - w.plan.full : 0) * w.plan.splits * w.plan.cg * 128 * w.plan.bn * 4;
  w.ldb = up(g.k, 8);
  w.plane = (uint32_t)up(depth, kDepth);
  w.conv_bytes = w.plan.conv ? 0 : (size_t)w.plane * w.ldb * 2;
  return w;
}

// Where the product kernel reads and writes.
struct Ends {
  const void* dy;
  const __nv_bfloat16* operand;
  float* part;
};

template <int CG, int BN, int PARTS, bool CONV, bool DW, class O>
cudaError_t launch(const GemmArgs& g, const Work& w, const Ends& at, int* err, int sms, cudaStream_t stream) {
  using S = GradShape<CG, BN, PARTS, CONV>;
  GradArgs a;
  const int8_t* q = DW ? g.xq : g.wq;
  const size_t ldq = DW ? g.ldx : g.ldw;
  a.scale = DW ? g.xs : g.ws;
  a.m = DW ? g.n : g.t;
  a.depth = (uint32_t)(DW ? g.t : g.n);
  a.n = g.k;
  a.ksteps = (a.depth + kDepth - 1) / kDepth;
  a.out = g.out;
  a.ldo = g.ldo;
  a.part = at.part;
  a.tiles = w.plan.tiles;
  a.full = w.plan.full;
  a.splits = w.plan.splits;
  a.tiles_m = (uint32_t)((a.m + 128 * CG - 1) / (128 * CG));
  a.aligned = copy_fits(g.out, g.k * sizeof(O), g.ldo * sizeof(O));
  a.err = err;
  CUtensorMap mg, mq, mo = {};
  cudaError_t e = make_tensor_map(&mg, at.dy, 2, g.t, g.n, w.lddy, DW ? 64 : 128, 64, true);
  if (e == cudaSuccess)
    e = CONV ? make_tensor_map(&mq, q, 1, a.depth, a.n, ldq, kDepth, S::kNB, false)
             : make_tensor_map(&mq, at.operand, 2, w.plane, a.n, w.ldb, kDepth, 64, true);
  if (e == cudaSuccess && a.aligned) e = make_tensor_map(&mo, g.out, sizeof(O), a.m, a.n, g.ldo, 32, 128 / sizeof(O), true);
  auto* kernel = q8_grad_kernel<CG, BN, PARTS, CONV, DW, O>;
  static std::atomic<uint64_t> seen;
  if (e == cudaSuccess) e = allow_smem(kernel, S::kSmem, g.device, seen);
  if (e != cudaSuccess) return e;
  const uint64_t items = a.full + (uint64_t)(a.tiles - a.full) * a.splits, most = sms / CG;
  return launch_with(kernel, (unsigned)(items < most ? items : most) * CG, S::kThreads, S::kSmem, CG, w.pitch || !w.plan.conv, stream, mg, mq, mo, a);
}

template <int PARTS, bool DW, class O>
cudaError_t by_shape(const GemmArgs& g, const Work& w, const Ends& at, int* err, int sms, cudaStream_t s) {
  if constexpr (PARTS == 1) {
    if (!w.plan.conv) return launch<2, 256, PARTS, false, DW, O>(g, w, at, err, sms, s);
    if (w.plan.bn == 256) return launch<2, 256, PARTS, true, DW, O>(g, w, at, err, sms, s);
    if (w.plan.bn == 128) return launch<1, 128, PARTS, true, DW, O>(g, w, at, err, sms, s);
  } else {
    if (w.plan.bn == 128) return launch<2, 128, PARTS, true, DW, O>(g, w, at, err, sms, s);
  }
  return launch<1, 64, PARTS, true, DW, O>(g, w, at, err, sms, s);
}

template <bool DW>
cudaError_t grad(const GemmArgs& g, void* ws, int sms, int* err, cudaStream_t stream, int* launches) {
  const Work w = work_of(g, DW, sms);
  const uint64_t m = DW ? g.n : g.t;
  const bool f32 = g.out_dtype == STQ_GRAD_F32;
  uint8_t* base = static_cast<uint8_t*>(ws);
  Ends at = {g.dy, nullptr, reinterpret_cast<float*>(base + w.pitch_bytes)};
  *launches = 1;
  if (w.pitch) {
    __nv_bfloat16* to = reinterpret_cast<__nv_bfloat16*>(base);
    const uint64_t items = g.t * ((g.n + 255) / 256);      // (a warp each)
    q8_pitch_kernel<<<(unsigned)((items + 7) / 8), 256, 0, stream>>>(static_cast<const __nv_bfloat16*>(g.dy), g.lddy, g.t, g.n, to, w.lddy);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    at.dy = to;
    ++*launches;
  }
  if (!w.plan.conv) {
    __nv_bfloat16* to = reinterpret_cast<__nv_bfloat16*>(base + w.pitch_bytes + w.part_bytes);
    const uint64_t items = (uint64_t)w.plane * ((w.ldb + 15) / 16);
    const cudaError_t e = launch_with(q8_convert_kernel, dim3((unsigned)((items + 255) / 256)), dim3(256), 0, 1, w.pitch, stream,
                                      DW ? g.xq : g.wq, DW ? g.ldx : g.ldw, DW ? g.xs : g.ws, (uint32_t)(DW ? g.t : g.n), g.k, w.plane, to, w.ldb);
    if (e != cudaSuccess) return e;
    at.operand = to;
    ++*launches;
  }
  cudaError_t e = f32 ? by_shape<3, DW, float>(g, w, at, err, sms, stream) : by_shape<1, DW, __nv_bfloat16>(g, w, at, err, sms, stream);
  if (e != cudaSuccess || w.plan.splits == 1) return e;
  const uint32_t count = w.plan.tiles - w.plan.full, tile_m = w.plan.cg * 128, tiles_m = (uint32_t)((m + tile_m - 1) / tile_m);
  const dim3 grid((unsigned)(((uint64_t)count * tile_m * (w.plan.bn / 4) + 255) / 256));
  e = f32 ? launch_with(q8_join_kernel<float>, grid, dim3(256), 0, 1, true, stream, (const float*)at.part, w.plan.splits, tile_m, (uint32_t)w.plan.bn,
                        w.plan.full, count, tiles_m, m, g.k, static_cast<float*>(g.out), g.ldo, rows_aligned(g.out, g.ldo * 4))
          : launch_with(q8_join_kernel<__nv_bfloat16>, grid, dim3(256), 0, 1, true, stream, (const float*)at.part, w.plan.splits, tile_m,
                        (uint32_t)w.plan.bn, w.plan.full, count, tiles_m, m, g.k, static_cast<__nv_bfloat16*>(g.out), g.ldo,
                        rows_aligned(g.out, g.ldo * 2));
  ++*launches;
  return e;
}

}  // namespace

size_t q8_grad_workspace(const GemmArgs& g, bool dw, int sms) {
  const Work w = work_of(g, dw, sms);
  return w.pitch_bytes + w.part_bytes + w.conv_bytes;
}
cudaError_t launch_q8_linear_dx(const GemmArgs& g, void* ws, int sms, int* err, cudaStream_t stream, int* launches) {
  return grad<false>(g, ws, sms, err, stream, launches);
}
cudaError_t launch_q8_linear_dw(const GemmArgs& g, void* ws, int sms, int* err, cudaStream_t stream, int* launches) {
  return grad<true>(g, ws, sms, err, stream, launches);
}

}  // namespace stq
