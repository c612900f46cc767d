// Cross entropy over a vocabulary without keeping the logits z[t][i] = x[t] . w[i] + b[i]:
//   lse[t] = log sum_i exp z[t][i],  loss[t] = lse[t] - z[t][target[t]],  dz[t][i] = dloss[t] (exp(z[t][i] - lse[t]) - [i = target[t]])
// One kernel forms the logits tile by tile in tensor memory and either reduces them (a maximum and a sum of exp a row and
// part of the vocabulary, joined by a second kernel) or, with lse known, turns them into their gradients, in bf16, for one
// piece of the vocabulary at a time; stq_vocab_grad.cu multiplies these with w and x.  The logits are formed twice that way:
// 2 t v d operations more, against 4 t v bytes held between the passes.
//
// Tokens without a loss (padding, what a masked language model does not predict) take no part: their rows are left out
// first (gather_kernel).  How many are left is known on the device alone, so every kernel reads it there.
#include <cuda_bf16.h>

#include "../../include/stq.h"
#include "stq_q8_mma.cuh"
#include "stq_q8_tma.h"
#include "stq_rowcopy.cuh"
#include "stq_vocab.h"

namespace stq {
namespace {

constexpr int kDepth = 64;             // length of the sum per stage: 128 bytes of bf16
constexpr int kStepK = 16;             // and per product instruction
constexpr uint32_t kChunk = 8;         // stages after which a logit's sum leaves the matrix unit, with more than 128 tokens
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// ---- rows ----------------------------------------------------------------------------------------------------------
constexpr int kGatherRows = 16;        // tokens to a CTA
constexpr int kScan = 8;               // targets that a thread has on the way

// Every CTA counts the targets before its tokens and in all, so that nothing has to be passed between CTAs.  That reads t^2 / 2 bytes of
// targets from the cache: 33 MB for 8192 tokens, but 0.5 GB for 32768 (48 us) and 34 GB for 262144 (2.5 ms).
__global__ void __launch_bounds__(256) gather_kernel(const GatherArgs a) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  __shared__ uint32_t sums[2][8];
  __shared__ float tops[8];
  __shared__ int32_t where[kGatherRows];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t t0 = blockIdx.x * kGatherRows;
  uint32_t before = 0, all = 0;
  float top = 0.f;
  const bool scan = a.scale && blockIdx.x == 0;
  for (uint32_t i0 = threadIdx.x; i0 < a.t; i0 += 256 * kScan) {
    int64_t to[kScan];
    float g[kScan];
#pragma unroll
    for (int j = 0; j < kScan; ++j) {
      const uint32_t i = i0 + 256 * j;
      to[j] = i < a.t ? __ldg(a.target + i) : a.ignore;
      g[j] = scan && i < a.t ? __ldg(a.dloss + i) : 0.f;
    }
#pragma unroll
    for (int j = 0; j < kScan; ++j) {
      const uint32_t counts = to[j] != a.ignore;
      all += counts;
      before += i0 + 256 * j < t0 ? counts : 0;
      if (counts) top = fmaxf(top, fabsf(g[j]));
    }
  }
  if (scan) {
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (lane == 0) tops[warp] = top;
  }
  before = __reduce_add_sync(0xffffffffu, before);
  all = __reduce_add_sync(0xffffffffu, all);
  if (lane == 0) { sums[0][warp] = before; sums[1][warp] = all; }
  __syncthreads();
  before = all = 0;
  for (int i = 0; i < 8; ++i) { before += sums[0][i]; all += sums[1][i]; }
  if (scan && threadIdx.x == 0) {
    for (int i = 1; i < 8; ++i) top = fmaxf(top, tops[i]);
    *a.scale = top > 0.f && top < INFINITY ? top : 1.f;
  }
  if (warp == 0) {
    const uint32_t t = t0 + lane;
    const bool mine = lane < kGatherRows && t < a.t, counts = mine && a.target[t] != a.ignore;
    const uint32_t mask = __ballot_sync(0xffffffffu, counts);
    const int32_t to = counts ? (int32_t)(before + __popc(mask & ((1u << lane) - 1))) : -1;
    if (lane < kGatherRows) where[lane] = to;
    if (mine) a.row[t] = to;
    if (counts) a.token[to] = t;
    if (blockIdx.x == 0 && lane == 0) *a.count = all;
  }
  __syncthreads();
  const uint16_t* x = static_cast<const uint16_t*>(a.x);
  uint16_t* out = static_cast<uint16_t*>(a.out);
  if (a.aligned) {
    const uint32_t per_row = a.d / 8;      // 16-byte pieces
    for (uint32_t i0 = threadIdx.x; i0 < kGatherRows * per_row; i0 += 256 * 4) {
      uint4 v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t i = i0 + 256 * j, r = i / per_row;
        if (i < kGatherRows * per_row && where[r] >= 0) v[j] = __ldg(reinterpret_cast<const uint4*>(x + (size_t)(t0 + r) * a.ldx) + (i - r * per_row));
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t i = i0 + 256 * j, r = i / per_row;
        if (i < kGatherRows * per_row && where[r] >= 0) *(reinterpret_cast<uint4*>(out + (size_t)where[r] * a.ldo) + (i - r * per_row)) = v[j];
      }
    }
  } else {
    const uint32_t per_row = (a.d + 255) / 256;
    for (uint32_t i0 = warp; i0 < kGatherRows * per_row; i0 += 8 * 4) {
      RowPart p[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t i = i0 + 8 * j, r = i / per_row;
        if (i < kGatherRows * per_row && where[r] >= 0) p[j].load(x + (size_t)(t0 + r) * a.ldx, a.d, (i - r * per_row) * 256, lane);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t i = i0 + 8 * j, r = i / per_row;
        if (i < kGatherRows * per_row && where[r] >= 0)
          p[j].store(x + (size_t)(t0 + r) * a.ldx, a.d, (i - r * per_row) * 256, out + (size_t)where[r] * a.ldo, lane);
      }
    }
  }
  // the rest of the last tile: what is multiplied with zeros must be finite
  const uint32_t end = min(a.most, (all + 255) / 256 * 256);
  for (uint32_t r = all + blockIdx.x; r < end; r += gridDim.x)
    for (uint32_t c = threadIdx.x * 8; c < a.ldo; c += 256 * 8) *reinterpret_cast<uint4*>(out + (size_t)r * a.ldo + c) = make_uint4(0, 0, 0, 0);
}

// ---- products ------------------------------------------------------------------------------------------------------
struct ScoreArgs {
  const uint32_t* count;
  uint32_t rows, most;
  uint32_t v0, v1, ksteps, tiles_n;
  uint32_t chunk;          // stages after which sums leave the matrix unit, a power of two
  uint32_t wide;           // entries of the vocabulary to a tile, at most BN
  int merge;               // the loss of a single tile of rows: a CTA's tiles make one part
  uint32_t stage_bytes;    // that are copied to a stage (of a CTA)
  const float* bias;
  const uint32_t* token;
  const int64_t* target;
  int64_t ignore;
  // loss
  float2* part;
  float* chosen;
  // gradients
  const float* lse;
  const float* dloss;
  const float* scale;
  float* dbias;
  size_t ldb;
  uint32_t panels;
  int* err;
};

// Warps that take results out of tensor memory, to each quarter of its lanes: with short sums the loss waits for them (for the latency
// of a maximum, of exp and of a sum that follow one another), and they need few registers.  (8192 tokens, 30000 entries, 64 and 256
// columns: 165 -> 143 and 143 -> 122 us; 4384 x 344 x 86592: 257 -> 272, there are twice as many parts to join.)
constexpr int kShort = 4, kLong = 2;
constexpr int shares_of(int planes, bool add) { return planes == 0 && !add ? kShort : kLong; }

// The matrix unit cuts its fp32 sums off instead of rounding them, always towards zero: over a sum of 4096 a logit lost 2e-6 of itself,
// and the loss 4e-6 where the vocabulary is small.  The sum therefore leaves the unit every `chunk` stages (VocabShape) and is added, rounded,
// in registers.  (The accumulators take turns, so the next part is multiplied meanwhile; 128 sums a thread leave a few registers short: 112
// bytes spilled in the loss, 152 in the gradients, 168 with dbias.)  So it is in the gradients, in one bf16 number too: what all logits of a
// row are off by alike is also in lse, and drops out of z - lse only where both passes cut off alike.  (With whole sums dx of tokens with p
// near 1 was off by 22 times what roundings explain.  They take 1 to 2 % less time: 8192 tokens, 50257 entries, 1600 columns, loss and
// gradients 4113 instead of 4168 us.)
// Sums of one part (512 columns at most) are taken from the unit as they are: the same numbers, without the registers that add parts up.
template <int CG, int BN, int PLANES, bool ADD>
struct ScoreShape {
  static constexpr int kShares = shares_of(PLANES, ADD), kWriters = 4 * kShares, kCols = BN / kShares;
  static constexpr int kThreads = 32 * (2 + kWriters);
  static constexpr int kA = 128 * kDepth * 2, kB = BN / CG * kDepth * 2, kStage = kA + kB;
  static constexpr int kOut = PLANES ? kWriters * 2 * 4096 : 0;
  static constexpr int kFit = ((PLANES ? 224 : 192) * 1024 - kOut) / kStage;      // (the loss leaves room for CTAs of the kernel after it)
  static constexpr int kStages = kFit < 8 ? kFit : 8;
  static constexpr int kSmem = kStages * kStage + kOut + 1024;
};

// Sums over the lanes: lane i gets that of v[i].
__device__ __forceinline__ float lane_sums(float (&v)[32], int lane) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const bool up = lane & o;
#pragma unroll
    for (int i = 0; i < o; ++i) {
      const float give = up ? v[i] : v[i + o], keep = up ? v[i + o] : v[i];
      v[i] = __fadd_rn(keep, __shfl_xor_sync(0xffffffffu, give, o));
    }
  }
  return v[0];
}

// PLANES = 0: the loss, else gradients; ADD: sums leave the unit in parts; SUMS: dbias, beside gradients in one number
template <int CG, int BN, int PLANES, bool ADD, bool SUMS>
__global__ void __launch_bounds__((ScoreShape<CG, BN, PLANES, ADD>::kThreads), 1)
score_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_p,
             const ScoreArgs a) {
  using S = ScoreShape<CG, BN, PLANES, ADD>;
  constexpr int kStages = S::kStages;
  extern __shared__ uint8_t raw[];
  __shared__ uint64_t bars[2 * kStages + 4];
  __shared__ uint32_t tmem_slot;
  const uint32_t ring = (smem_addr(raw) + 1023u) & ~1023u, outs = ring + kStages * S::kStage;
  // per stage: has landed (both CTAs, at the leader), is free; per accumulator: done, read (both CTAs, at the leader)
  const uint32_t full = smem_addr(bars), empty = full + 8 * kStages, done = empty + 8 * kStages, freed = done + 16;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CG == 2 ? cluster_rank() : 0;
  const bool leader = rank == 0;
  const uint32_t unit = blockIdx.x / CG, units = gridDim.x / CG;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      bar_init(full + 8 * i, 1);
      bar_init(empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      bar_init(done + 8 * i, 1);
      bar_init(freed + 8 * i, S::kWriters * CG);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc<CG>(smem_addr(&tmem_slot), 2 * BN);
  mma_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync_all();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  mma_fence_after();
  const uint32_t tmem = tmem_slot;
  const uint32_t count = a.count ? *a.count : a.rows;
  const float scale = PLANES > 0 ? *a.scale : 1.f;
  const uint32_t tiles_m = (count + 128 * CG - 1) / (128 * CG), tiles = tiles_m * a.tiles_n;

  bool ok = true;
  if (warp == 0) {
    if (elect_one()) {
      uint32_t it = 0;
      const uint32_t full0 = CG == 2 ? peer_addr(full, 0) : full;
      for (uint32_t w = unit; ok && w < tiles; w += units) {
        const int row = (int)(w % tiles_m * 128 * CG + 128 * rank), col = (int)(a.v0 + w / tiles_m * a.wide + a.wide / CG * rank);
        for (uint32_t k = 0; k < a.ksteps; ++k, ++it) {
          const uint32_t s = it % kStages, ph = (it / kStages) & 1;
          if (!(ok = bar_wait(empty + 8 * s, ph ^ 1))) break;
          const uint32_t at = ring + s * S::kStage;
          if (leader) bar_expect(full + 8 * s, CG * a.stage_bytes);
          tensor_load<CG>(at, &map_x, (int)(k * kDepth), row, full0 + 8 * s);
          tensor_load<CG>(at + S::kA, &map_w, (int)(k * kDepth), col, full0 + 8 * s);
        }
      }
      if (!ok && leader)      // leave no copy in flight
        for (uint32_t i = it > kStages ? it - kStages : 0; i < it; ++i) bar_wait(full + 8 * (i % kStages), (i / kStages) & 1);
    }
  } else if (warp == 1) {
    if (leader && elect_one()) {
      const uint32_t id = idesc(kIdescBf16, 128 * CG, (int)a.wide, false, false);
      uint32_t it = 0, n = 0;
      for (uint32_t w = unit; ok && w < tiles; w += units) {
        for (uint32_t k = 0; k < a.ksteps; ++k, ++it) {
          const uint32_t s = it % kStages, ph = (it / kStages) & 1, acc = n & 1, place = ADD ? k & (a.chunk - 1) : k;
          if (place == 0) {
            if (!(ok = bar_wait<CG == 2>(freed + 8 * acc, ((n >> 1) & 1) ^ 1))) break;
            mma_fence_after();
          }
          if (!(ok = bar_wait<CG == 2>(full + 8 * s, ph))) break;
          mma_fence_after();
          const uint64_t da = operand_desc(ring + s * S::kStage, 16, 1024), db = operand_desc(ring + s * S::kStage + S::kA, 16, 1024);
#pragma unroll
          for (int j = 0; j < kDepth / kStepK; ++j)
            mma<CG, false>(tmem + acc * BN, da + j * ((kStepK * 2) >> 4), db + j * ((kStepK * 2) >> 4), id, place != 0 || j != 0);
          mma_commit<CG>(empty + 8 * s);
          if ((ADD && place == a.chunk - 1) || k + 1 == a.ksteps) {
            mma_commit<CG>(done + 8 * acc);
            ++n;
          }
        }
      }
    }
  } else {
    const int quad = warp & 3, share = (warp - 2) / 4;
    const uint32_t freed0 = CG == 2 ? peer_addr(freed, 0) : freed;
    uint32_t n = 0, puts = 0;
    float m = -INFINITY, s = 0.f;      // the loss: maximum and sum of exp of this row over a part
    const uint32_t mine = tmem + ((uint32_t)(quad * 32) << 16) + share * S::kCols;
    // What a tile's row and columns come with.  With short sums the tiles follow one another so quickly that it would be waited for: it is
    // loaded a tile ahead, and which token the row is another tile ahead of that.  (8192 tokens, 64 columns, 30000 entries: loss 179 -> 164
    // us.  Where sums are added up there are no registers for that: 768 columns, 50257 entries, bias, 552 -> 610.)
    struct Row {
      int64_t to;
      float dloss, lse;
      float bias[S::kCols / 32];      // of column 32 i + lane
    };
    constexpr uint32_t kNone = 0xffffffffu;
    auto token_of = [&](uint32_t w) {
      if (w >= tiles) return kNone;
      const uint32_t row = w % tiles_m * 128 * CG + 128 * rank + quad * 32 + lane;
      return row >= count ? kNone : a.token ? a.token[row] : row;
    };
    auto fetch = [&](uint32_t w, uint32_t t) {
      Row r;
      r.to = t == kNone ? a.ignore : a.target[t];
      r.dloss = PLANES == 0 || t == kNone ? 0.f : a.dloss[t];
      r.lse = PLANES == 0 || t == kNone ? 0.f : a.lse[t];
      if (a.bias && w < tiles) {
        const uint32_t tile = w / tiles_m, col = a.v0 + tile * a.wide + share * S::kCols + lane, end = min(a.v1, a.v0 + (tile + 1) * a.wide);
#pragma unroll
        for (int i = 0; i < S::kCols / 32; ++i) r.bias[i] = col + 32 * i < end ? __ldg(a.bias + col + 32 * i) : 0.f;
      }
      return r;
    };
    Row next = {};
    uint32_t token = 0;
    if constexpr (!ADD) {
      next = fetch(unit, token_of(unit));
      token = token_of(unit + units);
    }
    for (uint32_t w = unit; ok && w < tiles; w += units) {
      const uint32_t row0 = w % tiles_m * 128 * CG + 128 * rank + quad * 32, row = row0 + lane;
      const uint32_t tile = w / tiles_m, col0 = a.v0 + tile * a.wide + share * S::kCols;
      // (nothing is read of rows behind the last one, or behind the stage of dw's sums that has it)
      const uint32_t end = row0 < (PLANES > 0 ? (count + kDepth - 1) / kDepth * kDepth : count) ? min(a.v1, a.v0 + (tile + 1) * a.wide) : 0;
      // this row's target, if it lies in these columns; gradients: what the row is multiplied with, and its normaliser
      const Row now = ADD ? fetch(w, token_of(w)) : next;
      if constexpr (!ADD) {
        next = fetch(w + units, token);
        token = token_of(w + 2 * units);
      }
      const bool real = now.to != a.ignore;
      const int32_t hit = real && now.to >= col0 && now.to < min(end, col0 + S::kCols) ? (int32_t)(now.to - col0) : -1;
      const float g = real ? __fdiv_rn(now.dloss, scale) : 0.f, lse = now.lse;
      float z[ADD ? S::kCols : 32];      // logits: of all columns of the tile, or of a block of them
      auto release = [&](uint32_t acc) {
        mma_fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive_leader<CG>(freed + 8 * acc, freed0 + 8 * acc, leader);
      };
      if constexpr (ADD) {
#pragma unroll
        for (int i = 0; i < S::kCols; ++i) z[i] = 0.f;
        for (uint32_t k = 0; k < a.ksteps; k += a.chunk, ++n) {
          ok = bar_wait(done + 8 * (n & 1), (n >> 1) & 1);
          if (!(ok = __all_sync(0xffffffffu, ok))) break;
          mma_fence_after();
#pragma unroll
          for (int c = 0; c < S::kCols; c += 32) {
            if (col0 + c >= end) break;
            float v[32];
            load_block(mine + (n & 1) * BN + c, v);
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              const float2 sum = __fadd2_rn(make_float2(z[c + i], z[c + i + 1]), make_float2(v[i], v[i + 1]));
              z[c + i] = sum.x;
              z[c + i + 1] = sum.y;
            }
          }
          release(n & 1);
        }
        if (!ok) break;
      } else {
        ok = bar_wait(done + 8 * (n & 1), (n >> 1) & 1);
        if (!(ok = __all_sync(0xffffffffu, ok))) break;
        mma_fence_after();
      }
      // the 32 logits from column c (a constant after unrolling) on, with their bias
      auto logits = [&](int c, float(&v)[32]) {
        if constexpr (ADD) {
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = z[c + i];
        } else {
          load_block(mine + (n & 1) * BN + c, v);
        }
        if (a.bias) {
#pragma unroll
          for (int i = 0; i < 32; ++i) v[i] = __fadd_rn(v[i], __shfl_sync(0xffffffffu, now.bias[c / 32], i));
        }
      };
      if constexpr (PLANES == 0) {
#pragma unroll
        for (int c = 0; c < S::kCols; c += 32) {
          const uint32_t col = col0 + c;
          if (col >= end) break;
          float v[32];
          logits(c, v);
          if (col + 32 > end) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (col + i >= end) v[i] = -INFINITY;
          }
          const int at = hit - c;      // (few rows have their target in the block)
          if (__any_sync(0xffffffffu, at >= 0 && at < 32)) {
            float z = 0.f;
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (at == i) z = v[i];
            if (at >= 0 && at < 32) a.chosen[row] = z;
          }
          float tops[4] = {m, m, m, m};
#pragma unroll
          for (int i = 0; i < 32; ++i) tops[i & 3] = fmaxf(tops[i & 3], v[i]);
          const float top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
          // (nothing but -inf so far, or NaN, which fmaxf passes over: measured from 0 they add 0 or NaN)
          // (subtracted before it is scaled: a logit may be the lowest number there is)
          const float ref = top == -INFINITY ? 0.f : top;
          s = s * ex2(__fmul_rn(__fadd_rn(m, -ref), kLog2e));
          float2 more[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
          const float2 less = make_float2(-ref, -ref), scale2 = make_float2(kLog2e, kLog2e);
#pragma unroll
          for (int i = 0; i < 32; i += 2) {
            const float2 e = __fmul2_rn(__fadd2_rn(make_float2(v[i], v[i + 1]), less), scale2);
            more[i / 2 & 1] = __fadd2_rn(more[i / 2 & 1], make_float2(ex2(e.x), ex2(e.y)));
          }
          s = __fadd_rn(s, __fadd_rn(__fadd_rn(more[0].x, more[0].y), __fadd_rn(more[1].x, more[1].y)));
          m = top;
        }
        const uint32_t part = a.merge ? unit : tile;
        if (!a.merge || w + units >= tiles) {
          if (row < a.most) a.part[(size_t)(S::kShares * part + share) * a.most + row] = make_float2(m, s);
          m = -INFINITY;
          s = 0.f;
        }
      } else {
        const uint32_t out = outs + (warp - 2) * 2 * 4096;
        const float2 less = make_float2(-lse, -lse), scale2 = make_float2(kLog2e, kLog2e), g2 = make_float2(g, g);
#pragma unroll
        for (int c = 0; c < S::kCols; c += 64) {
          const uint32_t col = col0 + c;
          if (col >= end) break;
          float v[64];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float(&b)[32] = *reinterpret_cast<float(*)[32]>(v + 32 * h);
            logits(c + 32 * h, b);
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              const float2 e = __fmul2_rn(__fadd2_rn(make_float2(b[i], b[i + 1]), less), scale2);
              b[i] = ex2(e.x);
              b[i + 1] = ex2(e.y);
            }
          }
          const int at = hit - c;      // (few rows have their target in the block)
          if (__any_sync(0xffffffffu, at >= 0 && at < 64)) {
#pragma unroll
            for (int i = 0; i < 64; ++i)
              if (at == i) v[i] = __fadd_rn(v[i], -1.f);
          }
#pragma unroll
          for (int i = 0; i < 64; i += 2) {
            const float2 z = __fmul2_rn(g2, make_float2(v[i], v[i + 1]));
            v[i] = z.x;
            v[i + 1] = z.y;
          }
          if (!real) {                 // (whatever the logits of a row that does not count are)
#pragma unroll
            for (int i = 0; i < 64; ++i) v[i] = 0.f;
          }
          if (col + 64 > end) {
#pragma unroll
            for (int i = 0; i < 64; ++i)
              if (col + i >= end) v[i] = 0.f;
          }
          if ((PLANES == 3 || SUMS) && a.dbias) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              float b[32];
#pragma unroll
              for (int i = 0; i < 32; ++i) b[i] = v[32 * h + i];
              const float sum = lane_sums(b, lane);
              a.dbias[(size_t)(row0 / 32) * a.ldb + (col - a.v0) + 32 * h + lane] = sum;
            }
          }
          // the next part holds what this one's rounding left (exactly: three parts of 8 bits are the 24 of fp32)
#pragma unroll
          for (int p = 0; p < PLANES; ++p) {
            put_block<__nv_bfloat16>(&map_p, 0, (int)((p * a.panels + (col - a.v0) / 64) * a.most + row0), v, lane, out, puts);
            if (p + 1 < PLANES) {
#pragma unroll
              for (int i = 0; i < 64; i += 2) {
                const uint32_t w = bf16_pair(v[i], v[i + 1]);      // (the words that have just been put)
                const float2 rest = __fadd2_rn(make_float2(v[i], v[i + 1]),
                                               make_float2(__uint_as_float((w << 16) ^ 0x80000000u), __uint_as_float((w & 0xffff0000u) ^ 0x80000000u)));
                v[i] = rest.x;
                v[i + 1] = rest.y;
              }
            }
          }
        }
      }
      if constexpr (!ADD) {
        release(n & 1);
        ++n;
      }
    }
    if constexpr (PLANES > 0) store_blocks_done(lane);
  }
  if (!ok) *a.err = 1;
  __syncwarp();
  mma_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync_all();
  if (warp == 1) {
    mma_fence_after();
    tmem_free<CG>(tmem, 2 * BN);
  }
}

__device__ __forceinline__ float2 join(float2 a, float2 b) {
  const float top = fmaxf(a.x, b.x), ref = top == -INFINITY ? 0.f : top;
  return make_float2(top, __fadd_rn(__fmul_rn(a.y, ex2((a.x - ref) * kLog2e)), __fmul_rn(b.y, ex2((b.x - ref) * kLog2e))));
}

// R tokens to a CTA: 256 / R threads share the parts of each.  The target's logit is the one that went into the sum: where the target has
// nearly all of it, lse and logit agree in all but their last bits, and what two products round differently would be the loss.  (929
// columns, loss 0.09, lse 7.6: off by 4e-6 with the logit formed apart in fp32.)  For the same reason the loss comes from the maximum, not
// from lse, whose rounding is larger.
template <int R>
__global__ void __launch_bounds__(256) finish_kernel(const VocabArgs a, const float2* part, uint32_t parts, const float* chosen, float* loss,
                                                     float* lse) {
  __shared__ float2 sums[8][R];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t t0 = blockIdx.x * R;
  constexpr int kGroups = 256 / R;
  const int mine = threadIdx.x % R, group = threadIdx.x / R;
  const uint32_t t = t0 + mine;
  // (targets and rows were there before the products began)
  const int64_t to = t < a.t ? a.target[t] : a.ignore;
  int32_t row = -1;
  if (to != a.ignore) row = a.r.row ? a.r.row[t] : (int32_t)t;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  float2 sum = make_float2(-INFINITY, 0.f);
  if (row >= 0) {
    for (uint32_t i0 = group; i0 < parts; i0 += 8 * kGroups) {
      float2 p[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        p[j] = i0 + j * kGroups < parts ? __ldcg(part + (size_t)(i0 + j * kGroups) * a.r.most + row) : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int o = 4; o > 0; o >>= 1)
#pragma unroll
        for (int j = 0; j < o; ++j) p[j] = join(p[j], p[j + o]);
      sum = join(sum, p[0]);
    }
  }
#pragma unroll
  for (int o = R; o < 32; o <<= 1) sum = join(sum, make_float2(__shfl_xor_sync(0xffffffffu, sum.x, o), __shfl_xor_sync(0xffffffffu, sum.y, o)));
  if (lane < R) sums[warp][lane] = sum;
  __syncthreads();
  if (threadIdx.x >= R || t >= a.t) return;
  for (int i = 1; i < 8; ++i) sum = join(sum, sums[i][mine]);
  float z = 0.f, top = 0.f, rest = 0.f;
  if (row >= 0) {
    // (the NaN of a target outside the vocabulary goes into lse as well: all gradients of the token are NaN)
    const bool inside = to >= 0 && to < (int64_t)a.v;
    z = inside ? __ldcg(chosen + row) : __int_as_float(0x7fc00000);
    top = !inside ? z : sum.x == -INFINITY ? 0.f : sum.x;
    rest = logf(sum.y);
  }
  lse[t] = top + rest;
  loss[t] = (top - z) + rest;
}

// ---- launches ------------------------------------------------------------------------------------------------------
// CTAs or pairs of them that a product is launched with.
uint32_t units_of(VocabShape s, uint32_t rows, uint32_t tiles_n, int sms) {
  const uint64_t items = (uint64_t)((rows + 128 * s.cg - 1) / (128 * s.cg)) * tiles_n, most = sms / s.cg;
  return (uint32_t)(items < most ? items : most);
}
bool merged(VocabShape s, uint32_t most) { return most <= 128u * s.cg; }

template <int CG, int BN, int PLANES, bool ADD, bool SUMS>
cudaError_t launch(const VocabArgs& a, VocabShape sh, ScoreArgs s, const VocabGradOut* o, int sms, cudaStream_t stream) {
  using S = ScoreShape<CG, BN, PLANES, ADD>;
  s.count = a.r.count;
  s.rows = a.r.rows;
  s.most = a.r.most;
  s.bias = a.bias;
  s.ksteps = (a.d + kDepth - 1) / kDepth;
  // few tokens: no more rows are copied than there are.  (Rows of zeros behind the matrix take longer than others: 17 tokens,
  // 1600 x 50257, 45 us with 128 rows, 30 with 17.  What a product reads behind them is what an earlier stage left, and stays in its
  // rows.)
  const uint32_t rows = CG == 1 && a.r.rows < 128 ? a.r.rows : 128;
  s.wide = sh.wide;
  s.chunk = sh.chunk;
  s.tiles_n = (s.v1 - s.v0 + s.wide - 1) / s.wide;
  s.stage_bytes = (rows + s.wide / CG) * kDepth * 2;
  CUtensorMap mx, mw, mp = {};
  cudaError_t e = make_tensor_map(&mx, a.r.x, 2, a.r.rows, a.d, a.r.ldx, rows, kDepth, true);
  if (e == cudaSuccess) e = make_tensor_map(&mw, a.w, 2, a.v, a.d, a.ldw, s.wide / CG, kDepth, true);
  if (e == cudaSuccess && o) e = make_tensor_map(&mp, o->p, 2, (uint64_t)a.r.most * o->panels * o->planes, 64, 64, 32, 64, true);
  auto* kernel = score_kernel<CG, BN, PLANES, ADD, SUMS>;
  static std::atomic<uint64_t> seen;
  if (e == cudaSuccess) e = allow_smem(kernel, S::kSmem, a.device, seen);
  if (e != cudaSuccess) return e;
  return launch_with(kernel, units_of(sh, a.r.rows, s.tiles_n, sms) * CG, S::kThreads, S::kSmem, CG, true, stream, mx, mw, mp, s);
}

template <int PLANES, bool ADD, bool SUMS>
cudaError_t by_shape(const VocabArgs& a, VocabShape sh, const ScoreArgs& s, const VocabGradOut* o, int sms, cudaStream_t stream) {
  constexpr int kPair = PLANES == 3 ? 128 : 256;
  return sh.cg == 2 ? launch<2, kPair, PLANES, ADD, SUMS>(a, sh, s, o, sms, stream)
                    : launch<1, 128, PLANES, ADD, SUMS>(a, sh, s, o, sms, stream);
}
template <int PLANES, bool SUMS = false>
cudaError_t by_length(const VocabArgs& a, VocabShape sh, const ScoreArgs& s, const VocabGradOut* o, int sms, cudaStream_t stream) {
  return a.d > sh.chunk * kDepth ? by_shape<PLANES, true, SUMS>(a, sh, s, o, sms, stream)
                                 : by_shape<PLANES, false, SUMS>(a, sh, s, o, sms, stream);
}

}  // namespace

cudaError_t launch_vocab_gather(const GatherArgs& a, cudaStream_t stream) {
  GatherArgs g = a;
  g.aligned = rows_aligned(a.x, a.ldx * 2) && a.d % 8 == 0;
  const uint32_t ctas = (a.t + kGatherRows - 1) / kGatherRows;      // (more of them for few tokens: there are rows of zeros to write)
  return launch_with(gather_kernel, dim3(ctas < 32 ? 32 : ctas), dim3(256), 0, 1, true, stream, g);
}

VocabShape vocab_shape(uint32_t rows, uint32_t v, uint32_t d, int planes, int sms, double* cost) {
  const uint32_t k = (d + kDepth - 1) / kDepth, step = planes ? 64 : 16;
  VocabShape best = {1, 128, 0};
  double least = 1e300;
  // A stage is 4096 multiply-adds a cycle and SM or, where that is longer, its copies at 62 bytes a cycle, and 400 cycles at least (the
  // ring holds six, and what is in flight must cover the memory's latency: 1 token, 1600 x 50257, 38 us in tiles of 64, 30 in tiles of
  // 128); a tile takes as long as its stages or, beside the next one's, as its results.  Of the widths, the one whose tiles fill their
  // last round best.  (`rows` are those that may count.  How many do is known on the device alone: a plan for tokens of which few count is
  // that of all.)
  for (int cg = rows > 128 ? 2 : 1; cg > 0; --cg)
    for (uint32_t wide = planes == 3 ? 128 : 128 * cg; wide >= (planes == 3 ? 128u : 64u * cg); wide -= step) {
      const uint64_t tiles = (uint64_t)((rows + 128 * cg - 1) / (128 * cg)) * ((v + wide - 1) / wide), units = sms / cg;
      const double copied = (rows < 128 ? rows : 128) * 128.0 + wide / cg * 128.0;
      double stage = 2.0 * wide > 400.0 ? 2.0 * wide : 400.0;
      if (copied / 62.0 > stage) stage = copied / 62.0;
      const double results = 500.0 + (cg == 2 ? 14.0 : 16.0) * (planes == 3 ? 2.0 : 1.0) * wide;
      // (of gradients in three parts the results take so long that a tile is the sum of both: 1024 and 4096 tokens, 256 to 2560 columns, 490
      // cycles a stage of a pair and 4000 a tile; 300 tokens, 540 of a CTA and 5000)
      if (planes == 3 && cg == 2) stage = 490.0;
      const double tile = planes == 3 ? k * stage + results : k * stage > results ? k * stage : results;
      const double c = (double)((tiles + units - 1) / units) * tile + results;
      if (c < 0.99 * least) {
        least = c;
        best = {cg, wide, 0};
      }
    }
  // (up to 128 tokens wait for memory, and have the time to add sums up twice as often: 1 token, 1600 x 50257, 0.1 us; 8192 tokens would
  // take 10 % longer)
  best.chunk = rows > 128 ? kChunk : kChunk / 2;
  if (cost) *cost = least;
  return best;
}

uint32_t vocab_parts_of_tile(uint32_t d) { return shares_of(0, d > kChunk * kDepth); }

uint32_t vocab_parts(const VocabArgs& a, VocabShape s, uint32_t most, int sms) {
  const uint32_t tiles = (a.v + s.wide - 1) / s.wide;
  return shares_of(0, a.d > s.chunk * kDepth) * (merged(s, most) ? units_of(s, most, tiles, sms) : tiles);
}

cudaError_t launch_vocab_parts(const VocabArgs& a, VocabShape sh, uint32_t most, float2* part, float* chosen, int sms, int* err,
                               cudaStream_t stream) {
  ScoreArgs s = {};
  s.v0 = 0;
  s.v1 = a.v;
  s.token = a.r.token;
  s.target = a.target;
  s.ignore = a.ignore;
  s.part = part;
  s.chosen = chosen;
  s.merge = merged(sh, most);
  s.err = err;
  return by_length<0>(a, sh, s, nullptr, sms, stream);
}

cudaError_t launch_vocab_finish(const VocabArgs& a, const float2* part, uint32_t parts, const float* chosen, float* loss, float* lse, int sms,
                                cudaStream_t stream) {
  // As many threads to a token as leave all CTAs resident at once, five to an SM.  The number of parts hardly matters to that.  (Whole losses
  // from a graph, 4, 8 and 32 tokens to a CTA: 2048 tokens, 64 columns, 30000 entries (470 parts) 33.0, 33.7 and 41.2 us, 576 columns, 8000
  // entries (63) 25.5, 25.2 and 25.9; 5000 tokens 74, 69 and 76, and 52.0, 47.4 and 48.0; 8192 tokens 120, 118 and 122, and 78, 74 and 73;
  // 16384 tokens 227, 222 and 221, and 146, 139 and 134.)
  auto go = [&](auto* kernel, uint32_t r) {
    return launch_with(kernel, dim3((a.t + r - 1) / r), dim3(256), 0, 1, true, stream, a, part, parts, chosen, loss, lse);
  };
  const uint32_t resident = 5 * sms;
  return a.t <= 4 * resident ? go(finish_kernel<4>, 4) : a.t <= 8 * resident ? go(finish_kernel<8>, 8) : go(finish_kernel<32>, 32);
}

cudaError_t launch_vocab_dlogits(const VocabArgs& a, VocabShape sh, uint32_t v0, uint32_t v1, const VocabGradOut& o, int sms, int* err,
                                 cudaStream_t stream) {
  ScoreArgs s = {};
  s.v0 = v0;
  s.v1 = v1;
  s.token = a.r.token;
  s.target = a.target;
  s.ignore = a.ignore;
  s.lse = o.lse;
  s.dloss = o.dloss;
  s.scale = a.r.scale;
  s.dbias = o.dbias;
  s.ldb = o.ldb;
  s.panels = o.panels;
  s.err = err;
  return o.planes == 3 ? by_length<3>(a, sh, s, &o, sms, stream)
         : o.dbias     ? by_length<1, true>(a, sh, s, &o, sms, stream)
                       : by_length<1>(a, sh, s, &o, sms, stream);
}

}  // namespace stq
