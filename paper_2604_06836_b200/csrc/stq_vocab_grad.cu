// Gradients of the vocabulary cross entropy from those of the logits, p (stq_vocab_scores.cu):
//   dw[i][:] = sum over rows r of p[r][i] x[r][:]      (rows of the result: entries of the vocabulary)
//   dx[r][:] = sum over entries i of p[r][i] w[i][:]   (rows of the result: tokens)
// p lies row by row, so dw reads it MN-major and dx K-major; x and w are read MN-major, as they lie.  Nothing is transposed.
//
// dw: its sum is over the tokens, complete within a piece of the vocabulary.  For a bf16 result p is bf16 too (2^-8 a term,
// random in sign, as large as the rounding of the result).  For an fp32 result p comes in three bf16 parts that are together
// exactly the fp32 gradient, and the sum leaves the matrix unit, which cuts its sums off instead of rounding them, every 128
// terms and is added, rounded, to a running sum in registers.
//
// dx: its sum is over the vocabulary, so every piece adds to it, in fp32 in memory (copies that add: nothing is read back).  It is
// bf16 at the end, so p enters as one bf16 number here, the first part where there are three.  The tiles are few (8192 x 1600:
// 112 of two blocks of rows for 74 pairs of CTAs): whole rounds of them run in step, the rest is cut into parts that run in step, and what
// is left then into ranges (stq_vocab_ranges.h).  A whole tile's sum goes to one plane, parts and ranges each to a segment of their own;
// a tile's segments are added in a fixed order at the end.
#include <cuda_bf16.h>

#include "../../include/stq.h"
#include "stq_q8.h"
#include "stq_q8_mma.cuh"
#include "stq_q8_tma.h"
#include "stq_vocab.h"
#include "stq_vocab_ranges.h"

namespace stq {
namespace {

constexpr int kDepth = 64;
constexpr int kStepK = 16;
constexpr int kWriters = 8;             // warps that take results out of tensor memory: two groups of four
constexpr int kMaxTilesN = 512;        // tiles along a row of dx

struct GradArgs {
  const uint32_t* count;
  uint32_t rows, most, panels;
  uint32_t n, bn;                      // columns of the result, and of a tile
  uint32_t units;
  // dw
  const float* scale;
  void* out;
  size_t ldo;
  uint32_t m;                          // rows of the result
  uint32_t tiles, full, splits;        // tiles from `full` on are shared by `splits` work items each
  float* part;
  int aligned;
  // dx
  uint32_t ksteps, first;              // stages of this piece and of the first one
  int begin, beside;
  int* err;
};

// MT: blocks of 128 * CG rows in a tile.  A pair's SMs take in 64 bytes a cycle each, which is what a tile of 256 x 256 needs (32 KB for
// 512 cycles of products); with two blocks of rows to one of columns it needs three quarters of that.  Both accumulators of the tensor
// memory then belong to one tile, so its results leave while nothing is multiplied: that pays where the sums are long.
template <int CG, int BN, int PARTS, int MT>
struct GradShape {
  static constexpr int kThreads = 32 * (2 + kWriters);
  static constexpr int kNB = BN / CG < 64 ? 64 : BN / CG;         // columns that are copied: whole 128-byte rows
  static constexpr int kA = 128 * kDepth * 2, kB = kDepth * kNB * 2;
  static constexpr int kStage = kA * PARTS * MT + kB;
  // A writing warp's blocks on their way out; two where there is room for them beside the stages.  (One ragged block takes 4.5 KB.)
  static constexpr int kPlaces = MT == 1 && PARTS == 1 ? 2 : 1;
  static constexpr bool kRagged = MT == 1;                        // rows that tensor copies cannot write
  static constexpr int kOut = kPlaces == 2 ? 8192 : kRagged ? kStageBytes : 4096;
  static constexpr int kFit = (224 * 1024 - kWriters * kOut) / kStage;
  static constexpr int kStages = kFit < 8 ? kFit : 8;
  static constexpr int kChunk = PARTS == 3 ? 2 : 1 << 30;         // stages to one accumulator
  static constexpr int kCols = 2 * BN;                            // two accumulators
  static constexpr int kSmem = kStages * kStage + kWriters * kOut + 1024;
  static_assert(MT == 1 || PARTS == 1, "a running sum is kept of one block of rows");
  static_assert(!kRagged || kOut >= 32 * kStageRow, "room for a ragged block");
};

// One work item: tile (its row and column), stages [k0, k1) of its sum, and where the result goes.
struct Item {
  uint32_t tile, row, col, k0, k1;
  int share;                           // number of the segment (dx) or of the partial result (dw), -1 for the whole sum
};

// DW: rows of the result are entries of the vocabulary.  O: type of dw (dx: float).
template <int CG, int BN, int PARTS, int MT, bool DW, class O>
__global__ void __launch_bounds__((GradShape<CG, BN, PARTS, MT>::kThreads), 1)
vocab_grad_kernel(const __grid_constant__ CUtensorMap map_p, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_o,
                  const __grid_constant__ CUtensorMap map_s, const GradArgs a) {
  using S = GradShape<CG, BN, PARTS, MT>;
  constexpr int kTileM = 128 * CG * MT;
  constexpr int kStages = S::kStages;
  extern __shared__ uint8_t raw[];
  __shared__ uint64_t bars[2 * kStages + 4];
  __shared__ uint32_t tmem_slot;
  const uint32_t ring = (smem_addr(raw) + 1023u) & ~1023u, outs = ring + kStages * S::kStage;
  const uint32_t full = smem_addr(bars), empty = full + 8 * kStages, done = empty + 8 * kStages, freed = done + 16;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CG == 2 ? cluster_rank() : 0;
  const bool leader = rank == 0;
  const uint32_t unit = blockIdx.x / CG;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      bar_init(full + 8 * i, 1);
      bar_init(empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      bar_init(done + 8 * i, 1);
      bar_init(freed + 8 * i, kWriters / MT * CG);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc<CG>(smem_addr(&tmem_slot), S::kCols);
  mma_fence_before();
  __syncthreads();
  if (CG == 2) cluster_sync_all();
  // dx does not need what the kernel before it, dw's, computes: once that one has begun, all that came before it is done.  It starts on
  // SMs that dw has no more work for, and ends after it (below).
  if (DW || !a.beside) asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  mma_fence_after();
  const uint32_t tmem = tmem_slot;
  const uint32_t count = a.count ? *a.count : a.rows;

  const uint32_t tiles_n = (a.n + a.bn - 1) / a.bn;
  const uint32_t ksteps = DW ? (count + kDepth - 1) / kDepth : a.ksteps;
  const Ranges ranges(DW ? 0 : count, kTileM, tiles_n, a.first, a.units);
  // calls f(item) for each of this unit's items, in order, until it returns false
  auto items = [&](auto&& f) {
    if constexpr (DW) {
      const uint32_t work = a.full + (a.tiles - a.full) * a.splits;
      for (uint32_t w = unit; w < work; w += a.units) {
        Item it = {w, 0, 0, 0, ksteps, -1};
        if (w >= a.full) {
          const uint32_t i = w - a.full, sp = i % a.splits;
          it.tile = a.full + i / a.splits;
          it.k0 = (uint32_t)((uint64_t)ksteps * sp / a.splits);
          it.k1 = (uint32_t)((uint64_t)ksteps * (sp + 1) / a.splits);
          it.share = (int)i;
        }
        it.row = it.tile / tiles_n * kTileM;      // (row by row: the tiles of a row read the same columns of p)
        it.col = it.tile % tiles_n * a.bn;
        if (!f(it)) return;
      }
    } else {
      for (uint32_t q = unit; q < ranges.whole; q += a.units)
        if (!f(Item{q, q / tiles_n * kTileM, q % tiles_n * a.bn, 0, a.ksteps, -1})) return;
      auto item = [&](uint32_t r, uint32_t k0, uint32_t k1, uint32_t segment) {
        const uint32_t q = ranges.whole + r;
        return Item{q, q / tiles_n * kTileM, q % tiles_n * a.bn, k0, k1, (int)segment};
      };
      if (unit < ranges.cut * ranges.parts) {
        const uint32_t r = unit % ranges.cut, part = unit / ranges.cut;
        if (!f(item(r, ranges.begin(part, a.ksteps), ranges.begin(part + 1, a.ksteps), ranges.segment(r) + part))) return;
      }
      if (ranges.left == 0 || unit >= ranges.U) return;
      for (uint32_t r = ranges.tile_first(unit); r <= ranges.tile_last(unit); ++r)
        if (!f(item(ranges.cut + r, ranges.begin(r, unit, a.ksteps), ranges.begin(r, unit + 1, a.ksteps), a.units + r + unit))) return;
    }
  };

  bool ok = true;
  if (warp == 0) {
    if (elect_one()) {
      uint32_t it = 0;
      const uint32_t full0 = CG == 2 ? peer_addr(full, 0) : full;
      items([&](const Item& w) {
        const int row = (int)(w.row + 128 * rank), col = (int)(w.col + a.bn / CG * rank);
        for (uint32_t k = w.k0; k < w.k1; ++k, ++it) {
          const uint32_t s = it % kStages, ph = (it / kStages) & 1;
          if (!(ok = bar_wait(empty + 8 * s, ph ^ 1))) return false;
          const uint32_t at = ring + s * S::kStage;
          const int c = (int)(k * kDepth);
          if (leader) bar_expect(full + 8 * s, CG * S::kStage);
#pragma unroll
          for (int i = 0; i < S::kNB / 64; ++i) tensor_load<CG>(at + S::kStage - S::kB + i * (kDepth * 128), &map_b, col + 64 * i, c, full0 + 8 * s);
#pragma unroll
          for (int p = 0; p < PARTS * MT; ++p) {      // (parts of a block, or blocks)
            const int r = row + (MT > 1 ? p * 128 * CG : 0), first = MT > 1 ? 0 : p * (int)a.panels;
            if constexpr (DW) {
              tensor_load<CG>(at + p * S::kA, &map_p, 0, (first + r / 64) * (int)a.most + c, full0 + 8 * s);
              tensor_load<CG>(at + p * S::kA + S::kA / 2, &map_p, 0, (first + r / 64 + 1) * (int)a.most + c, full0 + 8 * s);
            } else {
              tensor_load<CG>(at + p * S::kA, &map_p, 0, (int)k * (int)a.most + r, full0 + 8 * s);
            }
          }
        }
        return true;
      });
      if (!ok && leader)      // leave no copy in flight
        for (uint32_t i = it > kStages ? it - kStages : 0; i < it; ++i) bar_wait(full + 8 * (i % kStages), (i / kStages) & 1);
    }
  } else if (warp == 1) {
    if (leader && elect_one()) {
      const uint32_t id = idesc(kIdescBf16, 128 * CG, (int)a.bn, DW, true);
      uint32_t it = 0, n = 0;
      items([&](const Item& w) {
        for (uint32_t k = w.k0; k < w.k1; ++k, ++it) {
          const uint32_t s = it % kStages, ph = (it / kStages) & 1, place = (k - w.k0) % S::kChunk;
          const bool last = place == S::kChunk - 1 || k + 1 == w.k1;
          if (!(ok = bar_wait<CG == 2>(full + 8 * s, ph))) return false;
          const uint32_t at = ring + s * S::kStage;
          const uint64_t da = DW ? operand_desc(at, S::kA / 2, 1024) : operand_desc(at, 16, 1024);
          const uint64_t db = operand_desc(at + S::kStage - S::kB, kDepth * 128, 1024);
          constexpr uint32_t kStepA = DW ? (kStepK * 128) >> 4 : (kStepK * 2) >> 4, kStepB = (kStepK * 128) >> 4;
#pragma unroll
          for (int b = 0; b < MT; ++b) {
            // one block to a tile: the accumulators are used in turn; two: each has its own
            const uint32_t acc = MT == 1 ? n & 1 : b, use = MT == 1 ? n >> 1 : n;
            if (place == 0 && !(ok = bar_wait<CG == 2>(freed + 8 * acc, (use & 1) ^ 1))) return false;
            mma_fence_after();
#pragma unroll
            for (int p = PARTS - 1; p >= 0; --p)                  // the smallest part first
#pragma unroll
              for (int j = 0; j < kDepth / kStepK; ++j)
                mma<CG, false>(tmem + acc * BN, da + (b + p) * (S::kA >> 4) + j * kStepA, db + j * kStepB, id, place != 0 || p < PARTS - 1 || j != 0);
            if (last) mma_commit<CG>(done + 8 * acc);
          }
          mma_commit<CG>(empty + 8 * s);
          n += last;
        }
        return true;
      });
    }
  } else {
    // (a group has a block of rows or, of a single block, every other block of columns)
    const int quad = warp & 3, group = (warp - 2) / 4, block = MT == 1 ? 0 : group;
    const uint32_t lanes = (uint32_t)(quad * 32) << 16, stage = outs + (warp - 2) * S::kOut;
    const uint32_t freed0 = CG == 2 ? peer_addr(freed, 0) : freed;
    uint32_t n = 0, puts = 0;
    constexpr int kC = 128 / sizeof(O);
    const float scale = DW ? *a.scale : 1.f;
    items([&](const Item& w) {
      const uint32_t within = block * 128 * CG + 128 * rank + quad * 32, row = w.row + within;
      const uint32_t end = min(a.bn, a.n - w.col);
      const bool add = !DW && !a.begin;
      // Blocks of kC columns; the last one of a tile begins early where the tile is not a whole number of them (what is
      // written twice that way is the same, what is added must not be).
      auto blocks = [&](auto&& f) {
#pragma unroll 1
        for (uint32_t c = MT == 1 ? group * kC : 0; c < end; c += MT == 1 ? 2 * kC : kC) {
          const uint32_t over = c + kC > a.bn ? c + kC - a.bn : 0;
          f(c - over, over);
        }
      };
      auto emit = [&](uint32_t c, uint32_t over, float(&v)[kC]) {
        const uint32_t col = w.col + c;
        if constexpr (DW) {
#pragma unroll
          for (int i = 0; i < kC; ++i) v[i] = __fmul_rn(v[i], scale);
          O* out = static_cast<O*>(a.out) + (size_t)row * a.ldo + col;
          const int rows = row >= a.m ? 0 : (int)min(32u, a.m - row);
          if (w.share >= 0) {
            float* part = a.part + ((size_t)w.share * kTileM + within) * a.bn;
#pragma unroll
            for (int i = 0; i < kC; i += 32) store_part(part + c + i, a.bn, v + i, lane);
          } else if (S::kRagged && !a.aligned) {
            if (col < a.n) store_ragged(out, a.ldo, v, rows, (int)min((uint32_t)kC, a.n - col), lane, raw + (stage - smem_addr(raw)));
          } else if (rows > 0) {
            put_block<O, false, S::kPlaces>(&map_o, (int)col, (int)row, v, lane, stage, puts);
          }
        } else {
          const CUtensorMap* map = w.share < 0 ? &map_o : &map_s;
          const int x = (int)(w.share < 0 ? col : c), y = (int)(w.share < 0 ? row : (uint32_t)w.share * kTileM + within);
          if (add) {
#pragma unroll
            for (int i = 0; i < kC; ++i) v[i] = i < (int)over ? 0.f : v[i];
            put_block<float, true, S::kPlaces>(map, x, y, v, lane, stage, puts);
          } else {
            put_block<float, false, S::kPlaces>(map, x, y, v, lane, stage, puts);
          }
        }
      };
      if (w.k0 == w.k1) {                         // (no token counts, or fewer stages than shares)
        if (add) return true;
        blocks([&](uint32_t c, uint32_t over) {
          float v[kC];
#pragma unroll
          for (int i = 0; i < kC; ++i) v[i] = 0.f;
          emit(c, over, v);
        });
        return true;
      }
      float run[PARTS == 3 ? BN / 64 : 1][32];
      for (uint32_t k = w.k0; k < w.k1; k += min((uint32_t)S::kChunk, w.k1 - k), ++n) {
        const uint32_t acc = MT == 1 ? n & 1 : block, from = tmem + lanes + acc * BN;
        const bool first = k == w.k0;
        ok = bar_wait(done + 8 * acc, (MT == 1 ? n >> 1 : n) & 1);
        if (!(ok = __all_sync(0xffffffffu, ok))) return false;
        mma_fence_after();
        if constexpr (PARTS == 3) {      // to the running sum; the results leave below, while the next item is multiplied
#pragma unroll
          for (int b = 0; b < BN / 64; ++b) {
            const uint32_t c = (2 * b + group) * 32;
            if (c >= end) break;
            float v[32];
            load_block(from + c, v);
#pragma unroll
            for (int i = 0; i < 32; ++i) run[b][i] = first ? v[i] : __fadd_rn(run[b][i], v[i]);
          }
        } else {
          blocks([&](uint32_t c, uint32_t over) {
            float v[kC];
            load_block(from + c, v);
            emit(c, over, v);
          });
        }
        mma_fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive_leader<CG>(freed + 8 * acc, freed0 + 8 * acc, leader);
      }
      if constexpr (PARTS == 3) {
        static_assert(PARTS == 1 || kC == 32, "a block of columns to each part of the running sum");
#pragma unroll
        for (int b = 0; b < BN / 64; ++b) {
          const uint32_t c = (2 * b + group) * 32;
          if (c >= end) break;
          emit(c, 0, run[b]);
        }
      }
      return true;
    });
    store_blocks_done(lane);
  }
  if (!DW && a.beside) asm volatile("griddepcontrol.wait;" ::: "memory");
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

// Column sums of the partial sums of 32 rows each: 32 columns to a CTA, every eighth row to a warp.
struct DbiasArgs {
  const float* part;
  size_t ldb;
  const uint32_t* count;
  uint32_t rows;
  const float* scale;
  uint32_t cols;
  float* out;
};
__device__ __forceinline__ void dbias_block(const DbiasArgs& a, uint32_t block) {
  __shared__ float sums[8][33];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t groups = ((a.count ? *a.count : a.rows) + 31) / 32, c = block * 32 + lane;
  float s = 0.f;
  if (c < a.cols) {
#pragma unroll 4
    for (uint32_t g = warp; g < groups; g += 8) s += __ldcg(a.part + (size_t)g * a.ldb + c);
  }
  sums[warp][lane] = s;
  __syncthreads();
  if (warp != 0 || c >= a.cols) return;
  for (int i = 1; i < 8; ++i) s += sums[i][lane];
  a.out[c] = s * *a.scale;
}
__global__ void __launch_bounds__(256) dbias_kernel(const DbiasArgs a) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  dbias_block(a, blockIdx.x);
}

// dx of up to four tokens to a CTA, four columns to a thread: what the plane has of a whole tile, or the segments of one, added in order.
// (What does not depend on them was there before the kernel that writes them began: it is worked out while that one still runs.)
// CTAs behind those of the tokens have columns of dbias.
struct FinishArgs {
  const float *plane, *segments;
  size_t ldd;
  const uint32_t* count;
  uint32_t rows;
  const int32_t* row;
  uint32_t tile_m, bn, wide;      // wide: columns of a segment
  uint32_t first, units;
  const float* scale;
  uint32_t t, each, d;
  __nv_bfloat16* dx;
  size_t lddx;
  int aligned;
  uint32_t ctas;
};
__global__ void __launch_bounds__(256) dx_finish_kernel(const FinishArgs a, const DbiasArgs db) {
  if (blockIdx.x >= a.ctas) {
    asm volatile("griddepcontrol.wait;" ::: "memory");
    dbias_block(db, blockIdx.x - a.ctas);
    return;
  }
  __shared__ uint16_t start[2][kMaxTilesN];      // of a tile: its first segment,
  __shared__ uint8_t many[2][kMaxTilesN];        // and how many it has (0: it is whole)
  __shared__ int32_t row[4];
  __shared__ uint32_t lowest;
  const uint32_t count = a.count ? *a.count : a.rows, tiles_n = (a.d + a.bn - 1) / a.bn;
  const uint32_t t0 = (a.ctas - 1 - blockIdx.x) * a.each;      // (the last tiles have the most segments: they come first)
  const float scale = *a.scale;
  // (tokens that follow one another have rows in at most two tiles)
  if (threadIdx.x < 32) {
    const uint32_t i = t0 + threadIdx.x;
    const int32_t r = threadIdx.x >= a.each || i >= a.t ? -1 : a.row ? a.row[i] : (int32_t)i;
    if (threadIdx.x < 4) row[threadIdx.x] = r;
    const uint32_t lo = __reduce_min_sync(0xffffffffu, r < 0 ? 0xffffffffu : (uint32_t)r / a.tile_m);
    if (threadIdx.x == 0) lowest = lo;
  }
  __syncthreads();
  const uint32_t lo = lowest;
  if (lo != 0xffffffffu) {
    const Ranges r(count, a.tile_m, tiles_n, a.first, a.units);
    for (uint32_t i = threadIdx.x; i < 2 * tiles_n; i += 256) {
      const uint32_t m = i / tiles_n, n = i % tiles_n, q = (lo + m) * tiles_n + n;
      if (q < r.whole || q >= r.tiles) {
        many[m][n] = 0;
      } else {
        start[m][n] = (uint16_t)r.segment(q - r.whole);
        many[m][n] = (uint8_t)r.count(q - r.whole);
      }
    }
  }
  __syncthreads();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const uint32_t per_row = (a.d + 3) / 4;
  for (uint32_t i = threadIdx.x; i < a.each * per_row; i += 256) {
    const uint32_t k = i / per_row, tok = t0 + k, c = i % per_row * 4;
    if (tok >= a.t) break;
    const int32_t at = row[k];
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (at >= 0) {      // (a tile's columns are a multiple of 16: the four lie in one tile)
      const uint32_t m = at / a.tile_m - lo, col = c / a.bn, n = many[m][col];
      if (n == 0) {
        const float4 u = __ldcs(reinterpret_cast<const float4*>(a.plane + (size_t)at * a.ldd + c));
        s[0] = u.x; s[1] = u.y; s[2] = u.z; s[3] = u.w;
      } else {
        const size_t next = (size_t)a.tile_m * a.wide;
        const float* from = a.segments + start[m][col] * next + (size_t)(at % a.tile_m) * a.wide + (c - col * a.bn);
        for (uint32_t p = 0; p < n; p += 8, from += 8 * next) {
          float4 u[8];
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (p + j < n) u[j] = __ldcs(reinterpret_cast<const float4*>(from + j * next));
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (p + j < n) { s[0] += u[j].x; s[1] += u[j].y; s[2] += u[j].z; s[3] += u[j].w; }
        }
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] *= scale;
    }
    __nv_bfloat16* to = a.dx + (size_t)tok * a.lddx + c;
    if (a.aligned && c + 4 <= a.d) {
      *reinterpret_cast<uint2*>(to) = make_uint2(bf16_pair(s[0], s[1]), bf16_pair(s[2], s[3]));
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (c + j < a.d) to[j] = __float2bfloat16_rn(s[j]);
    }
  }
}

// ---- launches ------------------------------------------------------------------------------------------------------
uint32_t up(uint32_t v, uint32_t to) { return (v + to - 1) / to * to; }

// Columns of a tile: as many equal tiles as the widest allowed makes necessary.
uint32_t tile_columns(uint32_t n, uint32_t widest, uint32_t unit) {
  const uint32_t tiles = (n + widest - 1) / widest, bn = up((n + tiles - 1) / tiles, unit);
  return bn < 64 ? 64 : bn;
}

struct DwPlan {
  int cg, mt;
  uint32_t bn, tiles_m, tiles, full, splits;
  double cost;
};
// Time of a plan in clock cycles, as for the 8-bit products: a stage is 4096 multiply-adds a cycle and SM, a tile has a beginning
// and an end, partial results go through memory once more.  It goes by the tokens that may count, since how many do is known on the device
// alone (4096 tokens, 85 % masked: 64 stages in the plan, 10 in the run).
DwPlan dw_plan(const VocabDw& a, int sms) {
  const uint32_t ksteps = (a.r.most + kDepth - 1) / kDepth;
  // CTAs, widest tile, blocks of rows; time of the copies of a stage
  const struct { int cg, bn, mt; double copies; } shapes[2][3] = {{{2, 256, 2, 800.0}, {2, 256, 1, 530.0}, {1, 128, 1, 530.0}},
                                                                  {{2, 128, 1, 930.0}, {1, 64, 1, 930.0}, {0, 0, 0, 0.0}}};
  const int parts = a.f32 ? 3 : 1;
  const size_t e = a.f32 ? 4 : 2;
  DwPlan best = {};
  double least = 1e300;
  for (const auto& sh : shapes[a.f32]) {
    if (sh.cg == 0 || (sh.mt > 1 && !copy_fits(a.dw, a.d * e, a.lddw * e))) continue;      // (two blocks of rows: no room for ragged ones)
    const uint32_t tile_m = 128 * sh.cg * sh.mt;
    DwPlan p = {sh.cg, sh.mt, tile_columns(a.d, sh.bn, a.f32 ? 32 : 16), (a.cols + tile_m - 1) / tile_m, 0, 0, 0, 0.0};
    p.tiles = p.tiles_m * ((a.d + p.bn - 1) / p.bn);
    const double products = 2.0 * p.bn * parts * sh.mt, stage = products > sh.copies ? products : sh.copies;
    const uint64_t units = sms / p.cg, rounds = p.tiles / units, full = rounds * units, rest = p.tiles - full;
    for (uint32_t sp = 1; sp <= 32 && sp * 4 <= (ksteps < 4 ? 4 : ksteps); ++sp) {
      const double part = sp > 1 ? (double)rest * sp * tile_m * p.bn : 0.0;
      if (part * 4 > 128e6) break;      // (an eighth of a gigabyte of partial results at most)
      const double ends = 2500.0 * sh.mt;
      double c = rounds * (ksteps * stage + ends);
      if (rest) c += (double)((rest * sp + units - 1) / units) * ((ksteps + sp - 1) / sp * stage + ends);
      if (sp > 1) c += (part * 8 + (double)rest * tile_m * p.bn * e) / 3000.0 + 4000.0;
      if (c < least) {
        least = c;
        best = p;
        best.full = (uint32_t)(sp > 1 ? full : p.tiles);
        best.splits = sp;
        best.cost = c;
      }
      if (!rest) break;
    }
  }
  return best;
}

template <int CG, int BN, int PARTS, int MT, bool DW, class O>
cudaError_t launch(const VocabRows& r, const void* p, uint32_t panels, const void* b, uint64_t b_rows, uint32_t b_cols, size_t ldb, void* out,
                   uint64_t out_rows, size_t ldo, void* segments, uint64_t items, GradArgs g, int device, int sms, int* err, cudaStream_t stream) {
  using S = GradShape<CG, BN, PARTS, MT>;
  g.count = r.count;
  g.rows = r.rows;
  g.most = r.most;
  g.panels = panels;
  g.scale = r.scale;
  g.err = err;
  const uint64_t most = sms / CG;
  g.units = (uint32_t)(items < most ? items : most);
  CUtensorMap mp, mb, mo = {}, ms = {};
  cudaError_t e = make_tensor_map(&mp, p, 2, (uint64_t)r.most * panels * PARTS, 64, 64, DW ? 64 : 128, 64, true);
  if (e == cudaSuccess) e = make_tensor_map(&mb, b, 2, b_rows, b_cols, ldb, 64, 64, true);
  if (e == cudaSuccess && (!DW || g.aligned)) e = make_tensor_map(&mo, out, sizeof(O), out_rows, DW ? g.n : ldo, ldo, 32, 128 / sizeof(O), true);
  if (e == cudaSuccess && !DW) e = make_tensor_map(&ms, segments, 4, (uint64_t)Ranges::segments(sms / CG) * 128 * CG * MT, BN, BN, 32, 32, true);
  auto* kernel = vocab_grad_kernel<CG, BN, PARTS, MT, DW, O>;
  static std::atomic<uint64_t> seen;
  if (e == cudaSuccess) e = allow_smem(kernel, S::kSmem, device, seen);
  if (e != cudaSuccess) return e;
  return launch_with(kernel, g.units * CG, S::kThreads, S::kSmem, CG, true, stream, mp, mb, mo, ms, g);
}

DbiasArgs dbias_args(const VocabDbias& a, const VocabRows& r) { return {a.part, a.ldb, r.count, r.rows, r.scale, a.cols, a.out}; }

// Tiles of dx: a CTA's for few tokens, a pair's else, with one block of rows or two (dx_blocks).
struct DxShape {
  int cg, mt;
  uint32_t bn;
  uint32_t tile_m() const { return 128u * cg * mt; }
  uint32_t widest() const { return 128u * cg; }
};
DxShape dx_shape(uint32_t most, uint32_t d, int sms) {
  const int cg = most > 128 ? 2 : 1;
  const uint32_t bn = tile_columns(d, 128 * cg, 16);
  return {cg, cg == 2 ? dx_blocks(most, 256, (d + bn - 1) / bn, sms / 2) : 1, bn};
}

}  // namespace

size_t vocab_dw_partial(const VocabDw& a, int sms) {
  const DwPlan p = dw_plan(a, sms);
  return p.splits > 1 ? (size_t)(p.tiles - p.full) * p.splits * p.cg * p.mt * 128 * p.bn : 0;
}

double vocab_dw_cost(const VocabDw& a, int sms) { return dw_plan(a, sms).cost; }

cudaError_t launch_vocab_dw(const VocabDw& a, float* part, int sms, int* err, cudaStream_t stream) {
  const DwPlan p = dw_plan(a, sms);
  GradArgs g = {};
  g.n = a.d;
  g.bn = p.bn;
  g.out = a.dw;
  g.ldo = a.lddw;
  g.m = a.cols;
  g.tiles = p.tiles;
  g.full = p.full;
  g.splits = p.splits;
  g.part = part;
  const size_t e = a.f32 ? 4 : 2;
  g.aligned = copy_fits(a.dw, a.d * e, a.lddw * e);
  const uint64_t items = p.full + (uint64_t)(p.tiles - p.full) * p.splits;
  cudaError_t rc;
  const auto go = [&](auto launch_fn) {
    return launch_fn(a.r, a.p, a.panels, a.r.x, (uint64_t)a.r.rows, a.d, a.r.ldx, a.dw, (uint64_t)a.cols, a.lddw, nullptr, items, g, a.device, sms, err, stream);
  };
  if (a.f32)
    rc = p.cg == 2 ? go(launch<2, 128, 3, 1, true, float>) : go(launch<1, 64, 3, 1, true, float>);
  else
    rc = p.mt == 2   ? go(launch<2, 256, 1, 2, true, __nv_bfloat16>)
         : p.cg == 2 ? go(launch<2, 256, 1, 1, true, __nv_bfloat16>)
                     : go(launch<1, 128, 1, 1, true, __nv_bfloat16>);
  return rc;
}

cudaError_t launch_vocab_dw_join(const VocabDw& a, const float* part, int sms, cudaStream_t stream, int* launches) {
  const DwPlan p = dw_plan(a, sms);
  if (p.splits == 1) return cudaSuccess;
  ++*launches;
  return launch_join(part, p.splits, p.cg * p.mt * 128, p.bn, p.full, p.tiles - p.full, p.tiles / p.tiles_m, true, a.cols, a.d, a.dw, a.lddw, a.f32, stream);
}

void vocab_dx_space(uint32_t most, uint32_t d, size_t ldd, int sms, size_t* plane, size_t* segments) {
  const DxShape s = dx_shape(most, d, sms);
  *plane = (size_t)up(most, s.tile_m()) * ldd;
  *segments = (size_t)Ranges::segments(sms / s.cg) * s.tile_m() * s.widest();
}

cudaError_t launch_vocab_dx(const VocabDx& a, int sms, int* err, cudaStream_t stream) {
  const DxShape s = dx_shape(a.r.most, a.d, sms);
  GradArgs g = {};
  g.n = a.d;
  g.bn = s.bn;
  g.ksteps = (a.cols + kDepth - 1) / kDepth;
  g.first = (a.first + kDepth - 1) / kDepth;
  g.begin = a.begin;
  g.beside = a.beside;
  const auto go = [&](auto launch_fn) {
    return launch_fn(a.r, a.p, a.panels, a.w, (uint64_t)a.cols, a.d, a.ldw, a.plane, (uint64_t)up(a.r.most, s.tile_m()), a.ldd, a.segments,
                     (uint64_t)(sms / s.cg), g, a.device, sms, err, stream);
  };
  return s.mt == 2 ? go(launch<2, 256, 1, 2, false, float>) : s.cg == 2 ? go(launch<2, 256, 1, 1, false, float>) : go(launch<1, 128, 1, 1, false, float>);
}

cudaError_t launch_vocab_dx_finish(const VocabDx& a, uint32_t t, void* dx, size_t lddx, const VocabDbias* db, int sms, cudaStream_t stream) {
  const DxShape s = dx_shape(a.r.most, a.d, sms);
  // (few tokens: as many CTAs as there are SMs, to have enough loads on the way)
  uint32_t each = t / (4 * sms) < 1 ? 1 : t / (4 * sms);
  if (each > 4) each = 4;
  FinishArgs f;
  f.plane = a.plane;
  f.segments = a.segments;
  f.ldd = a.ldd;
  f.count = a.r.count;
  f.rows = a.r.rows;
  f.row = a.r.row;
  f.tile_m = s.tile_m();
  f.bn = s.bn;
  f.wide = s.widest();
  f.first = (a.first + kDepth - 1) / kDepth;
  f.units = (uint32_t)(sms / s.cg);
  f.scale = a.r.scale;
  f.t = t;
  f.each = each;
  f.d = a.d;
  f.dx = static_cast<__nv_bfloat16*>(dx);
  f.lddx = lddx;
  f.aligned = rows_aligned(dx, lddx * 2);
  f.ctas = (t + each - 1) / each;
  const DbiasArgs d = db ? dbias_args(*db, a.r) : DbiasArgs{};
  return launch_with(dx_finish_kernel, dim3(f.ctas + (d.cols + 31) / 32), dim3(256), 0, 1, true, stream, f, d);
}

cudaError_t launch_vocab_dbias(const VocabDbias& a, const VocabRows& r, cudaStream_t stream) {
  return launch_with(dbias_kernel, dim3((a.cols + 31) / 32), dim3(256), 0, 1, true, stream, dbias_args(a, r));
}

}  // namespace stq
