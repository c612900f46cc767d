// out[t][n] = xs[t] * ws[n] * sum_k xq[t][k] * wq[n][k] (+ bias[n]): products of 8-bit rows, sums in exact 32-bit integers.
//
// Four kernels, by the number of tokens (see by_shape):
//  - a batch: pairs of CTAs own tiles of 256 tokens x 128 or 256 channels and walk a list of them (q8_linear_kernel);
//  - tens to hundreds of tokens: one tile of 128 tokens x 32 to 128 channels to a cluster, whose CTAs share the sum
//    (q8_linear_split_kernel);
//  - up to 16 tokens: the weight is streamed from memory straight into register fragments (q8_linear_stream_kernel);
//  - one token: it is streamed through the integer dot products of the CUDA cores (q8_linear_few_kernel).
#include "../../include/stq.h"
#include "stq_internal.h"
#include "stq_q8.h"
#include "stq_q8_mma.cuh"
#include "stq_q8_tma.h"

namespace stq {
namespace {

constexpr int kBK = 128;               // bytes (= elements) of the sum per stage
constexpr int kMmaK = 32;              // elements of the sum per product instruction
constexpr int kThreads8 = 192;         // split kernel: two working warps and four that write
constexpr int kWriters = 8;            // pairs: writing warps, two to each quarter of the rows

struct LinearArgs {
  const float* xs;
  const float* ws;
  const float* bias;
  void* out;
  size_t ldo;
  uint64_t t;
  uint32_t n, ksteps;
  uint32_t tiles_m, tiles_n;
  uint32_t box;                        // split kernel: tokens per tensor copy
  int aligned;                         // tensor copies can write `out`: map_o describes it
  int* err;
};

// A result from its integer sum, the same in every kernel.  The scales are applied one after the other: their product may
// leave the range of fp32 where the result does not (two small scales lose digits, two large ones make a sum of 0 a NaN).
__device__ __forceinline__ float scaled(int sum, float xs, float ws, float bias) { return fmaf((float)sum * xs, ws, bias); }

// ---- batches ---------------------------------------------------------------------------------------------------------
// Warp 0 keeps a ring of shared-memory stages full with tensor copies (128 bytes of the sum at a time, 128-byte swizzle,
// out-of-range rows and columns read as zero), warp 1 issues the products into one of two accumulators in tensor
// memory, warps 2-9 turn the other accumulator into results.  Each CTA of a pair holds 128 tokens and half of the
// channels of the tile; the leader issues the products of both.  Where a tile has few stages the writing bounds the
// kernel: with four warps and stores by row it took as long as 20 stages of products; eight warps and tensor copies of
// whole lines take 8192 x 768 x 2304 from 22.7 to 17.1 us and 8192 x 1600 x 6400 (13 stages) from 84 to 76 at the power cap.
template <int BN>
struct LinearShape {
  static constexpr int kA = 128 * kBK, kB = BN / 2 * kBK, kStage = kA + kB;
  static constexpr int kFit = (180 * 1024) / kStage;
  static constexpr int kStages = kFit < 8 ? kFit : 8;
  static constexpr int kCols = 2 * BN;                         // tensor memory: two accumulators
  static constexpr int kSmem = kStages * kStage + kWriters * kStageBytes + 1024;      // (+ alignment of the swizzle atoms)
};

template <int BN, class O>
__global__ void __launch_bounds__(64 + 32 * kWriters, 1)
q8_linear_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_o,
                 const LinearArgs a) {
  using S = LinearShape<BN>;
  constexpr int kStages = S::kStages;
  extern __shared__ uint8_t raw[];
  __shared__ uint64_t bars[2 * kStages + 4];
  __shared__ uint32_t tmem_slot;
  __shared__ float4 scale_n[2][BN / 4], bias_n[2][BN / 4];
  const uint32_t ring = (smem_addr(raw) + 1023u) & ~1023u, stages = ring + kStages * S::kStage;
  const uint32_t full = smem_addr(bars), empty = full + 8 * kStages, done = empty + 8 * kStages;
  const uint32_t freed = done + 16;      // accumulators are read (both CTAs, at the leader)
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_rank();
  const bool leader = rank == 0;
  const uint32_t unit = blockIdx.x / 2, units = gridDim.x / 2, tiles = a.tiles_m * a.tiles_n;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      bar_init(full + 8 * i, 1);
      bar_init(empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      bar_init(done + 8 * i, 1);
      bar_init(freed + 8 * i, 2 * kWriters);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc<2>(smem_addr(&tmem_slot), S::kCols);
  mma_fence_before();
  __syncthreads();
  cluster_sync_all();
  mma_fence_after();
  const uint32_t tmem = tmem_slot;

  bool ok = true;
  if (warp == 0) {
    if (elect_one()) {
      uint32_t it = 0;
      const uint32_t full0 = peer_addr(full, 0);
      for (uint32_t tile = unit; ok && tile < tiles; tile += units) {
        const int row = (int)(tile % a.tiles_m) * 256 + 128 * rank, col = (int)(tile / a.tiles_m) * BN + (BN / 2) * rank;
        for (uint32_t k = 0; k < a.ksteps; ++k, ++it) {
          const uint32_t s = it % kStages, ph = (it / kStages) & 1;
          if (!(ok = bar_wait(empty + 8 * s, ph ^ 1))) break;
          if (leader) bar_expect(full + 8 * s, 2 * S::kStage);
          const uint32_t at = ring + s * S::kStage;
          tensor_load<2>(at, &map_x, (int)k * kBK, row, full0 + 8 * s);
          tensor_load<2>(at + S::kA, &map_w, (int)k * kBK, col, full0 + 8 * s);
        }
      }
      if (!ok && leader)      // leave no copy in flight
        for (uint32_t i = it > kStages ? it - kStages : 0; i < it; ++i) bar_wait<true>(full + 8 * (i % kStages), (i / kStages) & 1);
    }
  } else if (warp == 1) {
    if (leader && elect_one()) {
      constexpr uint32_t id = idesc(kIdescI8, 256, BN, false, false);
      uint32_t it = 0, n = 0;
      for (uint32_t tile = unit; ok && tile < tiles; tile += units, ++n) {
        const uint32_t acc = n & 1;
        if (!(ok = bar_wait<true>(freed + 8 * acc, ((n >> 1) & 1) ^ 1))) break;
        mma_fence_after();
        for (uint32_t k = 0; k < a.ksteps; ++k, ++it) {
          const uint32_t s = it % kStages, ph = (it / kStages) & 1;
          if (!(ok = bar_wait<true>(full + 8 * s, ph))) break;
          mma_fence_after();
          const uint32_t at = ring + s * S::kStage;
          const uint64_t da = operand_desc(at, 16, 1024), db = operand_desc(at + S::kA, 16, 1024);
#pragma unroll
          for (int j = 0; j < kBK / kMmaK; ++j)
            mma<2, true>(tmem + acc * BN, da + j * (kMmaK >> 4), db + j * (kMmaK >> 4), id, (k | j) != 0);
          mma_commit<2>(empty + 8 * s);
        }
        if (ok) mma_commit<2>(done + 8 * acc);
      }
    }
  } else {
    // a warp reaches the 32 lanes 32 * (warp % 4) of tensor memory; it takes half of their columns
    const int quad = warp & 3, half = (warp - 2) / 4, thread = threadIdx.x - 64;
    const uint32_t freed0 = peer_addr(freed, 0);
    uint32_t n = 0;
    for (uint32_t tile = unit; ok && tile < tiles; tile += units, ++n) {
      const uint32_t acc = n & 1;
      const uint64_t row = (uint64_t)(tile % a.tiles_m) * 256 + 128 * rank + quad * 32;
      const uint32_t col = tile / a.tiles_m * BN;
      for (int c = thread; c < BN; c += 32 * kWriters) {
        reinterpret_cast<float*>(scale_n[acc])[c] = col + c < a.n ? a.ws[col + c] : 0.f;
        reinterpret_cast<float*>(bias_n[acc])[c] = a.bias && col + c < a.n ? a.bias[col + c] : 0.f;
      }
      const float xs = row + lane < a.t ? a.xs[row + lane] : 0.f;
      ok = bar_wait(done + 8 * acc, (n >> 1) & 1);
      if (!(ok = all_of<32 * kWriters>(ok))) break;       // (the writing warps leave together; the scales above are visible to all)
      mma_fence_after();
      const uint32_t from = tmem + ((uint32_t)(quad * 32) << 16) + acc * BN;
      O* out = static_cast<O*>(a.out) + row * a.ldo + col;
      const int rows = row >= a.t ? 0 : (int)min((uint64_t)32, a.t - row);
      constexpr int kC = 128 / sizeof(O);
#pragma unroll 1
      for (int c = half * (BN / 2); c < (half + 1) * (BN / 2); c += kC) {
        if (col + c >= a.n) break;
        float v[kC];
        load_block(from + c, v);
#pragma unroll
        for (int i = 0; i < kC; i += 4) {
          const float4 ws = scale_n[acc][(c + i) / 4], b = bias_n[acc][(c + i) / 4];
          v[i] = scaled(__float_as_int(v[i]), xs, ws.x, b.x);
          v[i + 1] = scaled(__float_as_int(v[i + 1]), xs, ws.y, b.y);
          v[i + 2] = scaled(__float_as_int(v[i + 2]), xs, ws.z, b.z);
          v[i + 3] = scaled(__float_as_int(v[i + 3]), xs, ws.w, b.w);
        }
        if (!a.aligned)
          store_ragged(out + c, a.ldo, v, rows, (int)min((uint32_t)kC, a.n - col - c), lane, raw + (stages - smem_addr(raw)) + (warp - 2) * kStageBytes);
        else if (rows > 0)
          store_block<O>(&map_o, (int)(col + c), (int)row, v, lane, stages + (warp - 2) * kStageBytes);
      }
      mma_fence_before();
      __syncwarp();
      if (lane == 0) bar_arrive_leader<2>(freed + 8 * acc, freed0 + 8 * acc, leader);
    }
    store_blocks_done(lane);
  }
  if (!ok) *a.err = 1;
  __syncwarp();
  mma_fence_before();
  __syncthreads();
  cluster_sync_all();
  if (warp == 1) {
    mma_fence_after();
    tmem_free<2>(tmem, S::kCols);
  }
}

// ---- tens to hundreds of tokens ------------------------------------------------------------------------------------------
// A cluster owns a tile of 128 tokens x BN channels; its CTAs each take a share of the sum.  Their integer partial sums
// meet in shared memory: CTA j collects columns [j, j + 1) * BN / size from all, adds them (in any order: integers) and
// writes the results, a warp to a row.
template <int BN>
struct SplitShape {
  static constexpr int kA = 128 * kBK, kB = BN * kBK, kStage = kA + kB;
  static constexpr int kFit = (140 * 1024) / kStage;
  static constexpr int kStages = kFit < 6 ? kFit : 6;
  static constexpr int kMeet = 128 * (BN + 4 * 8) * 4;         // rows of BN / size + 4 words from each of up to 8 CTAs
  static constexpr int kSmem = kStages * kStage + kMeet + 1024;
};

template <int BN, class O>
__global__ void __launch_bounds__(kThreads8, 1)
q8_linear_split_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const LinearArgs a, int log_size) {
  using S = SplitShape<BN>;
  constexpr int kLog = BN == 128 ? 7 : BN == 64 ? 6 : 5;
  constexpr int kStages = S::kStages;
  extern __shared__ uint8_t raw[];
  __shared__ uint64_t bars[2 * kStages + 1];
  __shared__ uint32_t tmem_slot;
  __shared__ float scale_t[128];
  const int size = 1 << log_size;
  const uint32_t ring = (smem_addr(raw) + 1023u) & ~1023u, meet = ring + kStages * S::kStage;
  const uint32_t full = smem_addr(bars), empty = full + 8 * kStages, done = empty + 8 * kStages;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = size > 1 ? cluster_rank() : 0, tile = blockIdx.x >> log_size;
  const uint32_t row0 = tile % a.tiles_m * 128, col0 = tile / a.tiles_m * BN;
  const uint32_t k0 = a.ksteps * rank >> log_size, k1 = a.ksteps * (rank + 1) >> log_size;
  const int rows = (int)min((uint64_t)128, a.t - row0), slice = BN >> log_size, pitch = slice + 4;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      bar_init(full + 8 * i, 1);
      bar_init(empty + 8 * i, 1);
    }
    bar_init(done, 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc<1>(smem_addr(&tmem_slot), BN);
  mma_fence_before();
  __syncthreads();
  mma_fence_after();
  if (size > 1) cluster_arrive();
  const uint32_t tmem = tmem_slot;

  bool ok = true;
  if (warp == 0) {
    if (elect_one()) {
      uint32_t it = 0;
      const uint32_t boxes = (rows + a.box - 1) / a.box;      // (the rest of the tile's rows keep what they hold: not used)
      for (uint32_t k = k0; k < k1; ++k, ++it) {
        const uint32_t s = it % kStages, ph = (it / kStages) & 1;
        if (!(ok = bar_wait(empty + 8 * s, ph ^ 1))) break;
        bar_expect(full + 8 * s, S::kB + boxes * a.box * kBK);
        const uint32_t at = ring + s * S::kStage;
        tensor_load<1>(at + S::kA, &map_w, (int)k * kBK, (int)col0, full + 8 * s);
        for (uint32_t b = 0; b < boxes; ++b)
          tensor_load<1>(at + b * a.box * kBK, &map_x, (int)k * kBK, (int)(row0 + b * a.box), full + 8 * s);
      }
      if (!ok)      // leave no copy in flight
        for (uint32_t i = it > kStages ? it - kStages : 0; i < it; ++i) bar_wait(full + 8 * (i % kStages), (i / kStages) & 1);
    }
  } else if (warp == 1) {
    if (elect_one()) {
      constexpr uint32_t id = idesc(kIdescI8, 128, BN, false, false);
      uint32_t it = 0;
      for (uint32_t k = k0; k < k1; ++k, ++it) {
        const uint32_t s = it % kStages, ph = (it / kStages) & 1;
        if (!(ok = bar_wait(full + 8 * s, ph))) break;
        mma_fence_after();
        const uint32_t at = ring + s * S::kStage;
        const uint64_t da = operand_desc(at, 16, 1024), db = operand_desc(at + S::kA, 16, 1024);
#pragma unroll
        for (int j = 0; j < kBK / kMmaK; ++j) mma<1, true>(tmem, da + j * (kMmaK >> 4), db + j * (kMmaK >> 4), id, (it | j) != 0);
        mma_commit<1>(empty + 8 * s);
      }
      if (ok) mma_commit<1>(done);
    }
  } else {
    const int quad = warp & 3, row = quad * 32 + lane;
    scale_t[row] = row < rows ? a.xs[row0 + row] : 0.f;
    if (size > 1) cluster_wait();                  // (all CTAs of the cluster have started)
    if (quad * 32 < rows && (ok = bar_wait(done, 0))) {
      mma_fence_after();
      const uint32_t from = tmem + ((uint32_t)(quad * 32) << 16);
#pragma unroll 1
      for (int c = 0; c < BN; c += 32) {
        uint32_t r[32];
        tmem_load(from + c, r);
        tmem_load_wait();
#pragma unroll
        for (int i = 0; i < 32; i += 4) {
          const int to = (c + i) >> (kLog - log_size), at = (c + i) & (slice - 1);
          const uint32_t local = meet + (((int)rank * 128 + row) * pitch + at) * 4;
          const uint32_t addr = size > 1 ? peer_addr(local, to) : local;
          asm volatile("st.shared::cluster.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3])
                       : "memory");
        }
      }
    }
  }
  __syncwarp();
  if (size > 1 && warp < 2) cluster_wait();
  mma_fence_before();
  if (size > 1)
    cluster_sync_all();
  else
    __syncthreads();
  // A warp takes the slice's columns, 32 at a time, or several rows where the slice is narrower.
  const uint32_t c0 = col0 + slice * rank;
  const int width = slice < 32 ? slice : 32, per = 32 / width, sub = lane / width;
  for (int c = lane & (width - 1); c < slice; c += 32) {
    const bool in = c0 + c < a.n;
    const float ws = in ? a.ws[c0 + c] : 0.f, b = in && a.bias ? a.bias[c0 + c] : 0.f;
#pragma unroll 4
    for (int row = warp * per + sub; row < rows; row += 6 * per) {
      int sum = 0;
#pragma unroll
      for (int p = 0; p < 8; ++p) {
        int x = 0;
        if (p < size) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(meet + ((p * 128 + row) * pitch + c) * 4));
        sum += x;
      }
      if (in) static_cast<O*>(a.out)[(size_t)(row0 + row) * a.ldo + c0 + c] = static_cast<O>(scaled(sum, scale_t[row], ws, b));
    }
  }
  if (!ok) *a.err = 1;
  __syncthreads();
  if (warp == 1) {
    mma_fence_after();
    tmem_free<1>(tmem, BN);
  }
}

// ---- one token -------------------------------------------------------------------------------------------------------
// T tokens' codes lie in shared memory; a warp takes R channels at a time, 16 bytes of each to a lane and step, U steps
// in flight.  Bound by the reading of the weight.
template <int T, int R, class O>
__global__ void __launch_bounds__(256) q8_linear_few_kernel(const int8_t* xq, size_t ldx, const int8_t* wq, size_t ldw, uint32_t k,
                                                            const LinearArgs a) {
  constexpr int U = 4;
  extern __shared__ uint4 x[];                     // [T][pieces]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t pieces = (k + 15) / 16, n0 = (blockIdx.x * 8 + warp) * R;
  uint4 w[U][R];
  auto fetch = [&](uint32_t base) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const uint32_t p = base + u * 32 + lane;
        w[u][r] = make_uint4(0, 0, 0, 0);
        if (p < pieces && n0 + r < a.n) w[u][r] = reinterpret_cast<const uint4*>(wq + (size_t)(n0 + r) * ldw)[p];
      }
  };
  fetch(0);                                        // (on its way while the tokens are laid down)
  for (uint32_t i = threadIdx.x; i < T * pieces; i += 256) {
    const uint32_t t = i / pieces, p = i - t * pieces;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (t < a.t) {
      v = reinterpret_cast<const uint4*>(xq + t * ldx)[p];
      const int left = (int)(k - p * 16);          // bytes beyond k may hold anything
      if (left < 16) {
        uint32_t* e = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int b = left - 4 * j;
          if (b < 4) e[j] &= b <= 0 ? 0u : (1u << (8 * b)) - 1;
        }
      }
    }
    x[i] = v;
  }
  __syncthreads();
  int sum[T][R] = {};
  for (uint32_t base = 0;;) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t p = base + u * 32 + lane;
      if (p < pieces) {
#pragma unroll
        for (int t = 0; t < T; ++t) {
          const uint4 v = x[t * pieces + p];
#pragma unroll
          for (int r = 0; r < R; ++r) {
            sum[t][r] = __dp4a((int)v.x, (int)w[u][r].x, sum[t][r]);
            sum[t][r] = __dp4a((int)v.y, (int)w[u][r].y, sum[t][r]);
            sum[t][r] = __dp4a((int)v.z, (int)w[u][r].z, sum[t][r]);
            sum[t][r] = __dp4a((int)v.w, (int)w[u][r].w, sum[t][r]);
          }
        }
      }
    }
    base += U * 32;
    if (base >= pieces) break;
    fetch(base);
  }
  int mine = 0;                                    // lane t * R + r keeps the sum of token t and channel r
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int s = __reduce_add_sync(0xffffffffu, sum[t][r]);
      if (lane == t * R + r) mine = s;
    }
  const uint32_t t = lane / R, n = n0 + lane % R;
  if (lane < T * R && t < a.t && n < a.n)
    static_cast<O*>(a.out)[t * a.ldo + n] = static_cast<O>(scaled(mine, a.xs[t], a.ws[n], a.bias ? a.bias[n] : 0.f));
}

// ---- up to 16 tokens -----------------------------------------------------------------------------------------------------
// 16 MT channels x 8 NT tokens to a CTA; its eight warps share the sum, 64 bytes of every 512 to each, and add their
// integer partial sums up in shared memory.  Operands go from memory straight into the fragments of the products: a lane
// loads 16 bytes of its channel (token) and uses them as the k positions that the fragment layout gives it, the same
// positions in both operands, which is all that a sum over k needs.  U steps of loads are in flight, so that the weight
// streams at the rate of the memory.
__device__ __forceinline__ void mma_s8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <int MT, int NT, int U, class O>
__global__ void __launch_bounds__(256) q8_linear_stream_kernel(const int8_t* xq, size_t ldx, const int8_t* wq, size_t ldw, uint32_t k,
                                                               const LinearArgs a) {
  constexpr int kCh = 16 * MT, kTok = 8 * NT, kPitch = kCh + 1;
  extern __shared__ int part[];                    // [8][kTok][kPitch]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
  const uint32_t pieces = (k + 15) / 16, n0 = blockIdx.x * kCh;
  const uint64_t t0 = (uint64_t)blockIdx.y * kTok;
  int acc[MT][NT][4] = {};
  const uint4* wrow[MT][2];
  const uint4* xrow[NT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t n = n0 + m * 16 + h * 8 + g;
      wrow[m][h] = n < a.n ? reinterpret_cast<const uint4*>(wq + (size_t)n * ldw) : nullptr;
    }
#pragma unroll
  for (int t = 0; t < NT; ++t) xrow[t] = t0 + t * 8 + g < a.t ? reinterpret_cast<const uint4*>(xq + (t0 + t * 8 + g) * ldx) : nullptr;
  const int last = (int)(k - (pieces - 1) * 16);   // bytes of the last piece; beyond them anything may lie

  for (uint32_t base = warp * 4; base < pieces; base += 32 * U) {      // (the whole warp takes every step together)
    uint4 w[U][MT][2], x[U][NT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t p = base + u * 32 + q;
      const bool in = p < pieces;
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int h = 0; h < 2; ++h) w[u][m][h] = in && wrow[m][h] ? wrow[m][h][p] : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int t = 0; t < NT; ++t) x[u][t] = in && xrow[t] ? xrow[t][p] : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (last < 16 && base + u * 32 + 4 >= pieces) {      // (the same for the whole warp)
        const bool tail = base + u * 32 + q == pieces - 1;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          uint32_t* e = reinterpret_cast<uint32_t*>(&x[u][t]);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int b = last - 4 * j;
            const uint32_t keep = b >= 4 ? 0xffffffffu : b <= 0 ? 0u : (1u << (8 * b)) - 1;
            e[j] &= tail ? keep : 0xffffffffu;
          }
        }
      }
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          mma_s8(acc[m][t], w[u][m][0].x, w[u][m][1].x, w[u][m][0].y, w[u][m][1].y, x[u][t].x, x[u][t].y);
          mma_s8(acc[m][t], w[u][m][0].z, w[u][m][1].z, w[u][m][0].w, w[u][m][1].w, x[u][t].z, x[u][t].w);
        }
    }
  }
#pragma unroll
  for (int m = 0; m < MT; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        part[(warp * kTok + t * 8 + q * 2 + (i & 1)) * kPitch + m * 16 + (i >> 1) * 8 + g] = acc[m][t][i];
  __syncthreads();
  for (int i = threadIdx.x; i < kCh * kTok; i += 256) {
    const int c = i % kCh, t = i / kCh;
    if (n0 + c >= a.n || t0 + t >= a.t) continue;
    int sum = 0;
#pragma unroll
    for (int p = 0; p < 8; ++p) sum += part[(p * kTok + t) * kPitch + c];
    static_cast<O*>(a.out)[(t0 + t) * a.ldo + n0 + c] =
        static_cast<O>(scaled(sum, a.xs[t0 + t], a.ws[n0 + c], a.bias ? a.bias[n0 + c] : 0.f));
  }
}

// ---- launches -----------------------------------------------------------------------------------------------------------
template <class O>
LinearArgs args_of(const GemmArgs& g, int tile_m, int tile_n, int* err) {
  LinearArgs a;
  a.xs = g.xs; a.ws = g.ws; a.bias = g.bias;
  a.out = g.out; a.ldo = g.ldo;
  a.t = g.t; a.n = g.n; a.ksteps = (g.k + kBK - 1) / kBK;
  a.tiles_m = (uint32_t)((g.t + tile_m - 1) / tile_m);
  a.tiles_n = (g.n + tile_n - 1) / tile_n;
  a.aligned = copy_fits(g.out, g.n * sizeof(O), g.ldo * sizeof(O));
  a.err = err;
  return a;
}

template <int BN, class O>
cudaError_t launch_pairs(const GemmArgs& g, int sms, int* err, cudaStream_t stream) {
  using S = LinearShape<BN>;
  const LinearArgs a = args_of<O>(g, 256, BN, err);
  CUtensorMap mx, mw, mo = {};
  cudaError_t e = make_tensor_map(&mx, g.xq, 1, g.t, g.k, g.ldx, 128, kBK, true);
  if (e == cudaSuccess) e = make_tensor_map(&mw, g.wq, 1, g.n, g.k, g.ldw, BN / 2, kBK, true);
  if (e == cudaSuccess && a.aligned) e = make_tensor_map(&mo, g.out, sizeof(O), g.t, g.n, g.ldo, 32, 128 / sizeof(O), true);
  static std::atomic<uint64_t> seen;
  if (e == cudaSuccess) e = allow_smem(q8_linear_kernel<BN, O>, S::kSmem, g.device, seen);
  if (e != cudaSuccess) return e;
  const uint64_t tiles = (uint64_t)a.tiles_m * a.tiles_n, most = sms / 2;
  return launch_with(q8_linear_kernel<BN, O>, (unsigned)(tiles < most ? tiles : most) * 2, 64 + 32 * kWriters, S::kSmem, 2, false, stream, mx, mw, mo, a);
}

template <int BN, class O>
cudaError_t launch_split(const GemmArgs& g, int size, int* err, cudaStream_t stream) {
  using S = SplitShape<BN>;
  LinearArgs a = args_of<O>(g, 128, BN, err);
  // Rows outside the matrix make a copy slow (16 tokens in a box of 128: 470 ns a stage, as long as a box of 64 full
  // rows and more), so boxes hold no more than there are, or 64.
  a.box = g.t < 128 ? (uint32_t)(g.t + 7) / 8 * 8 : 64;
  CUtensorMap mx, mw;
  cudaError_t e = make_tensor_map(&mx, g.xq, 1, g.t, g.k, g.ldx, a.box, kBK, true);
  if (e == cudaSuccess) e = make_tensor_map(&mw, g.wq, 1, g.n, g.k, g.ldw, BN, kBK, true);
  static std::atomic<uint64_t> seen;
  if (e == cudaSuccess) e = allow_smem(q8_linear_split_kernel<BN, O>, S::kSmem, g.device, seen);
  if (e != cudaSuccess) return e;
  return launch_with(q8_linear_split_kernel<BN, O>, a.tiles_m * a.tiles_n * size, kThreads8, S::kSmem, size, false, stream, mx, mw, a, size == 8 ? 3 : size / 2);
}

template <int T, int R, class O>
cudaError_t launch_few(const GemmArgs& g, cudaStream_t stream) {
  const LinearArgs a = args_of<O>(g, 1, 1, nullptr);
  const size_t smem = (size_t)T * ((g.k + 15) / 16) * 16;
  q8_linear_few_kernel<T, R, O><<<(g.n + 8 * R - 1) / (8 * R), 256, smem, stream>>>(g.xq, g.ldx, g.wq, g.ldw, g.k, a);
  return cudaGetLastError();
}

template <int MT, int NT, int U, class O>
cudaError_t launch_stream(const GemmArgs& g, cudaStream_t stream) {
  const LinearArgs a = args_of<O>(g, 1, 1, nullptr);
  constexpr size_t smem = 8 * (8 * NT) * (16 * MT + 1) * 4;
  auto* kernel = q8_linear_stream_kernel<MT, NT, U, O>;
  static std::atomic<uint64_t> seen;
  const cudaError_t e = allow_smem(kernel, smem, g.device, seen);
  if (e != cudaSuccess) return e;
  kernel<<<dim3((g.n + 16 * MT - 1) / (16 * MT), (unsigned)((g.t + 8 * NT - 1) / (8 * NT))), 256, smem, stream>>>(
      g.xq, g.ldx, g.wq, g.ldw, g.k, a);
  return cudaGetLastError();
}

// The kernel by the number of tokens.  On a weight of 4096 x 4096 read from memory, in us:
//   tokens                    1      2      4      8     16     32     64    128    256
//   few                     2.9*   5.3    6.7    9.4                                       (* 1600 x 6400; stream 3.4)
//   stream, 8 or 16 tokens         5.0    4.9    5.0    6.8   11.3   18.3
//   split                                        7.3    7.5    8.3    9.3   11.4   16.0
//   pairs                                                                          11.1
template <class O>
cudaError_t by_shape(const GemmArgs& g, int sms, int* err, cudaStream_t stream) {
  if (g.t == 1 && ((size_t)g.k + 15) / 16 * 16 <= 48 * 1024) return launch_few<1, 2, O>(g, stream);
  if (g.t <= 8) return launch_stream<2, 1, 4, O>(g, stream);
  if (g.t <= 16) return launch_stream<2, 2, 4, O>(g, stream);
  // Beyond, the shape with the least time in clock cycles.  A stage takes its products (8192 multiply-adds a cycle and SM)
  // or, where that is longer, its copies: 28 bytes a cycle and SM in the split kernel, 42 in the pairs' deeper ring, and
  // 64 where tiles follow one another and find most operands in L2.  The partial sums of a split tile change hands at
  // 6 bytes a cycle.
  const double ksteps = (g.k + kBK - 1) / kBK, rows = g.t < 128 ? (double)g.t : 128.0;
  double least = 1e300;
  int bn = 0, size = 0;
  for (int b : {256, 128}) {
    const uint64_t tiles = ((g.t + 255) / 256) * ((g.n + b - 1) / b), rounds = (tiles + sms / 2 - 1) / (sms / 2);
    const double copy = (128.0 + b / 2) * kBK / (rounds > 1 ? 64 : 42), product = 2.0 * b;
    const double c = rounds * (ksteps * (copy > product ? copy : product) + 1500) + 3000;
    if (c < least) { least = c; bn = b; }
  }
  for (int b : {128, 64, 32})
    for (int s = 1; s <= 8 && s <= ksteps; s *= 2) {
      // (clusters of 4 and 8 do not fill every SM)
      const uint64_t ctas = ((g.t + 127) / 128) * ((g.n + b - 1) / b) * s, most = s <= 2 ? sms : s == 4 ? sms * 9 / 10 : sms * 8 / 10;
      const double each = (uint32_t)((ksteps + s - 1) / s) * (rows + b) * kBK / 28 + (s > 1 ? rows * b * 4 / 6 : 0) + 2500;
      const double c = (double)((ctas + most - 1) / most) * each + 3000;
      if (c < least) { least = c; bn = b; size = s; }
    }
  if (size == 0) return bn == 256 ? launch_pairs<256, O>(g, sms, err, stream) : launch_pairs<128, O>(g, sms, err, stream);
  if (bn == 128) return launch_split<128, O>(g, size, err, stream);
  if (bn == 64) return launch_split<64, O>(g, size, err, stream);
  return launch_split<32, O>(g, size, err, stream);
}

}  // namespace

cudaError_t launch_q8_linear(const GemmArgs& a, int sms, int* err, cudaStream_t stream) {
  return a.out_dtype == STQ_GRAD_F32 ? by_shape<float>(a, sms, err, stream) : by_shape<__nv_bfloat16>(a, sms, err, stream);
}

}  // namespace stq
