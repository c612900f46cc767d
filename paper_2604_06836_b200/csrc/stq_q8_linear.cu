// out[t][n] = xs[t] * ws[n] * sum_k xq[t][k] * wq[n][k] (+ bias[n]): products of 8-bit rows on the tensor cores.
//
// One CTA (CG = 1) or a pair of CTAs (CG = 2) owns a tile of 128 * CG tokens x BN channels at a time and walks a list
// of tiles.  Warp 0 keeps a ring of shared-memory stages full with tensor copies (128 bytes of the sum at a time, 128-
// byte swizzle, out-of-range rows and columns read as zero), warp 1 issues the products into one of two accumulators
// in tensor memory, warps 2-5 turn the other accumulator (exact 32-bit integers) into results.  In a pair, each CTA
// holds 128 tokens and half of the channels of the tile; the leader issues the products of both.
#include "../../include/stq.h"
#include "stq_internal.h"
#include "stq_q8.h"
#include "stq_q8_mma.cuh"
#include "stq_q8_tma.h"

namespace stq {
namespace {

constexpr int kBK = 128;               // bytes (= elements) of the sum per stage
constexpr int kMmaK = 32;              // elements of the sum per product instruction
constexpr int kThreads8 = 192;

struct LinearArgs {
  const float* xs;
  const float* ws;
  const float* bias;
  void* out;
  size_t ldo;
  uint64_t t;
  uint32_t n, ksteps;
  uint32_t tiles_m, tiles_n;
  int align;                           // bytes that the rows of `out` are aligned to (32, 16, or less)
  int* err;
};

template <int CG, int BN>
struct LinearShape {
  static constexpr int kA = 128 * kBK, kB = BN / CG * kBK, kStage = kA + kB;
  static constexpr int kFit = (200 * 1024) / kStage;
  static constexpr int kStages = kFit < 8 ? kFit : 8;
  static constexpr int kCols = 2 * BN < 32 ? 32 : 2 * BN;      // tensor memory: two accumulators
  static constexpr int kSmem = kStages * kStage + 1024;        // (+ alignment of the swizzle atoms)
};

template <int CG, int BN, class O>
__global__ void __launch_bounds__(kThreads8, 1)
q8_linear_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w, const LinearArgs a) {
  using S = LinearShape<CG, BN>;
  constexpr int kStages = S::kStages;
  extern __shared__ uint8_t raw[];
  __shared__ uint64_t bars[2 * kStages + 4];
  __shared__ uint32_t tmem_slot;
  __shared__ float scale_n[2][BN], bias_n[2][BN];
  __shared__ float stage[4][32 * 33];
  const uint32_t ring = (smem_addr(raw) + 1023u) & ~1023u;
  const uint32_t full = smem_addr(bars), empty = full + 8 * kStages, done = empty + 8 * kStages;
  const uint32_t freed = done + 16;      // accumulators are read (both CTAs, at the leader)
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = CG == 2 ? cluster_rank() : 0;
  const bool leader = rank == 0;
  const uint32_t unit = blockIdx.x / CG, units = gridDim.x / CG, tiles = a.tiles_m * a.tiles_n;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      bar_init(full + 8 * i, 1);
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
  mma_fence_after();
  const uint32_t tmem = tmem_slot;

  bool ok = true;
  if (warp == 0) {
    if (elect_one()) {
      uint32_t it = 0;
      const uint32_t full0 = CG == 2 ? peer_addr(full, 0) : full;
      for (uint32_t tile = unit; ok && tile < tiles; tile += units) {
        const int row = (int)(tile % a.tiles_m) * 128 * CG + 128 * rank, col = (int)(tile / a.tiles_m) * BN + (BN / CG) * rank;
        for (uint32_t k = 0; k < a.ksteps; ++k, ++it) {
          const uint32_t s = it % kStages, ph = (it / kStages) & 1;
          if (!(ok = bar_wait(empty + 8 * s, ph ^ 1))) break;
          if (leader) bar_expect(full + 8 * s, CG * S::kStage);
          const uint32_t at = ring + s * S::kStage;
          tensor_load<CG>(at, &map_x, (int)k * kBK, row, full0 + 8 * s);
          tensor_load<CG>(at + S::kA, &map_w, (int)k * kBK, col, full0 + 8 * s);
        }
      }
      if (!ok && leader)      // leave no copy in flight
        for (uint32_t s = 0; s < kStages && s < it; ++s) bar_wait(full + 8 * ((it - 1 - s) % kStages), ((it - 1 - s) / kStages) & 1);
    }
  } else if (warp == 1) {
    if (leader && elect_one()) {
      constexpr uint32_t id = idesc(kIdescI8, 128 * CG, BN, false, false);
      uint32_t it = 0, n = 0;
      for (uint32_t tile = unit; ok && tile < tiles; tile += units, ++n) {
        const uint32_t acc = n & 1;
        if (!(ok = bar_wait<CG == 2>(freed + 8 * acc, ((n >> 1) & 1) ^ 1))) break;
        mma_fence_after();
        for (uint32_t k = 0; k < a.ksteps; ++k, ++it) {
          const uint32_t s = it % kStages, ph = (it / kStages) & 1;
          if (!(ok = bar_wait(full + 8 * s, ph))) break;
          mma_fence_after();
          const uint32_t at = ring + s * S::kStage;
          const uint64_t da = operand_desc(at, 16, 1024), db = operand_desc(at + S::kA, 16, 1024);
#pragma unroll
          for (int j = 0; j < kBK / kMmaK; ++j)
            mma<CG, true>(tmem + acc * BN, da + j * (kMmaK >> 4), db + j * (kMmaK >> 4), id, (k | j) != 0);
          mma_commit<CG>(empty + 8 * s);
        }
        if (ok) mma_commit<CG>(done + 8 * acc);
      }
    }
  } else {
    const int quad = warp & 3, thread = threadIdx.x - 64;     // (a warp reaches the 32 lanes 32 * (warp % 4) of tensor memory)
    const uint32_t freed0 = CG == 2 ? peer_addr(freed, 0) : freed;
    uint32_t n = 0;
    for (uint32_t tile = unit; ok && tile < tiles; tile += units, ++n) {
      const uint32_t acc = n & 1;
      const uint64_t row = (uint64_t)(tile % a.tiles_m) * 128 * CG + 128 * rank + quad * 32 + lane;
      const uint32_t col = tile / a.tiles_m * BN;
      for (int c = thread; c < BN; c += 128) {
        scale_n[acc][c] = col + c < a.n ? a.ws[col + c] : 0.f;
        bias_n[acc][c] = a.bias && col + c < a.n ? a.bias[col + c] : 0.f;
      }
      const float xs = row < a.t ? a.xs[row] : 0.f;
      ok = bar_wait(done + 8 * acc, (n >> 1) & 1);
      if (!(ok = all_of_128(ok))) break;       // (the four warps leave together; the scales above are visible to all)
      mma_fence_after();
      const uint32_t from = tmem + ((uint32_t)(quad * 32) << 16) + acc * BN;
      O* out = static_cast<O*>(a.out) + (row - lane) * a.ldo + col;
      const int rows = row - lane >= a.t ? 0 : (int)min((uint64_t)32, a.t - (row - lane));
      constexpr int kC = BN < 32 ? BN : 32;
#pragma unroll 2
      for (int c = 0; c < BN; c += kC) {
        if (col + c >= a.n) break;
        uint32_t r[kC];
        tmem_load(from + c, r);
        tmem_load_wait();
        float v[kC];
#pragma unroll
        for (int i = 0; i < kC; ++i) v[i] = fmaf((float)(int)r[i], xs * scale_n[acc][c + i], bias_n[acc][c + i]);
        store_block<O, kC>(out + c, a.ldo, v, rows, (int)min((uint32_t)kC, a.n - col - c), a.align, lane, stage[quad]);
      }
      mma_fence_before();
      __syncwarp();
      if (lane == 0) bar_arrive_leader<CG>(freed + 8 * acc, freed0 + 8 * acc, leader);
    }
  }
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

template <int CG, int BN, class O>
cudaError_t launch(const GemmArgs& g, int sms, int* err, cudaStream_t stream) {
  using S = LinearShape<CG, BN>;
  LinearArgs a;
  a.xs = g.xs; a.ws = g.ws; a.bias = g.bias;
  a.out = g.out; a.ldo = g.ldo;
  a.t = g.t; a.n = g.n; a.ksteps = (g.k + kBK - 1) / kBK;
  a.tiles_m = (uint32_t)((g.t + 128 * CG - 1) / (128 * CG));
  a.tiles_n = (g.n + BN - 1) / BN;
  a.align = row_alignment(g.out, g.ldo * sizeof(O));
  a.err = err;
  CUtensorMap mx, mw;
  cudaError_t e = make_tensor_map(&mx, g.xq, 1, g.t, g.k, g.ldx, 128, kBK, true);
  if (e == cudaSuccess) e = make_tensor_map(&mw, g.wq, 1, g.n, g.k, g.ldw, BN / CG, kBK, true);
  static std::atomic<uint64_t> seen;
  if (e == cudaSuccess) e = allow_smem(q8_linear_kernel<CG, BN, O>, S::kSmem, g.device, seen);
  if (e != cudaSuccess) return e;
  const uint64_t tiles = (uint64_t)a.tiles_m * a.tiles_n, most = sms / CG;
  return launch_cluster(q8_linear_kernel<CG, BN, O>, (unsigned)(tiles < most ? tiles : most) * CG, kThreads8, S::kSmem, CG,
                        stream, mx, mw, a);
}

template <class O>
cudaError_t by_shape(const GemmArgs& g, int sms, int* err, cudaStream_t stream) {
  // Clock cycles of a tile by its slower side: products (8192 multiply-adds a cycle and SM), or the copies of its
  // operands; and the fixed cost of a tile's beginning and end.  The shape with the least time over all rounds wins.
  auto cost = [&](int cg, int bn) {
    const uint64_t tm = (g.t + 128 * cg - 1) / (128 * cg), tn = (g.n + bn - 1) / bn, rounds = (tm * tn + sms / cg - 1) / (sms / cg);
    const uint64_t rows = g.t < 128 ? g.t : 128, product = 2 * (uint64_t)bn / cg < 64 ? 64 : 2 * (uint64_t)bn, copy = (rows + bn / cg) * 2;
    return rounds * ((product > copy ? product : copy) * ((g.k + kBK - 1) / kBK) + 1500);
  };
  const uint64_t c[] = {cost(2, 256), cost(2, 128), cost(1, 128), cost(1, 64), cost(1, 32), cost(1, 16)};
  int best = 0;
  for (int i = 1; i < 6; ++i)
    if (c[i] < c[best]) best = i;
  switch (best) {
    case 0: return launch<2, 256, O>(g, sms, err, stream);
    case 1: return launch<2, 128, O>(g, sms, err, stream);
    case 2: return launch<1, 128, O>(g, sms, err, stream);
    case 3: return launch<1, 64, O>(g, sms, err, stream);
    case 4: return launch<1, 32, O>(g, sms, err, stream);
    default: return launch<1, 16, O>(g, sms, err, stream);
  }
}

}  // namespace

cudaError_t launch_q8_linear(const GemmArgs& a, int sms, int* err, cudaStream_t stream) {
  return a.out_dtype == STQ_GRAD_F32 ? by_shape<float>(a, sms, err, stream) : by_shape<__nv_bfloat16>(a, sms, err, stream);
}

}  // namespace stq
