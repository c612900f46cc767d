// Device helpers of the matrix kernels: barriers, tensor copies, tcgen05 instructions and their descriptors.
//
// Every wait is bounded; a wait that runs out returns false, the caller raises the handle's error flag and leaves.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <stdint.h>

namespace stq {

constexpr long long kMmaWaitCycles = 4000000000ll;   // ~2 s: far beyond any copy or product; then give up

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cta.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Arrival on a barrier of another CTA of the cluster (address from peer_addr).  What has to come before it are this thread's
// reads of tensor memory (complete, tcgen05.wait::ld) or writes to its own CTA's shared memory (behind a proxy fence), which
// the pair's products touch once the other side has waited.  The release is at CTA scope, so the PTX memory model, which asks
// for a scope that includes both sides, promises nothing here: that the arrival is seen after them rests on the hardware.  At
// cluster scope an arrival also waits for every global access in flight: 1400 cycles measured behind the loads of the scales
// (dx 8192 x 4096 x 8192: 798 instead of 484 us).
__device__ __forceinline__ void bar_arrive_peer(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cta.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ uint32_t peer_addr(uint32_t local, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(local), "r"(rank));
  return a;
}
template <bool CLUSTER>
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  if constexpr (CLUSTER)
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
  return ok != 0;
}
// CLUSTER: arrivals come from another CTA of the cluster too.
template <bool CLUSTER = false>
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {
  if (bar_try<CLUSTER>(bar, parity)) return true;
  const long long t0 = clock64();
  while (!bar_try<CLUSTER>(bar, parity))
    if (clock64() - t0 > kMmaWaitCycles) return false;
  return true;
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Arrival on the barrier of a pair's leader (or of the CTA itself): `bar` in this CTA, `bar0` its address at the leader.
template <int CG>
__device__ __forceinline__ void bar_arrive_leader(uint32_t bar, uint32_t bar0, bool leader) {
  if (CG == 1 || leader)
    bar_arrive(bar);
  else
    bar_arrive_peer(bar0);
}
// The two halves of that: a CTA may write to another's shared memory once that one has arrived, so once it has started.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0;
}

// Box of a 2-D tensor map -> shared memory of this CTA, bytes counted on `bar`.  In a pair of CTAs (CG = 2) the
// barrier may be the pair leader's.
template <int CG>
__device__ __forceinline__ void tensor_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  if constexpr (CG == 1)
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
  else
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], "
        "[%4];" ::"r"(dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}

// ---- tensor memory ----------------------------------------------------------------------------------------------
template <int CG>
__device__ __forceinline__ void tmem_alloc(uint32_t slot, uint32_t cols) {   // one whole warp (of each CTA of a pair)
  if constexpr (CG == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  } else {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  }
}
template <int CG>
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t cols) {
  if constexpr (CG == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols));
  else
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols));
}
__device__ __forceinline__ void mma_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void mma_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }

// 32 columns of this warp's 32 lanes
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
      "%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
        "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_store(uint32_t addr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
      "%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(addr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
      "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// N columns as they are (accumulators of fp32)
template <int N>
__device__ __forceinline__ void load_block(uint32_t addr, float (&v)[N]) {
  uint32_t r[N / 32][32];
#pragma unroll
  for (int i = 0; i < N / 32; ++i) tmem_load(addr + 32 * i, r[i]);
  tmem_load_wait();
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = __uint_as_float(r[i / 32][i % 32]);
}

// ---- products -------------------------------------------------------------------------------------------------
// Shared-memory operand in the 128-byte swizzle.  K-major: rows of 128 bytes, groups of 8 rows 1024 bytes apart
// (`stride`); `lead` is not used.  MN-major: 64 two-byte elements along the row, 8 rows along the sum to an atom of
// 1024 bytes, `lead` bytes between atoms along the row, `stride` bytes between atoms along the sum.
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr, uint32_t lead, uint32_t stride) {
  return (uint64_t)((addr & 0x3ffff) >> 4) | ((uint64_t)(lead >> 4) << 16) | ((uint64_t)(stride >> 4) << 32) | (1ull << 46) |
         (2ull << 61);
}
// Instruction descriptor: accumulator and operand formats, transposed (MN-major) operands, extent of the result.
constexpr uint32_t kIdescI8 = (2u << 4) | (1u << 7) | (1u << 10);      // s32 += s8 * s8
constexpr uint32_t kIdescBf16 = (1u << 4) | (1u << 7) | (1u << 10);    // f32 += bf16 * bf16
__host__ __device__ constexpr uint32_t idesc(uint32_t kind, int m, int n, bool a_mn, bool b_mn) {
  return kind | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

template <int CG, bool I8>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t id, bool add) {
  const uint32_t acc = add ? 1u : 0u;
  if constexpr (CG == 1 && I8)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
                 "l"(a), "l"(b), "r"(id), "r"(acc)
                 : "memory");
  else if constexpr (CG == 2 && I8)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
                 "l"(a), "l"(b), "r"(id), "r"(acc)
                 : "memory");
  else if constexpr (CG == 1)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
                 "l"(a), "l"(b), "r"(id), "r"(acc)
                 : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
                 "l"(a), "l"(b), "r"(id), "r"(acc)
                 : "memory");
}
// The barrier (the same offset in both CTAs of a pair) gets one arrival when the products issued so far are done.
template <int CG>
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  if constexpr (CG == 1)
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
  else
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                 "h"((uint16_t)3)
                 : "memory");
}

// 32 bytes to an address aligned to them
__device__ __forceinline__ void store32(void* p, const uint32_t (&v)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]),
               "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
               : "memory");
}
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// True if `ok` is true in all of the N threads that share barrier 1 (whole warps); a barrier for them too.
template <int N>
__device__ __forceinline__ bool all_of(bool ok) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(r)
      : "r"((uint32_t)ok), "n"(N)
      : "memory");
  return r != 0;
}

// ---- results ------------------------------------------------------------------------------------------------------
// A warp's block of 32 rows x 128 bytes, lane = row.
constexpr int kStageRow = 144, kStageBytes = 5 * 1024;      // shared memory for it, a multiple of the swizzle's 1024 bytes

// To a matrix whose rows are aligned to 16 bytes and whole numbers of them: through shared memory (128-byte swizzle: eight lanes write eight
// different pieces) and one tensor copy, which leaves out what lies outside the matrix.  The next block waits until the
// copy has read this one.
template <class O>
__device__ __forceinline__ void block_words(const float (&v)[128 / sizeof(O)], uint32_t (&w)[32]) {
  constexpr int C = 128 / sizeof(O);
#pragma unroll
  for (int i = 0; i < 32; ++i) w[i] = sizeof(O) == 2 ? bf16_pair(v[2 * i % C], v[(2 * i + 1) % C]) : __float_as_uint(v[i % C]);
}
template <class O>
__device__ __forceinline__ void store_block(const CUtensorMap* map, int x, int y, const float (&v)[128 / sizeof(O)], int lane, uint32_t stage) {
  if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
  uint32_t w[32];
  block_words<O>(v, w);
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 8; ++i)
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(stage + lane * 128 + ((i ^ (lane & 7)) << 4)), "r"(w[4 * i]),
                 "r"(w[4 * i + 1]), "r"(w[4 * i + 2]), "r"(w[4 * i + 3])
                 : "memory");
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
  if (lane == 0) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(stage)
                 : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
  }
}
// The same through one of PLACES in shared memory, 4096 bytes each, in turn (n counts the blocks): with two, a copy has the time
// of a whole block to read its own.  ADD: added to what is there (fp32).
template <class O, bool ADD = false, int PLACES = 2>
__device__ __forceinline__ void put_block(const CUtensorMap* map, int x, int y, const float (&v)[128 / sizeof(O)], int lane, uint32_t stages, uint32_t& n) {
  if (lane == 0) asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(PLACES - 1) : "memory");
  const uint32_t stage = stages + n++ % PLACES * 4096;
  uint32_t w[32];
  block_words<O>(v, w);
  __syncwarp();
#pragma unroll
  for (int i = 0; i < 8; ++i)
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(stage + lane * 128 + ((i ^ (lane & 7)) << 4)), "r"(w[4 * i]),
                 "r"(w[4 * i + 1]), "r"(w[4 * i + 2]), "r"(w[4 * i + 3])
                 : "memory");
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  __syncwarp();
  if (lane == 0) {
    if constexpr (ADD)
      asm volatile("cp.reduce.async.bulk.tensor.2d.global.shared::cta.add.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(stage)
                   : "memory");
    else
      asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(stage)
                   : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
  }
}
// Before a warp ends (or reuses its shared memory for anything else): its copies are done.
__device__ __forceinline__ void store_blocks_done(int lane) {
  if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
  __syncwarp();
}

// To workspace rows of `ld` floats, aligned to 32 bytes.
__device__ __forceinline__ void store_part(float* base, size_t ld, const float* v, int lane) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = __float_as_uint(v[8 * i + j]);
    store32(base + lane * ld + 8 * i, w);
  }
}

// To a matrix whose rows are not: `rows` x `cols` of the block lie inside it.  A row is laid down in shared memory as far
// from a 16-byte boundary as it lies in global memory, so that all but its first and last pieces move 16 bytes at a time,
// eight neighbouring lanes to a row.
template <class O>
__device__ __forceinline__ void store_ragged(O* base, size_t ld, const float (&v)[128 / sizeof(O)], int rows, int cols, int lane,
                                             uint8_t* stage) {
  constexpr int C = 128 / sizeof(O), kPiece = 16 / sizeof(O);
  auto off = [&](int r) { return (int)(reinterpret_cast<uintptr_t>(base + (size_t)r * ld) & 15); };
  __syncwarp();
  {
    const int mis = off(lane);
    uint32_t* to = reinterpret_cast<uint32_t*>(stage + lane * kStageRow + (mis & ~3));
    if constexpr (sizeof(O) == 2) {
      const bool odd = mis & 2;                                  // (a word holds an odd and the next even column then)
#pragma unroll
      for (int i = 0; i < 33; ++i) {
        const float e0 = i < 32 ? v[2 * i % C] : 0.f, o0 = i < 32 ? v[(2 * i + 1) % C] : 0.f, before = i > 0 ? v[(2 * i - 1) % C] : 0.f;
        if (i < 32 || odd) to[i] = odd ? bf16_pair(before, e0) : bf16_pair(e0, o0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 32; ++i) to[i] = __float_as_uint(v[i % C]);
    }
  }
  __syncwarp();
  if (cols == C) {
#pragma unroll
    for (int it = 0; it < 8; ++it) {                             // whole pieces, four rows at a time
      const int r = it * 4 + lane / 8, mis = off(r), piece = lane % 8 + (mis != 0);
      if (r < rows && piece < 8)
        *reinterpret_cast<uint4*>(reinterpret_cast<uint8_t*>(base + (size_t)r * ld) - mis + piece * 16) =
            *reinterpret_cast<const uint4*>(stage + r * kStageRow + piece * 16);
    }
#pragma unroll
    for (int it = 0; it < kPiece; ++it) {                        // what is left at both ends of a row: a piece's worth
      const int r = it * (32 / kPiece) + lane / kPiece, k = lane % kPiece, mis = off(r), head = (16 - mis) / (int)sizeof(O);
      const int e = k < head ? k : C - kPiece + k;
      if (r < rows && mis != 0) base[(size_t)r * ld + e] = *reinterpret_cast<const O*>(stage + r * kStageRow + mis + e * sizeof(O));
    }
  } else {
    for (int r = 0; r < rows; ++r)
      for (int e = lane; e < cols; e += 32)
        base[(size_t)r * ld + e] = *reinterpret_cast<const O*>(stage + r * kStageRow + off(r) + e * sizeof(O));
  }
}

}  // namespace stq
