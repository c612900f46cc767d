// Maxima and sums of exp of the logits of up to 16 tokens (stq_vocab_scores.cu has the formulas and the form for more of them).
//
// Bound by the matrix, which is read once: 2 v d bytes.  A tile of the matrix units would spend its copies on rows of tokens that are not
// there, and its boxes of 128 bytes a row reach 3.8 TB/s.  Here a warp loads 16 rows of the matrix straight into the fragments of
// mma.m16n8k16 (the sum may run over the columns in any order, so a lane takes 16 neighbouring bytes of a row and uses them for two
// products), eight warps share a row's columns in turns of 64 bytes, and the next rows are on the way while these are multiplied:
// 64 to 96 KB in flight on each SM.
#include <cuda_bf16.h>

#include "../../include/stq.h"
#include "stq_q8_tma.h"
#include "stq_vocab.h"

namespace stq {
namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kRows = 16;              // rows of the matrix to a group
constexpr int kPiece = 32;             // columns that a warp takes at a time: 16 bytes for each of four lanes
constexpr int kAhead = 4;              // pieces to a step
constexpr int kStep = kWarps * kAhead * kPiece;
constexpr float kLog2e = 1.4426950408889634f;

struct FewArgs {
  const uint16_t* x;
  size_t ldx;
  const uint16_t* w;
  size_t ldw;
  const float* bias;
  uint32_t t, v, d;
  uint32_t steps, groups;
  uint32_t pitch;          // bytes of a token's row in shared memory
  bool aligned;            // rows of x are 16-byte pieces
  float2* part;
  uint32_t most;
};

__device__ __forceinline__ float ex2(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ void product(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 load_stream(const uint16_t* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// NT: groups of eight tokens.
template <int NT>
__global__ void __launch_bounds__(kThreads, 2) few_kernel(const FewArgs a) {
  extern __shared__ __align__(16) uint8_t raw[];
  float* parts = reinterpret_cast<float*>(raw);                       // [2][kWarps][kRows][8 NT]
  uint8_t* xs = raw + 2 * kWarps * kRows * 8 * NT * sizeof(float);    // tokens [8 NT] of `pitch` bytes
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");

  // lane: row lane / 4 (and that + 8) of the group, 8 columns from (lane % 4) * 8 of the piece
  const uint32_t r0 = lane >> 2, c0 = (lane & 3) * 8;
  uint4 next[kAhead][2], now[kAhead][2];
  auto load = [&](uint32_t i) {      // step i of this CTA: its group, and which columns
    const uint32_t group = blockIdx.x + i / a.steps * gridDim.x, k0 = i % a.steps * kStep + warp * kPiece + c0;
    const uint32_t top = a.v - 1, r = min(group * kRows + r0, top), r8 = min(group * kRows + r0 + 8, top);
    const uint16_t *p = a.w + (size_t)r * a.ldw + k0, *q = a.w + (size_t)r8 * a.ldw + k0;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const uint32_t k = k0 + j * kWarps * kPiece;
      const bool in = group < a.groups && k < a.d;
      next[j][0] = in ? load_stream(p + j * kWarps * kPiece) : make_uint4(0, 0, 0, 0);
      next[j][1] = in ? load_stream(q + j * kWarps * kPiece) : make_uint4(0, 0, 0, 0);
    }
  };
  load(0);

  // tokens to shared memory, with zeros behind their last column and in the rows of tokens that are not there
  const uint32_t wide = a.pitch / 16;
  for (uint32_t i = threadIdx.x; i < 8 * NT * wide; i += kThreads) {
    const uint32_t t = i / wide, c = (i - t * wide) * 8;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (t < a.t && c < a.d) {
      const uint16_t* p = a.x + (size_t)t * a.ldx + c;
      if (a.aligned && c + 8 <= a.d) {
        v = *reinterpret_cast<const uint4*>(p);
      } else {
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (c + j < a.d) w[j / 2] |= (uint32_t)p[j] << (16 * (j & 1));
        v = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
    *reinterpret_cast<uint4*>(xs + (size_t)t * a.pitch + c * 2) = v;
  }
  __syncthreads();

  // this thread's logits: row threadIdx / (8 NT) of each group, token threadIdx % (8 NT)
  const uint32_t mine_row = threadIdx.x / (8 * NT), mine_tok = threadIdx.x % (8 * NT);
  float m = -INFINITY, s = 0.f;
  float c[NT][4] = {};
  uint32_t turn = 0;
  const uint32_t mine_groups = blockIdx.x < a.groups ? (a.groups - 1 - blockIdx.x) / gridDim.x + 1 : 0, count = mine_groups * a.steps;
  for (uint32_t i = 0; i < count; ++i) {
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      now[j][0] = next[j][0];
      now[j][1] = next[j][1];
    }
    load(i + 1);
    const uint32_t step = i % a.steps, k0 = step * kStep + warp * kPiece + c0;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const uint32_t k = k0 + j * kWarps * kPiece;
      if (k - c0 >= a.d) break;
      uint4 u = now[j][0], v = now[j][1];
      if (k + 8 > a.d) {      // what lies behind a row's last column may be anything
        uint32_t keep[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) keep[e] = k + 2 * e + 1 < a.d ? 0xffffffffu : k + 2 * e < a.d ? 0xffffu : 0u;
        u.x &= keep[0]; u.y &= keep[1]; u.z &= keep[2]; u.w &= keep[3];
        v.x &= keep[0]; v.y &= keep[1]; v.z &= keep[2]; v.w &= keep[3];
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const uint4 b = *reinterpret_cast<const uint4*>(xs + (size_t)(8 * n + r0) * a.pitch + k * 2);
        product(c[n], u.x, v.x, u.y, v.y, b.x, b.y);
        product(c[n], u.z, v.z, u.w, v.w, b.z, b.w);
      }
    }
    if (step + 1 < a.steps) continue;
    // the warps' sums of the group, added in their order; a thread keeps the maximum and the sum of exp of its own logits
    float* out = parts + (turn * kWarps + warp) * kRows * 8 * NT;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float* o = out + 8 * n + 2 * (lane & 3);
      *reinterpret_cast<float2*>(o + r0 * 8 * NT) = make_float2(c[n][0], c[n][1]);
      *reinterpret_cast<float2*>(o + (r0 + 8) * 8 * NT) = make_float2(c[n][2], c[n][3]);
#pragma unroll
      for (int e = 0; e < 4; ++e) c[n][e] = 0.f;
    }
    __syncthreads();
    if (mine_row < kRows) {
      float z = 0.f;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) z = __fadd_rn(z, parts[((turn * kWarps + w) * kRows + mine_row) * 8 * NT + mine_tok]);
      const uint32_t row = (blockIdx.x + i / a.steps * gridDim.x) * kRows + mine_row;
      if (row < a.v) {
        if (a.bias) z = __fadd_rn(z, __ldg(a.bias + row));
        const float top = fmaxf(m, z), ref = top == -INFINITY ? 0.f : top;
        s = __fadd_rn(__fmul_rn(s, ex2(__fmul_rn(__fadd_rn(m, -ref), kLog2e))), ex2(__fmul_rn(__fadd_rn(z, -ref), kLog2e)));
        m = top;
      }
    }
    turn ^= 1;      // (the next group's sums go elsewhere, so one barrier a group is enough)
  }
  __syncthreads();
  float2* all = reinterpret_cast<float2*>(parts);
  if (mine_row < kRows) all[mine_row * 8 * NT + mine_tok] = make_float2(m, s);
  __syncthreads();
  if (threadIdx.x < a.t) {
    float2 p = all[threadIdx.x];
    for (int r = 1; r < kRows; ++r) {
      const float2 q = all[r * 8 * NT + threadIdx.x];
      const float top = fmaxf(p.x, q.x), ref = top == -INFINITY ? 0.f : top;
      p = make_float2(top, __fadd_rn(__fmul_rn(p.y, ex2((p.x - ref) * kLog2e)), __fmul_rn(q.y, ex2((q.x - ref) * kLog2e))));
    }
    a.part[(size_t)blockIdx.x * a.most + threadIdx.x] = p;
  }
}

uint32_t pitch_of(uint32_t d) { return (d + kPiece - 1) / kPiece * kPiece * 2 + 64 - ((d + kPiece - 1) / kPiece & 1) * 64; }
size_t smem_of(uint32_t t, uint32_t d) {
  const size_t nt = t <= 8 ? 1 : 2;
  return nt * 8 * pitch_of(d) + 2 * kWarps * kRows * 8 * nt * sizeof(float);
}

}  // namespace

uint32_t vocab_few_parts(uint32_t t, uint32_t v, uint32_t d, int sms) {
  if (t > 16 || smem_of(t, d) > 110 * 1024) return 0;      // (two CTAs to an SM)
  const uint32_t groups = (v + kRows - 1) / kRows;
  return groups < 2u * sms ? groups : 2 * sms;
}

cudaError_t launch_vocab_few(const VocabArgs& a, const void* x, size_t ldx, float2* part, int sms, cudaStream_t stream) {
  FewArgs f;
  f.x = static_cast<const uint16_t*>(x);
  f.ldx = ldx;
  f.w = static_cast<const uint16_t*>(a.w);
  f.ldw = a.ldw;
  f.bias = a.bias;
  f.t = a.t; f.v = a.v; f.d = a.d;
  f.steps = (a.d + kStep - 1) / kStep;
  f.groups = (a.v + kRows - 1) / kRows;
  f.pitch = pitch_of(a.d);
  f.aligned = rows_aligned(x, a.t > 1 ? ldx * 2 : 0);
  f.part = part;
  f.most = a.r.most;
  const size_t smem = smem_of(a.t, a.d);
  auto go = [&](auto* kernel, std::atomic<uint64_t>& seen) {
    const cudaError_t e = allow_smem(kernel, 112 * 1024, a.device, seen);
    return e != cudaSuccess ? e : launch_with(kernel, dim3(vocab_few_parts(a.t, a.v, a.d, sms)), dim3(kThreads), smem, 1, true, stream, f);
  };
  static std::atomic<uint64_t> seen[2];
  return a.t <= 8 ? go(few_kernel<1>, seen[0]) : go(few_kernel<2>, seen[1]);
}

}  // namespace stq
