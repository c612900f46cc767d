// Rows of bf16 numbers at any 2-byte address, copied to rows aligned to 16 bytes.
#pragma once
#include <stdint.h>

namespace stq {

// A warp moves columns [base, base + 256) of a row of `cols`: its lanes load the 16-byte pieces that hold them (the first and last
// may reach outside the row, never outside the piece of an element of it), take the next piece from the next lane and shift
// the two into place.  `row`: the row's first element; `out`: its place in the aligned rows (whole pieces are written, so up
// to 7 elements behind the row).
struct RowPart {
  uint4 v, next;
  __device__ __forceinline__ void load(const void* row, uint32_t cols, uint32_t base, int lane) {
    const uintptr_t from = reinterpret_cast<uintptr_t>(row) + 2 * (uintptr_t)base, end = reinterpret_cast<uintptr_t>(row) + 2 * (uintptr_t)cols;
    const uint32_t off = from & 15;
    const uintptr_t piece = from - off + 16 * lane;
    v = next = make_uint4(0, 0, 0, 0);
    if (piece < end) v = *reinterpret_cast<const uint4*>(piece);
    if (lane == 31 && off && piece + 16 < end) next = *reinterpret_cast<const uint4*>(piece + 16);
  }
  __device__ __forceinline__ void store(const void* row, uint32_t cols, uint32_t base, void* out, int lane) const {
    const uint32_t off = (reinterpret_cast<uintptr_t>(row) + 2 * (uintptr_t)base) & 15;
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
    if (c < cols) *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(out) + c) = make_uint4(w[0], w[1], w[2], w[3]);
  }
};
__device__ __forceinline__ void copy_row_part(const void* row, uint32_t cols, uint32_t base, void* out, int lane) {
  RowPart p;
  p.load(row, cols, base, lane);
  p.store(row, cols, base, out, lane);
}

}  // namespace stq
