// Barriers that tell a ring of shared-memory stages' readers of arrivals, where the readers take the stages in turn.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define STQ_HOST_DEVICE __host__ __device__
#else
#define STQ_HOST_DEVICE
#endif

namespace stq {

// Stage i lies in slot i % SLOTS and is read by group i % GROUPS alone.  A wait by parity tells only whether the latest
// phase of a barrier has the parity asked for, so a reader may not fall two phases behind.  With a barrier to each slot it
// could where SLOTS is not a multiple of GROUPS: the slot's next stage belongs to another group and does not wait for this
// one.  So there are enough barriers that each belongs to one group: the next stage of barrier i % kBars is loaded into a
// slot that stage i was read from, which only this group's having read it sets free.
template <int SLOTS, int GROUPS>
struct ArrivalRing {
  static constexpr int kBars = SLOTS % GROUPS == 0 ? SLOTS : SLOTS * GROUPS;
  static_assert(kBars % GROUPS == 0 && kBars % SLOTS == 0, "a barrier belongs to one group and one slot");
  STQ_HOST_DEVICE static constexpr uint32_t bar(uint32_t stage) { return stage % kBars; }
  STQ_HOST_DEVICE static constexpr uint32_t parity(uint32_t stage) { return stage / kBars & 1; }
};

}  // namespace stq
