// The order of psrl_kv_move's large moves: which parts may be stored when.  Plain arithmetic, shared by the kernel and by a
// model of it on the CPU (tests/test_move_order.py), where warps may be late by any amount.
//
// The rows (slots of one pool and head) to be moved are cut into parts, handed out in ascending order, 32 parts to a group.
// A warp takes a part, loads it, counts it in its group and stores it once all groups up to wait_until() are complete.
// The counts are kept modulo kRing and never reset, so a count of 32 in a group's first round of the ring, 64 in its second, ...
// says that the group is complete, as long as no part of a group kRing later has been counted by then.
//
// How far back a group can be incomplete while a part of group G is at work: let Q be an incomplete group.  Every part of a
// group from Q + kAhead on waits for Q before it is stored, so it is still held by the warp that took it.  All parts of the
// groups Q + kAhead ... G - 1 have been handed out before G's, and at most kSpan groups' worth of warps exist, one of them with
// the part of G: G - Q - kAhead < kSpan.  So all groups before G - (kSpan + kAhead) + 1 are complete, whatever a warp has seen
// of them and however late it is, and the groups whose counts still change fit the ring.
#pragma once
#include <cstdint>

#ifdef __CUDACC__
#define PSRL_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define PSRL_HOST_DEVICE inline
#endif

namespace psrl {

constexpr uint32_t kGroup = 32;                    // parts of a group
constexpr uint32_t kRing = 32, kSpan = 15, kAhead = 15;
static_assert(kSpan + kAhead + 1 < kRing && kRing <= 32, "a lane polls one group, all that may be incomplete in one go");

// the last of n extents that starts at or before `at` (the first one if none does)
PSRL_HOST_DEVICE int extent_of(const int32_t* starts, int n, int at) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (starts[mid] <= at) lo = mid; else hi = mid;
  }
  return lo;
}

// The last group that has to be complete before the part of rows [.., end) is stored: what the part overwrites must have been
// loaded, i.e. the sources below its last destination slot.  They are rows of this part or of parts before it; the last
// of them decides.  (No source at or below that slot: then nothing of this head is overwritten that anybody reads, and the
// rows of the head before, if the part has any, end before the head's first row.)  Nor may a part run kAhead groups ahead.
template <class List>
PSRL_HOST_DEVICE uint32_t wait_until(const List& list, uint32_t part, uint32_t end, uint32_t part_rows) {
  const uint32_t last_row = end - 1, ph = last_row / uint32_t(list.slots);
  const int s_last = int(last_row - ph * uint32_t(list.slots)), e_last = extent_of(list.first, list.n, s_last);
  const int dst_last = list.dst[e_last] + s_last - list.first[e_last];
  const int e_src = extent_of(list.src, list.n, dst_last);
  int s_src = 0;
  if (list.src[e_src] <= dst_last) {
    s_src = list.first[e_src] + dst_last - list.src[e_src];
    if (s_src >= list.first[e_src + 1]) s_src = list.first[e_src + 1] - 1;
  }
  const uint32_t group = part / kGroup, needed = (ph * uint32_t(list.slots) + uint32_t(s_src)) / part_rows / kGroup;
  const uint32_t ahead = group > kAhead ? group - kAhead : 0;
  return needed > ahead ? needed : ahead;
}

// The first group to look at before a part of `group` is stored, when those below `seen` are known to be complete: with the 31
// that may still be incomplete, 32 lanes see them all, however many have gone by since the warp's last part.
PSRL_HOST_DEVICE uint32_t poll_from(uint32_t seen, uint32_t group) {
  const uint32_t oldest = group > kSpan + kAhead ? group - (kSpan + kAhead) : 0;
  return seen > oldest ? seen : oldest;
}

// the count at which group g is complete
PSRL_HOST_DEVICE uint32_t full_count(uint32_t g, uint32_t n_parts) {
  const uint32_t before = g * kGroup < n_parts ? g * kGroup : n_parts, here = n_parts - before;
  return g / kRing * kGroup + (here < kGroup ? here : kGroup);
}

}  // namespace psrl
