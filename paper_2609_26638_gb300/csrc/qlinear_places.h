// qlinear_places.h -- which barrier hands a group's place in tensor memory back (plain C++).
//
// Group q's products are summed in place q % places and added from there; then group q +
// places overwrites it.  A wait tells a barrier's phases apart by their parity alone, so
// whoever waits has to see every phase.  With four groups to a stage and four places the two
// issuing warps take turns at each place: on one barrier a place each would see every other
// phase, and take the addition before the last for the last one.  Nor would waiting for both
// do: the earlier one may be two phases back by then, and the wait never end.  So a place has two
// barriers, for its even and its odd uses.  Whatever the groups of a stage, one warp waits
// for all phases of each.
#pragma once

namespace gs {

// The barrier on which group q is told to be added.
constexpr int place_barrier(int q, int places) { return q / places % 2 * places + q % places; }
// The parity of that phase.
constexpr int place_phase(int q, int places) { return q / places / 2 % 2; }

}  // namespace gs
