// The ring of tiles of the attention over 4-bit caches (k_attend4.cu): how the warps that multiply walk it.
//
// Tiles of kPart steps fill the slots in order, over all segments of a CTA, and a warp takes every kWarps-th step of
// that run (a segment's last tile may have fewer steps; a warp's steps go on from one segment to the next as if
// nobody knew of segments).  So a warp uses some tiles of a slot and never sees the others.  A parity wait tells a
// phase only from its neighbours: one for fill k of a slot (k fills came before it) also passes where only k - 1 fills
// have landed.  Before it a warp therefore waits for the slot's empty barrier: fill k - 1 was used up, as the loads themselves
// wait before fill k.  That wait has one meaning, as
//   - no more than k fills were used up: the warp's own arrival for fill k is outstanding;
//   - no fewer than k - 1 were: between two steps of a warp lie kWarps - 1 others, of at most four tiles, so the warp's
//     last tile, or the join of the segments before the last, landed after every slot's fill before the last had been
//     used up (the loads are issued in order).
// With fill k - 1 used up the wait for fill k has one meaning too.
#pragma once

#if defined(__CUDACC__)
#define BKV_RING_FN __host__ __device__ __forceinline__
#else
#define BKV_RING_FN inline
#endif

namespace bkv {

// kWarps: warps at work on steps; kPart: steps of a tile; kSlots: tiles of the ring.
template <int D, int NB>
struct Ring4 {
  static constexpr int kWarps = NB == 1 ? 12 : 8, kPart = 4;
  static constexpr int kSlots = D == 64 ? 16 : NB == 1 ? 8 : 7;
};

template <typename R>
struct RingWalk {
  static_assert(R::kWarps % R::kPart == 0, "a warp takes the same part of every tile of a segment");
  // Of two neighbouring steps of a warp the second's tile is at most 1 + (kWarps - 1 + kPart - 1) / kPart tiles on.
  static_assert(R::kSlots >= 2 + (R::kWarps - 1 + R::kPart - 1) / R::kPart, "see above");
  int step;       // of the present segment, the warp's next one
  int tiles = 0;  // of the segments before
  int slot = 0, turn = 0;  // where that step's tile lies, and how many tiles lay there before it
  BKV_RING_FN explicit RingWalk(int warp) : step(warp) {}
  BKV_RING_FN void begin() {  // of a segment
    const int tile = tiles + step / R::kPart;
    slot = tile % R::kSlots;
    turn = tile / R::kSlots;
  }
  BKV_RING_FN void next() {
    step += R::kWarps;
    slot += R::kWarps / R::kPart;
    if (slot >= R::kSlots) {
      slot -= R::kSlots;
      ++turn;
    }
  }
  BKV_RING_FN void end(int n_steps) {  // of a segment of n_steps, with all its steps taken
    step -= n_steps;
    tiles += (n_steps + R::kPart - 1) / R::kPart;
  }
  // Whether the step's tile is there: empty(slot, parity) and full(slot, parity) test a phase of a barrier, in this
  // order, which gives the second its meaning.
  template <typename Empty, typename Full>
  BKV_RING_FN bool there(Empty&& empty, Full&& full) const {
    const bool used = turn == 0 || empty(slot, (turn - 1) & 1), landed = full(slot, turn & 1);
    return used && landed;
  }
  // The same, where they wait for it.
  template <typename Empty, typename Full>
  BKV_RING_FN void await(Empty&& empty, Full&& full) const {
    if (turn > 0) empty(slot, (turn - 1) & 1);
    full(slot, turn & 1);
  }
};

}  // namespace bkv
