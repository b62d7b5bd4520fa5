// Who waits for whom among the warps of the prefix kernel where more than one segment is concerned.
// Plain C++, so that the kernel's own rules can be walked through on the host in every order that two
// warps can come in.
#pragma once

#ifdef __CUDACC__
#define SEPLLM_HD __host__ __device__ __forceinline__
#else
#define SEPLLM_HD inline
#endif

namespace sepllm {

// Turns at the exponentials of the n_both key tiles of a segment that both slots have.  Two barriers, one
// of each slot: a slot waits for its turn at its own and hands over at the other slot's.  Slot 0
// begins, and after every tile the turn passes to the other slot; behind the last one slot 0 takes it back,
// so that a segment leaves no hand-over behind: a second one on the same barrier, before slot 1 has come
// for the first, would complete it without slot 1, which would then wait for good.
//
// Slot x waits for its turn before tile j of the segment,
SEPLLM_HD bool turn_waits(int x, int j, int n_both) { return x == 1 ? j < n_both : j > 0 && j < n_both; }
// hands it over behind that tile's exponentials,
SEPLLM_HD bool turn_passes(int j, int n_both) { return j < n_both; }
// and takes it back at the segment's end.
SEPLLM_HD bool turn_returns(int x, int n_both) { return x == 0 && n_both > 0; }

// V rows behind the longest prefix, in the last of a segment's n_tiles key tiles: each slot that multiplies
// with that tile asks a fourth warp to have them cleared, once the tile has landed, and waits for the
// answer.  Request and answer have a barrier for each slot, so that a slot is never more than one phase
// away from the warp that clears, whatever the other slot is at: one that leaves a last tile to the other
// goes on to the next segments at once.
//
// Slot x multiplies with the last tile (n_mine: its tiles of the segment; alt: the slots take them in turn).
SEPLLM_HD bool uses_last(bool alt, int x, int n_tiles, int n_mine) {
  return alt ? ((n_tiles - 1) & 1) == x : n_mine == n_tiles;
}

}  // namespace sepllm
