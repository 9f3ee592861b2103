// The turns of the attention kernel's two issuing warps (heads over 64), host and device.
//
// Warp t issues the products of query tile t of a piece in n goes; n_other are the other tile's, and tile 0 has no more
// than tile 1.  A go of one tile follows one of the other: 0, 1, 0, 1, ... until tile 0 has no more.  turn[t] is a barrier
// of one arrival, given by the other warp; a phase's parity tells it from the next one only, so no turn may be given
// before the one before it has been taken.  Every turn therefore follows one of the other tile: tile 1 hands one over
// after its last go beside tile 0 too, and tile 0 takes it before its first go of the next piece of two tiles.
#pragma once

namespace geocache {

// Go j of tile t waits for its turn.  `first`: the block has had no piece of two tiles with keys before.
constexpr bool turn_taken(int t, int j, int n_other, bool first) {
    return t == 0 ? n_other > 0 && !(first && j == 0) : j < n_other;
}
// Go j of tile t hands the turn over.
constexpr bool turn_given(int t, int j, int n_other) { return t == 0 ? n_other > 0 : j < n_other; }
// ... as soon as it has taken its own: nothing of this go has to come before the next piece's.
constexpr bool turn_given_at_once(int t, int j, int n_other) { return t == 1 && j + 1 == n_other; }

}  // namespace geocache
