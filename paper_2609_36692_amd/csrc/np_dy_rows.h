// How the weight gradient may read the rows of dy (np_checkpoint.hip), apart from
// the kernels so that a host program can check it.
#pragma once

#include <stdint.h>

namespace np {

// Tokens of one tile.
constexpr int64_t kDyTile = 32;

// dy is read in pieces of `piece` elements (16 bytes), from column 0 or, past the
// last column, from that one.
//   Whole : a row is a whole number of pieces, so no piece leaves its row.
//   Ragged: a piece may run past its row's last column.  It runs at most piece - 1
//           elements past it, and where a row starts that many elements after the
//           one before it, one row more holds them: every tile of a share of tokens
//           but the last one has such a row after it.  The last tile is read
//           element by element at the edge.
//   Narrow: rows are closer than that; every tile is read element by element.
enum class DyRows { Whole, Ragged, Narrow };

inline DyRows dy_rows(int64_t outer, int64_t ld, int64_t piece) {
    return outer % piece == 0 ? DyRows::Whole : ld >= piece - 1 ? DyRows::Ragged : DyRows::Narrow;
}

}  // namespace np
