// An entry of a plan, and the rows that it stands for.  Plain C++, so that a host
// program can check it.
#pragma once

#include <stdint.h>

namespace np {

// Rows of a block: queries in the forward and the dq pass, keys in the dk/dv
// pass.  One entry of a plan covers that many rows of one sequence.
constexpr int kAttnRows = 128;

// {first token, length of the sequence, tile within it, 0}
struct AttnTile { int32_t start, len, tile, zero; };

// Row 0 <= `within` < kAttnRows of the tile, as a row of its sequence, in row0; false
// if there is none.  Plans lie in device memory that a caller may have given to
// something else by now: whatever the entry holds, a row that this finds lies in a
// sequence that lies in the batch (tiles below 2^24: row0 fits).
constexpr bool tile_row(const AttnTile& t, int64_t tokens, int within, int& row0) {
    row0 = (int)((uint32_t)t.tile * kAttnRows + (uint32_t)within);
    return t.start >= 0 && t.len > 0 && t.tile >= 0 && t.tile < 1 << 24 && row0 < t.len && (int64_t)t.start + t.len <= tokens;
}

}  // namespace np
