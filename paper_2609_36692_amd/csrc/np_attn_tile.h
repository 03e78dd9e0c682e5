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

// The key tiles of bn rows that a block of queries from row q0 on meets, of the keys
// before row `end`: those of the first keys (sinks), `near` of them, then those from the
// window of its first query on, `skip` tiles later.
struct KeyWalk {
    int steps, near, skip;
    constexpr int tile(int n) const { return n < near ? n : n + skip; }
};
constexpr KeyWalk key_walk(int q0, int end, int window, int sinks, int bn) {
    const int first = (q0 < window ? 0 : q0 - (window - 1)) / bn;
    const int wanted = sinks / bn + (sinks % bn != 0), near = wanted < first ? wanted : first;
    return {(end - 1) / bn + 1 - (first - near), near, first - near};
}

// With a window, what follows a plan's 2 x tiles entries: for each key tile with keys that
// queries past their windows see (sinks) an AttnSink, and for each piece of those queries
// an AttnPiece.  The key tile's own entry then has 1 + the number of its AttnSink for zero.
// Sums of a piece go to its slot (each share of it, as of any block, to one of its own); those of
// the tile's windows to the slot behind its last, where there is one share.
struct AttnSink { AttnTile tile; int32_t pieces, zero[3]; };      // tile.zero: the first piece's slot
struct AttnPiece { int32_t sink, piece, slot, zero; };

// The queries of piece `piece` of a sink tile: steps [from, to) over the bm-row tiles
// of queries from tile `first` on, `per` of them, once for each of `group` heads.  Queries
// before the window of the tile's first key has passed see it as any key; the others
// are the pieces'.
struct PieceSteps { int first, per, from, to; };
constexpr PieceSteps piece_steps(const AttnTile& t, int window, int pieces, int piece, int group, int bm) {
    const int kt = t.tile * kAttnRows;
    const int past = t.len - kt > window ? kt + window : t.len;
    const int first = past / bm, per = past < t.len ? (t.len - 1) / bm + 1 - first : 0;
    const int64_t all = (int64_t)per * group;
    return {first, per, (int)(all * piece / pieces), (int)(all * (piece + 1) / pieces)};
}

}  // namespace np
