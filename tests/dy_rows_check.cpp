// Driver of tests/test_dy_rows.py: the elements of dy that the weight gradient's
// tiles read (csrc/np_dy_rows.h), for every small shape, against those there are.
#include "np_dy_rows.h"

#include <algorithm>
#include <cstdio>

using namespace np;

// Index of the last element read of dy [tokens][outer], rows ld apart, in shares of
// `chunk` tokens.
static int64_t last_read(DyRows rows, int64_t tokens, int64_t outer, int64_t ld, int64_t piece, int64_t chunk) {
    int64_t top = -1;
    for (int64_t t0 = 0; t0 < tokens; t0 += chunk) {
        const int64_t t1 = std::min(tokens, t0 + chunk);
        for (int64_t t = t0; t < t1; t += kDyTile) {
            const bool last = t + kDyTile >= t1, guarded = rows == DyRows::Narrow || (rows == DyRows::Ragged && last);
            for (int64_t r = t; r < t + kDyTile; ++r) {
                const int64_t row = std::min(r, t1 - 1);      // past the last token: a copy of it
                for (int64_t c = 0; c < outer + 2 * piece; c += piece) {
                    const int64_t from = std::min(c, rows == DyRows::Whole ? outer - piece : outer - 1);
                    const int64_t n = guarded ? std::min(piece, outer - c) : piece;
                    if (n > 0) top = std::max(top, row * ld + from + n - 1);
                }
            }
        }
    }
    return top;
}

int main() {
    int failures = 0, past = 0;
    for (int64_t piece : {4, 8})
        for (int64_t outer = 1; outer <= 20; ++outer)
            for (int64_t ld = outer; ld <= outer + 9; ++ld)
                for (int64_t tokens = 1; tokens <= 131; ++tokens)
                    for (int64_t chunk : {kDyTile, 2 * kDyTile, 4 * kDyTile, 8 * kDyTile}) {
                        const int64_t end = (tokens - 1) * ld + outer;
                        const DyRows rows = dy_rows(outer, ld, piece);
                        if (last_read(rows, tokens, outer, ld, piece, chunk) >= end) {
                            if (failures++ < 10)
                                std::printf("%lld tokens of %lld, rows %lld apart, pieces of %lld, shares of %lld: read past the end\n",
                                            (long long)tokens, (long long)outer, (long long)ld, (long long)piece, (long long)chunk);
                        }
                        // That the narrow rows are no more than they must be.
                        if (rows == DyRows::Narrow)
                            past += last_read(DyRows::Ragged, tokens, outer, ld, piece, chunk) >= end;
                    }
    std::printf("%d narrow shapes would be read past their end in whole pieces\n%d failure(s)\n", past, failures);
    return failures != 0 || past == 0;
}
