// Driver of tests/test_attn_tile.py: an entry of a plan finds the rows that it stands
// for (csrc/np_attn_tile.h), and one that no plan holds none.
#include "np_attn_tile.h"

#include <cstdio>
#include <initializer_list>

using namespace np;

int main() {
    int failures = 0;
    auto expect = [&](bool ok, const AttnTile& t, int64_t tokens, int within) {
        if (!ok && failures++ < 10)
            std::printf("{%d, %d, %d} of %lld tokens, row %d\n", t.start, t.len, t.tile, (long long)tokens, within);
    };
    const int32_t ends[] = {INT32_MIN, -1000, -129, -128, -1, 0, 1, 2, 127, 128, 129, 1000, 1 << 23, (1 << 24) - 1, 1 << 24,
                            (1 << 24) + 1, 1 << 25, 33554433, 1 << 30, INT32_MAX - 128, INT32_MAX - 1, INT32_MAX};
    for (int32_t start : ends)
        for (int32_t len : ends)
            for (int32_t tile : ends)
                for (int64_t tokens : {int64_t(0), int64_t(1), int64_t(129), int64_t(5000), int64_t(INT32_MAX)})
                    for (int within : {0, 32, 64, 96}) {
                        const AttnTile t{start, len, tile, 0};
                        int row = -7;
                        const bool found = tile_row(t, tokens, within, row);
                        const bool holds = start >= 0 && len > 0 && (int64_t)start + len <= tokens && tile >= 0 &&
                                           (int64_t)tile * kAttnRows + within < len;
                        expect(found == holds, t, tokens, within);
                        if (found) expect(row == (int64_t)tile * kAttnRows + within && start + (int64_t)row < tokens, t, tokens, within);
                    }
    std::printf("%d failure(s)\n", failures);
    return failures != 0;
}
