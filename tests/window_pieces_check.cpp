// The pieces of the queries past the windows (paper_2609_36692_amd/csrc/np_attn_tile.h) in the largest
// batches that the host side admits: num_tiles * heads up to 2^23 - 1.  One after the other, none empty, and
// together all steps.
#include "../paper_2609_36692_amd/csrc/np_attn_tile.h"

#include <cstdio>
#include <initializer_list>

using namespace np;

int main() {
    long long failures = 0, checked = 0;
    for (int group : {1, 3, 64, 1024, 8388607}) {
        const int64_t tiles = ((int64_t(1) << 23) - 1) / group, most = tiles * kAttnRows;
        for (int64_t len : {most, most - 1, most - 127})
            for (int64_t window : {int64_t(1), int64_t(1000), most / 2, most - 130})
                for (int tile : {0, 1})
                    for (int bm : {32, 64})
                        // Pieces of a tile, up to 512 and one more a tile, times up to 4 shares.
                        for (int pieces : {1, 2, 511, 2048}) {
                            const int64_t kt = (int64_t)tile * kAttnRows, past = len - kt - window;
                            if (window < 1 || past < 1 || past < pieces * (int64_t)bm) continue;
                            const AttnTile t{0, (int32_t)len, tile, 0};
                            int64_t at = 0, per = 0;
                            for (int p = 0; p < pieces; ++p) {
                                const PieceSteps s = piece_steps(t, (int)window, pieces, p, group, bm);
                                const int64_t first = (kt + window) / bm, count = (len - 1) / bm + 1 - first;
                                if (s.first != first || s.per != count || s.from != at || s.to <= s.from) {
                                    if (failures++ < 10)
                                        std::printf("group %d len %lld window %lld bm %d piece %d of %d: first %d per %d steps %d %d\n", group,
                                                    (long long)len, (long long)window, bm, p, pieces, s.first, s.per, s.from, s.to);
                                }
                                at = s.to;
                                per = s.per;
                            }
                            if (at != per * group) {
                                if (failures++ < 10) std::printf("group %d len %lld: %lld of %lld steps\n", group, (long long)len, (long long)at, (long long)per * group);
                            }
                            ++checked;
                        }
    }
    std::printf("%lld batches, %lld failure(s)\n", checked, failures);
    return failures != 0 || checked < 200;
}
