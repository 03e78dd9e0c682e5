// Which tiles the passes of attention with a window go through
// (paper_2609_36692_amd/csrc/np_attn_tile.h), against the pairs that it has, over small
// sequences, windows and numbers of first tokens.
#include "../paper_2609_36692_amd/csrc/np_attn_tile.h"

#include <algorithm>
#include <cstdio>
#include <vector>

using namespace np;

static long long failures = 0;
static void fail(const char* what, int len, int window, int sinks, int a, int b) {
    if (failures++ < 10) std::printf("%s: len %d window %d sinks %d at %d %d\n", what, len, window, sinks, a, b);
}

static bool sees(int i, int j, int window, int sinks) { return j <= i && (j > i - window || j < sinks); }

// Blocks of queries: every key that one of them sees is met once, and tiles of the first keys
// alone hold no key of a window.
static void queries(int len, int window, int sinks, int rows, int bn) {
    for (int q0 = 0; q0 < len; q0 += rows) {
        const int end = std::min(len, q0 + rows);
        const KeyWalk w = key_walk(q0, end, window, sinks, bn);
        std::vector<int> met(len + bn, 0);
        int before = -1;
        for (int n = 0; n < w.steps; ++n) {
            const int t = w.tile(n);
            if (t <= before || t * bn >= end) fail("order of tiles", len, window, sinks, q0, n);
            before = t;
            const int limit = n < w.near ? std::min(sinks, w.near * bn) : len;
            if (limit <= t * bn) fail("empty tile", len, window, sinks, q0, t);
            for (int j = t * bn; j < std::min(limit, t * bn + bn); ++j) ++met[j];
            // What is met and not seen lies in the tiles of the windows.
            if (n < w.near)
                for (int j = t * bn; j < std::min(limit, t * bn + bn); ++j)
                    if (!sees(q0, j, window, sinks)) fail("unseen key", len, window, sinks, q0, j);
        }
        for (int i = q0; i < end; ++i)
            for (int j = 0; j <= i; ++j)
                if (sees(i, j, window, sinks) && met[j] != 1) fail("key of a query", len, window, sinks, i, j);
    }
}

// Blocks of keys: every query that sees one is met once, by the block of its windows or by
// one of the pieces of those past them.
static void keys(int len, int window, int sinks, int group, int pieces, int bm) {
    for (int tile = 0; tile * kAttnRows < len; ++tile) {
        const AttnTile t{0, len, tile, 0};
        const int kt = tile * kAttnRows, kend = std::min(len, kt + kAttnRows);
        std::vector<int> windows(len + bm, 0), past((size_t)(len + bm) * group, 0);
        const int last = kt + (int)std::min<int64_t>((int64_t)window + kAttnRows - 1, len - kt);
        for (int n = kt / bm; n * bm < last; ++n)
            for (int i = n * bm; i < n * bm + bm; ++i) ++windows[i];
        if (kt < sinks && len - kt > window)
            for (int p = 0; p < pieces; ++p) {
                const PieceSteps s = piece_steps(t, window, pieces, p, group, bm);
                for (int it = s.from; it < s.to; ++it) {
                    const int h = it / s.per, q0 = (s.first + it % s.per) * bm;
                    if (h >= group || q0 >= len) { fail("step of a piece", len, window, sinks, tile, it); continue; }
                    for (int i = q0; i < q0 + bm; ++i) ++past[(size_t)h * (len + bm) + i];
                }
            }
        for (int j = kt; j < kend; ++j)
            for (int i = j; i < len; ++i)
                for (int h = 0; h < group; ++h) {
                    // As the kernel masks them: by the distance alone, and past it sinks alone.
                    const int n = (i - j < window ? windows[i] : 0) +
                                  (i - j >= window && j < sinks ? past[(size_t)h * (len + bm) + i] : 0);
                    if (n != sees(i, j, window, sinks)) fail("query of a key", len, window, sinks, i, j);
                }
    }
}

int main() {
    for (int len : {1, 2, 31, 63, 64, 65, 127, 128, 129, 200, 257, 300})
        for (int window : {1, 2, 3, 31, 32, 33, 63, 64, 65, 100, 128, 129, 250, 299, 2147483647})
            for (int sinks : {0, 1, 2, 31, 33, 64, 65, 127, 128, 130, 200, 2147483647}) {
                for (int rows : {64, 128})
                    for (int bn : {32, 64}) queries(len, window, sinks, rows, bn);
                for (int bm : {32, 64})
                    for (int pieces : {1, 2, 5}) keys(len, window, sinks, pieces == 2 ? 3 : 1, pieces, bm);
            }
    // The longest sequence that there is.
    const int most = 2147483647;
    const KeyWalk w = key_walk(most - 100, most, 1000, 4, 64);
    if (w.near != 1 || w.tile(w.steps - 1) != (most - 1) / 64 || w.tile(1) != (most - 100 - 999) / 64) fail("far walk", most, 1000, 4, w.steps, w.skip);
    const PieceSteps s = piece_steps({0, most, 0, 0}, 1, 512, 511, 64, 32);
    if (s.to != (int64_t)s.per * 64 && (int64_t)s.per * 64 <= most) fail("far piece", most, 1, 1, s.from, s.to);
    std::printf("%lld failure(s)\n", failures);
    return failures != 0;
}
