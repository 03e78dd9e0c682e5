// Host side of attention with a sliding window of the C ABI (include/normpre.h):
// its plan, argument checks and the calls of the kernels' launchers.
#include "np_checks.h"

#include <algorithm>
#include <cstring>
#include <new>
#include <vector>

using namespace np;

namespace {

// Blocks of the pieces, at most about this many: enough for every CU with one key head.
constexpr int64_t kMostPieces = 512;

int check_window(const normpre_window* w) {
    if (!w) return bad("the window is null");
    if (w->window < 1) return bad("window < 1");
    if (w->sinks < 0) return bad("sinks < 0");
    return NORMPRE_OK;
}

// Sequences have fewer than 2^31 tokens: larger numbers mean the same.
int clipped(int64_t n) { return (int)std::min<int64_t>(n, INT32_MAX); }

// Queries past the window of the first key of tile `tile`, where it is a sink.
int64_t past(int64_t len, int64_t tile, int window, int sinks) {
    const int64_t kt = tile * kAttnRows;
    return kt < sinks ? std::max<int64_t>(len - kt - window, 0) : 0;
}

// Queries of a piece: about as many as other blocks of keys have, not so few that the
// sums of the pieces cost more than they, and not more than kMostPieces of them.
int64_t piece_length(int64_t num_seqs, const int64_t* lens, int window, int sinks) {
    int64_t all = 0;
    for (int64_t i = 0; i < num_seqs; ++i)
        for (int64_t k = 0; k * kAttnRows < std::min<int64_t>(lens[i], sinks); ++k) all += past(lens[i], k, window, sinks);
    return std::max<int64_t>({(int64_t)window + kAttnRows, 256, (all + kMostPieces - 1) / kMostPieces});
}

// f(first token, length, tile, pieces) of every sink tile.
template <class F>
void each_sink(int64_t num_seqs, const int64_t* lens, int window, int sinks, F f) {
    const int64_t n = piece_length(num_seqs, lens, window, sinks);
    int64_t start = 0;
    for (int64_t i = 0; i < num_seqs; start += lens[i++])
        for (int64_t k = 0; k * kAttnRows < std::min<int64_t>(lens[i], sinks); ++k)
            if (const int64_t q = past(lens[i], k, window, sinks)) f(start, lens[i], k, (q + n - 1) / n);
}

int sink_rows(int sinks) { return std::min(kAttnRows, sinks > kAttnRows ? kAttnRows : (sinks + 31) / 32 * 32); }

int check_block(const normpre_attention* a, const normpre_window* w) {
    NP_CHECK(check_window(w));
    NP_CHECK(check_attention_sizes(a));
    if (a->causal != 1) return bad("a window is causal");
    if (w->sink_tiles < 0 || w->sink_tiles > a->num_tiles || w->sink_pieces < w->sink_tiles ||
        w->sink_pieces > w->sink_tiles + kMostPieces || (w->sink_tiles == 0 && w->sink_pieces != 0) ||
        (w->sinks == 0 && w->sink_tiles != 0))
        return bad("sink_tiles and sink_pieces are not the plan's");
    if ((a->num_tiles + w->sink_pieces) * a->heads > kMaxBlocks)
        return fail(NORMPRE_ERR_UNSUPPORTED, "more than 2^23 - 1 blocks of 128 rows");
    return NORMPRE_OK;
}

AttnArgs sizes(const normpre_attention* a, const normpre_window* w) {
    AttnArgs k = attention_sizes(a);
    // No sequence is longer: larger numbers mean the same.
    k.window = (int)std::clamp<int64_t>(w->window, 1, std::max<int64_t>(a->tokens, 1));
    k.sinks = (int)std::min(w->sinks, a->tokens);
    k.sink_tiles = (int)w->sink_tiles;
    k.sink_pieces = (int)w->sink_pieces;
    k.sink_rows = sink_rows(k.sinks);
    k.splits = window_splits((DType)a->dtype, k);
    return k;
}

// Floats in front of first_keys, and of it.
int64_t before(const AttnArgs& k) { return (attention_workspace(k) + 3) / 4 * 4; }
int64_t first_keys(const AttnArgs& k) {
    return 2 * ((int64_t)k.sink_pieces + k.sink_tiles) * k.splits * k.kv_heads * k.sink_rows * (k.dim <= 64 ? 64 : 128);
}

int attention(const normpre_attention* a, const normpre_window* w, bool backward, void* stream) {
    NP_CHECK(check_block(a, w));
    NP_CHECK(check_attention(a, backward));
    if (a->tokens == 0) return NORMPRE_OK;
    AttnArgs k = sizes(a, w);
    attention_operands(a, backward, k);
    const DType dt = (DType)a->dtype;
    if (!backward) return launched(launch_window_forward(dt, k, (hipStream_t)stream));
    float* ws = static_cast<float*>(a->workspace);
    if (!ws || !on(ws, 16) || a->workspace_bytes < 4 * (before(k) + first_keys(k)))
        return bad("workspace is null, misaligned or too small");
    attention_parts(ws, k);
    k.first_keys = ws + before(k);
    return launched(launch_window_backward(dt, k, (hipStream_t)stream));
}

}  // namespace

extern "C" {

int normpre_window_attention_plan_sizes(int64_t num_seqs, const int64_t* lens, normpre_window* window,
                                        int64_t* num_tiles) {
    NP_CHECK(check_window(window));
    if (!num_tiles) return bad("num_tiles is null");
    int64_t tiles, tokens;
    NP_CHECK(count_tiles(num_seqs, lens, tiles, tokens));
    *num_tiles = tiles;
    window->sink_tiles = window->sink_pieces = 0;
    each_sink(num_seqs, lens, clipped(window->window), clipped(window->sinks),
              [&](int64_t, int64_t, int64_t, int64_t pieces) {
                  ++window->sink_tiles;
                  window->sink_pieces += pieces;
              });
    return NORMPRE_OK;
}

int normpre_window_attention_plan(int64_t num_seqs, const int64_t* lens, const normpre_window* window, int32_t* plan,
                                  int64_t capacity) {
    NP_CHECK(check_window(window));
    int64_t n, tokens;
    NP_CHECK(count_tiles(num_seqs, lens, n, tokens));
    const int win = clipped(window->window), sinks = clipped(window->sinks);
    int64_t sink_tiles = 0, sink_pieces = 0;
    each_sink(num_seqs, lens, win, sinks, [&](int64_t, int64_t, int64_t, int64_t pieces) {
        ++sink_tiles;
        sink_pieces += pieces;
    });
    if (sink_tiles != window->sink_tiles || sink_pieces != window->sink_pieces)
        return bad("sink_tiles and sink_pieces are not those of these sequences");
    if (capacity < 8 * n + 8 * sink_tiles + 4 * sink_pieces) return bad("the plan does not fit");
    if (n == 0) return NORMPRE_OK;
    if (!plan) return bad("plan is null");
    try {
        // Rows that the other side streams past one tile.
        struct Item { AttnTile t; int64_t work; };
        std::vector<Item> items((size_t)n);
        for (int side = 0; side < 2; ++side) {
            size_t at = 0;
            int64_t start = 0, sink = 0;
            for (int64_t i = 0; i < num_seqs; start += lens[i++])
                for (int64_t k = 0; k * kAttnRows < lens[i]; ++k) {
                    const int64_t first = k * kAttnRows, end = std::min(lens[i], first + kAttnRows);
                    const int64_t from = std::max<int64_t>(first - win + 1, 0);
                    const int64_t met = side == 0 ? end - from + std::min<int64_t>(sinks, from)
                                                  : std::min<int64_t>(lens[i] - first, (int64_t)win + kAttnRows - 1);
                    const bool is_sink = side == 1 && past(lens[i], k, win, sinks) > 0;
                    items[at++] = {{(int32_t)start, (int32_t)lens[i], (int32_t)k, is_sink ? (int32_t)++sink : 0}, met};
                }
            std::stable_sort(items.begin(), items.end(), [](const Item& x, const Item& y) { return x.work > y.work; });
            for (size_t i = 0; i < items.size(); ++i)
                std::memcpy(plan + 4 * (side * (size_t)n + i), &items[i].t, sizeof(AttnTile));
        }
        // Sinks, and their pieces: longest sequences first, as the kernel takes them.
        std::vector<AttnSink> tiles;
        std::vector<AttnPiece> all;
        tiles.reserve((size_t)sink_tiles);
        all.reserve((size_t)sink_pieces);
        int32_t slot = 0;
        each_sink(num_seqs, lens, win, sinks, [&](int64_t start, int64_t len, int64_t tile, int64_t pieces) {
            for (int32_t p = 0; p < pieces; ++p) all.push_back({(int32_t)tiles.size(), p, slot + p, 0});
            tiles.push_back({{(int32_t)start, (int32_t)len, (int32_t)tile, slot}, (int32_t)pieces, {0, 0, 0}});
            slot += (int32_t)pieces + 1;             // and that of the tile's windows
        });
        auto length = [&](const AttnPiece& p) {
            const AttnSink& s = tiles[(size_t)p.sink];
            return past(s.tile.len, s.tile.tile, win, sinks) / s.pieces;
        };
        std::stable_sort(all.begin(), all.end(), [&](const AttnPiece& x, const AttnPiece& y) { return length(x) > length(y); });
        if (!tiles.empty()) {                        // and then there are pieces
            std::memcpy(plan + 8 * n, tiles.data(), tiles.size() * sizeof(AttnSink));
            std::memcpy(plan + 8 * n + 8 * sink_tiles, all.data(), all.size() * sizeof(AttnPiece));
        }
    } catch (const std::bad_alloc&) {
        return fail(NORMPRE_ERR_OOM, "no memory for the plan");
    }
    return NORMPRE_OK;
}

int normpre_window_attention_workspace(const normpre_attention* a, const normpre_window* window, int64_t* bytes) {
    if (!bytes) return bad("bytes is null");
    NP_CHECK(check_block(a, window));
    const AttnArgs k = sizes(a, window);
    *bytes = 4 * (before(k) + first_keys(k));
    return NORMPRE_OK;
}

int normpre_window_attention_forward(const normpre_attention* a, const normpre_window* window, void* stream) {
    return attention(a, window, false, stream);
}

int normpre_window_attention_backward(const normpre_attention* a, const normpre_window* window, void* stream) {
    return attention(a, window, true, stream);
}

}  // extern "C"
