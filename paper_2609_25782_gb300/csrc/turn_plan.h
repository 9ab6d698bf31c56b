// How the work of an attention call over several new tokens per session is laid
// out and shared among the CTAs: plain integer code, for the kernel and for
// tests without a GPU.
//
// A row tile is 128 rows of one kv-head: 128 / G tokens times the G query heads
// that share it. An item is one (session, kv-head, pair of row tiles); it reads
// key tiles of 128: the cached tokens', then those of the call's own tokens that
// its rows can see. An item whose tokens fit one row tile is narrow: the CTA's two
// streams then take every other key tile of it instead of a row tile each.
//
// All items in order (session, kv-head, pair) make one line of costs, cut into
// equal pieces, one per CTA. A cut may fall between any two key tiles of an item:
// its pieces leave partial results, which the last one to finish merges. So every
// CTA has the same work whatever the lengths are, and at most two pieces of its
// own need merging.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define KVT_PLAN __host__ __device__ inline
#else
#define KVT_PLAN inline
#endif

namespace kvt {

constexpr int kTurnRows = 128;    // rows of a row tile
constexpr int kTurnKeys = 128;    // keys of a key tile
// Costs of a key tile of a pair, of a narrow item, and of an item's start and end.
constexpr int kCostPair = 4, kCostNarrow = 3, kCostItem = 4;
// Least cost of a CTA's piece. Over kCostItem + kCostPair no piece is empty.
constexpr int kCostPiece = 12;
static_assert(kCostPiece > kCostItem + kCostPair, "every piece has a key tile");

struct TurnSession {
    int32_t n, P, lo;   // new tokens (0: skipped), cached tokens before them, first row
};

// A key tile of an item; b == B: the end.
struct TurnPos {
    int32_t b, g, pair, t;
};

struct TurnShape {
    int32_t tokens;     // of a row tile, 128 / G
    int32_t Hkv;
    bool causal;
};

KVT_PLAN int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

KVT_PLAN int turn_pairs(const TurnShape &s, const TurnSession &x) {
    return static_cast<int>(ceil_div(x.n, 2 * s.tokens));
}
KVT_PLAN bool turn_narrow(const TurnShape &s, const TurnSession &x, int pair) {
    return x.n - pair * 2 * s.tokens <= s.tokens;
}
// Own tokens that the item's rows can see.
KVT_PLAN int turn_own_keys(const TurnShape &s, const TurnSession &x, int pair) {
    const int64_t end = static_cast<int64_t>(pair + 1) * 2 * s.tokens;
    return s.causal && end < x.n ? static_cast<int>(end) : x.n;
}
KVT_PLAN int turn_cached_tiles(const TurnSession &x) {
    return static_cast<int>(ceil_div(x.P, kTurnKeys));
}
KVT_PLAN int turn_tiles(const TurnShape &s, const TurnSession &x, int pair) {
    return turn_cached_tiles(x) + static_cast<int>(ceil_div(turn_own_keys(s, x, pair), kTurnKeys));
}
KVT_PLAN int turn_tile_cost(const TurnShape &s, const TurnSession &x, int pair) {
    return turn_narrow(s, x, pair) ? kCostNarrow : kCostPair;
}
KVT_PLAN int64_t turn_item_cost(const TurnShape &s, const TurnSession &x, int pair) {
    return static_cast<int64_t>(turn_tile_cost(s, x, pair)) * turn_tiles(s, x, pair) + kCostItem;
}
// Cost of the first p pairs of a kv-head, p below the number of pairs: all of
// them full, so the own key tiles of a causal pair i are ceil((i + 1) * 2 tokens / 128).
KVT_PLAN int64_t turn_cost_before(const TurnShape &s, const TurnSession &x, int64_t p) {
    const int64_t cached = turn_cached_tiles(x);
    int64_t own;
    if (!s.causal) {
        own = p * ceil_div(x.n, kTurnKeys);
    } else if (2 * s.tokens >= kTurnKeys) {
        own = 2 * s.tokens / kTurnKeys * (p * (p + 1) / 2);
    } else {
        const int64_t r = kTurnKeys / (2 * s.tokens), a = p / r;   // r pairs a key tile
        own = r * (a * (a + 1) / 2) + (p - a * r) * (a + 1);
    }
    return kCostPair * (p * cached + own) + kCostItem * p;
}
KVT_PLAN int64_t turn_head_cost(const TurnShape &s, const TurnSession &x) {
    const int pairs = turn_pairs(s, x);
    return pairs == 0 ? 0 : turn_cost_before(s, x, pairs - 1) + turn_item_cost(s, x, pairs - 1);
}

// Pieces that work of cost W makes, and where piece c begins.
KVT_PLAN int turn_pieces(int64_t W, int ctas) {
    const int64_t n = W / kCostPiece;
    return n < 1 ? 1 : n < ctas ? static_cast<int>(n) : ctas;
}
KVT_PLAN int64_t turn_cut(int64_t W, int pieces, int c) { return W * c / pieces; }
// The last piece that begins at or before cost x.
KVT_PLAN int turn_piece_of(int64_t W, int pieces, int64_t x) {
    return static_cast<int>(((x + 1) * pieces - 1) / W);
}

// The key tile at cost o of session b's work (o below Hkv times its head cost), and the cost at
// which its item begins, from the session's start. t may be the item's number of key tiles: its end.
KVT_PLAN TurnPos turn_locate(const TurnShape &s, const TurnSession &x, int b, int64_t o, int64_t *item_at) {
    const int64_t head = turn_head_cost(s, x);
    TurnPos p;
    p.b = b;
    p.g = static_cast<int>(o / head);
    o -= p.g * head;
    int lo = 0, hi = turn_pairs(s, x) - 1;   // the last pair that begins at or before o
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (turn_cost_before(s, x, mid) <= o) lo = mid;
        else hi = mid - 1;
    }
    p.pair = lo;
    const int64_t at = turn_cost_before(s, x, lo);
    *item_at = p.g * head + at;
    const int64_t in = o - at - kCostItem;
    p.t = in <= 0 ? 0 : static_cast<int>(ceil_div(in, turn_tile_cost(s, x, lo)));
    return p;
}

// Pieces that the item at cost U, of `tiles` key tiles, is cut into: first .. last.
KVT_PLAN void turn_item_pieces(int64_t W, int pieces, int64_t U, int tiles, int tile_cost, int *first, int *last) {
    *first = turn_piece_of(W, pieces, U + kCostItem);
    *last = turn_piece_of(W, pieces, U + kCostItem + static_cast<int64_t>(tiles - 1) * tile_cost);
}

}  // namespace kvt
