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
// its pieces leave partial results, which a second kernel merges. So every CTA has
// the same work whatever the lengths are, and at most two partial results.
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
// Costs of a key tile, and of an item's start and end.
constexpr int kCostTile = 4, kCostItem = 4;
// Least cost of a CTA's piece. Places where a cut moves on by a key tile are at most
// kCostItem + kCostTile apart (from an item's last tile to the next one's first), so no
// piece of so much is empty, and items of one key tile each get a CTA of their own.
constexpr int kCostPiece = kCostItem + kCostTile;

struct TurnSession {
    int32_t n, P, lo;   // new tokens (0: skipped), cached tokens before them, first row
};

// A key tile of an item; b == B: the end.
struct TurnPos {
    int32_t b, g, pair, t;
};

struct TurnShape {
    int32_t shift;      // tokens of a row tile, 128 / G, as a power of two
    int32_t Hkv;
    bool causal;
};

KVT_PLAN int turn_tiles_of(int keys) { return static_cast<int>((static_cast<uint32_t>(keys) + kTurnKeys - 1) / kTurnKeys); }
KVT_PLAN int turn_pairs(const TurnShape &s, const TurnSession &x) {
    return static_cast<int>((static_cast<uint32_t>(x.n) + (2u << s.shift) - 1) >> (s.shift + 1));
}
KVT_PLAN bool turn_narrow(const TurnShape &s, const TurnSession &x, int pair) {
    return x.n - (pair << (s.shift + 1)) <= 1 << s.shift;
}
// Own tokens that the item's rows can see.
KVT_PLAN int turn_own_keys(const TurnShape &s, const TurnSession &x, int pair) {
    const int64_t end = (static_cast<int64_t>(pair) + 1) << (s.shift + 1);
    return s.causal && end < x.n ? static_cast<int>(end) : x.n;
}
KVT_PLAN int turn_tiles(const TurnShape &s, const TurnSession &x, int pair) {
    return turn_tiles_of(x.P) + turn_tiles_of(turn_own_keys(s, x, pair));
}
// Costs are counted in I, 32 bits where all of a call's fit them (the device has no others; a plan in 64
// bits takes twice as long).
template <typename I>
KVT_PLAN I turn_item_cost(const TurnShape &s, const TurnSession &x, int pair) {
    return static_cast<I>(kCostTile) * turn_tiles(s, x, pair) + kCostItem;
}
// Cost of the first p pairs of a kv-head, p below the number of pairs: all of
// them full, so the own key tiles of a causal pair i are ceil((i + 1) * 2 tokens / 128).
template <typename I>
KVT_PLAN I turn_cost_before(const TurnShape &s, const TurnSession &x, I p) {
    I own;
    if (!s.causal) {
        own = p * turn_tiles_of(x.n);
    } else if ((2 << s.shift) >= kTurnKeys) {
        own = (2 << s.shift) / kTurnKeys * (p * (p + 1) / 2);
    } else {
        const int r_shift = 6 - s.shift;   // 128 / (2 tokens) pairs a key tile
        const I a = p >> r_shift;
        own = ((a * (a + 1) / 2) << r_shift) + (p - (a << r_shift)) * (a + 1);
    }
    return kCostTile * (p * turn_tiles_of(x.P) + own) + kCostItem * p;
}
template <typename I>
KVT_PLAN I turn_head_cost(const TurnShape &s, const TurnSession &x) {
    const int pairs = turn_pairs(s, x);
    return pairs == 0 ? 0 : turn_cost_before<I>(s, x, pairs - 1) + turn_item_cost<I>(s, x, pairs - 1);
}
// No call's cost is above this, and none of its parts.
KVT_PLAN int64_t turn_cost_bound(const TurnShape &s, int64_t total, int64_t B, int64_t longest) {
    return ((total >> (s.shift + 1)) + B) * s.Hkv * ((longest / kTurnKeys + 2) * kCostTile + kCostItem);
}

// Pieces that work of cost W makes, and where piece c begins: the first W % pieces
// are one longer than the others.
template <typename I>
KVT_PLAN int turn_pieces(I W, int ctas) {
    const I n = W / kCostPiece;
    return n < 1 ? 1 : n < ctas ? static_cast<int>(n) : ctas;
}
template <typename I>
KVT_PLAN I turn_cut(I W, int pieces, int c) {
    const I each = W >> 30 ? W / pieces : static_cast<I>(static_cast<uint32_t>(W) / static_cast<uint32_t>(pieces));
    const I longer = W - each * pieces;
    return each * c + (c < longer ? c : longer);
}

// The key tile at cost o of session b's work (o below Hkv times `head`, its head cost). t may be the item's
// number of key tiles: its end.
template <typename I>
KVT_PLAN TurnPos turn_locate(const TurnShape &s, const TurnSession &x, int b, I head, I o) {
    TurnPos p = {b, 0, 0, 0};
    for (; o >= head; o -= head) ++p.g;      // at most 8 kv-heads
    int lo = 0, hi = turn_pairs(s, x) - 1;   // the last pair that begins at or before o
    while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (turn_cost_before<I>(s, x, mid) <= o) lo = mid;
        else hi = mid - 1;
    }
    p.pair = lo;
    const I in = o - turn_cost_before<I>(s, x, lo) - kCostItem;
    p.t = in <= 0 ? 0 : static_cast<int>((in + kCostTile - 1) / kCostTile);
    return p;
}

}  // namespace kvt
