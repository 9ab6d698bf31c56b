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
// Costs of a key tile of a wide and of a narrow item, of an item's start and end, and the least cost of a
// CTA's piece. Places where a cut moves on by a key tile are at most an item's and a tile's cost apart
// (from an item's last tile to the next one's first), so no piece of that much is empty.
struct TurnCosts {
    int32_t tile, narrow_tile, item, piece;
};
// With little work the shortest piece counts, and items of one key tile have a CTA each (one prompt of 37
// tokens 9.1 us; 12 with the other costs). With much, what the parts take: a wide item's tile 3 250 to 3 500
// cycles, a narrow one's 2 500, an item's end and the next one's start 6 000. What that gave when it was
// chosen (present times: turn_kernels.cu): 32 sessions of 20-60 drafts 140 -> 124 us, chunks of 1-200 tokens on 1K-40K
// 282 -> 236, turns of 300-3K tokens 935 -> 910.
constexpr TurnCosts kCostsFew = {4, 4, 4, 8}, kCostsMany = {4, 3, 8, 12};

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
    bool causal, many;   // many: the costs of much work
};

KVT_PLAN TurnCosts turn_costs(const TurnShape &s) {
    return {s.many ? kCostsMany.tile : kCostsFew.tile, s.many ? kCostsMany.narrow_tile : kCostsFew.narrow_tile,
            s.many ? kCostsMany.item : kCostsFew.item, s.many ? kCostsMany.piece : kCostsFew.piece};
}

KVT_PLAN int turn_tiles_of(int keys) { return static_cast<int>((static_cast<uint32_t>(keys) + kTurnKeys - 1) / kTurnKeys); }
// The longest session that a call takes: what a table row holds, and so that a position in a last key tile,
// or a group of 16 keys that a lane of a warp past it would have, still is a 32-bit one.
KVT_PLAN int32_t turn_longest(int64_t max_blocks, int block_tokens) {
    const int64_t holds = max_blocks * block_tokens, most = INT32_MAX - 4 * kTurnKeys;
    return static_cast<int32_t>(holds < most ? holds : most);
}
// Whether items of such sessions may be cut: those of at most two key tiles are not, which saves the merge's
// launch (a prompt of 37 tokens: 9.9 us with it, 9.1 without).
KVT_PLAN bool turn_cuts(int64_t longest) { return longest > kTurnKeys; }
KVT_PLAN int turn_pairs(const TurnShape &s, const TurnSession &x) {
    return static_cast<int>((static_cast<uint32_t>(x.n) + (2u << s.shift) - 1) >> (s.shift + 1));
}
KVT_PLAN bool turn_narrow(const TurnShape &s, const TurnSession &x, int pair) {
    return x.n - (pair << (s.shift + 1)) <= 1 << s.shift;
}
// Row tiles of q that an item loads, q[0] and (wide) q[1], and those whose copies a stream's products wait
// for, a bit each. The barrier of a q tile is one parity: a wait for its phase k passes at once while phase
// k - 1 is still on its way, unless that one has been waited for. So whoever waits for a barrier waits for
// each of its phases: stream 1 for q[0] in wide items too, which it does not read there, since it reads it
// in narrow ones, and a session's last item is often narrow.
KVT_PLAN int turn_q_tiles(bool narrow) { return narrow ? 1 : 2; }
KVT_PLAN int turn_q_waits(int stream, bool narrow) { return stream == 0 || narrow ? 1 : 3; }
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
    const TurnCosts cost = turn_costs(s);
    return static_cast<I>(turn_narrow(s, x, pair) ? cost.narrow_tile : cost.tile) * turn_tiles(s, x, pair) + cost.item;
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
    return turn_costs(s).tile * (p * turn_tiles_of(x.P) + own) + turn_costs(s).item * p;
}
template <typename I>
KVT_PLAN I turn_head_cost(const TurnShape &s, const TurnSession &x) {
    const int pairs = turn_pairs(s, x);
    return pairs == 0 ? 0 : turn_cost_before<I>(s, x, pairs - 1) + turn_item_cost<I>(s, x, pairs - 1);
}
// No call's cost is above this, and none of its parts.
KVT_PLAN int64_t turn_cost_bound(const TurnShape &s, int64_t total, int64_t B, int64_t longest) {
    return ((total >> (s.shift + 1)) + B) * s.Hkv * ((longest / kTurnKeys + 2) * turn_costs(s).tile + turn_costs(s).item);
}
// Whether a call has much work, by the bound of its cost with the costs of little: so much that, were it all
// narrow items' tiles, every CTA would have a piece. (The launch knows the tables' width, not the lengths.)
KVT_PLAN bool turn_many(int64_t bound, int ctas) {
    return bound >= int64_t(1) * kCostsMany.piece * kCostsFew.tile / kCostsMany.narrow_tile * ctas;
}

// Pieces that work of cost W makes, and where piece c begins: the first W % pieces
// are one longer than the others.
template <typename I>
KVT_PLAN int turn_pieces(const TurnShape &s, I W, int ctas) {
    const I n = s.many ? W / kCostsMany.piece : W / kCostsFew.piece;
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
    const I in = o - turn_cost_before<I>(s, x, lo) - turn_costs(s).item;
    if (in <= 0) p.t = 0;
    else if (!s.many) p.t = static_cast<int>((in + kCostsFew.tile - 1) / kCostsFew.tile);
    else if (turn_narrow(s, x, lo)) p.t = static_cast<int>((in + kCostsMany.narrow_tile - 1) / kCostsMany.narrow_tile);
    else p.t = static_cast<int>((in + kCostsMany.tile - 1) / kCostsMany.tile);
    return p;
}

}  // namespace kvt
