// The plan of attention calls over several new tokens, for tests/test_turn_plan_host.py.
#include "turn_plan.h"

using namespace kvt;

static TurnShape shape(int tokens, int Hkv, int causal, int many = 0) {
    int shift = 0;
    while (1 << shift < tokens) ++shift;
    return {shift, Hkv, causal != 0, many != 0};
}

extern "C" {
int32_t pairs(int tokens, int causal, int n) { return turn_pairs(shape(tokens, 1, causal), {n, 0, 0}); }
int32_t narrow(int tokens, int n, int pair) { return turn_narrow(shape(tokens, 1, 1), {n, 0, 0}, pair); }
int32_t tiles(int tokens, int causal, int n, int P, int pair) {
    return turn_tiles(shape(tokens, 1, causal), {n, P, 0}, pair);
}
int64_t cost_before(int tokens, int causal, int many, int n, int P, int pair) {
    return turn_cost_before<int64_t>(shape(tokens, 1, causal, many), {n, P, 0}, pair);
}
int64_t head_cost(int tokens, int causal, int many, int n, int P) {
    return turn_head_cost<int64_t>(shape(tokens, 1, causal, many), {n, P, 0});
}
int64_t head_cost_32(int tokens, int causal, int many, int n, int P) {
    return turn_head_cost<int32_t>(shape(tokens, 1, causal, many), {n, P, 0});
}
int64_t cost_bound(int tokens, int Hkv, int many, int64_t total, int64_t B, int64_t longest) {
    return turn_cost_bound(shape(tokens, Hkv, 1, many), total, B, longest);
}
static void put(const TurnPos &p, int32_t *pos) {
    pos[0] = p.g;
    pos[1] = p.pair;
    pos[2] = p.t;
}
void locate(int tokens, int Hkv, int causal, int many, int n, int P, int64_t o, int32_t *pos) {
    const TurnShape s = shape(tokens, Hkv, causal, many);
    const TurnSession x = {n, P, 0};
    put(turn_locate<int64_t>(s, x, 0, turn_head_cost<int64_t>(s, x), o), pos);
}
void locate_32(int tokens, int Hkv, int causal, int many, int n, int P, int64_t o, int32_t *pos) {
    const TurnShape s = shape(tokens, Hkv, causal, many);
    const TurnSession x = {n, P, 0};
    put(turn_locate<int32_t>(s, x, 0, turn_head_cost<int32_t>(s, x), static_cast<int32_t>(o)), pos);
}
int32_t pieces(int many, int64_t W, int ctas) { return turn_pieces(shape(16, 1, 1, many), W, ctas); }
int32_t is_many(int64_t W, int ctas) { return turn_many(W, ctas); }
int64_t cut(int64_t W, int n, int c) { return turn_cut(W, n, c); }
int64_t cut_32(int64_t W, int n, int c) { return turn_cut(static_cast<int32_t>(W), n, c); }
int32_t tile_cost(int many, int narrow) {
    const TurnCosts c = turn_costs(shape(16, 1, 1, many));
    return narrow ? c.narrow_tile : c.tile;
}
int32_t longest(int64_t max_blocks, int bt) { return turn_longest(max_blocks, bt); }
int32_t tiles_of(int keys) { return turn_tiles_of(keys); }
int32_t q_tiles(int narrow) { return turn_q_tiles(narrow != 0); }
int32_t q_waits(int stream, int narrow) { return turn_q_waits(stream, narrow != 0); }
int32_t item_cost(int many) { return turn_costs(shape(16, 1, 1, many)).item; }
}
