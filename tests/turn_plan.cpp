// The plan of attention calls over several new tokens, for tests/test_turn_plan_host.py.
#include "turn_plan.h"

using namespace kvt;

static TurnShape shape(int tokens, int Hkv, int causal) { return {tokens, Hkv, causal != 0}; }

extern "C" {
int32_t pairs(int tokens, int causal, int n) { return turn_pairs(shape(tokens, 1, causal), {n, 0, 0}); }
int32_t tiles(int tokens, int causal, int n, int P, int pair) {
    return turn_tiles(shape(tokens, 1, causal), {n, P, 0}, pair);
}
int32_t tile_cost(int tokens, int causal, int n, int pair) {
    return turn_tile_cost(shape(tokens, 1, causal), {n, 0, 0}, pair);
}
int64_t cost_before(int tokens, int causal, int n, int P, int pair) {
    return turn_cost_before(shape(tokens, 1, causal), {n, P, 0}, pair);
}
int64_t head_cost(int tokens, int causal, int n, int P) {
    return turn_head_cost(shape(tokens, 1, causal), {n, P, 0});
}
int64_t locate(int tokens, int Hkv, int causal, int n, int P, int64_t o, int32_t *pos) {
    int64_t at;
    const TurnPos p = turn_locate(shape(tokens, Hkv, causal), {n, P, 0}, 0, o, &at);
    pos[0] = p.g;
    pos[1] = p.pair;
    pos[2] = p.t;
    return at;
}
int32_t pieces(int64_t W, int ctas) { return turn_pieces(W, ctas); }
int64_t cut(int64_t W, int n, int c) { return turn_cut(W, n, c); }
void item_pieces(int64_t W, int n, int64_t U, int tiles, int cost, int32_t *out) {
    turn_item_pieces(W, n, U, tiles, cost, &out[0], &out[1]);
}
int32_t item_overhead() { return kCostItem; }
}
