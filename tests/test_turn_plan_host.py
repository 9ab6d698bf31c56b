"""The line of items of prompt and draft attention, and its pieces, without a GPU: whatever the
lengths, every key tile of every item lies in exactly one piece, no piece is empty, and a piece that
holds part of an item knows which others hold the rest."""
import ctypes
import functools
import os
import random
import subprocess
import tempfile

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2609_25782_gb300", "csrc")


@functools.cache
def lib():
    with tempfile.TemporaryDirectory() as d:
        so = os.path.join(d, "turn_plan.so")
        subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-I", CSRC,
                        os.path.join(HERE, "turn_plan.cpp"), "-o", so], check=True)
        x = ctypes.CDLL(so)
    i32, i64 = ctypes.c_int32, ctypes.c_int64
    for name in ("cost_before", "head_cost", "locate", "cut"):
        getattr(x, name).restype = i64
    x.locate.argtypes = [i32] * 5 + [i64, ctypes.POINTER(i32)]
    x.pieces.argtypes = [i64, i32]
    x.cut.argtypes = [i64, i32, i32]
    x.item_pieces.argtypes = [i64, i32, i64, i32, i32, ctypes.POINTER(i32)]
    return x


def own_tiles(tokens, causal, n, pair):
    last = min((pair + 1) * 2 * tokens, n) if causal else n
    return -(-last // 128)


@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("tokens", [16, 32, 64, 128])
def test_costs_add_up(tokens, causal):
    x, r = lib(), random.Random(tokens)
    for _ in range(60):
        n = r.choice([1, 15, 16, 17, 64, r.randint(1, 64)]) if not causal else int(2 ** r.uniform(0, 12))
        P = r.choice([0, 1, 127, 128, 129, r.randint(0, 5000)])
        pairs = x.pairs(tokens, causal, n)
        assert pairs == -(-n // (2 * tokens))
        total = 0
        for p in range(pairs):
            assert x.cost_before(tokens, causal, n, P, p) == total
            t = x.tiles(tokens, causal, n, P, p)
            assert t == -(-P // 128) + own_tiles(tokens, causal, n, p)
            narrow = n - p * 2 * tokens <= tokens
            assert x.tile_cost(tokens, causal, n, p) == (3 if narrow else 4)
            total += t * (3 if narrow else 4) + x.item_overhead()
        assert x.head_cost(tokens, causal, n, P) == total


def layout(sessions, tokens, hkv, causal):
    """[(session, head, pair, cost at its start, tiles, cost of a tile)], and the whole cost."""
    x, at, items = lib(), 0, []
    for b, (n, P) in enumerate(sessions):
        for g in range(hkv):
            for p in range(x.pairs(tokens, causal, n)):
                t, c = x.tiles(tokens, causal, n, P, p), x.tile_cost(tokens, causal, n, p)
                items.append((b, g, p, at, t, c))
                at += t * c + x.item_overhead()
    return items, at


@pytest.mark.parametrize("seed", range(40))
def test_pieces_cover_the_line(seed):
    x, r = lib(), random.Random(seed)
    causal, tokens, hkv = r.random() < 0.6, r.choice([16, 32, 64, 128]), r.choice([1, 2, 4, 8])
    B = r.choice([1, 2, 5, 40])
    sessions = [(r.choice([0, 1, 16, 17, 40, 64]) if not causal else r.choice([0, int(2 ** r.uniform(0, 10))]),
                 r.choice([0, 1, 128, 129, r.randint(0, 6000)])) for _ in range(B)]
    items, W = layout(sessions, tokens, hkv, int(causal))
    if W == 0:
        return
    index = {i[:3]: k for k, i in enumerate(items)}
    starts, at = [], 0
    for n, P in sessions:
        starts.append(at)
        at += hkv * x.head_cost(tokens, int(causal), n, P)
    assert at == W
    for ctas in (1, 2, 7, 152):
        m = x.pieces(W, ctas)
        assert 1 <= m <= ctas
        cuts = []
        for c in range(m):
            u = x.cut(W, m, c)
            b = max(i for i in range(B) if starts[i] <= u and sessions[i][0] > 0)
            pos = (ctypes.c_int32 * 3)()
            item_at = x.locate(tokens, hkv, int(causal), *sessions[b], u - starts[b], pos)
            k = index[(b, pos[0], pos[1])]
            assert items[k][3] == starts[b] + item_at and 0 <= pos[2] <= items[k][4]
            cuts.append((k, pos[2]) if pos[2] < items[k][4] else (k + 1, 0))
        cuts.append((len(items), 0))
        assert cuts[0] == (0, 0) and all(a < b for a, b in zip(cuts, cuts[1:])), "an empty piece"
        # which pieces hold tiles of each item, by the cuts themselves
        for k, (_, _, _, U, t, cost) in enumerate(items):
            held = [c for c in range(m) if cuts[c] < (k, t) and cuts[c + 1] > (k, 0)]
            out = (ctypes.c_int32 * 2)()
            x.item_pieces(W, m, U, t, cost, out)
            assert held == list(range(out[0], out[1] + 1))
