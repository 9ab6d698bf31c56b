"""The line of items of prompt and draft attention, and its pieces, without a GPU: whatever the
lengths, every key tile of every item lies in exactly one piece, and no piece is empty."""
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
    for name in ("cost_before", "head_cost", "head_cost_32", "cut", "cut_32", "cost_bound"):
        getattr(x, name).restype = i64
    for name in ("locate", "locate_32"):
        getattr(x, name).restype = None
        getattr(x, name).argtypes = [i32] * 6 + [i64, ctypes.POINTER(i32)]
    x.pieces.argtypes = [i32, i64, i32]
    x.longest.argtypes = [i64, i32]
    x.is_many.argtypes = [i64, i32]
    x.cut.argtypes = x.cut_32.argtypes = [i64, i32, i32]
    x.cost_bound.argtypes = [i32, i32, i32, i64, i64, i64]
    return x


def own_tiles(tokens, causal, n, pair):
    last = min((pair + 1) * 2 * tokens, n) if causal else n
    return -(-last // 128)


@pytest.mark.parametrize("many", [0, 1])
@pytest.mark.parametrize("causal", [0, 1])
@pytest.mark.parametrize("tokens", [16, 32, 64, 128])
def test_costs_add_up(tokens, causal, many):
    x, r = lib(), random.Random(tokens)
    for _ in range(60):
        n = r.choice([1, 15, 16, 17, 64, r.randint(1, 64)]) if not causal else int(2 ** r.uniform(0, 12))
        P = r.choice([0, 1, 127, 128, 129, r.randint(0, 5000)])
        pairs = x.pairs(tokens, causal, n)
        assert pairs == -(-n // (2 * tokens))
        total = 0
        for p in range(pairs):
            assert x.cost_before(tokens, causal, many, n, P, p) == total
            t = x.tiles(tokens, causal, n, P, p)
            assert t == -(-P // 128) + own_tiles(tokens, causal, n, p)
            narrow = n - p * 2 * tokens <= tokens
            assert x.narrow(tokens, n, p) == narrow
            total += t * x.tile_cost(many, narrow) + x.item_cost(many)
        assert x.head_cost(tokens, causal, many, n, P) == x.head_cost_32(tokens, causal, many, n, P) == total


def layout(sessions, tokens, hkv, causal, many):
    """[(session, head, pair, cost at its start, tiles, cost of a tile)], and the whole cost."""
    x, at, items = lib(), 0, []
    for b, (n, P) in enumerate(sessions):
        for g in range(hkv):
            for p in range(x.pairs(tokens, causal, n)):
                t = x.tiles(tokens, causal, n, P, p)
                tile = x.tile_cost(many, x.narrow(tokens, n, p))
                items.append((b, g, p, at, t, tile))
                at += t * tile + x.item_cost(many)
    return items, at


@pytest.mark.parametrize("many", [0, 1])
@pytest.mark.parametrize("seed", range(60))
def test_pieces_cover_the_line(seed, many):
    x, r = lib(), random.Random(seed)
    causal, tokens, hkv = r.random() < 0.6, r.choice([16, 32, 64, 128]), r.choice([1, 2, 4, 8])
    B = r.choice([1, 2, 5, 40])
    sessions = [(r.choice([0, 1, 16, 17, 40, 64]) if not causal else r.choice([0, int(2 ** r.uniform(0, 10))]),
                 r.choice([0, 1, 128, 129, r.randint(0, 6000)])) for _ in range(B)]
    items, W = layout(sessions, tokens, hkv, int(causal), many)
    if W == 0:
        return
    index = {i[:3]: k for k, i in enumerate(items)}
    starts, at = [], 0
    for n, P in sessions:
        starts.append(at)
        at += hkv * x.head_cost(tokens, int(causal), many, n, P)
    assert at == W
    longest = max(P + (n if causal else 0) for n, P in sessions)
    assert W <= x.cost_bound(tokens, hkv, many, sum(n for n, _ in sessions), B, longest) < 2 ** 30
    for ctas in (1, 2, 7, 152):
        m = x.pieces(many, W, ctas)
        assert 1 <= m <= ctas and x.cut(W, m, 0) == 0 and x.cut(W, m, m) == W
        if x.is_many(layout(sessions, tokens, hkv, int(causal), 0)[1], ctas) and many:
            assert m == ctas, "a CTA without work"
        lengths = [x.cut(W, m, c + 1) - x.cut(W, m, c) for c in range(m)]
        assert max(lengths) - min(lengths) <= 1
        cuts = []
        for c in range(m):
            u = x.cut(W, m, c)
            b = max(i for i in range(B) if starts[i] <= u and sessions[i][0] > 0)
            pos = (ctypes.c_int32 * 3)()
            x.locate(tokens, hkv, int(causal), many, *sessions[b], u - starts[b], pos)
            again = (ctypes.c_int32 * 3)()
            x.locate_32(tokens, hkv, int(causal), many, *sessions[b], u - starts[b], again)
            assert list(pos) == list(again) and x.cut_32(W, m, c) == u
            k = index[(b, pos[0], pos[1])]
            assert 0 <= pos[2] <= items[k][4]
            # the tile whose cost contains the cut, or the one after it
            into = u - items[k][3] - x.item_cost(many)
            assert pos[2] == max(0, -(-into // items[k][5]))
            cuts.append((k, pos[2]) if pos[2] < items[k][4] else (k + 1, 0))
        cuts.append((len(items), 0))
        assert cuts[0] == (0, 0) and all(a < b for a, b in zip(cuts, cuts[1:])), "an empty piece"


@pytest.mark.parametrize("items", [1, 8, 100, 152])
def test_items_of_one_tile_have_a_piece_each(items):
    """A short prompt's items, all of one key tile: no CTA has two of them."""
    x = lib()
    W = items * (x.tile_cost(0, 0) + x.item_cost(0))
    m = x.pieces(0, W, 152)
    assert x.tile_cost(0, 0) == x.tile_cost(0, 1) and not x.is_many(W, 152)
    assert m == items and all(x.cut(W, m, c) == c * W // items for c in range(m + 1))


def test_cuts_of_work_past_32_bits():
    x = lib()
    for W in (2 ** 31 - 1, 2 ** 31, 2 ** 40 + 7):
        cuts = [x.cut(W, 152, c) for c in range(153)]
        assert cuts[0] == 0 and cuts[-1] == W
        assert max(b - a for a, b in zip(cuts, cuts[1:])) - min(b - a for a, b in zip(cuts, cuts[1:])) <= 1


def test_no_wait_for_a_q_tile_passes_a_phase_early():
    """A barrier of one parity lets a wait for phase k through after k phases less one, too. So in any order
    of wide and narrow items, each wait of a stream for a q tile's phase k comes after its wait for k - 1;
    and a stream waits for what it reads: its own tile in wide items, the only one in narrow ones."""
    x, r = lib(), random.Random(5)
    assert (x.q_tiles(0), x.q_tiles(1)) == (2, 1)
    for stream in (0, 1):
        assert x.q_waits(stream, 1) & 1 and x.q_waits(stream, 0) >> stream & 1
        for _ in range(200):
            loaded, done = [0, 0], [0, 0]                # phases begun; those that the stream knows to be over
            for narrow in [r.random() < 0.4 for _ in range(12)]:
                for tile in range(x.q_tiles(narrow)):
                    phase = loaded[tile]
                    loaded[tile] += 1
                    if not x.q_waits(stream, narrow) >> tile & 1:
                        continue
                    least, most = done[tile], loaded[tile]
                    passes = [n for n in range(least, most + 1) if n & 1 != phase & 1]   # phases over by then
                    assert passes and all(n > phase for n in passes), "a wait that the phase before lets through"
                    done[tile] = phase + 1


@pytest.mark.parametrize("bt", [16, 64])
def test_positions_of_the_longest_session_fit_32_bits(bt):
    """Tables may have rows of 2^26 blocks; a lane's group of 16 keys lies up to 496 past a tile's start."""
    x = lib()
    for blocks in (1, 7, 1 << 20, (1 << 25) - 1, 1 << 25, 1 << 26):
        longest = x.longest(blocks, bt)
        assert longest == blocks * bt or blocks * bt > longest > 2 ** 31 - 1024
        assert (x.tiles_of(longest) - 1) * 128 + 31 * 16 < 2 ** 31
