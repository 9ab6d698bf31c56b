"""Selection of blocks against the definition: whole numbers, ties to the lowest block."""
import pytest
import torch

from sparse_cases import Cache

pytestmark = pytest.mark.gpu

HEADS = [(32, 4), (8, 8), (8, 4), (8, 2), (8, 1), (64, 8), (6, 6)]


@pytest.mark.parametrize("bt", [16, 64])
@pytest.mark.parametrize("T,top,first,last", [
    ([1], 1, 0, 1), ([1, 16, 17, 0], 2, 1, 1), ([15, 200, 3000, 64], 5, 0, 0), ([700] * 3, 7, 3, 4),
    ([9000, 40, 2000], 64, 1, 2), ([5000, 4999, 1], 200, 2, 8), ([300, 1000], 400, 1, 1), ([12345], 129, 0, 1),
])
def test_selection(cuda_dev, T, top, first, last, bt):
    c = Cache(T, bt=bt, seed=len(T) + top, q_std=2.0)
    c.make_bounds()
    c.check_selection(top, first, last)


@pytest.mark.parametrize("hq,hkv", HEADS)
def test_head_layouts_and_strides(cuda_dev, hq, hkv):
    c = Cache([2000, 333, 50], hq=hq, hkv=hkv, layers=3, layer=1, fused=True, seed=hq + hkv)
    c.make_bounds()
    c.check_selection(11, 1, 1)


@pytest.mark.parametrize("n", [500, 3000])
def test_ties_go_to_the_lowest_blocks(cuda_dev, n):
    """Scores of few values, and all of one."""
    c = Cache([16 * n, 16 * 300], seed=3)
    g = torch.Generator(device="cuda").manual_seed(1)
    c.codes.copy_(torch.randint(-1, 2, (*c.steps.shape, 1, 1), device="cuda", generator=g, dtype=torch.int8))
    c.steps.fill_(0.25)
    for top in (1, 7, 100, 256, n - 1):
        c.check_selection(top, 0, 0)
    c.codes.zero_()
    c.check_selection(33, 1, 2)
    c.q.zero_()
    c.codes.fill_(5)
    c.check_selection(33, 1, 2)


@pytest.mark.parametrize("spread", [0, 1, 40])
def test_steps_of_every_size(cuda_dev, spread):
    """Equal and very unequal steps, infinite ones among them, scores that overflow or vanish."""
    c = Cache([16 * 700, 16 * 90], seed=4)
    g = torch.Generator(device="cuda").manual_seed(2)
    c.codes.copy_(torch.randint(-127, 128, c.codes.shape, device="cuda", generator=g, dtype=torch.int32).to(torch.int8))
    e = torch.randint(-3 * spread - 1, 3 * spread + 1, c.steps.shape, device="cuda", generator=g)
    c.steps.copy_(torch.exp2(e.clamp(-132, 122).double()))
    c.steps[:, :, ::29] = float("inf")
    c.check_selection(20, 1, 1)
    c.check_selection(60, 2, 2)
    c.steps.fill_(2.0 ** 122)
    c.check_selection(20, 0, 0)
    c.steps.fill_(2.0 ** -132)
    c.check_selection(20, 0, 0)


def test_queries_of_every_size(cuda_dev):
    """Subnormal, huge, zero and not finite; one head far above the others of its group."""
    c = Cache([1600, 1600, 1600, 1600, 1600, 800], seed=5)
    c.make_bounds()
    c.q[0] *= 1e-39
    c.q[1] *= 1e37
    c.q[2, 5, 3], c.q[2, 6, 100], c.q[2, 20] = float("nan"), float("inf"), -float("inf")
    c.q[3].zero_()
    c.q[4, ::8] *= 1000
    c.q[5] = 2.0 ** -133
    c.check_selection(17, 1, 1)


def test_scores_bound_the_products(cuda_dev):
    """A block's score, in q's units, is at least the group's sum of products of each of its tokens."""
    c = Cache([1000], seed=6, q_std=3.0)
    c.make_bounds()
    c.select(10, 0, 0)
    for g in range(4):
        q = c.q[0, 8 * g:8 * g + 8].double()
        e = torch.floor(torch.log2(q.abs().max()))
        whole = torch.round(q * torch.exp2(10 - e))
        for j in range(c.blocks(0)):
            n = min(16, 1000 - 16 * j)
            k = c.hot[int(c.tab[0, j]), 0, 0, g, :n].double()
            most = (k @ whole.T).sum(1).max()
            # the sum's one rounding to 24 bits
            assert float(c.scores[0, g, j]) >= float(most) * (1 - 2 ** -24 * (1 if most > 0 else -1))


def test_bounds_of_forced_blocks_are_not_read(cuda_dev):
    c = Cache([500], seed=7)
    c.make_bounds()
    want = c.select(9, 2, 3).clone(), c.scores.clone()
    blk = torch.from_numpy(c.tab[0]).long().cuda()
    for j in (0, 1, 29, 30, 31):
        c.steps[:, :, blk[j]] = float("nan")
        c.codes[:, :, blk[j]] = 99
    c.select(9, 2, 3)
    assert torch.equal(c.selected, want[0]) and torch.equal(c.scores, want[1])


def test_bad_lengths_and_ids(cuda_dev):
    from paper_2609_25782_gb300 import kvtier
    c = Cache([500, 300, 400], seed=8)
    c.make_bounds()
    want = c.select(9).clone()
    for bad in (-1, c.width * 16 + 1, 2 ** 31 - 1):
        c.lens[1] = bad
        c.select(9)
        assert c.pool.check_device() == kvtier.KV_DEVICE_BAD_LENGTH
        assert torch.equal(c.selected[0], want[0]) and torch.equal(c.selected[2], want[2])
        assert (c.selected[1] == -1).all() and (c.scores[1] == 7).all()
    c.lens[1] = 300
    for bad in (-1, c.nb):
        c.tables[1, 5] = bad
        c.select(9)
        assert c.pool.check_device() == kvtier.KV_DEVICE_BAD_BLOCK
        assert torch.equal(c.selected[0], want[0]) and torch.equal(c.selected[2], want[2])


@pytest.mark.parametrize("width", [5000, 12288, 49152])
def test_wide_tables(cuda_dev, width):
    """Short rows in a wide table, and a row that fills it (all of one block's bounds)."""
    c = Cache([100, 16 * 40], seed=9, hq=8, hkv=2)
    c.make_bounds()
    wide = torch.full((2, width), -1, dtype=torch.int32, device="cuda")
    wide[:, :c.tables.shape[1]] = c.tables
    import numpy as np
    r = np.random.RandomState(1)
    c.tab = np.concatenate([c.tab, np.full((2, width - c.tab.shape[1]), -1, np.int32)], 1)
    c.tab[1] = r.randint(0, c.nb, width)
    c.tables, c.width, c.T[1] = torch.from_numpy(c.tab).cuda(), width, width * 16 - 3
    c.steps.copy_(torch.where(c.steps == 0, 1.0, c.steps))
    c.lens.copy_(torch.tensor(c.T, dtype=torch.int32))
    c.check_selection(300, 1, 1)


def test_many_rows_and_calls_at_once(cuda_dev):
    """Calls on several streams, without the scores as well; the same every time."""
    c = Cache([(97 * i) % 1500 for i in range(60)], seed=10)
    c.make_bounds()
    c.check_selection(24, 1, 1)
    want = c.selected.clone()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(4)]
    outs = [torch.zeros_like(want) for _ in streams]
    for _ in range(10):
        for st, o in zip(streams, outs):
            c.pool.select_blocks(0, c.q, c.bounds, c.tables, c.lens, c.B, c.width, o, first=1, last=1, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


@pytest.mark.parametrize("width", [24000, 28000, 49152])
@pytest.mark.parametrize("B", [20, 60])
def test_many_units_in_wide_tables(cuda_dev, B, width):
    """Tables too wide for two CTAs' keys on an SM, and just not; rows of one block to some thousands."""
    T = [(37 * i * i) % 900 + 1 for i in range(B)]
    T[3], T[B - 1], T[7] = 40000, 17, 0
    c = Cache(T, seed=31, hq=8, hkv=4, extra_width=width - 2500)
    assert c.width == width
    c.make_bounds()
    c.check_selection(9, 1, 2)
    assert c.scores[3, 0, 2500:].eq(-float("inf")).all()
