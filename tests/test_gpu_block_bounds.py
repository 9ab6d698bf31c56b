"""Bounds of blocks' keys against the definition in 64 bits."""
import pytest
import torch

from sparse_cases import D, Cache, bounds_of

pytestmark = pytest.mark.gpu


def check(c, layers, since=None, before=None):
    """All blocks that the call does; the others as they were."""
    codes, steps = before if before else (torch.zeros_like(c.codes), torch.zeros_like(c.steps))
    for b in range(c.B):
        if since and since[b] >= c.T[b]:
            continue
        for j in range((since[b] if since else 0) // c.bt, c.blocks(b)):
            for layer in layers:
                blk = int(c.tab[b, j])
                codes[layer, :, blk], steps[layer, :, blk] = c.reference_bounds(b, j, layer)
    assert c.pool.check_device() == 0
    assert torch.equal(c.codes, codes) and torch.equal(c.steps, steps)


@pytest.mark.parametrize("bt", [16, 64])
@pytest.mark.parametrize("hq,hkv", [(32, 4), (8, 8), (8, 4), (4, 2), (8, 1)])
def test_lengths_and_heads(cuda_dev, bt, hq, hkv):
    c = Cache([1, 0, 15, 16, 17, 63, 64, 65, 200, 1000], hq=hq, hkv=hkv, bt=bt, layers=3, seed=hkv)
    c.make_bounds()
    check(c, range(3))


@pytest.mark.parametrize("bt", [16, 64])
def test_one_layer_and_since(cuda_dev, bt):
    c = Cache([500, 64, 70, 0, 33], bt=bt, layers=2, seed=2)
    c.make_bounds(layer=1)
    check(c, [1])
    for since in ([0, 64, 65, 0, 32], [500, 0, 69, 0, 33], [16, 1, 64, 0, 0]):
        c.codes.fill_(3)
        c.steps.fill_(5.0)
        before = c.codes.clone(), c.steps.clone()
        c.make_bounds(since=since)
        check(c, range(2), since, before)


def test_bounds_hold_and_are_tight(cuda_dev):
    c = Cache([777], seed=3)
    c.make_bounds()
    values = c.codes.double() * c.steps.double()[..., None, None]
    for j in range(c.blocks(0)):
        n = min(16, 777 - 16 * j)
        k = c.hot[int(c.tab[0, j]), 0, 0, :, :n].double()
        hi, lo = values[0, :, int(c.tab[0, j])].unbind(1)
        step = c.steps[0, :, int(c.tab[0, j])].double()[:, None]
        assert (hi >= k.amax(1)).all() and (lo <= k.amin(1)).all()
        assert (hi - k.amax(1) < step).all() and (k.amin(1) - lo < step).all()


def test_values_of_every_size(cuda_dev):
    """Subnormal, tiny beside huge, all fraction bits set, zeros, one sign; each block its own kind."""
    c = Cache([16 * 64 + 5], layers=2, seed=4)
    g = torch.Generator(device="cuda").manual_seed(5)
    for j in range(c.blocks(0)):
        n = min(16, c.T[0] - 16 * j)
        bits = torch.randint(0, 1 << 15, (2, 4, n, D), device="cuda", generator=g, dtype=torch.int32)
        if j % 8 == 0:
            bits &= 0x7F                                  # subnormal
        elif j % 8 == 1:
            bits = bits % 0x7F80                          # every finite magnitude
        elif j % 8 == 2:
            bits = (bits & 0x3F80) | 0x7F                 # 255/128 of a power of two
        elif j % 8 == 3:
            bits = torch.zeros_like(bits)
        elif j % 8 == 4:
            bits = bits * 0 + torch.randint(0, 2, bits.shape, device="cuda", generator=g, dtype=torch.int32)
        elif j % 8 == 5:
            bits = (bits % 0x300) + 0x3E00
        elif j % 8 == 6:
            bits = bits * 0 + 0x7F7F                      # the largest
        else:
            bits = bits % 0x4000
        if j % 3:
            bits |= torch.randint(0, 2, bits.shape, device="cuda", generator=g, dtype=torch.int32) << 15
        elif j % 2:
            bits |= 1 << 15
        bits = torch.where(bits >= 1 << 15, bits - (1 << 16), bits).to(torch.int16)
        c.hot[int(c.tab[0, j]), :, 0, :, :n] = bits.view(torch.bfloat16)
    c.make_bounds()
    check(c, range(2))


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_keys_that_are_not_finite(cuda_dev, value):
    """Only their own block and head; what lies past the end may be anything."""
    c = Cache([100, 40], layers=2, seed=6)
    c.make_bounds()
    codes, steps = c.codes.clone(), c.steps.clone()
    blk = int(c.tab[0, 2])
    c.hot[blk, 1, 0, 2, 5, 77] = value
    c.make_bounds()
    assert (c.codes[1, 2, blk, 0] == 127).all() and (c.codes[1, 2, blk, 1] == -127).all()
    assert c.steps[1, 2, blk] == float("inf")
    codes[1, 2, blk], steps[1, 2, blk] = c.codes[1, 2, blk], c.steps[1, 2, blk]
    assert torch.equal(c.codes, codes) and torch.equal(c.steps, steps)
    assert bounds_of(c.hot[blk, 1, 0, 2, :16])[1] == float("inf")


def test_bad_lengths_ids_and_wide_tables(cuda_dev):
    from paper_2609_25782_gb300 import kvtier
    c = Cache([100, 40, 70], seed=7, extra_width=3000)
    good = c.lens.clone()
    for change in ([-1, 40, 70], [100, c.width * 16 + 1, 70], [100, 40, 2 ** 31 - 1]):
        c.lens.copy_(torch.tensor(change, dtype=torch.int32))
        c.codes.zero_(), c.steps.zero_()
        c.make_bounds()
        assert c.pool.check_device() == kvtier.KV_DEVICE_BAD_LENGTH
        for b in range(3):
            some = c.steps[0, :, torch.from_numpy(c.tab[b, :c.blocks(b)]).long()]
            assert ((some != 0).all() if change[b] == c.T[b] else (some == 0).all())
    c.lens.copy_(good)
    for since in ([101, 0, 0], [0, -1, 0]):
        c.make_bounds(since=since)
        assert c.pool.check_device() == kvtier.KV_DEVICE_BAD_LENGTH
    c.codes.zero_(), c.steps.zero_()
    c.tables[1, 1] = c.nb
    c.make_bounds()
    assert c.pool.check_device() == kvtier.KV_DEVICE_BAD_BLOCK
    c.tab[1, 1] = c.tab[1, 0]                             # (the reference's: not looked at)
    assert (c.steps[0, :, int(c.tab[1, 0])] != 0).all() and (c.steps[0, :, int(c.tab[2, 4])] != 0).all()


def test_many_rows(cuda_dev):
    """More rows than a CTA has threads, several of them empty."""
    T = [(37 * i) % 90 for i in range(700)]
    c = Cache(T, hq=2, hkv=1, seed=8)
    c.make_bounds()
    check(c, [0])


def test_captured_and_replayed(cuda_dev):
    c = Cache([300, 120, 5], layers=2, seed=9)
    since = torch.tensor([0, 0, 0], dtype=torch.int32, device="cuda")
    c.make_bounds(since=since)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.make_bounds(since=since, stream=torch.cuda.current_stream())
    for now in ([0, 0, 0], [290, 100, 5]):
        since.copy_(torch.tensor(now, dtype=torch.int32))
        c.codes.fill_(1), c.steps.fill_(2.0)
        before = c.codes.clone(), c.steps.clone()
        graph.replay()
        check(c, range(2), now, before)
