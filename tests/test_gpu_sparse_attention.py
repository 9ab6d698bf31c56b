"""Attention of one new token over listed blocks against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from sparse_cases import Cache

pytestmark = pytest.mark.gpu

HEADS = [(32, 4), (8, 8), (8, 4), (8, 2), (8, 1), (64, 8), (6, 6)]


@pytest.mark.parametrize("bt", [16, 64])
@pytest.mark.parametrize("T,top", [
    ([1], 1), ([2, 16, 17], 1), ([0, 5, 64], 3), ([65, 1000, 31], 10), ([3000] * 3, 40), ([5000, 1, 700], 129),
    ([9000], 500), ([250] * 40, 12), ([2000] * 70, 33),
])
@pytest.mark.parametrize("new", [False, True])
def test_lists_in_any_order(cuda_dev, T, top, bt, new):
    c = Cache(T, bt=bt, seed=len(T) + top, q_std=2.0)
    c.random_lists(top, seed=top)
    c.check(new)


@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("new", [False, True])
def test_head_layouts_and_strides(cuda_dev, hq, hkv, new):
    c = Cache([2000, 333, 50], hq=hq, hkv=hkv, layers=3, layer=1, fused=True, seed=hq + hkv, q_std=4.0)
    c.random_lists(20, seed=1)
    c.check(new)


def test_out_fp32(cuda_dev):
    c = Cache([2000, 1, 130], seed=3, dtype=torch.float32)
    c.random_lists(60, seed=2)
    c.check(True)


@pytest.mark.parametrize("scale", [-0.3, 0.0, 1e-3, 2.0])
def test_scales(cuda_dev, scale):
    c = Cache([1000, 40], seed=4)
    c.scale = scale
    c.random_lists(33, seed=3)
    c.check()


def test_large_scores(cuda_dev):
    """Scores of several hundred: one key takes nearly all, running maxima jump."""
    c = Cache([1500, 3000, 90], seed=5, q_std=60.0)
    c.random_lists(80, seed=4)
    c.check()


def test_rows_that_see_nothing_are_zeros(cuda_dev):
    c = Cache([500, 0, 300], seed=6)
    c.random_lists(9, seed=5)
    c.selected[0, 1:3] = -1
    c.selected[2] = -7
    for new in (False, True):
        c.out.fill_(7.0)
        c.check(new)                                     # the new token is written all the same
        assert (c.out[0, 8:24] == 0).all() and (c.out[1:] == 0).all() and (c.out[0, :8] != 0).any()


def test_a_block_named_twice_counts_twice(cuda_dev):
    c = Cache([200], seed=7)
    c.selected = torch.tensor([3, 5, 3, 12, 12, 12], dtype=torch.int32, device="cuda").expand(1, 4, 6).contiguous()
    c.check(True)


def test_what_lies_past_the_end_is_not_seen(cuda_dev):
    """Infinities and NaN behind the last token, whole blocks of them not listed."""
    c = Cache([77, 130], seed=8)
    c.selected = torch.tensor([[4, 1], [8, 0]], dtype=torch.int32, device="cuda")[:, None].expand(2, 4, 2).contiguous()
    for j in (0, 2, 3):
        c.hot[int(c.tab[0, j])] = float("inf")
    c.check()
    c.check(True)


def test_all_blocks_is_the_decode_step(cuda_dev):
    c = Cache([777, 1, 2000], seed=9, dtype=torch.float32)
    n = c.width
    lists = torch.arange(n, device="cuda").int().expand(3, 4, n).clone()
    for b in range(3):
        lists[b, :, c.blocks(b):] = -1
    c.selected = lists
    c.check()
    from paper_2609_25782_gb300 import Pool
    pool = Pool(num_layers=1, num_hot_blocks=c.nb, cold_bytes=256, max_sessions=1, max_batch=3, max_context=n * 16)
    pool.hot.copy_(c.pool.hot)
    out = torch.empty_like(c.out)
    pool.decode_attention(0, c.q, c.tables, c.lens, 3, n, c.scale, out)
    torch.testing.assert_close(c.out, out, rtol=0, atol=8e-3)


def test_bad_lengths_blocks_and_ids(cuda_dev):
    from paper_2609_25782_gb300 import kvtier
    c = Cache([500, 300, 400], seed=10)
    c.random_lists(9, seed=6, holes=0.0)
    refs = [c.reference(b) for b in range(3)]
    for bad in (-1, c.width * 16 + 1, 2 ** 31 - 1):
        c.lens[1] = bad
        c.out.fill_(7.0)
        c.attend()
        assert c.pool.check_device() == kvtier.KV_DEVICE_BAD_LENGTH
        assert (c.out[1] == 7).all()
        c.assert_right(0, *refs[0]), c.assert_right(2, *refs[2])
    c.lens[1] = 300
    keep = c.selected.clone()
    for bad in (19, 2 ** 26, 2 ** 31 - 1):               # the row has 19 blocks: they are skipped
        c.selected[1, 2, 4] = bad
        c.attend()
        assert c.pool.check_device() == kvtier.KV_DEVICE_BAD_BLOCK
        got = c.out.clone()
        c.selected[1, 2, 4] = -1
        c.check()
        assert torch.equal(got, c.out)
        c.selected.copy_(keep)
    for bad in (-1, c.nb, 2 ** 31 - 1):
        c.tables[1, int(c.selected[1, 0, 0])] = bad
        c.attend()
        assert c.pool.check_device() == kvtier.KV_DEVICE_BAD_BLOCK
        c.assert_right(0, *refs[0]), c.assert_right(2, *refs[2])
        assert torch.isfinite(c.out[1]).all()


def test_lists_longer_than_the_sessions_and_wide_tables(cuda_dev):
    c = Cache([40, 900, 17], seed=11, extra_width=5000)
    c.random_lists(4000, seed=7)
    c.check(True)


def test_one_rows_nan_stays_its_own(cuda_dev):
    c = Cache([300, 200, 100], seed=12)
    c.random_lists(15, seed=8, holes=0.0)
    c.selected[1] = torch.arange(15, device="cuda").int().where(torch.arange(15, device="cuda") < 13, torch.tensor(-1, device="cuda").int())
    clean = c.attend().clone()
    c.hot[int(c.tab[1, 3])] = float("nan")
    c.out.fill_(7.0)
    c.attend()
    assert torch.equal(c.out[0], clean[0]) and torch.equal(c.out[2], clean[2]) and c.out[1].isnan().all()


def test_same_from_run_to_run_and_several_calls_at_once(cuda_dev):
    c = Cache([(211 * i) % 4000 for i in range(24)], seed=13, q_std=2.0)
    c.random_lists(100, seed=9)
    want = c.attend().clone()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(4)]
    outs = [torch.zeros_like(want) for _ in streams]
    for _ in range(20):
        for st, o in zip(streams, outs):
            c.pool.sparse_attention(0, c.q, c.selected, c.tables, c.lens, c.B, c.width, c.scale, o, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs) and c.pool.check_device() == 0


def test_captured_steps_with_padding(cuda_dev):
    """A graph of selection and attention, replayed for other lengths; a padded row has length 0."""
    c = Cache([700, 333, 90], seed=14)
    c.make_bounds()
    c.selected = torch.zeros(3, 4, 12, dtype=torch.int32, device="cuda")

    def step():
        st = torch.cuda.current_stream()
        c.pool.select_blocks(0, c.q, c.bounds, c.tables, c.lens, 3, c.width, c.selected, first=1, last=1, stream=st)
        c.pool.sparse_attention(0, c.q, c.selected, c.tables, c.lens, 3, c.width, c.scale, c.out, c.k, c.v, st)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for T in ([700, 333, 90], [650, 0, 33], [0, 0, 1]):
        c.T = T
        c.lens.copy_(torch.tensor(T, dtype=torch.int32))
        c.out.fill_(7.0)
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        for b in range(3):
            for g in range(4):
                assert c.selected[b, g].tolist() == c.reference_selection(b, g, 12)[0]
            c.assert_right(b, *c.reference(b, True))
    assert c.pool.check_device() == 0


def test_pool_of_over_32_bits_of_elements(cuda_dev):
    """Blocks past 2^32 elements of the arena and 2^31 bytes of bounds."""
    from paper_2609_25782_gb300 import Pool
    L, nb, bt = 48, 6000, 16                             # 9.4 GB
    pool = Pool(num_layers=L, num_hot_blocks=nb, cold_bytes=256, max_sessions=1, max_batch=1, max_context=16 * 64)
    pool.hot.zero_()
    hot, bounds = pool.hot_view(), pool.new_bounds()
    codes, steps = pool.bounds_views(bounds)
    g = torch.Generator(device="cuda").manual_seed(1)
    rows = torch.tensor([list(range(nb - 40, nb))], dtype=torch.int32, device="cuda")
    hot[nb - 40:] = torch.randn(40, L, 2, 4, bt, 128, device="cuda", generator=g).bfloat16()
    lens = torch.tensor([639], dtype=torch.int32, device="cuda")
    pool.block_bounds(-1, rows, lens, 1, 40, bounds)
    from sparse_cases import bounds_of
    want = bounds_of(hot[nb - 1, L - 1, 0, :, :15])
    assert torch.equal(codes[L - 1, :, nb - 1], want[0]) and torch.equal(steps[L - 1, :, nb - 1], want[1])
    q = torch.randn(1, 32, 128, device="cuda", generator=g).bfloat16()
    selected = torch.zeros(1, 4, 40, dtype=torch.int32, device="cuda")
    pool.select_blocks(L - 1, q, bounds, rows, lens, 1, 40, selected)
    assert (selected == torch.arange(40, device="cuda")).all()
    out = torch.zeros(1, 32, 128, device="cuda")
    pool.sparse_attention(L - 1, q, selected, rows, lens, 1, 40, 0.1, out)
    k, v = (hot[nb - 40:, L - 1, w].transpose(0, 1).reshape(4, 640, 128)[:, :639].double() for w in (0, 1))
    w = torch.softmax(q[0].double().view(4, 8, 128) @ k.transpose(1, 2) * 0.1, -1)
    torch.testing.assert_close(out[0].double(), (w @ v).view(32, 128), rtol=0, atol=4e-3)
    assert pool.check_device() == 0


def test_numpy_int_arguments_are_plain_numbers(cuda_dev):
    c = Cache([100], seed=15)
    c.random_lists(3, seed=1)
    c.pool.sparse_attention(0, c.q, c.selected, c.tables, c.lens, int(np.int64(1)), c.width, c.scale, c.out)
    assert c.pool.check_device() == 0


@pytest.mark.parametrize("kind", [np.int64, np.int32])
def test_numpy_numbers_give_the_same_results(cuda_dev, kind):
    c = Cache([400, 90], seed=15)
    c.make_bounds()
    c.select(6)
    want = c.selected.clone(), c.scores.clone(), c.attend().clone()
    c.selected.fill_(12345), c.scores.fill_(7.0), c.out.fill_(7.0)
    c.pool.select_blocks(kind(0), c.q, c.bounds, c.tables, c.lens, kind(2), kind(c.width), c.selected, first=kind(1), last=kind(1),
                         scores=c.scores)
    c.pool.sparse_attention(kind(0), c.q, c.selected, c.tables, c.lens, kind(2), kind(c.width), np.float64(c.scale), c.out)
    assert c.pool.check_device() == 0
    assert torch.equal(c.selected, want[0]) and torch.equal(c.scores, want[1]) and torch.equal(c.out, want[2])
    for b in range(2):
        c.assert_right(b, *c.reference(b))


def test_a_wait_that_runs_out(cuda_dev):
    """The hook's one call reports it and ends, the next ones are right; a context that goes on."""
    from paper_2609_25782_gb300 import kvtier
    for T, top in (([1000], 40), ([2000] * 130, 20)):    # few units and many
        c = Cache(T, seed=16)
        c.random_lists(top, seed=2, holes=0.0)
        kvtier.kv_pool_inject_decode_timeout(c.pool.handle, 1)
        c.attend()
        assert c.pool.check_device() == kvtier.KV_DEVICE_TIMEOUT
        for b in range(1, c.B):
            c.assert_right(b, *c.reference(b))
        c.check(True)


def test_infinite_keys_and_values(cuda_dev):
    """A score of -inf has no weight, whatever came before it; of +inf or with an infinite value nothing is finite."""
    c = Cache([400], seed=17, hq=8, hkv=1)
    c.selected = torch.arange(25, device="cuda").int().view(1, 1, 25)
    blk = [int(x) for x in c.tab[0]]
    c.q[0] = c.q[0].abs() + 0.1
    for j in (0, 1, 2, 13):
        c.hot[blk[j], 0, 0, 0, :, 5] = -float("inf")     # q is positive there
    c.hot[blk[14], 0, 0, 0, 3, 5] = -float("inf")
    seen = torch.tensor([t for t in range(400) if t // 16 not in (0, 1, 2, 13) and t != 14 * 16 + 3], device="cuda")
    k, v = (torch.stack([c.hot[blk[int(t) // 16], 0, w, 0, int(t) % 16] for t in seen]).double() for w in (0, 1))
    w = torch.softmax(c.q[0].double() @ k.T * c.scale, 1)
    c.attend()
    c.assert_right(0, w @ v, torch.sqrt((w * w) @ (v * v).sum(1)))
    c.hot[blk[9], 0, 1, 0, 2, 7] = float("inf")
    c.attend()
    assert (c.out[0, :, 7] == float("inf")).all() and torch.isfinite(c.out[0, :, 8]).all()
    c.hot[blk[9], 0, 1, 0, 2, 7] = 0
    c.hot[blk[9], 0, 0, 0, 2, 7] = float("inf")
    c.attend()
    assert c.out.isnan().all() and c.pool.check_device() == 0


def test_a_captured_step_behind_copies_and_two_streams(cuda_dev):
    """What a step waits for: a copy, kernels of two streams that meet, the step before it."""
    c = Cache([900, 333, 90], seed=18)
    c.make_bounds()
    c.selected = torch.zeros(3, 4, 12, dtype=torch.int32, device="cuda")
    qs = [torch.randn_like(c.q.float()).bfloat16() for _ in range(2)]
    source, big = qs[0].clone(), torch.zeros(64 << 20, device="cuda")
    side = torch.cuda.Stream()

    def step():
        st = torch.cuda.current_stream()
        side.wait_stream(st)
        with torch.cuda.stream(side):                    # slow, and q comes from it
            big.add_(1)
            c.q.copy_(source)
        big2 = big[:1 << 20] * 2
        st.wait_stream(side)
        c.pool.select_blocks(0, c.q, c.bounds, c.tables, c.lens, 3, c.width, c.selected, stream=st)
        c.pool.sparse_attention(0, c.q, c.selected, c.tables, c.lens, 3, c.width, c.scale, c.out, stream=st)
        c.q.copy_(-source)                               # the next step's begins with other values
        c.pool.select_blocks(0, c.q, c.bounds, c.tables, c.lens, 3, c.width, c.selected, stream=st)
        c.pool.sparse_attention(0, c.q, c.selected, c.tables, c.lens, 3, c.width, c.scale, c.out, stream=st)
        return big2

    first = torch.cuda.Stream()
    with torch.cuda.stream(first):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=first):
        step()
    for q in qs:
        source.copy_(q)
        for replay in (False, True):
            c.out.fill_(7.0)
            if replay:
                graph.replay()
            else:
                torch.cuda.synchronize()
                with torch.cuda.stream(first):
                    step()
            torch.cuda.synchronize()
            for b in range(3):
                for g in range(4):
                    assert c.selected[b, g].tolist() == c.reference_selection(b, g, 12)[0]
                c.assert_right(b, *c.reference(b))
    assert c.pool.check_device() == 0


def test_as_many_rows_as_a_call_takes(cuda_dev):
    """65 535 rows, each of one block of a few that they share, and their q rows apart."""
    from paper_2609_25782_gb300 import KVError
    c = Cache([16, 40, 5, 0], seed=20, hq=2, hkv=1)
    c.make_bounds()
    B, width = 65535, 3
    which = torch.arange(B + 1, device="cuda") % 4
    tables, lens = c.tables[:, :width][which].contiguous(), c.lens[which].contiguous()
    q = torch.randn(B + 1, 4, 128, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).bfloat16()[:, 1:3]
    selected = torch.zeros(B, 1, 2, dtype=torch.int32, device="cuda")
    out = torch.zeros(B, 2, 128, device="cuda")
    c.pool.select_blocks(0, q[:B], c.bounds, tables, lens, B, width, selected)
    want = torch.tensor([[0, -1], [0, 2], [0, -1], [-1, -1]], dtype=torch.int32, device="cuda")
    assert torch.equal(selected[:, 0], want[which[:B]])
    c.pool.sparse_attention(0, q[:B], selected, tables, lens, B, width, c.scale, out)
    for kind in range(4):
        rows = torch.nonzero(which[:B] == kind)[:, 0]
        pos = [t for t in range(c.T[kind]) if t // 16 in want[kind].tolist()]
        if not pos:
            assert (out[rows] == 0).all()
            continue
        at = torch.tensor(pos, device="cuda")
        blk = torch.from_numpy(c.tab[kind]).cuda().long()[at // 16]
        k, v = (c.hot[blk, 0, w, 0, at % 16].double() for w in (0, 1))
        w = torch.softmax(q[rows].double() @ k.T * c.scale, -1)
        ref, noise = w @ v, torch.sqrt((w * w) @ (v * v).sum(1))
        from turn_cases import ROW
        assert ((out[rows].double() - ref).norm(dim=2) <= ROW * (noise + ref.norm(dim=2))).all()
    assert c.pool.check_device() == 0
    with pytest.raises(KVError):
        c.pool.sparse_attention(0, q, torch.zeros(B + 1, 1, 2, dtype=torch.int32, device="cuda"), tables, lens, B + 1, width, c.scale,
                                torch.zeros(B + 1, 2, 128, device="cuda"))


def test_calls_on_a_closed_pool_are_refused(cuda_dev):
    from paper_2609_25782_gb300 import KVError
    c = Cache([100], seed=19)
    c.make_bounds()
    c.select(4)
    c.attend()
    assert c.pool.check_device() == 0
    c.pool.close()
    for call in (lambda: c.select(4), c.attend, c.make_bounds):
        with pytest.raises(KVError, match="null pool"):
            call()


FIRST_CALLS = """
import sys
sys.path[:0] = [ROOT, ROOT + "/tests"]
import torch
from sparse_cases import Cache
c = Cache([700, 333, 90], seed=14)
c.selected = torch.zeros(3, 4, 12, dtype=torch.int32, device="cuda")
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    st = torch.cuda.current_stream()
    c.make_bounds(stream=st)
    c.pool.select_blocks(0, c.q, c.bounds, c.tables, c.lens, 3, c.width, c.selected, stream=st)
    c.pool.sparse_attention(0, c.q, c.selected, c.tables, c.lens, 3, c.width, c.scale, c.out, c.k, c.v, st)
graph.replay()
torch.cuda.synchronize()
for b in range(3):
    for g in range(4):
        assert c.selected[b, g].tolist() == c.reference_selection(b, g, 12)[0]
    c.assert_right(b, *c.reference(b, True))
assert c.pool.check_device() == 0
print("as they should be")
"""


def test_first_calls_of_a_process_in_a_capture(cuda_dev):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    run = subprocess.run([sys.executable, "-c", FIRST_CALLS.replace("ROOT", repr(root))], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "as they should be" in run.stdout, run.stderr[-2000:]
