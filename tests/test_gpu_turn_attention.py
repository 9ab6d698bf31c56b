"""Prompt and draft-tree attention over the paged cache against the definition in 64 bits."""
import pytest
import torch

from turn_cases import Call, tree_masks

pytestmark = pytest.mark.gpu

HEADS = [(32, 4), (8, 8), (8, 4), (8, 2), (8, 1)]        # groups of 8, 1, 2, 4 and 8


@pytest.mark.parametrize("bt", [16, 64])
@pytest.mark.parametrize("n,p", [
    ([1], [0]), ([2], [0]), ([15, 16, 17], [0, 0, 0]), ([31, 32, 33], [0, 5, 16]),
    ([1, 1, 1], [1, 127, 128]), ([1, 64, 3], [129, 15, 4000]), ([127, 128, 129], [0, 128, 1]),
    ([255, 257], [256, 300]), ([700, 1, 65], [0, 2048, 1000]), ([1500], [777]),
    ([0, 5, 0, 40], [100, 200, 0, 0]),
])
def test_prefill(cuda_dev, n, p, bt):
    if all(x == 0 for x in n):
        pytest.skip("nothing to do")
    Call("prefill", n, p, bt=bt, seed=len(n) * 100 + n[0], q_std=2.0).check()


@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("n,p", [([5, 130, 260], [70, 0, 513]), ([64, 1], [64, 1023])])
def test_prefill_head_layouts(cuda_dev, hq, hkv, n, p):
    Call("prefill", n, p, hq=hq, hkv=hkv, seed=hq + hkv, q_std=4.0, fused=True).check()


@pytest.mark.parametrize("bt", [16, 64])
@pytest.mark.parametrize("n,p", [
    ([1], [1]), ([1], [16]), ([7], [3001]), ([16, 17], [0, 1]), ([64, 64], [128, 4000]),
    ([3, 0, 33, 16], [127, 50, 129, 2047]), ([16] * 12, list(range(100, 1300, 100))),
])
def test_tree(cuda_dev, n, p, bt):
    Call("tree", n, p, bt=bt, seed=n[0] * 7 + p[0], q_std=4.0).check()


@pytest.mark.parametrize("hq,hkv", HEADS)
def test_tree_head_layouts(cuda_dev, hq, hkv):
    Call("tree", [64, 9, 31], [700, 40, 2500], hq=hq, hkv=hkv, seed=hkv, fused=True).check()


def test_tree_masks_of_every_kind(cuda_dev):
    """Bits past the session's drafts do nothing, a draft need not see itself, and one that sees
    nothing gets zeros."""
    n, p = [4, 64, 5], [0, 0, 33]
    full = (1 << 64) - 1
    masks = [0, 1, full, 0b1000] + [1 << 63] * 32 + [0] * 16 + [full] * 16 + [0, 0, full << 5 & full, 1, 0b10110]
    c = Call("tree", n, p, masks=masks, seed=4)
    c.check()
    zero = [0] + list(range(4 + 32, 4 + 48))
    assert (c.out[zero] == 0).all() and (c.out[[1, 2, 3, 4, 60, 68]] != 0).any(2).all()


@pytest.mark.parametrize("kind", ["prefill", "tree"])
def test_out_fp32_and_one_layer_of_several(cuda_dev, kind):
    Call(kind, [40, 64, 2], [1000, 3, 260], layers=3, layer=1, dtype=torch.float32, seed=11, q_std=3.0).check()


@pytest.mark.parametrize("kind", ["prefill", "tree"])
def test_large_scores(cuda_dev, kind):
    """Scores of several hundred: one key takes nearly all, running maxima jump."""
    c = Call(kind, [33, 64], [900, 200], seed=12, q_std=60.0)
    c.check()


@pytest.mark.parametrize("scale", [-0.3, 0.0, 1e-3, 2.0])
@pytest.mark.parametrize("kind", ["prefill", "tree"])
def test_scales(cuda_dev, kind, scale):
    """Negative: the smallest product weighs most. Zero: all that a row sees weighs the same."""
    c = Call(kind, [33, 64, 3], [900, 0, 200], seed=27)
    c.scale = scale
    c.check()


@pytest.mark.parametrize("blocks,B", [(3000, 3), (1 << 24, 40)])
@pytest.mark.parametrize("kind", ["prefill", "tree"])
def test_tables_much_wider_than_the_sessions(cuda_dev, kind, blocks, B):
    """The launch goes by the tables' width, the plan by the lengths: little work in a plan for much, and
    one whose costs could pass 32 bits."""
    c = Call(kind, [5, 40, 1, 17][:min(B, 4)] * max(1, B // 4), [100, 3, 129, 700][:min(B, 4)] * max(1, B // 4), seed=28)
    wide = torch.full((B, blocks), -1, dtype=torch.int32, device="cuda")
    wide[:, :c.width] = c.tables
    c.tables, c.width = wide, blocks
    c.check()
    assert c.pool.check_device() == 0


@pytest.mark.parametrize("kind", ["prefill", "tree"])
def test_one_sessions_nan_stays_its_own(cuda_dev, kind):
    n, p = [20, 37, 50], [300, 40, 0]
    c = Call(kind, n, p, seed=13)
    clean = c.run().clone()
    c.k[20:57], c.v[20:57] = float("nan"), float("inf")
    blk, slot = c.slots(1, 0, p[1])
    c.hot[blk, 0, :, :, slot] = float("nan")
    c.out.fill_(7.0)
    c.run()
    assert torch.equal(c.out[:20], clean[:20]) and torch.equal(c.out[57:], clean[57:])
    assert c.out[20:57].isnan().all()


@pytest.mark.parametrize("kind", ["prefill", "tree"])
def test_same_from_run_to_run_and_on_other_streams(cuda_dev, kind):
    n, p = ([200, 64, 1, 300], [900, 5000, 70, 0]) if kind == "prefill" else ([16, 64, 1, 30], [900, 5000, 70, 0])
    c = Call(kind, n, p, seed=14, q_std=2.0)
    first = c.run().clone()
    for _ in range(3):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        c.out.fill_(7.0)
        side.wait_stream(torch.cuda.current_stream())
        c.run(side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(c.out, first)


@pytest.mark.parametrize("kind,hq,hkv,bt", [("tree", 32, 4, 16), ("tree", 32, 8, 64), ("prefill", 32, 8, 64)])
def test_many_calls_in_a_row(cuda_dev, kind, hq, hkv, bt):
    """Hundreds of calls queued behind each other, of items that fill one row tile and items that fill
    two: the same output every time, no wait that runs out."""
    n = [20, 31, 32, 52, 16, 60, 29, 7, 58, 33] * 2
    p = [500 + 397 * i for i in range(20)]
    c = Call(kind, n, p, hq=hq, hkv=hkv, bt=bt, seed=26, q_std=2.0)
    first = c.run().clone()
    outs = [torch.empty_like(c.out) for _ in range(8)]
    for _ in range(40):
        for o in outs:
            c.out = o
            c.run()
        assert all(torch.equal(o, first) for o in outs)
    assert c.pool.check_device() == 0


@pytest.mark.parametrize("hq,hkv,n", [(32, 4, 48), (32, 8, 70), (8, 4, 150)])
def test_short_wide_items_before_narrow_ones(cuda_dev, hq, hkv, n):
    """Each CTA goes through several items of one or two key tiles, a pair of row tiles and then a single one
    in turn: q tiles of both kinds follow each other faster than a stream's products."""
    c = Call("prefill", [n] * 60, [0] * 60, hq=hq, hkv=hkv, seed=30, q_std=2.0)
    c.check()
    first = c.out.clone()
    outs = [torch.empty_like(c.out) for _ in range(8)]
    for _ in range(25):
        for o in outs:
            c.out = o
            c.run()
        assert all(torch.equal(o, first) for o in outs)
    assert c.pool.check_device() == 0


def test_prefill_of_one_token_is_the_decode_step(cuda_dev):
    """n = 1 over the same cache: the decode kernel's result, both within their rounding."""
    p = [77, 1, 2000]
    c = Call("prefill", [1, 1, 1], p, seed=15, dtype=torch.float32)
    c.check()
    out = torch.empty_like(c.out)
    from paper_2609_25782_gb300 import Pool
    pool = Pool(num_layers=1, num_hot_blocks=c.hot.shape[0], cold_bytes=256, max_sessions=1, max_batch=3,
                max_context=c.width * c.bt)
    pool.hot.copy_(c.pool.hot)
    pool.decode_attention(0, c.q, c.tables, c.lens, 3, c.width, c.scale, out)
    torch.testing.assert_close(c.out, out, rtol=0, atol=8e-3)
    assert pool.check_device() == 0


def test_bad_device_data_is_flagged_and_skipped(cuda_dev):
    """Offsets and lengths out of range: that session's rows stay, the others are right."""
    from paper_2609_25782_gb300 import kvtier
    c = Call("prefill", [20, 30, 40], [100, 100, 100], seed=16)
    refs = [c.reference(b) for b in range(3)]
    for change in ("long", "short", "negative", "past"):
        lens, cu = c.lens.clone(), c.cu.clone()
        if change == "long":
            lens[1] = c.width * c.bt + 1
        elif change == "short":
            lens[1] = 29
        elif change == "negative":
            lens[1] = -5
        else:
            cu[1], cu[2] = 20, 20                        # the last session has 70 tokens of 140
        c.out.fill_(7.0)
        c.pool.prefill_attention(0, c.q, c.k, c.v, cu, c.tables, lens, 3, c.width, c.scale, c.out)
        if change != "past":
            assert c.pool.check_device() == kvtier.KV_DEVICE_BAD_LENGTH
            assert (c.out[20:50] == 7).all()
            c.assert_right(2, *refs[2])
        else:
            assert c.pool.check_device() == 0
        c.assert_right(0, *refs[0])
    c.out.fill_(7.0)
    cu = torch.tensor([0, 20, 10, 1 << 30], dtype=torch.int32, device="cuda")
    c.pool.prefill_attention(0, c.q, c.k, c.v, cu, c.tables, c.lens, 3, c.width, c.scale, c.out)
    assert c.pool.check_device() == kvtier.KV_DEVICE_BAD_LENGTH
    assert (c.out[20:] == 7).all()
    c.assert_right(0, *refs[0])
    t = Call("tree", [64, 1], [10, 10], seed=17)
    cu = torch.tensor([0, 65, 65], dtype=torch.int32, device="cuda")
    t.pool.tree_attention(0, t.q, t.k, t.v, t.masks, cu, t.tables, t.lens, 2, t.width, t.scale, t.out)
    assert t.pool.check_device() == kvtier.KV_DEVICE_BAD_LENGTH and (t.out == 7).all()


def test_bad_block_ids_are_flagged(cuda_dev):
    from paper_2609_25782_gb300 import kvtier
    c = Call("tree", [16, 16], [200, 200], seed=18)
    want = c.run().clone()
    c.tables[1, 3] = 1 << 30
    c.tables[1, 5] = -1
    c.run()
    assert c.pool.check_device() & kvtier.KV_DEVICE_BAD_BLOCK
    assert torch.equal(c.out[:16], want[:16])


def test_reserve_then_prefill_then_decode(cuda_dev):
    """Sessions of the pool's own: two turns each, then a decode step; the cache holds every token."""
    import __graft_entry__
    __graft_entry__.build()
    from paper_2609_25782_gb300 import Pool
    for lru in (False, True):
        L, bt, turns = 2, 16, [[37, 16, 130], [100, 1, 48]]
        pool = Pool(num_layers=L, num_hot_blocks=40, cold_bytes=1 << 24, max_sessions=4, max_batch=4,
                    max_context=400, alloc_seed=3, lru_residency=lru)
        sids = [pool.session_create(400) for _ in range(3)]
        tables = torch.zeros(3, 25, dtype=torch.int32, device="cuda")
        lens = torch.zeros(3, dtype=torch.int32, device="cuda")
        g = torch.Generator(device="cuda").manual_seed(1)
        kv = [[] for _ in sids]
        for counts in turns:
            pool.batch_reserve(sids, tables, 25, lens, counts=counts)
            N = sum(counts)
            cu = torch.tensor([0] + [sum(counts[:i + 1]) for i in range(3)], dtype=torch.int32, device="cuda")
            x = torch.randn(L, 2, N, 4, 128, device="cuda", generator=g).bfloat16()
            q = torch.randn(N, 32, 128, device="cuda", generator=g).bfloat16()
            out = torch.empty(N, 32, 128, device="cuda", dtype=torch.bfloat16)
            for layer in range(L):
                pool.prefill_attention(layer, q, x[layer, 0], x[layer, 1], cu, tables, lens, 3, 25, 0.09, out)
            for i in range(3):
                kv[i].append(x[:, :, cu[i]:cu[i + 1]])
            if counts is turns[0] and not lru:
                pool.session_pause(sids[1])
                pool.session_resume(sids[1])
        assert lens.tolist() == [137, 17, 178]
        hot = pool.hot_view()
        for i, sid in enumerate(sids):
            row = torch.as_tensor(pool.session_block_table(sid), device="cuda", dtype=torch.int64)
            T = pool.session_info(sid).tokens
            got = hot[row].permute(1, 2, 0, 4, 3, 5).reshape(L, 2, -1, 4, 128)[:, :, :T]
            assert torch.equal(got, torch.cat(kv[i], 2))
        assert pool.check_device() == 0


@pytest.mark.parametrize("hq,hkv", [(24, 3), (5, 5), (24, 6), (14, 7)])
@pytest.mark.parametrize("kind", ["prefill", "tree"])
def test_every_number_of_kv_heads(cuda_dev, kind, hq, hkv):
    """3, 5, 6 and 7 KV heads, in groups of 8, 1, 4 and 2; the powers of two are above."""
    n = [5, 130, 260] if kind == "prefill" else [64, 9, 31]
    Call(kind, n, [70, 0, 513], hq=hq, hkv=hkv, seed=hq + hkv, q_std=3.0, fused=True).check()


@pytest.mark.parametrize("bad", [-1, 1 << 30])
@pytest.mark.parametrize("place", [2, 7])
def test_prefill_with_a_bad_block_id_writes_what_it_may(cuda_dev, place, bad):
    """A block id out of range, of cached tokens (place 2) or of reserved slots (place 7, tokens 112 to 127):
    it is flagged, no other row of the arena changes, and the other sessions come out right."""
    from paper_2609_25782_gb300 import kvtier
    c = Call("prefill", [20, 30, 40], [100, 100, 100], seed=32)
    refs = [c.reference(b) for b in (0, 2)]
    want = c.hot.clone()
    for b, (n, p) in enumerate(zip(c.n, c.p)):
        t = [x for x in range(p, p + n) if b != 1 or x // c.bt != place]
        lo = sum(c.n[:b])
        blk, slot = (x[t] for x in c.slots(b, 0, p + n))
        rows = [lo + x - p for x in t]
        want[blk, 0, 0, :, slot], want[blk, 0, 1, :, slot] = c.k[rows], c.v[rows]
    c.tables[1, place] = bad
    c.run()
    assert c.pool.check_device() & kvtier.KV_DEVICE_BAD_BLOCK
    assert torch.equal(c.hot.view(torch.int16), want.view(torch.int16))
    for b, ref in zip((0, 2), refs):
        c.assert_right(b, *ref)


def attended(q, k, v, scale):
    """(out, noise) of rows q [n][Hq][D], the newest of k, v [m][Hkv][D], in 64 bits: as Call.reference."""
    n, m, G = q.shape[0], k.shape[0], q.shape[1] // k.shape[1]
    k, v = (x.double().repeat_interleave(G, dim=1) for x in (k, v))
    x = torch.einsum("nhd,mhd->nhm", q.double(), k) * scale
    hidden = torch.arange(m, device=q.device)[None, :] > torch.arange(m - n, m, device=q.device)[:, None]
    w = torch.softmax(x.masked_fill(hidden[:, None], float("-inf")), 2)
    return torch.einsum("nhm,mhd->nhd", w, v), torch.sqrt(torch.einsum("nhm,mh->nh", w * w, (v * v).sum(2)))


@pytest.mark.parametrize("lru", [False, True])
def test_turns_and_a_decode_step_of_the_pools_own_sessions(cuda_dev, lru):
    """Reserve and prefill twice, a pause and a resume between, then a reserved decode step: every output
    against the session's whole history in 64 bits. (Decode rounds as these do, its result in 32 bits.)"""
    from turn_cases import ROW
    import __graft_entry__
    __graft_entry__.build()
    from paper_2609_25782_gb300 import Pool
    L, B, width, scale = 2, 3, 25, 0.09
    # 18 of the sessions' blocks at the end; in residency mode the other session's have to leave for them
    pool = Pool(num_layers=L, num_hot_blocks=24, cold_bytes=1 << 24, max_sessions=5, max_batch=4, max_context=400,
                alloc_seed=3, lru_residency=lru)
    other = pool.session_create(400)
    if lru:
        x = torch.zeros(L, 200, 4, 128, dtype=torch.bfloat16, device="cuda")
        pool.session_append(other, x, x)
    sids = [pool.session_create(400) for _ in range(B)]
    tables = torch.zeros(B, width, dtype=torch.int32, device="cuda")
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(2)
    history = [torch.zeros(L, 2, 0, 4, 128, dtype=torch.bfloat16, device="cuda") for _ in sids]

    def assert_right(layer, q, out, bounds):
        for i, (lo, hi) in enumerate(bounds):
            ref, noise = attended(q[lo:hi], history[i][layer, 0], history[i][layer, 1], scale)
            assert ((out[lo:hi].double() - ref).norm(dim=2) <= ROW * (noise + ref.norm(dim=2))).all(), (layer, i)

    for counts in ([37, 16, 90], [60, 1, 48]):
        pool.batch_reserve(sids, tables, width, lens, counts=counts)
        at = [sum(counts[:i]) for i in range(B + 1)]
        cu = torch.tensor(at, dtype=torch.int32, device="cuda")
        x = torch.randn(L, 2, at[-1], 4, 128, device="cuda", generator=g).bfloat16()
        history = [torch.cat([h, x[:, :, lo:hi]], 2) for h, lo, hi in zip(history, at, at[1:])]
        for layer in range(L):
            q = torch.randn(at[-1], 32, 128, device="cuda", generator=g).bfloat16()
            out = torch.empty(at[-1], 32, 128, device="cuda")
            pool.prefill_attention(layer, q, x[layer, 0], x[layer, 1], cu, tables, lens, B, width, scale, out)
            assert_right(layer, q, out, list(zip(at, at[1:])))
        pool.session_pause(sids[1])
        pool.session_resume(sids[1])
    pool.batch_reserve(sids, tables, width, lens)
    x = torch.randn(L, 2, B, 4, 128, device="cuda", generator=g).bfloat16()
    history = [torch.cat([h, x[:, :, i:i + 1]], 2) for i, h in enumerate(history)]
    for layer in range(L):
        q = torch.randn(B, 32, 128, device="cuda", generator=g).bfloat16()
        out = torch.empty(B, 32, 128, device="cuda")
        pool.decode_append_attention(layer, q, x[layer, 0], x[layer, 1], tables, lens, B, width, scale, out)
        assert_right(layer, q, out, [(i, i + 1) for i in range(B)])
    assert lens.tolist() == [98, 18, 139] and pool.check_device() == 0
    if lru:
        assert pool.stats()["blocks_evicted"] > 0


def test_capture_and_replay_with_longer_contexts(cuda_dev):
    """A draft verification recorded in a CUDA graph: lengths are read when it runs."""
    c = Call("tree", [16, 16], [2000, 900], seed=19)
    want = c.run().clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        graph.capture_begin()
        c.run(side)
        graph.capture_end()
    torch.cuda.current_stream().wait_stream(side)
    shorter = c.lens.clone()
    shorter[0] = 300
    full = c.lens.clone()
    c.lens.copy_(shorter)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(c.out[16:], want[16:]) or (c.out[16:].float() - want[16:].float()).abs().max() < 0.02
    assert not torch.equal(c.out[:16], want[:16])
    c.lens.copy_(full)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(c.out, want)


@pytest.mark.parametrize("kind", ["prefill", "tree"])
def test_the_first_call_of_a_pool_is_recorded(cuda_dev, kind):
    """The call that allocates the pool's workspace, while a graph is recorded; decodes need none of it."""
    c = Call(kind, [16, 40], [2000, 900], seed=31)
    refs = [c.reference(b) for b in range(2)]
    c.pool.decode_attention(0, c.q[:1], c.tables, torch.tensor([5], dtype=torch.int32, device="cuda"), 1, 1, c.scale,
                            torch.empty(1, c.hq, 128, device="cuda"))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        graph.capture_begin()
        c.run(side)
        graph.capture_end()
    for _ in range(2):
        c.out.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for b, (ref, noise) in enumerate(refs):
            c.assert_right(b, ref, noise)
    assert c.pool.check_device() == 0


@pytest.mark.slow
@pytest.mark.parametrize("kind", ["prefill", "tree"])
def test_arena_past_32_bit_offsets(cuda_dev, kind):
    """Blocks beyond 2^32 bytes and 2^32 elements of the arena."""
    c = Call(kind, [64, 20], [3000, 2500], layers=48, layer=47, hkv=8, hq=64, bt=64, seed=20, spare=1000)
    assert c.hot.numel() > 1 << 32 and int(c.tab.max()) * c.hot[0].numel() > 1 << 32
    refs = [c.reference(b) for b in range(2)]
    c.run()
    assert c.pool.check_device() == 0
    for b, (ref, noise) in enumerate(refs):
        lo = sum(c.n[:b])
        err = (c.out[lo:lo + c.n[b]].double() - ref).norm(dim=2)
        assert (err <= 4e-3 * (noise + ref.norm(dim=2))).all()


@pytest.mark.slow
def test_long_prompt(cuda_dev):
    Call("prefill", [5000], [3001], hq=8, hkv=1, seed=21, q_std=2.0).check()
    Call("prefill", [6001], [0], hq=8, hkv=8, seed=22, q_std=2.0).check()


@pytest.mark.slow
def test_many_sessions(cuda_dev):
    n = [1 + (i * 7) % 40 for i in range(150)]
    p = [(i * 37) % 500 for i in range(150)]
    Call("prefill", n, p, hq=8, hkv=2, seed=23).check()
    Call("tree", n, p, hq=8, hkv=2, seed=24).check()


def test_refusals(cuda_dev):
    c = Call("tree", [4, 4], [20, 20], seed=25)
    from paper_2609_25782_gb300 import kvtier

    def call(**kw):
        a = dict(layer=0, q=c.q, k=c.k, v=c.v, masks=c.masks, cu=c.cu, tables=c.tables, lens=c.lens, B=2,
                 width=c.width, scale=0.1, out=c.out, qs=0, kvs=0, total=8, flags=kvtier.KV_DECODE_OUT_BF16)
        a.update(kw)
        kvtier.tree_attention(c.pool.handle, a["layer"], a["q"], a["qs"], a["k"], a["v"], a["kvs"], a["masks"],
                              a["cu"], a["total"], a["tables"], a["lens"], a["B"], a["width"], a["scale"],
                              a["out"], a["flags"])

    call()
    call(total=0, q=None, k=None, v=None, out=None, masks=None)
    bad = [dict(layer=-1), dict(layer=1), dict(B=0), dict(B=65536), dict(total=-1), dict(total=(1 << 28) + 1),
           dict(width=0), dict(scale=float("nan")), dict(scale=float("inf")), dict(flags=1), dict(flags=4),
           dict(qs=4), dict(qs=32 * 128 - 8), dict(kvs=4 * 128 + 4), dict(kvs=8), dict(qs=-4096)]
    bad += [{x: None} for x in ("q", "k", "v", "masks", "cu", "tables", "lens", "out")]
    bad += [{x: getattr(c, x).data_ptr() + 8} for x in ("q", "k", "v", "out")]
    bad += [dict(cu=c.cu.data_ptr() + 2), dict(tables=c.tables.data_ptr() + 1), dict(lens=c.lens.data_ptr() + 2),
            dict(masks=c.masks.data_ptr() + 4)]
    for kw in bad:
        with pytest.raises(kvtier.KVError) as e:
            call(**kw)
        assert e.value.code == kvtier.KV_ERR_INVALID_ARG, kw
    for args in ((c.q[:, :, :64], c.k, c.v), (c.q.float(), c.k, c.v), (c.q, c.k, c.v[:, :2]),
                 (c.q, c.k, c.v[:7]), (c.q.transpose(1, 2), c.k, c.v)):
        with pytest.raises(ValueError):
            c.pool.tree_attention(0, *args, c.masks, c.cu, c.tables, c.lens, 2, c.width, 0.1, c.out)
    for out in (c.out[:, :4], c.out.half(), c.out.transpose(0, 1)):
        with pytest.raises(ValueError):
            c.pool.tree_attention(0, c.q, c.k, c.v, c.masks, c.cu, c.tables, c.lens, 2, c.width, 0.1, out)
    for masks in (c.masks[:7], c.masks.int()):
        with pytest.raises(ValueError):
            c.pool.tree_attention(0, c.q, c.k, c.v, masks, c.cu, c.tables, c.lens, 2, c.width, 0.1, c.out)
    assert len(tree_masks([3], 0)) == 3
