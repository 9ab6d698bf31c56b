"""Forks, truncation and compaction on the device: the sessions' tokens against a model of them."""
import math

import numpy as np
import pytest
import torch

from sparse_cases import D, generator

pytestmark = pytest.mark.gpu


class Model:
    """A pool and, for each session, the tokens that it should hold: [L][2][Hkv][T][D]."""

    def __init__(self, nb=80, *, L=3, hq=8, hkv=4, bt=16, lru=False, int8=False, sessions=12, cap=640, seed=0):
        import __graft_entry__
        __graft_entry__.build()
        from paper_2609_25782_gb300 import Pool
        self.L, self.hq, self.hkv, self.bt, self.cap, self.lru, self.int8 = L, hq, hkv, bt, cap, lru, int8
        row = 129 if int8 else 256
        self.pool = Pool(num_layers=L, num_hot_blocks=nb, cold_bytes=sessions * (cap * L * 2 * hkv * row + 256),
                         num_q_heads=hq, num_kv_heads=hkv, block_tokens=bt, max_sessions=sessions, max_batch=sessions,
                         max_context=cap, alloc_seed=seed, lru_residency=lru, cold_int8=int8)
        self.hot, self.g, self.want = self.pool.hot_view(), generator(seed + 1), {}
        self.hot.fill_(float("nan"))

    def tokens(self, n):
        return torch.randn(self.L, 2, self.hkv, n, D, device="cuda", generator=self.g).bfloat16()

    def create(self, n):
        sid = self.pool.session_create(self.cap)
        self.want[sid] = self.tokens(0)
        if n:
            self.append(sid, n)
        return sid

    def append(self, sid, n, stream=None):
        x = self.tokens(n)
        k, v = (x[:, i].transpose(1, 2).contiguous() for i in (0, 1))
        torch.cuda.synchronize()
        self.pool.session_append(sid, k, v, stream)
        self.keep = k, v
        self.want[sid] = torch.cat([self.want[sid], x], 3)

    def fork(self, sid, n=1, tokens=None, stream=None):
        kids = self.pool.session_fork(sid, n, tokens, stream=stream)
        for k in kids:
            self.want[k] = self.want[sid][:, :, :, :tokens]
        return kids

    def truncate(self, sid, tokens, stream=None):
        self.pool.session_truncate(sid, tokens, stream)
        self.want[sid] = self.want[sid][:, :, :, :tokens]

    def lists(self, sid, n, prefix, one=False, seed=0):
        T = self.want[sid].shape[3]
        r = np.random.RandomState(seed)
        k = np.sort(np.argsort(r.rand(self.L * self.hkv, T - prefix), axis=1)[:, :n], axis=1) + prefix
        k = torch.from_numpy(k.astype(np.int32)).cuda().view(self.L, self.hkv, n)
        return k[0, 0].contiguous() if one else k

    def compact(self, sid, keep, prefix, stream=None):
        self.pool.session_compact(sid, keep, prefix, stream)
        w = self.want[sid]
        at = keep.long().expand(self.L, self.hkv, -1)[:, None, :, :, None].expand(-1, 2, -1, -1, D)
        self.want[sid] = torch.cat([w[:, :, :, :prefix], w.gather(3, at)], 3)

    def table(self, sids, stream=None):
        """Rows and lengths from the device; in residency mode evicted blocks come back."""
        width = self.cap // self.bt + 1
        rows = torch.zeros(len(sids), width, dtype=torch.int32, device="cuda")
        lens = torch.zeros(len(sids), dtype=torch.int32, device="cuda")
        self.pool.batch_tables(sids, rows, width, lens, stream)
        return rows, lens

    def check(self, *sids):
        for sid in sids or list(self.want):
            w = self.want[sid]
            info = self.pool.session_info(sid)
            assert info.tokens == w.shape[3]
            if not info.tokens or info.state != 1:
                continue
            rows, lens = self.table([sid])
            torch.cuda.synchronize()
            blocks = self.pool.session_block_table(sid)
            assert rows[0, :len(blocks)].tolist() == blocks and lens[0] == info.tokens
            assert len(blocks) == -(-info.tokens // self.bt) and (rows[0, len(blocks):] == -1).all()
            got = self.hot[torch.tensor(blocks, device="cuda")].permute(1, 2, 3, 0, 4, 5).flatten(3, 4)
            assert torch.equal(got[:, :, :, :info.tokens], w), sid
        assert self.pool.check_device() == 0


@pytest.mark.parametrize("bt", [16, 64])
@pytest.mark.parametrize("lru", [False, True])
@pytest.mark.parametrize("hq,hkv", [(8, 4), (2, 1), (8, 8)])
def test_fork(cuda_dev, lru, bt, hq, hkv):
    m = Model(90, bt=bt, lru=lru, hq=hq, hkv=hkv)
    p = m.create(200)
    for tokens in (None, 0, 1, 63, 64, 65, 129):
        used = m.pool.session_block_table(p)
        before = m.hot.clone()
        kids = m.fork(p, 2, tokens)
        m.check(p, *kids)
        new = {b for k in kids for b in m.pool.session_block_table(k)} - set(used)
        same = torch.tensor([b not in new for b in range(90)], device="cuda")
        assert torch.equal(m.hot[same].view(torch.int16), before[same].view(torch.int16))   # (NaN among it)
        for i, k in enumerate(kids):
            m.append(k, 5 + 20 * i)
        m.check(p, *kids)
        for k in kids:
            if lru:
                m.truncate(k, 0)
            m.pool.session_destroy(k)
            del m.want[k]


@pytest.mark.parametrize("int8", [False, True])
def test_fork_out_of_the_parents_image(cuda_dev, int8):
    m = Model(24, lru=True, int8=int8)
    p, o = m.create(100), m.create(10)
    m.append(o, 374)                                     # 24 blocks: all of p leaves
    assert m.pool.session_info(p).num_blocks == 0
    m.truncate(o, 100)                                   # 17 free
    kid, = m.fork(p, 1, 90)
    assert m.pool.session_info(p).num_blocks == 0
    m.check(o)
    if not int8:
        m.check(kid, p)
        return
    m.table([kid])
    blocks = torch.tensor(m.pool.session_block_table(kid), device="cuda")
    mine = m.hot[blocks].permute(1, 2, 3, 0, 4, 5).flatten(3, 4)[:, :, :, :90].clone()
    m.table([p])                                         # 8 bits: the values that a fetch gives
    blocks = torch.tensor(m.pool.session_block_table(p), device="cuda")
    theirs = m.hot[blocks].permute(1, 2, 3, 0, 4, 5).flatten(3, 4)[:, :, :, :90]
    assert torch.equal(mine, theirs) and m.pool.check_device() == 0


@pytest.mark.parametrize("bt", [16, 64])
def test_many_branches_at_once(cuda_dev, bt):
    """More copies and children than a launch's parameters hold."""
    m = Model(1700, L=1, hq=1, hkv=1, bt=bt, sessions=1500, cap=192)
    p = m.create(2 * bt + 3)
    kids = m.fork(p, 1450)
    m.check(p, *kids[::7], kids[-1])
    rows = [m.pool.session_block_table(k) for k in kids]
    assert len({r[2] for r in rows}) == 1450 and all(r[:2] == rows[0][:2] for r in rows)


@pytest.mark.parametrize("bt", [16, 64])
def test_truncate_and_grow(cuda_dev, bt):
    m = Model(90, bt=bt)
    p = m.create(3 * bt + 5)
    kids = m.fork(p, 3)
    for k, t in zip(kids, (3 * bt, 2 * bt + 7, 1)):      # a block's end, the middle of shared ones
        m.truncate(k, t)
        m.check()
        m.append(k, 2 * bt)
        m.check()
    m.truncate(p, bt + 1)
    m.append(p, bt)
    m.check()


@pytest.mark.parametrize("bt", [16, 64])
@pytest.mark.parametrize("lru", [False, True])
@pytest.mark.parametrize("T,n,prefix", [(200, 50, 0), (200, 1, 199), (200, 1, 0), (129, 127, 1), (333, 200, 70),
                                        (64, 30, 16), (640, 639, 0), (640, 64, 512), (17, 15, 0)])
def test_compact(cuda_dev, T, n, prefix, lru, bt):
    m = Model(90, bt=bt, lru=lru)
    p, o = m.create(T), m.create(100)
    for one in (False, True):
        keep = m.lists(p, n, prefix, one, seed=T)
        m.compact(p, keep, prefix)
        m.check(p, o)
        if n + prefix < T:
            m.append(p, T - n - prefix)
        m.check(p, o)


def test_compact_that_keeps_the_newest_and_the_oldest(cuda_dev):
    m = Model(90)
    p = m.create(600)
    m.compact(p, torch.arange(571, 600, dtype=torch.int32, device="cuda"), 4)
    m.check()
    m.append(p, 500)
    m.compact(p, torch.arange(4, 200, dtype=torch.int32, device="cuda"), 4)      # nothing moves
    m.check()
    m.compact(p, torch.zeros(0, dtype=torch.int32, device="cuda"), 33)
    m.check()


@pytest.mark.parametrize("order", ["heads", "tokens", "shared"])
def test_strides_of_lists(cuda_dev, order):
    m = Model(90, seed=3)
    p = m.create(300)
    keep = m.lists(p, 77, 11, seed=4)
    if order == "heads":
        keep = keep.transpose(0, 1).contiguous().transpose(0, 1)
    elif order == "tokens":
        wide = torch.zeros(m.L, m.hkv, 90, dtype=torch.int32, device="cuda")
        wide[:, :, 7:84] = keep
        keep = wide[:, :, 7:84]
    else:
        keep = keep[:, :1].expand(-1, m.hkv, -1)
    m.compact(p, keep, 11)
    m.check()


@pytest.mark.parametrize("bt", [16, 64])
@pytest.mark.parametrize("n,prefix", [(100, 0), (100, 70), (3, 200), (236, 1), (20, 128)])
def test_compact_of_shared_blocks(cuda_dev, n, prefix, bt):
    m = Model(90, bt=bt)
    p = m.create(240)
    a, b = m.fork(p, 2)
    m.compact(a, m.lists(a, n, prefix, seed=n), prefix)
    m.check()
    m.compact(p, m.lists(p, n, prefix, seed=n + 1), prefix)
    m.append(a, 50)
    m.check()


def test_long_sessions_of_shared_blocks(cuda_dev):
    """More new blocks than a launch names: the second one reads what the first has left."""
    m = Model(7000, L=1, hq=1, hkv=1, cap=50000, sessions=2)
    p = m.create(48000)
    k, = m.fork(p)
    m.compact(k, m.lists(k, 44000, 100, seed=1), 100)
    m.check()


def test_images_after_changes(cuda_dev):
    """What a pause writes, and a resume brings back."""
    m = Model(90)
    p = m.create(200)
    kids = m.fork(p, 2, 150)
    for s in (p, *kids):
        m.pool.session_pause(s)
        m.pool.session_resume(s)
    m.check()
    m.truncate(p, 90)
    m.compact(kids[0], m.lists(kids[0], 60, 33, seed=2), 33)
    m.append(p, 20), m.append(kids[0], 30)
    m.pool.session_pause(kids[1])
    m.truncate(kids[1], 77)
    m.pool.session_resume(kids[1])
    for s in (p, kids[0], kids[1]):
        m.pool.session_pause(s)
    for s in (kids[0], p, kids[1]):
        m.pool.session_resume(s)
    m.check()


def test_evictions_after_changes(cuda_dev):
    m = Model(40, lru=True)
    p, o = m.create(300), m.create(200)                  # 19 + 13 blocks
    m.append(o, 300)                                     # some of p leave
    m.compact(p, m.lists(p, 80, 50, seed=5), 50)
    m.append(o, 100)
    m.truncate(o, 350)
    kid, = m.fork(p, 1, 100)
    m.append(kid, 40)
    m.append(o, 200)
    m.check()
    m.append(p, 60)
    m.check()


def test_positions_that_do_not_ascend(cuda_dev):
    from paper_2609_25782_gb300 import kvtier
    m = Model(90)
    p, o = m.create(200), m.create(100)
    other = m.want[o]
    for i, bad in enumerate((0, 199 + 1, -1, 2 ** 31 - 1, -2 ** 31)):
        keep = torch.arange(100, 150, dtype=torch.int32, device="cuda").expand(m.L, m.hkv, 50).clone()
        keep[1, 2, 30] = bad
        m.pool.session_compact(p, keep, 10)
        assert m.pool.check_device() == kvtier.KV_DEVICE_BAD_INDEX
        m.want[p] = m.want[p].new_zeros(m.L, 2, m.hkv, 60, D)
        m.append(p, 140)
        m.want[o] = other
        m.check(o)


@pytest.mark.parametrize("lru", [False, True])
def test_other_streams_wait(cuda_dev, lru):
    """A fork or a compaction behind a spin on one stream; the session goes on, or ends, on another."""
    m = Model(36 if lru else 44, lru=lru, seed=7)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    held = []                                            # what queued work still reads

    def append(sid, n):
        x = m.tokens(n)
        held.append([x[:, i].transpose(1, 2).contiguous() for i in (0, 1)])
        b.wait_stream(torch.cuda.current_stream())
        m.pool.session_append(sid, *held[-1], b)
        m.want[sid] = torch.cat([m.want[sid], x], 3)

    for spin in (0, 20_000_000):
        p = m.create(205)                                # 13 blocks
        torch.cuda.synchronize()
        with torch.cuda.stream(a):
            torch.cuda._sleep(spin)
        kid, = m.fork(p, stream=a)
        append(p, 30)
        m.pool.session_pause(p, b)
        o = m.create(0)
        append(o, 200)                                   # into the blocks that the pause has freed
        torch.cuda.synchronize()
        m.check(kid, o)
        m.pool.session_resume(p)
        m.check(p)
        held.append(m.lists(kid, 100, 50, seed=8))
        torch.cuda.synchronize()
        with torch.cuda.stream(a):
            torch.cuda._sleep(spin)
        m.compact(kid, held[-1], 50, stream=a)
        append(kid, 9)
        torch.cuda.synchronize()
        m.check(kid, p, o)
        for s in (p, kid, o):
            m.truncate(s, 0)
            m.pool.session_destroy(s)
            del m.want[s]
        torch.cuda.synchronize()


@pytest.mark.parametrize("stay", ["compact", "truncate", "third stream"])
@pytest.mark.parametrize("leave", ["pause", "compact", "truncate"])
@pytest.mark.parametrize("bt", [16, 64])
def test_who_keeps_a_shared_block_waits_for_who_left_it(cuda_dev, bt, leave, stay):
    """A session leaves shared blocks behind a spin on one stream; its fork, the last holder, writes them in place on
    another. Nothing waits between the calls but the pool's own events."""
    m = Model(60, bt=bt, seed=17)
    a, b, c = (torch.cuda.Stream() for _ in range(3))
    n = 13 * bt if bt == 16 else 8 * bt
    p = m.create(n)
    kid, = m.fork(p)                                     # all blocks are shared
    short = m.lists(p, n - 40, 3, seed=1)
    most = m.lists(kid, n - 1, 0, seed=2)                # gives back no block
    x = m.tokens(5)
    k, v = (x[:, i].transpose(1, 2).contiguous() for i in (0, 1))
    torch.cuda.synchronize()
    with torch.cuda.stream(a):
        torch.cuda._sleep(20_000_000)
    if leave == "pause":
        m.pool.session_pause(p, a)
    elif leave == "compact":
        m.compact(p, short, 3, stream=a)
    else:
        m.truncate(p, n - 3, a)                          # copies the last block's part
    if stay == "compact":
        m.compact(kid, most, 0, stream=b)
    else:
        m.truncate(kid, n - 8, b)
    m.pool.session_append(kid, k, v, c if stay == "third stream" else b)
    m.want[kid] = torch.cat([m.want[kid], x], 3)
    torch.cuda.synchronize()
    if leave == "pause":
        m.pool.session_resume(p)
    m.check()


@pytest.mark.parametrize("call", ["resume", "tables"])
def test_residency_mode_still_waits_after_a_resume(cuda_dev, call):
    """A compaction behind a spin; the session is paused and resumed on another stream (or has a block fetched
    there), and then grows: its ready event still covers the compaction."""
    m = Model(30, lru=True, seed=9)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    p, o = m.create(300), m.create(50)                   # 19 and 4 blocks
    keep = m.lists(p, 120, 60, seed=1)
    torch.cuda.synchronize()
    with torch.cuda.stream(a):
        torch.cuda._sleep(20_000_000)
    m.compact(p, keep, 60, stream=a)
    if call == "resume":
        m.pool.session_pause(p)
        m.pool.session_resume(p, b)
    else:
        m.pool.prefetch([p], (), b)
    x = m.tokens(40)
    k, v = (x[:, i].transpose(1, 2).contiguous() for i in (0, 1))
    b.wait_stream(torch.cuda.current_stream())
    m.pool.session_append(p, k, v, b)
    m.want[p] = torch.cat([m.want[p], x], 3)
    torch.cuda.synchronize()
    m.check(p, o)


def test_random_calls(cuda_dev):
    import random
    from paper_2609_25782_gb300 import KVError, kvtier
    for lru in (False, True):
        m, r, done = Model(70, lru=lru, seed=11), random.Random(5), 0
        for step in range(150):
            ids = list(m.want)
            op = r.choice(["create", "fork", "append", "append", "truncate", "compact", "pause", "drop"])
            s = r.choice(ids) if ids else None
            try:
                if op == "create" or s is None:
                    m.create(r.randrange(1, 120))
                elif op == "drop":
                    m.truncate(s, 0)
                    m.pool.session_destroy(s)
                    del m.want[s]
                elif op == "append":
                    m.append(s, r.randrange(1, 40))
                elif op == "fork":
                    m.fork(s, r.choice([1, 2]), r.randrange(0, m.want[s].shape[3] + 1))
                elif op == "truncate":
                    m.truncate(s, r.randrange(0, m.want[s].shape[3] + 1))
                elif op == "pause":
                    m.pool.session_pause(s)
                    m.pool.session_resume(s)
                elif m.want[s].shape[3] > 2:
                    prefix = r.randrange(0, m.want[s].shape[3] - 1)
                    n = r.randrange(1, m.want[s].shape[3] - prefix)
                    m.compact(s, m.lists(s, n, prefix, r.random() < 0.3, seed=step), prefix)
            except KVError as e:                         # full, or paused because a resume found no blocks
                assert e.code in (kvtier.KV_ERR_NO_HOT_BLOCKS, kvtier.KV_ERR_NO_COLD_SPACE, kvtier.KV_ERR_BAD_STATE,
                                  kvtier.KV_ERR_INVALID_ARG)
                done -= 1
            done += 1
            if step % 10 == 9:
                m.check()
        m.check()
        assert done > 60


# ---- the calls together ---------------------------------------------------------------------

def answers(m, rows, lens, q, selected, layer):
    """Attention of each row's last token over its listed blocks, in 64 bits, from the model's tokens."""
    out = torch.zeros(len(rows), m.hq, D, dtype=torch.float64, device="cuda")
    noise = torch.zeros(len(rows), m.hq, dtype=torch.float64, device="cuda")
    G = m.hq // m.hkv
    for b, sid in enumerate(rows):
        w = m.want[sid][layer].double()
        for g in range(m.hkv):
            j = selected[b, g][selected[b, g] >= 0].long()
            pos = (j[:, None] * m.bt + torch.arange(m.bt, device="cuda")).flatten()
            pos = pos[pos < int(lens[b])]
            kk, vv = w[0, g, pos], w[1, g, pos]
            h = slice(g * G, (g + 1) * G)
            p = torch.softmax(q[b, h].double() @ kk.T / math.sqrt(D), 1)
            out[b, h], noise[b, h] = p @ vv, torch.sqrt((p * p) @ (vv * vv).sum(1))
    return out, noise


@pytest.mark.parametrize("lru", [False, True])
@pytest.mark.parametrize("bt", [16, 64])
def test_branches_decode_sparsely_and_shrink(cuda_dev, bt, lru):
    """An agent branches, each branch decodes over the blocks that its bounds select, one is undone, one
    compacted, and they go on; bounds are made anew from the place of each change on."""
    from sparse_cases import bounds_of
    from turn_cases import ROW
    m = Model(160, bt=bt, lru=lru, seed=13)
    parent = m.create(300)
    bounds = m.pool.new_bounds()
    codes, steps = m.pool.bounds_views(bounds)
    width, top = m.cap // bt + 1, 6
    since = {parent: 0}

    def step(sids):
        B = len(sids)
        rows = torch.zeros(B, width, dtype=torch.int32, device="cuda")
        lens = torch.zeros(B, dtype=torch.int32, device="cuda")
        m.pool.batch_reserve(sids, rows, width, lens, torch.cuda.current_stream())
        before = lens - 1                                # bounds of what is there; the new token's block is always read
        old = torch.tensor([min(since[s], m.want[s].shape[3]) for s in sids], dtype=torch.int32, device="cuda")
        m.pool.block_bounds(-1, rows, before, B, width, bounds, since=old)
        x = torch.randn(m.L, B, m.hq + 2 * m.hkv, D, device="cuda", generator=m.g).bfloat16()
        selected = torch.zeros(B, m.hkv, top, dtype=torch.int32, device="cuda")
        out = torch.zeros(m.L, B, m.hq, D, dtype=torch.bfloat16, device="cuda")
        chosen = []
        for layer in range(m.L):
            q, k, v = x[layer, :, :m.hq], x[layer, :, m.hq:m.hq + m.hkv], x[layer, :, m.hq + m.hkv:]
            m.pool.select_blocks(layer, q, bounds, rows, lens, B, width, selected)
            m.pool.sparse_attention(layer, q, selected, rows, lens, B, width, 1 / math.sqrt(D), out[layer], k, v)
            chosen.append(selected.clone())
        for b, s in enumerate(sids):
            new = torch.stack([x[:, b, m.hq:m.hq + m.hkv], x[:, b, m.hq + m.hkv:]], 1)[:, :, :, None]
            m.want[s] = torch.cat([m.want[s], new], 3)
            since[s] = m.want[s].shape[3] - 1
        for layer in range(m.L):
            ref, noise = answers(m, sids, lens, x[layer, :, :m.hq], chosen[layer], layer)
            err = (out[layer].double() - ref).norm(dim=2)
            assert (err <= ROW * (noise + ref.norm(dim=2))).all()
            for b, s in enumerate(sids):                 # the bounds that the selection went by
                t = m.want[s].shape[3] - 1
                for j in range(-(-t // bt)):
                    blk = int(rows[b, j])
                    c, st = bounds_of(m.want[s][layer, 0, :, j * bt:min(t, (j + 1) * bt)])
                    assert torch.equal(codes[layer, :, blk], c) and torch.equal(steps[layer, :, blk], st), (s, j)
                last = (int(lens[b]) - 1) // bt
                assert (chosen[layer][b] == 0).any() and (chosen[layer][b] == last).any(dim=1).all()

    step([parent])
    kids = m.fork(parent, 3)
    for k in kids:                                       # shared blocks' bounds are there; copied blocks' are not
        since[k] = 0 if lru else m.want[k].shape[3] // bt * bt
    for _ in range(3):
        step([parent, *kids])
    m.truncate(kids[0], 250)
    since[kids[0]] = 250 // bt * bt
    m.compact(kids[1], m.lists(kids[1], 90, 40, seed=3), 40)
    since[kids[1]] = 40
    m.pool.session_pause(kids[2])
    step([kids[0], parent, kids[1]])
    m.pool.session_resume(kids[2])
    since[kids[2]] = 0                                   # back in other blocks
    for _ in range(2):
        step([kids[2], kids[0], parent, kids[1]])
    m.check()


@pytest.mark.parametrize("back", ["prefetch", "resume"])
def test_tables_of_blocks_that_another_stream_is_bringing(cuda_dev, back):
    """Fetches behind a spin on one stream; a kernel behind the batch's tables on another reads the blocks."""
    m = Model(30, lru=True, seed=19)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    p, o = m.create(300), m.create(50)                   # 19 and 4 blocks
    m.append(o, 330)                                     # 24: 13 of p's leave
    m.truncate(o, 16)
    assert m.pool.session_info(p).num_blocks < 19
    rows = torch.zeros(1, 41, dtype=torch.int32, device="cuda")
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(a):
        torch.cuda._sleep(20_000_000)
    if back == "prefetch":
        m.pool.prefetch([p], (), a)
    else:
        m.pool.session_pause(p)
        m.pool.session_resume(p, a)
    m.pool.batch_tables([p], rows, 41, lens, b)
    with torch.cuda.stream(b):
        got = m.hot[rows[0, :19].long()]
    torch.cuda.synchronize()
    assert rows[0, :19].tolist() == m.pool.session_block_table(p) and int(lens[0]) == 300
    assert torch.equal(got.permute(1, 2, 3, 0, 4, 5).flatten(3, 4)[:, :, :, :300], m.want[p])
    m.check()
