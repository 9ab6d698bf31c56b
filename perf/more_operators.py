"""Timed operators over the paged cache, in their plain form and through the package.

bounds   channelwise bounds of the keys of blocks: for each block, layer and KV head the largest and the
         smallest K of its tokens, in 8 bits with a power-of-two step, rounded outwards
select   the blocks of each session that one new token's heads may need most: a score per block and KV
         head from the bounds, the `top` largest, the first and last ones always among them
attend   attention of one new token per session over the listed blocks of each KV head
step     a decode step of a layer that does both; the token's K and V go into its reserved slot
fork     sessions that begin with another one's tokens: full blocks are shared and the last, partly
         filled one is copied; in residency mode, where a block has one owner, all are copied
compact  a session keeps the listed tokens of its newest part, a list for each layer and KV head, or one
         list for all

A block's bounds are codes in -127..127 and a step 2^(E - 133), E the biased exponent of the block's
largest magnitude (one more where a code would pass 127). The scores are whole numbers times a step, so
that they do not depend on an order of sums.

Shapes are the repository's: head_dim 128, 32 query and 4 KV heads, 48 layers, blocks of 16 or 64
tokens, contexts from a few tokens to 128K. Attention and selection are one layer's call, as a model
makes it.
"""
import math

import numpy as np
import torch

own = False     # False: elementary torch operations; True: the package's operators

D = 128


def _case(name, kind, **kw):
    c = {"name": name, "kind": kind, "layers": 1, "hq": 32, "hkv": 4, "bt": 16, "batch": 1, "q_std": 1.0}
    c.update(kw)
    return c


def listed():
    return [
        # a prompt's keys have just been cached
        _case("bounds_1x2100", "bounds", layers=48, tmin=2100, tmax=2100, fresh=1.0, lens_seed=1),
        # several long sessions have come back into other blocks
        _case("bounds_3x8k-24k", "bounds", layers=48, batch=3, tmin=8000, tmax=24000, fresh=1.0, lens_seed=2),
        # one agent early in its task: latency (the scores are kept, to see what else to bring back)
        _case("select_1x6k", "select", tmin=6001, tmax=6001, first=1, last=2, top=64, lens_seed=3),
        # agents with long histories
        _case("select_8x10k-120k", "select", batch=8, tmin=10000, tmax=120000, first=1, last=4, top=256,
              lens_seed=4),
        # the layers after one that has selected: latency
        _case("attend_1x30k", "attend", tmin=30001, tmax=30001, first=1, last=4, top=128, lens_seed=5),
        # the same for a serving batch of very unequal lengths, 8 KV heads in groups of 4, 64-token
        # blocks, q as a view of a fused projection
        _case("attend_48x4k-60k_bt64", "attend", hkv=8, bt=64, batch=48, tmin=4000, tmax=60000, first=1, last=2,
              top=64, fused=True, lens_seed=6),
        # a decode step of one very long session
        _case("step_1x100k", "step", tmin=100003, tmax=100003, first=1, last=8, top=256, lens_seed=7),
        # the agentic trace's batch; peaked scores, as trained heads have
        _case("step_16x2k-30k", "step", batch=16, tmin=2048, tmax=30000, first=1, last=4, top=128, q_std=4.0,
              lens_seed=8),
        # an agent tries eight ways on from where it is
        _case("fork_1to8_of_20k", "fork", layers=48, tmin=20011, tmax=20011, ways=8, lru=False, lens_seed=9),
        # two branches of a session in a pool that evicts block by block
        _case("fork_copies_1to2_of_9k", "fork", layers=48, tmin=9007, tmax=9007, ways=2, lru=True, lens_seed=10),
        # a long tool result shrinks to the tokens that each head has looked at
        _case("compact_8k_to_2k", "compact", layers=48, tmin=8200, tmax=8200, prefix=40, keep=0.25, lists=True,
              lens_seed=11),
        # three sessions of a smaller model with 8 KV heads, one list each, 64-token blocks
        _case("compact_3x1k-6k_bt64", "compact", layers=16, hkv=8, bt=64, batch=3, tmin=1000, tmax=6000, prefix=0,
              keep=0.5, lists=False, lens_seed=12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above, no dearer than the largest of its kind."""
    kind = rng.choice(["bounds", "select", "select", "attend", "attend", "step", "step", "fork", "compact"])
    hkv, hq = rng.choice([(4, 32), (4, 32), (4, 32), (8, 32), (4, 16), (8, 64), (2, 16), (8, 8)])
    c = {"kind": kind, "layers": 1, "hq": hq, "hkv": hkv, "bt": rng.choice([16, 16, 64]), "q_std": rng.choice([1.0, 2.0, 4.0]),
         "lens_seed": rng.randrange(1 << 20)}
    if kind in ("select", "attend", "step"):
        c["tmax"] = _log_int(rng, 20, 128000)
        most = min(64, 4e9 / (c["tmax"] * _token_bytes(c)))
        c["top"] = _log_int(rng, 4, 4096 // c["bt"] * 2)
        c["first"], c["last"] = rng.choice([0, 1, 2]), rng.choice([1, 1, 2])
        c["fused"] = rng.random() < 0.4
    else:
        c["layers"] = rng.choice([4, 16, 28, 48])
        c["tmax"] = _log_int(rng, 30, 24000)
        limit = {"bounds": 3e9, "fork": 1.5e9, "compact": 1e9}[kind]
        if c["tmax"] * _token_bytes(c) > limit:
            c["layers"] = max(1, int(c["layers"] * limit / (c["tmax"] * _token_bytes(c))))
        most = min(6, limit / (c["tmax"] * _token_bytes(c)))
        if kind == "bounds":
            c["fresh"] = rng.choice([1.0, 1.0, 0.3])
        elif kind == "fork":
            most, c["lru"] = 1, rng.random() < 0.4
            c["ways"] = rng.choice([1, 2]) if c["lru"] else _log_int(rng, 1, 16)
        else:
            c["lists"], c["keep"] = rng.random() < 0.6, rng.choice([0.1, 0.3, 0.6, 0.9])
            c["prefix"] = rng.choice([0, 4, 16, 70])
    c["tmin"] = _log_int(rng, 20, c["tmax"]) if rng.random() < 0.7 else c["tmax"]
    c["batch"] = _log_int(rng, 1, max(1, int(most)))
    return c


# ---- sizes ---------------------------------------------------------------------------------

def _token_bytes(c):
    return c["layers"] * 2 * c["hkv"] * D * 2


def _lengths(c):
    """Tokens of each session, the same for every seed of the values."""
    r = np.random.RandomState(c["lens_seed"])
    n = np.rint(np.exp(r.uniform(math.log(c["tmin"]), math.log(c["tmax"]), c["batch"])))
    return [int(x) for x in n]


def _blocks(t, bt):
    return -(-t // bt)


def _old(c):
    """Tokens whose bounds are there already."""
    return [t - max(1, int(t * c["fresh"])) for t in _lengths(c)]


def _kept(c):
    """(prefix, kept tokens behind it) of each session of a compaction."""
    p = [min(c["prefix"], t - 1) for t in _lengths(c)]
    return [(x, max(1, int((t - x) * c["keep"]))) for t, x in zip(_lengths(c), p)]


def work(c):
    lens, bt, hkv, row = _lengths(c), c["bt"], c["hkv"], D * 2
    blocks = [_blocks(t, bt) for t in lens]
    if c["kind"] == "bounds":
        n = [(t, o // bt * bt) for t, o in zip(lens, _old(c))]
        b = sum((t - o) * row + _blocks(t - o, bt) * (2 * D + 2) for t, o in n) * hkv * c["layers"]
        return {"bytes": b, "flops": 0}
    if c["kind"] == "fork":
        copied = lens[0] if c["lru"] else lens[0] % bt
        return {"bytes": 2 * copied * c["ways"] * _token_bytes(c) + (1 + c["ways"]) * blocks[0] * 4, "flops": 0}
    if c["kind"] == "compact":
        n = sum(k for _, k in _kept(c))
        return {"bytes": 2 * n * _token_bytes(c) + n * 4 * (c["layers"] * hkv if c["lists"] else 1), "flops": 0}
    b, f = len(lens) * c["hq"] * row, 0
    if c["kind"] != "attend":
        seen = [max(0, n - c["first"] - c["last"]) for n in blocks]
        b += sum(seen) * hkv * (2 * D + 2 + 4) + sum(min(n, c["top"]) for n in blocks) * hkv * 4
        b += sum(blocks) * hkv * 4 if c["kind"] == "select" else 0
        f += sum(seen) * hkv * 4 * D
    if c["kind"] != "select":
        tokens = sum(min(t, c["top"] * bt) for t in lens)
        b += tokens * hkv * 2 * row + len(lens) * c["hq"] * row
        f += 4 * D * c["hq"] * tokens
    return {"bytes": b, "flops": f}


# ---- inputs --------------------------------------------------------------------------------

def _gen(seed, salt):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 1000003 + salt) & 0x7FFFFFFF)


def _fill(t, seed, salt, std=1.0):
    """N(0, std) values in place, from the seed alone."""
    g, flat, piece = _gen(seed, salt), t.view(-1), 1 << 30
    for i in range(0, flat.numel(), piece):
        flat[i:i + piece].normal_(0.0, std, generator=g)
    return t


def _normal(shape, seed, salt, std=1.0):
    return _fill(torch.empty(shape, dtype=torch.bfloat16, device="cuda"), seed, salt, std)


def _tables(c, seed):
    """Block tables of sessions at random places of an arena that they fill."""
    bt, lens = c["bt"], _lengths(c)
    n = [_blocks(t, bt) for t in lens]
    perm = np.random.RandomState(seed & 0x7FFFFFFF).permutation(sum(n))
    tab = np.full((len(n), max(n)), -1, dtype=np.int32)
    ends = np.cumsum([0] + n)
    for b, m in enumerate(n):
        tab[b, :m] = perm[ends[b]:ends[b + 1]]
    return tab, int(ends[-1])


def _fill_arena(hot, seed):
    """Keys and values; tokens that are cached together are near each other, so that blocks differ."""
    _fill(hot, seed, 1)
    if hot.shape[1] == 1:
        hot[:, :, 0] += _normal((hot.shape[0], 1, hot.shape[3], 1, D), seed, 6, 0.7)
    return hot


def _pool(c, blocks, max_context, sessions=1, lru=False, seed=0):
    from paper_2609_25782_gb300 import Pool
    return Pool(num_layers=c["layers"], num_hot_blocks=blocks, cold_bytes=sessions * (max_context * _token_bytes(c) + 512)
                if c["kind"] in ("fork", "compact") else 256, num_q_heads=c["hq"], num_kv_heads=c["hkv"],
                block_tokens=c["bt"], max_sessions=sessions, max_batch=max(c["batch"], 1), max_context=max_context,
                alloc_seed=int(seed), lru_residency=lru)


def _arena(c, blocks):
    """A hot arena, [blocks][L][2][Hkv][bt][D]."""
    return torch.empty((blocks, c["layers"], 2, c["hkv"], c["bt"], D), dtype=torch.bfloat16, device="cuda")


def _empty_bounds(c, blocks):
    shape = (c["layers"], c["hkv"], blocks)
    return (torch.zeros((*shape, 2, D), dtype=torch.int8, device="cuda"),
            torch.zeros(shape, dtype=torch.bfloat16, device="cuda"))


def _cached(c, seed):
    """Sessions in an arena: what bounds, selections and attention begin with."""
    lens = _lengths(c)
    tab, blocks = _tables(c, seed)
    return {"case": c, "n": lens, "tab": tab, "width": tab.shape[1], "blocks": blocks,
            "tables": torch.from_numpy(tab).cuda(), "lens": torch.tensor(lens, dtype=torch.int32, device="cuda")}


def _token_inputs(s, seed):
    """q, and for a step k and v, of one new token per session (the last of its length)."""
    c = s["case"]
    B, hq, hkv = c["batch"], c["hq"], c["hkv"]
    qkv = _normal((B, hq + 2 * hkv, D), seed, 2)
    qkv[:, :hq] *= c["q_std"]
    s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    if not c.get("fused"):
        s["q"], s["k"], s["v"] = (x.contiguous() for x in (s["q"], s["k"], s["v"]))
    s["out"] = torch.zeros((B, hq, D), dtype=torch.bfloat16, device="cuda")
    s["selected"] = torch.zeros((B, hkv, c["top"]), dtype=torch.int32, device="cuda")
    s["scores"] = torch.zeros((B, hkv, s["width"]), dtype=torch.float32, device="cuda") if c["kind"] == "select" else None
    return s


def _prepare_cached(c, seed):
    s = _cached(c, seed)
    if own:
        s["pool"] = _pool(c, s["blocks"], s["width"] * c["bt"])
        s["hot"] = s["pool"].hot_view()
        s["bounds"] = s["pool"].new_bounds()
        s["codes"], s["steps"] = s["pool"].bounds_views(s["bounds"])
    else:
        s["hot"] = _arena(c, s["blocks"])
        s["codes"], s["steps"] = _empty_bounds(c, s["blocks"])
    _fill_arena(s["hot"], seed)
    if c["kind"] == "bounds":
        s["since"] = torch.tensor(_old(c), dtype=torch.int32, device="cuda")
        s["codes"].zero_()
        s["steps"].zero_()
        return s
    _token_inputs(s, seed)
    if c["kind"] == "attend":       # what an earlier layer has selected
        s["selected"].copy_(torch.from_numpy(_some_blocks(c, seed)))
        return s
    s["since"] = torch.zeros_like(s["lens"])
    _plain_bounds(s)
    return s


def _some_blocks(c, seed):
    """A selection: the first and last blocks and some between them, ascending, -1 behind."""
    r = np.random.RandomState((seed + 77) & 0x7FFFFFFF)
    out = np.full((c["batch"], c["hkv"], c["top"]), -1, dtype=np.int32)
    for b, t in enumerate(_lengths(c)):
        n = _blocks(t, c["bt"])
        for g in range(c["hkv"]):
            weight = r.rand(n)
            weight[:c["first"]] = weight[max(0, n - c["last"]):] = 2
            pick = np.sort(np.argsort(-weight)[:c["top"]])
            out[b, g, :len(pick)] = pick
    return out


def _free_order(n, seed):
    """The order in which blocks leave a new pool's free list: 0..n-1 shuffled from the top by
    splitmix64 draws, taken from its end."""
    mask, st, v = (1 << 64) - 1, int(seed) & ((1 << 64) - 1), list(range(n))
    for i in range(n - 1, 0, -1):
        st = (st + 0x9E3779B97F4A7C15) & mask
        z = st
        z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & mask
        z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & mask
        z ^= z >> 31
        j = (z * (i + 1)) >> 64
        v[i], v[j] = v[j], v[i]
    return v[::-1]


def _prepare_sessions(c, seed):
    """Active sessions in a pool that has just been made, and what a fork or a compaction needs beside
    them. `rows`: each session's blocks; `free`: those behind them, in the order of their use."""
    lens, bt = _lengths(c), c["bt"]
    held = [_blocks(t, bt) for t in lens]
    more = 0
    if c["kind"] == "fork":
        more = c["ways"] * (held[0] if c["lru"] else 1)
    blocks = sum(held) + more
    order, ends = _free_order(blocks, seed), np.cumsum([0] + held)
    rows = [order[ends[i]:ends[i + 1]] for i in range(len(held))]
    width, B = max(held), len(lens) + c.get("ways", 0)
    s = {"case": c, "n": lens, "rows": rows, "free": order[ends[-1]:], "width": width, "B": B,
         "tables": torch.zeros((B, width), dtype=torch.int32, device="cuda"),
         "lens": torch.zeros(B, dtype=torch.int32, device="cuda")}
    if c["kind"] == "compact":
        s["keep"] = [torch.from_numpy(k).cuda() for k in _lists(c, seed)]
        s["kept"], s["gone"] = _kept(c), None
    if own:
        pool = s["pool"] = _pool(c, blocks, width * bt, sessions=B, lru=bool(c.get("lru")), seed=seed)
        s["sids"] = [pool.session_create(t) for t in lens]
        pool.batch_reserve(s["sids"], s["tables"], width, s["lens"], torch.cuda.current_stream(), counts=lens)
        s["branches"] = []
        s["hot"] = pool.hot_view()
    else:
        s["hot"] = _arena(c, blocks)
    _fill(s["hot"], seed, 1)
    return s


def _lists(c, seed):
    """Ascending positions behind the prefix, [L][Hkv][kept] or [kept], of each session."""
    r = np.random.RandomState((seed + 5) & 0x7FFFFFFF)
    out = []
    for t, (p, k) in zip(_lengths(c), _kept(c)):
        lists = c["layers"] * c["hkv"] if c["lists"] else 1
        pick = np.sort(np.argsort(r.rand(lists, t - p), axis=1)[:, :k], axis=1).astype(np.int32) + p
        out.append(pick.reshape(c["layers"], c["hkv"], k) if c["lists"] else pick[0])
    return out


def prepare(case, seed):
    return (_prepare_sessions if case["kind"] in ("fork", "compact") else _prepare_cached)(case, seed)


# ---- one pass ------------------------------------------------------------------------------

def run(state):
    return (_run_own if own else _run_plain)[state["case"]["kind"]](state)


def _own_bounds(s):
    c = s["case"]
    s["pool"].block_bounds(-1, s["tables"], s["lens"], c["batch"], s["width"], s["bounds"], since=s["since"],
                           stream=torch.cuda.current_stream())
    return [s["codes"] * s["steps"][..., None, None]]


def _own_select(s):
    c = s["case"]
    s["pool"].select_blocks(0, s["q"], s["bounds"], s["tables"], s["lens"], c["batch"], s["width"], s["selected"],
                            first=c["first"], last=c["last"], scores=s["scores"], stream=torch.cuda.current_stream())
    return [s["selected"]] + ([s["scores"]] if c["kind"] == "select" else [])


def _own_attend(s):
    s["pool"].sparse_attention(0, s["q"], s["selected"], s["tables"], s["lens"], s["case"]["batch"], s["width"],
                               1 / math.sqrt(D), s["out"], stream=torch.cuda.current_stream())
    return [s["out"]]


def _own_step(s):
    selected = _own_select(s)
    s["pool"].sparse_attention(0, s["q"], s["selected"], s["tables"], s["lens"], s["case"]["batch"], s["width"],
                               1 / math.sqrt(D), s["out"], k_new=s["k"], v_new=s["v"],
                               stream=torch.cuda.current_stream())
    return selected + [s["out"], s["hot"]]


def _own_fork(s):
    c, pool, st = s["case"], s["pool"], torch.cuda.current_stream()
    for sid in reversed(s["branches"]):     # the branches of the pass before have ended
        if c["lru"]:
            pool.session_truncate(sid, 0, st)
        pool.session_destroy(sid)
    s["branches"] = pool.session_fork(s["sids"][0], c["ways"], stream=st)
    pool.batch_tables(s["sids"] + s["branches"], s["tables"], s["width"], s["lens"], st)
    return [s["hot"], s["tables"], s["lens"]]


def _own_compact(s):
    pool, st = s["pool"], torch.cuda.current_stream()
    if s["gone"]:                           # the next turn's slots, after an earlier pass
        pool.batch_reserve(s["sids"], s["tables"], s["width"], s["lens"], st, counts=s["gone"])
    for sid, keep, (p, _) in zip(s["sids"], s["keep"], s["kept"]):
        pool.session_compact(sid, keep, prefix=p, stream=st)
    s["gone"] = [t - p - k for t, (p, k) in zip(s["n"], s["kept"])]
    pool.batch_tables(s["sids"], s["tables"], s["width"], s["lens"], st)
    return [s["hot"], s["tables"], s["lens"]]


def _plain_bounds(s):
    bt = s["case"]["bt"]
    j = torch.arange(s["width"], device="cuda")
    lens, since = s["lens"].long()[:, None], s["since"].long()[:, None]
    b, j = torch.nonzero((j * bt < lens) & (j >= since // bt) & (since < lens), as_tuple=True)
    blk = s["tables"][b, j].long()
    valid = j[:, None] * bt + torch.arange(bt, device="cuda") < lens[b]             # [P][bt]
    k = s["hot"][:, :, 0][blk].float()                                              # [P][L][Hkv][bt][D]
    off = ~valid[:, None, None, :, None]
    hi = k.masked_fill(off, -math.inf).amax(dim=3).double()
    lo = k.masked_fill_(off, math.inf).amin(dim=3).double()
    top = torch.maximum(hi.abs(), lo.abs()).amax(dim=-1)                            # [P][L][Hkv]
    bits = top.float().view(torch.int32)
    e = (bits >> 23).clamp_(min=1) + ((bits >> 16 & 127) == 127).int()
    step = torch.exp2(e.double() - 133)
    codes = torch.stack([torch.ceil(hi / step[..., None]), torch.floor(lo / step[..., None])], dim=3)
    fine = torch.isfinite(top)
    limit = torch.tensor([127.0, -127.0], device="cuda", dtype=torch.float64)[:, None]
    codes = torch.where(fine[..., None, None], codes, limit)
    s["codes"][:, :, blk] = codes.to(torch.int8).permute(1, 2, 0, 3, 4)
    s["steps"][:, :, blk] = torch.where(fine, step, math.inf).to(torch.bfloat16).permute(1, 2, 0)
    return [s["codes"] * s["steps"][..., None, None]]


def _plain_select(s):
    c, lens = s["case"], s["lens"].long()
    B, hkv, bt = c["batch"], c["hkv"], c["bt"]
    q = s["q"].float().reshape(B, hkv, -1)
    q = torch.where(torch.isfinite(q), q, 0.0)
    e = (q.abs().amax(dim=-1, keepdim=True).view(torch.int32) >> 23).clamp_(min=1)
    q = torch.round(q.double() * torch.exp2(137 - e.double())).view(B, hkv, -1, D)
    q = torch.stack([q.clamp(min=0).sum(dim=2), q.clamp(max=0).sum(dim=2)], dim=2).flatten(2)    # [B][Hkv][2 D]
    blk = s["tables"].long().clamp(min=0)                                           # [B][width]
    codes = s["codes"][0][:, blk].flatten(3).double().transpose(0, 1)               # [B][Hkv][width][2 D]
    x = torch.matmul(codes, q[..., None])[..., 0].float()       # whole numbers: exact up to here
    step = s["steps"][0][:, blk].float().transpose(0, 1)
    x = torch.where(torch.isinf(step), math.inf, x * step)
    n = ((lens + bt - 1) // bt)[:, None, None]
    j = torch.arange(s["width"], device="cuda")
    always = (j < c["first"]) | (j >= n - c["last"])
    x = torch.where(always, math.inf, x)
    x = torch.where(j < n, x, -math.inf).expand(B, hkv, -1)
    rank = torch.where(always & (j < n), 1, 0).expand_as(x)
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices
    order = order.gather(-1, torch.sort(rank.gather(-1, order), dim=-1, descending=True, stable=True).indices)
    top = order[..., :c["top"]]
    top = torch.where(top < n, top, 1 << 30).sort(dim=-1).values
    s["selected"].fill_(-1)
    s["selected"][..., :top.shape[-1]] = torch.where(top == 1 << 30, -1, top)
    if c["kind"] == "select":
        s["scores"].copy_(x)
        return [s["selected"], s["scores"]]
    return [s["selected"]]


def _plain_attend(s):
    c = s["case"]
    B, hq, hkv, bt = c["batch"], c["hq"], c["hkv"], c["bt"]
    j = s["selected"].long()                                                        # [B][Hkv][top]
    blk = s["tables"].long().gather(1, j.clamp(min=0).flatten(1)).view_as(j)
    pos = j[..., None] * bt + torch.arange(bt, device="cuda")
    seen = ((j >= 0)[..., None] & (pos < s["lens"].long()[:, None, None, None])).flatten(2)
    kv = s["hot"][blk, 0, :, torch.arange(hkv, device="cuda")[:, None]]             # [B][Hkv][top][2][bt][D]
    k, v = (kv[:, :, :, i].flatten(2, 3).float() for i in (0, 1))                   # [B][Hkv][top * bt][D]
    q = s["q"].float().reshape(B, hkv, hq // hkv, D)
    x = torch.matmul(q, k.transpose(2, 3)) * (1 / math.sqrt(D))
    x = x.masked_fill(~seen[:, :, None], -math.inf)
    x = torch.exp(x - x.amax(dim=-1, keepdim=True).clamp(min=-3e38))
    y = torch.matmul(x, v.masked_fill(~seen[..., None], 0.0)) / x.sum(dim=-1, keepdim=True).clamp(min=1e-38)
    s["out"].copy_(y.view(B, hq, D))
    return [s["out"]]


def _plain_step(s):
    last = s["lens"].long() - 1
    blk = s["tables"].long().gather(1, (last // s["case"]["bt"])[:, None])[:, 0]
    s["hot"][blk, 0, 0, :, last % s["case"]["bt"]] = s["k"]
    s["hot"][blk, 0, 1, :, last % s["case"]["bt"]] = s["v"]
    return _plain_select(s) + _plain_attend(s) + [s["hot"]]


def _tables_of(s, rows, lens):
    tab = np.full((len(rows), s["width"]), -1, dtype=np.int32)
    tab[np.arange(s["width"]) < np.array([len(r) for r in rows])[:, None]] = np.concatenate(rows)
    s["tables"].copy_(torch.from_numpy(tab))
    s["lens"].copy_(torch.tensor(lens, dtype=torch.int32))


def _branches(s):
    """The block rows of the forked sessions, one after the other."""
    c, row, t = s["case"], s["rows"][0], s["n"][0]
    shared = 0 if c["lru"] else t // c["bt"]
    own_blocks = len(row) - shared
    return shared, [row[:shared] + s["free"][w * own_blocks:(w + 1) * own_blocks] for w in range(c["ways"])]


def _plain_fork(s):
    c, row, t = s["case"], s["rows"][0], s["n"][0]
    bt, hot = c["bt"], s["hot"]
    shared, rows = _branches(s)
    full = len(row) - shared - (t % bt > 0)
    to = torch.tensor([r[shared:] for r in rows], device="cuda")
    source = torch.tensor(row[shared:], device="cuda")
    if full:
        hot[to[:, :full]] = hot[source[:full]]
    if t % bt:
        hot[to[:, full], :, :, :, :t % bt] = hot[source[full], :, :, :, :t % bt]
    _tables_of(s, [row] + rows, [t] * (1 + c["ways"]))
    return [hot, s["tables"], s["lens"]]


def _plain_compact(s):
    c, hot, bt = s["case"], s["hot"], s["case"]["bt"]
    li, g = (torch.arange(x, device="cuda") for x in (c["layers"], c["hkv"]))
    li, g = li[:, None, None], g[:, None]
    for row, keep, (p, k) in zip(s["rows"], s["keep"], s["kept"]):
        blk = torch.tensor(row, device="cuda")
        at = torch.arange(p, p + k, device="cuda")
        hot[blk[at // bt], li, :, g, at % bt] = hot[blk[keep.long() // bt], li, :, g, keep.long() % bt]
    total = [p + k for p, k in s["kept"]]
    _tables_of(s, [r[:_blocks(t, bt)] for r, t in zip(s["rows"], total)], total)
    return [hot, s["tables"], s["lens"]]


_run_own = {"bounds": _own_bounds, "select": _own_select, "attend": _own_attend, "step": _own_step,
            "fork": _own_fork, "compact": _own_compact}
_run_plain = {"bounds": _plain_bounds, "select": _plain_select, "attend": _plain_attend, "step": _plain_step,
              "fork": _plain_fork, "compact": _plain_compact}


# ---- in 64 bits ----------------------------------------------------------------------------

def _exact_bounds(c, seed):
    """A session's block at a time, all layers and heads."""
    s = _cached(c, seed)
    if s["blocks"] > 60000:
        return None                 # over 20 seconds, block by block
    hot = _fill_arena(_arena(c, s["blocks"]), seed)
    values = torch.zeros((c["layers"], c["hkv"], s["blocks"], 2, D), dtype=torch.float64, device="cuda")
    for b, (t, o) in enumerate(zip(s["n"], _old(c))):
        for j in range(o // c["bt"], _blocks(t, c["bt"])):
            blk = int(s["tab"][b, j])
            k = hot[blk, :, 0, :, :t - j * c["bt"]].double()
            hi, lo = k.amax(dim=2), k.amin(dim=2)
            largest = torch.maximum(hi, -lo).amax(dim=2, keepdim=True)
            unit = torch.exp2(torch.floor(torch.log2(largest)) - 6)     # none of these keys is zero
            unit = torch.where(largest / unit > 127, 2 * unit, unit)
            values[:, :, blk, 0] = torch.ceil(hi / unit) * unit
            values[:, :, blk, 1] = torch.floor(lo / unit) * unit
    return [values]


def _exact_selection(c, s, hot):
    """(selected, scores): for each session and head the bounds by the definition, whole numbers and a sort."""
    bt, G = c["bt"], c["hq"] // c["hkv"]
    selected = torch.full((c["batch"], c["hkv"], c["top"]), -1, dtype=torch.int32, device="cuda")
    scores = torch.full((c["batch"], c["hkv"], s["width"]), -math.inf, dtype=torch.float64, device="cuda")
    for b, t in enumerate(s["n"]):
        n = _blocks(t, bt)
        blk = torch.from_numpy(s["tab"][b, :n].astype(np.int64)).cuda()
        for g in range(c["hkv"]):
            q = s["q"][b, g * G:(g + 1) * G].double()
            q = torch.round(q * 2.0 ** (10 - math.floor(math.log2(float(q.abs().max()))))).long()
            k = hot[blk, 0, 0, g].double()                              # [n][bt][D]
            some = (torch.arange(n * bt, device="cuda") < t).view(n, bt, 1)
            hi = torch.where(some, k, -math.inf).amax(dim=1)
            lo = torch.where(some, k, math.inf).amin(dim=1)
            largest = torch.maximum(hi, -lo).amax(dim=1, keepdim=True)
            unit = torch.exp2(torch.floor(torch.log2(largest)) - 6)
            unit = torch.where(largest / unit > 127, 2 * unit, unit)
            hi, lo = torch.ceil(hi / unit).long(), torch.floor(lo / unit).long()
            total = torch.zeros(n, dtype=torch.int64, device="cuda")
            for h in range(G):
                total += torch.where(q[h] > 0, q[h] * hi, q[h] * lo).sum(dim=1)
            x = total.float().double() * unit[:, 0]                     # a score has 24 bits
            x[:c["first"]] = x[max(0, n - c["last"]):] = math.inf
            scores[b, g, :n] = x
            pick = torch.sort(x, descending=True, stable=True).indices[:c["top"]].sort().values
            selected[b, g, :len(pick)] = pick.int()
    return selected, scores


def _exact_attention(c, s, hot, selected):
    """A session and KV head at a time."""
    bt, G = c["bt"], c["hq"] // c["hkv"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    for b, t in enumerate(s["n"]):
        row = torch.from_numpy(s["tab"][b].astype(np.int64)).cuda()
        for g in range(c["hkv"]):
            j = selected[b, g][selected[b, g] >= 0].long()
            pos = (j[:, None] * bt + torch.arange(bt, device="cuda")).flatten()
            pos = pos[pos < t]
            k, v = (hot[row[pos // bt], 0, w, g, pos % bt].double() for w in (0, 1))
            x = s["q"][b, g * G:(g + 1) * G].double() @ k.T / math.sqrt(D)
            out[b, g * G:(g + 1) * G] = torch.softmax(x, dim=1) @ v
    return out


def _exact_cached(c, seed):
    s = _token_inputs(_cached(c, seed), seed)
    hot = _fill_arena(_arena(c, s["blocks"]), seed)
    if c["kind"] == "attend":
        return [_exact_attention(c, s, hot, torch.from_numpy(_some_blocks(c, seed)).cuda())]
    # a step's bounds are from before its token: its block is among the last ones, which need none
    selected, scores = _exact_selection(c, s, hot)
    if c["kind"] == "select":
        return [selected, scores]
    for b, t in enumerate(s["n"]):
        at = int(s["tab"][b, (t - 1) // c["bt"]]), (t - 1) % c["bt"]
        hot[at[0], 0, 0, :, at[1]], hot[at[0], 0, 1, :, at[1]] = s["k"][b], s["v"][b]
    return [selected, _exact_attention(c, s, hot, selected), None]


def _exact_sessions(c, seed):
    """The arena token by token of the definition; a token of all layers and heads at a time where it can be."""
    lens, bt = _lengths(c), c["bt"]
    if c["kind"] == "fork" and lens[0] * (1 + (c["ways"] if c["lru"] else 0)) * _token_bytes(c) > 4e9:
        return None                 # an arena of over 16 GB in 64 bits
    s = _prepare_sessions(c, seed)
    hot = s["hot"].double()
    if c["kind"] == "fork":
        _, rows = _branches(s)
        for row in rows:
            for j, blk in enumerate(row):
                n = min(bt, lens[0] - j * bt)
                hot[blk, :, :, :, :n] = s["hot"][s["rows"][0][j], :, :, :, :n].double()
        return [hot, None, None]
    for row, keep, (p, k) in zip(s["rows"], _lists(c, seed), _kept(c)):
        blk = torch.tensor(row, device="cuda")
        to = torch.arange(p, p + k, device="cuda")
        for layer in range(c["layers"]):
            for g in range(c["hkv"]):
                at = torch.from_numpy((keep[layer, g] if c["lists"] else keep).astype(np.int64)).cuda()
                for w in (0, 1):
                    hot[blk[to // bt], layer, w, g, to % bt] = s["hot"][blk[at // bt], layer, w, g, at % bt].double()
    return [hot, None, None]


def exact(c, seed):
    """Outputs by the definition, in 64 bits."""
    if c["kind"] == "bounds":
        return _exact_bounds(c, seed)
    if c["kind"] in ("fork", "compact"):
        return _exact_sessions(c, seed)
    return _exact_cached(c, seed)
