"""Timed operators of a turn over the tiered cache, in their plain form and through the package.

prefill  attention of a turn's new tokens (or of whole first prompts): causal, grouped heads, packed
         sequences of different lengths, over each session's cached prefix; the new tokens' K and V
         are written into their reserved slots of the hot pool as well
tree     attention of drafted tokens, each over the whole cached context and over the drafts that
         its bit mask names (its ancestors in the draft tree, and itself)
turn8    a turn's context is appended, the session pauses into an 8-bit image, and comes back
resume8  paused sessions come back from 8-bit images while others leave

An 8-bit image holds a row (token, layer, K or V, kv-head) of 128 values as codes in -127..127 and
the biased exponent E of its largest magnitude (at least 1): value = code * 2^(E - 133).

Shapes are the repository's: head_dim 128, 32 query and 4 KV heads, 48 layers, blocks of 16 or 64
tokens, contexts from a few tokens to 128K. Attention cases are one layer's call, as a model makes it.
"""
import math

import numpy as np
import torch

own = False     # False: elementary torch operations; True: the package's operators

D = 128


def _case(name, kind, **kw):
    c = {"name": name, "kind": kind, "layers": 1, "hq": 32, "hkv": 4, "bt": 16, "pmin": 0, "pmax": 0,
         "q_std": 1.0}
    c.update(kw)
    return c


def listed():
    return [
        # the first, short message of a chat: the smallest call, all latency
        _case("prompt_1x37", "prefill", batch=1, nmin=37, nmax=37, lens_seed=1),
        # a batch of first prompts of very unequal lengths, nothing cached yet
        _case("prompts_8x100-4k", "prefill", batch=8, nmin=100, nmax=4000, lens_seed=2),
        # the agentic trace's turns: tool results appended to long contexts
        _case("turns_4x300-3k_on_2k-24k", "prefill", batch=4, nmin=300, nmax=3000, pmin=2048,
              pmax=24576, q_std=2.0, lens_seed=3),
        # one whole long prompt: the tensor cores' case
        _case("prompt_1x16k", "prefill", batch=1, nmin=16391, nmax=16391, lens_seed=4),
        # a mixed step of a serving engine: short chunks and single tokens over long contexts, q, k
        # and v as views of one fused projection, 8 KV heads in groups of 4, 64-token blocks
        _case("chunks_16x1-200_on_1k-40k_bt64", "prefill", hkv=8, bt=64, batch=16, nmin=1, nmax=200,
              pmin=1000, pmax=40000, fused=True, lens_seed=5),
        # one agent verifying a short chain of drafts early in its task: latency
        _case("draft_1x7_on_3k", "tree", batch=1, nmin=7, nmax=7, pmin=3001, pmax=3001, branch=0.0,
              lens_seed=6),
        # the agentic trace's batch, 16 drafts a session; peaked scores, as trained heads have
        _case("draft_16x16_on_2k-30k", "tree", batch=16, nmin=16, nmax=16, pmin=2048, pmax=30000,
              branch=0.5, q_std=4.0, lens_seed=7),
        # wide draft trees over many shorter sessions, 8 KV heads in groups of 4, 64-token blocks
        _case("draft_32x20-60_on_200-9k_bt64", "tree", hkv=8, bt=64, batch=32, nmin=20, nmax=60,
              pmin=200, pmax=9000, branch=0.7, lens_seed=8),
        # one turn of the paper's model: appended, paused for a tool call, brought back
        _case("turn8_1x1536", "turn8", layers=48, batch=1, nmin=1536, nmax=1536, lens_seed=9),
        # three short turns of a smaller model with 8 KV heads, odd lengths
        _case("turn8_3x200-900_bt64", "turn8", layers=16, hkv=8, bt=64, batch=3, nmin=200, nmax=900,
              lens_seed=10),
        # one short session leaves, another comes back
        _case("resume8_1x2100", "resume8", layers=48, batch=1, nmin=2100, nmax=2100, lens_seed=11),
        # several long sessions come back at once
        _case("resume8_3x12k-32k", "resume8", layers=48, batch=3, nmin=12000, nmax=32768,
              lens_seed=12),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges above, no dearer than the largest of its kind."""
    kind = rng.choice(["prefill"] * 4 + ["tree"] * 3 + ["turn8", "resume8"])
    hkv, hq = rng.choice([(4, 32), (4, 32), (4, 32), (8, 32), (4, 16), (8, 64), (2, 16), (8, 8)])
    c = {"kind": kind, "layers": 1, "hq": hq, "hkv": hkv, "bt": rng.choice([16, 16, 64]), "pmin": 0,
         "pmax": 0, "q_std": rng.choice([1.0, 2.0, 4.0]), "lens_seed": rng.randrange(1 << 20)}
    if kind in ("prefill", "tree"):
        c["nmax"] = _log_int(rng, 1, 16000 if kind == "prefill" else 64)
        c["nmin"] = _log_int(rng, 1, c["nmax"]) if rng.random() < 0.7 else c["nmax"]
        if kind == "tree" or rng.random() < 0.6:
            c["pmax"] = _log_int(rng, 100, 100000)
            c["pmin"] = _log_int(rng, 100, c["pmax"]) if rng.random() < 0.7 else c["pmax"]
        if kind == "tree":
            c["branch"] = rng.choice([0.0, 0.5, 0.9])
        else:
            c["fused"] = rng.random() < 0.4
        # at most the pairs of the longest prompt, and 4 GB of cached K and V
        pairs = c["nmax"] * (c["pmax"] + c["nmax"] / 2) * hq
        most = min(1.3e8 * 32 / pairs, 4e9 / ((c["pmax"] + c["nmax"]) * hkv * 4 * D), 64)
        while most < 1:             # one session is too much by itself: fewer new tokens
            c["nmax"] = max(1, int(c["nmax"] * 0.7))
            c["nmin"] = min(c["nmin"], c["nmax"])
            pairs = c["nmax"] * (c["pmax"] + c["nmax"] / 2) * hq
            most = min(1.3e8 * 32 / pairs, 64)
        c["batch"] = _log_int(rng, 1, max(1, int(most)))
    else:
        c["layers"] = rng.choice([4, 16, 28, 48])
        limit = 2e9 if kind == "turn8" else 6e9
        c["nmax"] = _log_int(rng, 30, 32768)
        token = _token_bytes(c)
        if c["nmax"] * token > limit:
            c["layers"] = max(1, int(c["layers"] * limit / (c["nmax"] * token)))
            token = _token_bytes(c)
        c["nmin"] = _log_int(rng, 20, c["nmax"]) if rng.random() < 0.7 else c["nmax"]
        c["batch"] = _log_int(rng, 1, max(1, min(8, int(limit / (c["nmax"] * token)))))
    return c


# ---- sizes ---------------------------------------------------------------------------------

def _token_bytes(c):
    return c["layers"] * 2 * c["hkv"] * D * 2


def _lengths(c):
    """(new or drafted tokens, cached tokens) of each session, the same for every seed of the values."""
    r = np.random.RandomState(c["lens_seed"])
    lo, hi = math.log(c["nmin"]), math.log(c["nmax"])
    n = np.rint(np.exp(r.uniform(lo, hi, c["batch"]))).astype(np.int64)
    p = r.randint(c["pmin"], c["pmax"] + 1, c["batch"]) if c["pmax"] else np.zeros(c["batch"], int)
    return [int(x) for x in n], [int(x) for x in p]


def _blocks(t, bt):
    return -(-t // bt)


def work(c):
    n, p = _lengths(c)
    rows = sum(n)
    if c["kind"] in ("turn8", "resume8"):
        # 8-bit rows are 129 bytes for 256 in bf16; a turn: k and v read, blocks written (append),
        # blocks read, image written (pause), image read, blocks written (resume)
        head_rows = rows * c["layers"] * 2 * c["hkv"]
        per = 2 * 256 + 2 * (256 + 129) if c["kind"] == "turn8" else 2 * (256 + 129)
        return {"bytes": head_rows * per, "flops": 0}
    b = rows * c["hq"] * D * 2 * 2 + rows * c["hkv"] * D * 2 * 2 + sum(p) * c["hkv"] * D * 2 * 2
    if c["kind"] == "prefill":
        b += rows * c["hkv"] * D * 2 * 2            # K and V into the pool
        pairs = sum(x * y + x * (x + 1) // 2 for x, y in zip(n, p))
    else:
        b += rows * 8
        pairs = sum(x * y for x, y in zip(n, p)) + _masks(c)[1]
    return {"bytes": b, "flops": 4 * D * c["hq"] * pairs}


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


def _masks(c):
    """Each draft's bit mask over its session's drafts (its ancestors and itself), and the bits' sum.
    A draft follows the one before it, or with probability `branch` any earlier one or the context."""
    r = np.random.RandomState(c["lens_seed"] + 1)
    masks, bits = [], 0
    for n in _lengths(c)[0]:
        mine = []
        for i in range(n):
            parent = r.randint(-1, i) if r.rand() < c["branch"] else i - 1
            mine.append((mine[parent] if parent >= 0 else 0) | (1 << i))
        masks += mine
        bits += sum(bin(m).count("1") for m in mine)
    return np.array(masks, dtype=np.uint64).view(np.int64), bits


def _attention_inputs(c, seed):
    """Everything but the hot arena's values. A prefill's tables and lengths have its tokens' slots."""
    n, p = _lengths(c)
    own_slots = n if c["kind"] == "prefill" else [0] * len(n)
    total = [x + y for x, y in zip(own_slots, p)]
    bt = c["bt"]
    width = max(max(_blocks(t, bt) for t in total), 1)
    blocks = sum(_blocks(t, bt) for t in total)
    perm = np.random.RandomState(seed & 0x7FFFFFFF).permutation(blocks)
    tab = np.full((len(n), width), -1, dtype=np.int32)
    at = 0
    for i, t in enumerate(total):
        tab[i, :_blocks(t, bt)] = perm[at:at + _blocks(t, bt)]
        at += _blocks(t, bt)
    rows, hq, hkv = sum(n), c["hq"], c["hkv"]
    if c.get("fused"):              # one projection's output: [rows][hq + 2 hkv][D]
        qkv = _normal((rows, hq + 2 * hkv, D), seed, 2)
        qkv[:, :hq] *= c["q_std"]
        q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    else:
        q = _normal((rows, hq, D), seed, 2, c["q_std"])
        k, v = _normal((rows, hkv, D), seed, 3), _normal((rows, hkv, D), seed, 4)
    s = {"case": c, "n": n, "p": p, "blocks": max(blocks, 1), "width": width, "tab": tab,
         "tables": torch.from_numpy(tab).cuda(), "q": q, "k": k, "v": v,
         "lens": torch.tensor(total, dtype=torch.int32, device="cuda"),
         "cu": torch.tensor(np.concatenate([[0], np.cumsum(n)]), dtype=torch.int32, device="cuda"),
         "out": torch.zeros((rows, hq, D), dtype=torch.bfloat16, device="cuda")}
    if c["kind"] == "tree":
        s["masks"] = torch.from_numpy(_masks(c)[0]).cuda()
    return s


def _arena(c, blocks):
    """An empty hot arena, [blocks][L][2][Hkv][bt][D]."""
    return torch.zeros((blocks, c["layers"], 2, c["hkv"], c["bt"], D), dtype=torch.bfloat16,
                       device="cuda")


def _prepare_attention(c, seed):
    s = _attention_inputs(c, seed)
    if own:
        from paper_2609_25782_gb300 import Pool
        s["pool"] = Pool(num_layers=1, num_hot_blocks=s["blocks"], cold_bytes=256,
                         num_q_heads=c["hq"], num_kv_heads=c["hkv"], block_tokens=c["bt"],
                         max_sessions=1, max_batch=c["batch"],
                         max_context=s["width"] * c["bt"])
        s["hot"] = s["pool"].hot_view()
    else:
        s["hot"] = _arena(c, s["blocks"])
    _fill(s["hot"], seed, 1)
    return s


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


def _session_pool(c, seed, blocks, images):
    from paper_2609_25782_gb300 import Pool
    pool = Pool(num_layers=c["layers"], num_hot_blocks=blocks,
                cold_bytes=sum(t * _token_bytes(c) + 512 for t in images), num_q_heads=c["hq"],
                num_kv_heads=c["hkv"], block_tokens=c["bt"], max_sessions=len(images),
                max_batch=c["batch"], max_context=max(images), alloc_seed=int(seed),
                cold_int8=True)
    pool.hot.zero_()
    return pool


def _prepare_sessions(c, seed):
    """turn8: the turns' K and V. resume8: two groups of sessions' images (codes and exponents), the
    hot pool as large as one of them, which it holds."""
    lens = _lengths(c)[0]
    bt, L, hkv = c["bt"], c["layers"], c["hkv"]
    blocks, width = sum(_blocks(t, bt) for t in lens), max(_blocks(t, bt) for t in lens)
    s = {"case": c, "n": lens, "width": width, "blocks": blocks, "seed": int(seed),
         "tables": torch.zeros((len(lens), width), dtype=torch.int32, device="cuda"),
         "lens": torch.zeros(len(lens), dtype=torch.int32, device="cuda")}
    if c["kind"] == "turn8":
        s["kv"] = [(_normal((L, t, hkv, D), seed, 10 + 2 * i), _normal((L, t, hkv, D), seed, 11 + 2 * i))
                   for i, t in enumerate(lens)]
        images = []
    else:
        images = [_image8(c, t, seed, 10 + 2 * i) for i, t in enumerate(lens + lens)]
    if not own:
        s["hot"], s["images"] = _arena(c, blocks), images
        return s
    pool = s["pool"] = _session_pool(c, seed, blocks, lens if c["kind"] == "turn8" else lens + lens)
    s["hot"] = pool.hot_view()
    st = torch.cuda.current_stream()
    if c["kind"] == "turn8":
        s["sids"] = [pool.session_create(t) for t in lens]
        return s
    sids = [pool.session_create_paused(t, t) for t in lens + lens]
    for sid, (codes, exps) in zip(sids, images):
        to_codes, to_exps = pool.image_int8(sid)
        to_codes.copy_(codes)
        to_exps.copy_(exps)
    s["away"], s["sids"] = sids[:len(lens)], sids[len(lens):]
    for sid in s["sids"]:
        pool.session_resume(sid, st)
    return s


def _image8(c, t, seed, salt):
    """Codes and exponents as a pause leaves them: rows of N(0, 1) values have their largest in
    [1, 4) mostly, so exponents of 127 and 128, and codes up to 127 with most of them small."""
    g = _gen(seed, salt)
    shape = (c["layers"], 2, c["hkv"], t, D)
    codes = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(0.0, 32.0, generator=g)
    codes = codes.clamp_(-127, 127).to(torch.int8)
    exps = torch.empty(shape[:-1], dtype=torch.uint8, device="cuda").random_(126, 130, generator=g)
    return codes, exps


def prepare(case, seed):
    return (_prepare_attention if case["kind"] in ("prefill", "tree") else _prepare_sessions)(case, seed)


# ---- one pass ------------------------------------------------------------------------------

def run(state):
    return (_run_own if own else _run_plain)[state["case"]["kind"]](state)


def _own_prefill(s):
    s["pool"].prefill_attention(0, s["q"], s["k"], s["v"], s["cu"], s["tables"], s["lens"],
                                s["case"]["batch"], s["width"], 1 / math.sqrt(D), s["out"],
                                torch.cuda.current_stream())
    return [s["out"], s["hot"]]


def _own_tree(s):
    s["pool"].tree_attention(0, s["q"], s["k"], s["v"], s["masks"], s["cu"], s["tables"], s["lens"],
                             s["case"]["batch"], s["width"], 1 / math.sqrt(D), s["out"],
                             torch.cuda.current_stream())
    return [s["out"]]


def _own_turn8(s):
    pool, st = s["pool"], torch.cuda.current_stream()
    for sid in reversed(s["sids"]):     # the sessions of the pass before have ended
        pool.session_destroy(sid)
    s["sids"] = [pool.session_create(t) for t in s["n"]]
    for sid, (k, v) in zip(s["sids"], s["kv"]):
        pool.session_append(sid, k, v, st)
    for sid in reversed(s["sids"]):
        pool.session_pause(sid, st)
    for sid in s["sids"]:
        pool.session_resume(sid, st)
    pool.batch_tables(s["sids"], s["tables"], s["width"], s["lens"], st)
    return [s["hot"], s["tables"], s["lens"]]


def _own_resume8(s):
    pool, st = s["pool"], torch.cuda.current_stream()
    for out, back in ((s["sids"], s["away"]), (s["away"], s["sids"])):
        for sid in reversed(out):       # nothing new since the resume: the pause writes nothing
            pool.session_pause(sid, st)
        for sid in back:
            pool.session_resume(sid, st)
    pool.batch_tables(s["sids"], s["tables"], s["width"], s["lens"], st)
    return [s["hot"], s["tables"], s["lens"]]


def _cached(hot, row, p, bt):
    """K and V [Hkv][p][D] of a session's first p cached tokens."""
    idx = row[:_blocks(p, bt)].long()
    k, v = hot[idx, 0].permute(1, 2, 0, 3, 4).flatten(2, 3)[:, :, :p].float()
    return k, v


def _attend(q, k, v, keep):
    """q [n][Hq][D] over k, v [Hkv][m][D]; keep(first row, last row): which of the LAST n keys each
    of those rows sees (all earlier keys are seen). As many rows at a time as fit 1 GB of scores."""
    n, hq, _ = q.shape
    hkv, m, _ = k.shape
    q = q.float().view(n, hkv, hq // hkv, D).permute(1, 2, 0, 3)
    out = torch.empty((n, hq, D), dtype=torch.bfloat16, device=q.device)
    step = max(1, (1 << 28) // (hq * m))
    for i in range(0, n, step):
        rows = q[:, :, i:i + step]
        x = torch.matmul(rows.flatten(1, 2), k.transpose(1, 2)).view(hkv, hq // hkv, -1, m)
        x *= 1 / math.sqrt(D)
        x[..., m - n:].masked_fill_(~keep(i, min(n, i + step)), -math.inf)
        x -= x.amax(dim=-1, keepdim=True)
        x.exp_()
        y = torch.matmul(x.flatten(1, 2), v).view(hkv, hq // hkv, -1, D)
        y /= x.sum(dim=-1, keepdim=True)
        out[i:i + step] = y.permute(2, 0, 1, 3).reshape(-1, hq, D).to(torch.bfloat16)
    return out


def _plain_attention(s, masked):
    at = 0
    for b, (n, p) in enumerate(zip(s["n"], s["p"])):
        k, v = _cached(s["hot"], s["tables"][b], p, s["case"]["bt"])
        new = [x[at:at + n].float().transpose(0, 1) for x in (s["k"], s["v"])]
        s["out"][at:at + n] = _attend(s["q"][at:at + n], torch.cat([k, new[0]], 1),
                                      torch.cat([v, new[1]], 1), masked(s, at, n))
        at += n
    return s["out"]


def _causal(s, at, n):
    j = torch.arange(n, device="cuda")
    return lambda lo, hi: j[None, :] <= j[lo:hi, None]


def _ancestors(s, at, n):
    j = torch.arange(n, device="cuda")
    bits = ((s["masks"][at:at + n, None] >> j) & 1) == 1
    return lambda lo, hi: bits[lo:hi]


def _plain_prefill(s):
    bt, row_of = s["case"]["bt"], s["tables"].long()
    n, p = (torch.tensor(x, device="cuda") for x in (s["n"], s["p"]))
    which = torch.repeat_interleave(torch.arange(len(s["n"]), device="cuda"), n)
    pos = torch.arange(len(which), device="cuda") - s["cu"].long()[which] + p[which]
    blk = row_of[which, pos // bt]
    s["hot"][blk, 0, 0, :, pos % bt] = s["k"]
    s["hot"][blk, 0, 1, :, pos % bt] = s["v"]
    return [_plain_attention(s, _causal), s["hot"]]


def _plain_tree(s):
    return [_plain_attention(s, _ancestors)]


def _power(x, e):
    """x * 2^e, in two factors that 32 bits hold."""
    h = torch.div(e, 2, rounding_mode="floor")
    return torch.ldexp(torch.ldexp(x, h), e - h)


def _quantise(x):
    """Codes and exponents of rows of finite bf16 values."""
    x = x.float()
    e = (x.abs().amax(dim=-1).view(torch.int32) >> 23).clamp_(min=1)
    return _power(x, (133 - e)[..., None]).round_().clamp_(-127, 127).to(torch.int8), e.to(torch.uint8)


def _values(codes, exps):
    return _power(codes.float(), exps.int()[..., None] - 133).to(torch.bfloat16)


def _place(hot, blocks, kv, bt):
    """[L][2][Hkv][t][D] into its blocks of the arena."""
    t = kv.shape[3]
    full, idx = t // bt, torch.tensor(blocks, device="cuda")
    if full:
        hot[idx[:full]] = kv[:, :, :, :full * bt].unflatten(3, (full, bt)).permute(3, 0, 1, 2, 4, 5)
    if t > full * bt:
        hot[idx[full], :, :, :, :t - full * bt] = kv[:, :, :, full * bt:]


def _tables_of(s, rows):
    tab = np.full((len(rows), s["width"]), -1, dtype=np.int32)
    for i, r in enumerate(rows):
        tab[i, :len(r)] = r
    s["tables"].copy_(torch.from_numpy(tab))
    s["lens"].copy_(torch.tensor(s["n"], dtype=torch.int32))


def _take(free, lens, bt):
    """Blocks popped from the free list's end, session by session."""
    return [[free.pop() for _ in range(_blocks(t, bt))] for t in lens]


def _plain_turn8(s):
    """The free list is a stack: a pause pushes a session's blocks in order, a resume pops them."""
    bt, free = s["case"]["bt"], _free_order(s["blocks"], s["seed"])[::-1]
    first = _take(free, s["n"], bt)
    for blocks, (k, v) in zip(first, s["kv"]):
        _place(s["hot"], blocks, torch.stack([k, v], 1).transpose(2, 3), bt)
    for blocks in reversed(first):
        free += blocks
    images = [_quantise(torch.stack([k, v], 1).transpose(2, 3)) for k, v in s["kv"]]
    back = _take(free, s["n"], bt)
    for blocks, image in zip(back, images):
        _place(s["hot"], blocks, _values(*image), bt)
    _tables_of(s, back)
    return [s["hot"], s["tables"], s["lens"]]


def _plain_resume8(s):
    """Both groups of sessions come back once; the second one's blocks are those it had before."""
    bt, free = s["case"]["bt"], _free_order(s["blocks"], s["seed"])[::-1]
    here = _take(free, s["n"], bt)
    m = len(s["n"])
    for images in (s["images"][:m], s["images"][m:]):
        for blocks in reversed(here):
            free += blocks
        here = _take(free, s["n"], bt)
        for blocks, image in zip(here, images):
            _place(s["hot"], blocks, _values(*image), bt)
    _tables_of(s, here)
    return [s["hot"], s["tables"], s["lens"]]


_run_own = {"prefill": _own_prefill, "tree": _own_tree, "turn8": _own_turn8, "resume8": _own_resume8}
_run_plain = {"prefill": _plain_prefill, "tree": _plain_tree, "turn8": _plain_turn8,
              "resume8": _plain_resume8}


# ---- in 64 bits ----------------------------------------------------------------------------

def _exact_turn8(c, seed):
    """The arena after one pass over an empty one: the turns as appended, then as read back."""
    lens, bt = _lengths(c)[0], c["bt"]
    free = _free_order(sum(_blocks(t, bt) for t in lens), seed)[::-1]
    hot = _arena(c, len(free)).double()
    first = _take(free, lens, bt)
    back = _take([b for blocks in reversed(first) for b in blocks], lens, bt)
    for read_back in (False, True):
        for i, (t, blocks) in enumerate(zip(lens, back if read_back else first)):
            for w in (0, 1):
                x = _normal((c["layers"], t, c["hkv"], D), seed, 10 + 2 * i + w).double()
                if read_back:       # the step: a 64th of the power of two that the largest reaches
                    top = torch.floor(torch.log2(x.abs().amax(dim=-1, keepdim=True)))
                    unit = torch.exp2(top - 6)
                    x = torch.minimum(torch.round(x / unit).abs(), torch.tensor(127.0, device="cuda")) \
                        * torch.sign(x) * unit
                for j, b in enumerate(blocks):
                    part = x[:, j * bt:(j + 1) * bt].transpose(1, 2)
                    hot[b, :, w, :, :part.shape[2]] = part
    return [hot, None, None]


def _exact_resume8(c, seed):
    """The arena after one pass over one that is empty but for the second group's values."""
    lens, bt = _lengths(c)[0], c["bt"]
    if sum(lens) * _token_bytes(c) > 3e9:
        return None                 # an arena of over 12 GB in 64 bits, and as much on the way
    order = _free_order(sum(_blocks(t, bt) for t in lens), seed)
    hot = _arena(c, len(order)).double()
    there = _take(order[::-1], lens, bt)            # the second group's blocks, the other's backwards
    for group, places in ((1, there), (0, [b[::-1] for b in there]), (1, there)):
        for i, (t, blocks) in enumerate(zip(lens, places)):
            codes, exps = _image8(c, t, seed, 10 + 2 * (i + group * len(lens)))
            x = codes.double() * torch.exp2(exps.double() - 133)[..., None]
            for j, b in enumerate(blocks):
                part = x[:, :, :, j * bt:(j + 1) * bt]
                hot[b, :, :, :, :part.shape[3]] = part
    return [hot, None, None]


def exact(c, seed):
    """Outputs by the definition, in 64 bits: attention a session and head at a time."""
    if c["kind"] == "turn8":
        return _exact_turn8(c, seed)
    if c["kind"] == "resume8":
        return _exact_resume8(c, seed)
    n, p = _lengths(c)
    if c["hq"] * sum(x * (x + y) for x, y in zip(n, p)) > 1e10:
        return None                 # over 20 seconds in 64 bits
    s = _attention_inputs(c, seed)
    hot = _fill(_arena(c, s["blocks"]), seed, 1)
    group = c["hq"] // c["hkv"]
    out = torch.empty(s["out"].shape, dtype=torch.float64, device="cuda")
    for b in range(c["batch"]):
        lo = sum(n[:b])
        i = torch.arange(n[b], device="cuda")
        if c["kind"] == "prefill":
            seen = i[:, None] >= i
        else:
            m = [int(x) & ((1 << 64) - 1) for x in s["masks"][lo:lo + n[b]].tolist()]
            seen = torch.tensor([[x >> j & 1 for j in range(n[b])] for x in m], device="cuda").bool()
        pos = torch.arange(p[b], device="cuda")
        blk = torch.from_numpy(s["tab"][b].astype(np.int64)).cuda()[pos // c["bt"]]
        for g in range(c["hkv"]):
            k, v = (torch.cat([hot[blk, 0, w, g, pos % c["bt"]], x[lo:lo + n[b], g]]).double()
                    for w, x in ((0, s["k"]), (1, s["v"])))
            for h in range(g * group, (g + 1) * group):
                for r in range(0, n[b], 2048):
                    part = seen[r:r + 2048]
                    x = s["q"][lo + r:lo + r + len(part), h].double() @ k.T / math.sqrt(D)
                    x[:, p[b]:][~part] = -math.inf
                    out[lo + r:lo + r + len(part), h] = torch.softmax(x, dim=1) @ v
    return [out, None] if c["kind"] == "prefill" else [out]
