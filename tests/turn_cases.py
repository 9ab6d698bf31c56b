"""Inputs, a 64-bit reference and bounds for attention of several new tokens per session.

The reference is the definition: a softmax over the keys that a row sees, in 64 bits, one session
and head at a time.

Bounds, per output row (a token and head) of 128 values. The kernels hold scores and sums in 32
bits and round the weights p_j once to bf16 (relative 2^-9 at most, and independent), so the error
has a norm of about 2^-9 / sqrt(3) * 0.7 of sqrt(sum_j p_j^2 |V_j|^2) and never more than 2^-9 of
sum_j p_j |V_j|; outputs in bf16 add 2^-9 / sqrt(3) of the row's own norm, 2^-9 at most. One
weight carrying a whole row is the worst: 2^-9 and 2^-9 / sqrt(3), 2.3e-3 together. ROW = 4e-3 of
sqrt(sum_j p_j^2 |V_j|^2) + |out| leaves 32-bit sums (under 5e-4 with scores of the sizes here) their
room, and is well below what one key too few or too many changes.
"""
import math

import numpy as np
import torch

D = 128
ROW = 4e-3


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


class Call:
    """Sessions of n[b] new tokens on p[b] cached ones, blocks at random places of an arena whose
    other rows are NaN. kind: "prefill" or "tree"."""

    def __init__(self, kind, n, p, *, hq=32, hkv=4, bt=16, seed=0, q_std=1.0, layers=1, layer=0,
                 fused=False, masks=None, spare=3, dtype=torch.bfloat16, pool_kw=None):
        import __graft_entry__
        __graft_entry__.build()
        from paper_2609_25782_gb300 import Pool
        self.kind, self.n, self.p, self.hq, self.hkv, self.bt = kind, list(n), list(p), hq, hkv, bt
        self.layer, self.B = layer, len(n)
        g, r = generator(seed), np.random.RandomState(seed)
        self.T = [a + b for a, b in zip(n, p)] if kind == "prefill" else list(p)
        blocks = [-(-t // bt) for t in self.T]
        self.width = max(max(blocks), 1)
        nb = sum(blocks) + spare
        perm = r.permutation(nb)
        tab = np.full((self.B, self.width), -1, dtype=np.int32)
        at = 0
        for i, m in enumerate(blocks):
            tab[i, :m] = perm[at:at + m]
            at += m
        self.tab = tab
        self.pool = Pool(num_layers=layers, num_hot_blocks=nb, cold_bytes=256, num_q_heads=hq,
                         num_kv_heads=hkv, block_tokens=bt, max_sessions=1, max_batch=1,
                         max_context=self.width * bt, **(pool_kw or {}))
        self.hot = self.pool.hot_view()
        self.hot.fill_(float("nan"))
        for i, c in enumerate(self.p):                   # cached tokens of this layer
            if c:
                blk, slot = self.slots(i, 0, c)
                self.hot[blk, layer, :, :, slot] = torch.randn(c, 2, hkv, D, device="cuda", generator=g).bfloat16()
        rows = sum(self.n)
        qkv = torch.randn(rows, hq + 2 * hkv, D, device="cuda", generator=g)
        qkv[:, :hq] *= q_std
        qkv = qkv.bfloat16()
        self.q, self.k, self.v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        if not fused:
            self.q, self.k, self.v = (x.contiguous() for x in (self.q, self.k, self.v))
        self.cu = torch.tensor(np.concatenate([[0], np.cumsum(self.n)]), dtype=torch.int32, device="cuda")
        self.tables = torch.from_numpy(tab).cuda()
        self.lens = torch.tensor(self.T, dtype=torch.int32, device="cuda")
        self.out = torch.full((rows, hq, D), 7.0, dtype=dtype, device="cuda")
        self.scale = 1 / math.sqrt(D)
        if kind == "tree":
            m = masks if masks is not None else tree_masks(self.n, seed)
            self.bits = [int(x) for x in m]
            self.masks = torch.tensor([x - (1 << 64) if x >> 63 else x for x in self.bits],
                                      dtype=torch.int64, device="cuda")

    def slots(self, b, lo, hi):
        t = torch.arange(lo, hi, device="cuda")
        return torch.from_numpy(self.tab[b].astype(np.int64)).cuda()[t // self.bt], t % self.bt

    def run(self, stream=None):
        if self.kind == "prefill":
            self.pool.prefill_attention(self.layer, self.q, self.k, self.v, self.cu, self.tables, self.lens,
                                        self.B, self.width, self.scale, self.out, stream)
        else:
            self.pool.tree_attention(self.layer, self.q, self.k, self.v, self.masks, self.cu, self.tables,
                                     self.lens, self.B, self.width, self.scale, self.out, stream)
        return self.out

    def seen(self, b):
        """Which of the session's own tokens each of them sees, [n][n]."""
        n, lo = self.n[b], sum(self.n[:b])
        i = torch.arange(n, device="cuda")
        if self.kind == "prefill":
            return i[None, :] <= i[:, None]
        return torch.tensor([[self.bits[lo + r] >> c & 1 for c in range(n)] for r in range(n)],
                            device="cuda").bool().view(n, n)

    def reference(self, b):
        """(out [n][Hq][D], noise [n][Hq]) of session b; the arena as it was before the call."""
        n, p, lo, G = self.n[b], self.p[b], sum(self.n[:b]), self.hq // self.hkv
        out = torch.zeros(n, self.hq, D, dtype=torch.float64, device="cuda")
        noise = torch.zeros(n, self.hq, dtype=torch.float64, device="cuda")
        seen = torch.cat([torch.ones(n, p, dtype=torch.bool, device="cuda"), self.seen(b)], 1)
        some = seen.any(1)
        blk, slot = self.slots(b, 0, p)
        for h in range(self.hq):
            g = h // G
            k, v = (torch.cat([self.hot[blk, self.layer, w, g, slot], x[lo:lo + n, g]]).double()
                    for w, x in ((0, self.k), (1, self.v)))
            x = self.q[lo:lo + n, h].double() @ k.T * self.scale
            x = x.masked_fill(~seen, -math.inf)
            x[~some] = 0.0
            w = torch.softmax(x, 1) * some[:, None]
            out[:, h] = w @ v
            noise[:, h] = torch.sqrt((w * w) @ (v * v).sum(1))
        return out, noise

    def assert_right(self, b, ref, noise):
        """Session b's rows of `out` against reference(b)."""
        lo = sum(self.n[:b])
        got = self.out[lo:lo + self.n[b]].double()
        bound = ROW * (noise + ref.norm(dim=2))
        err = (got - ref).norm(dim=2)
        worst = (err - bound).max() if err.numel() else torch.tensor(-1.0)
        assert torch.isfinite(got).all(), f"session {b}: not finite"
        assert worst <= 0, f"session {b} (n {self.n[b]}, p {self.p[b]}): error over its bound by {worst:.3e}, " \
            f"rows {torch.nonzero(err > bound)[:6].tolist()}"

    def check(self):
        """Every row against the reference; for a prefill the slots as well, and nothing else written."""
        refs = [self.reference(b) for b in range(self.B)]
        before = self.hot.clone()
        self.run()
        assert self.pool.check_device() == 0
        for b, (ref, noise) in enumerate(refs):
            self.assert_right(b, ref, noise)
        if self.kind == "prefill":
            for b, p in enumerate(self.p):
                lo = sum(self.n[:b])
                blk, slot = self.slots(b, p, p + self.n[b])
                before[blk, self.layer, 0, :, slot] = self.k[lo:lo + self.n[b]]
                before[blk, self.layer, 1, :, slot] = self.v[lo:lo + self.n[b]]
        assert torch.equal(self.hot.view(torch.int16), before.view(torch.int16)), "the arena"


def tree_masks(n, seed, branch=0.5):
    """Random draft trees: bit masks of each draft's ancestors and itself."""
    r = np.random.RandomState(seed + 99)
    out = []
    for m in n:
        mine = []
        for i in range(m):
            parent = r.randint(-1, i) if r.rand() < branch else i - 1
            mine.append((mine[parent] if parent >= 0 else 0) | 1 << i)
        out += mine
    return out
