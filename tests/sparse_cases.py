"""Inputs and 64-bit references for bounds of blocks, selection and attention over listed blocks.

Bounds and selections are whole numbers: the kernels' have to be equal. Attention is held to the
bound of turn_cases.ROW, whose derivation holds here as well (32-bit scores and sums, weights rounded
once to bf16, outputs in bf16).
"""
import math

import numpy as np
import torch

D = 128


def generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


class Cache:
    """Sessions of T[b] tokens at random places of an arena whose other rows are NaN."""

    def __init__(self, T, *, hq=32, hkv=4, bt=16, seed=0, q_std=1.0, layers=1, layer=0, fused=False, spare=3,
                 dtype=torch.bfloat16, drift=0.7, extra_width=0):
        import __graft_entry__
        __graft_entry__.build()
        from paper_2609_25782_gb300 import Pool
        self.T, self.hq, self.hkv, self.bt, self.layer, self.B = list(T), hq, hkv, bt, layer, len(T)
        self.G = hq // hkv
        g, r = generator(seed), np.random.RandomState(seed)
        blocks = [-(-max(t, 0) // bt) for t in T]
        self.width = max(max(blocks), 1) + extra_width
        nb = sum(blocks) + spare
        perm = r.permutation(nb)
        tab = np.full((self.B, self.width), -1, dtype=np.int32)
        at = 0
        for i, m in enumerate(blocks):
            tab[i, :m] = perm[at:at + m]
            at += m
        self.tab, self.nb = tab, nb
        self.pool = Pool(num_layers=layers, num_hot_blocks=nb, cold_bytes=256, num_q_heads=hq, num_kv_heads=hkv,
                         block_tokens=bt, max_sessions=1, max_batch=1, max_context=self.width * bt)
        self.hot = self.pool.hot_view()
        self.hot.fill_(float("nan"))
        for i, t in enumerate(self.T):
            for j in range(blocks[i]):
                n = min(bt, t - j * bt)
                kv = torch.randn(layers, 2, hkv, n, D, device="cuda", generator=g)
                kv[:, 0] += drift * torch.randn(layers, hkv, 1, D, device="cuda", generator=g)
                self.hot[tab[i, j], :, :, :, :n] = kv.bfloat16()
        qkv = torch.randn(self.B, hq + 2 * hkv, D, device="cuda", generator=g)
        qkv[:, :hq] *= q_std
        qkv = qkv.bfloat16()
        self.q, self.k, self.v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        if not fused:
            self.q, self.k, self.v = (x.contiguous() for x in (self.q, self.k, self.v))
        self.tables = torch.from_numpy(tab).cuda()
        self.lens = torch.tensor(self.T, dtype=torch.int32, device="cuda")
        self.out = torch.full((self.B, hq, D), 7.0, dtype=dtype, device="cuda")
        self.scale = 1 / math.sqrt(D)
        self.bounds = self.pool.new_bounds()
        self.codes, self.steps = self.pool.bounds_views(self.bounds)

    def blocks(self, b):
        return -(-self.T[b] // self.bt)

    # bounds -------------------------------------------------------------------------
    def make_bounds(self, layer=-1, since=None, stream=None):
        if since is not None and not hasattr(since, "data_ptr"):
            since = torch.tensor(since, dtype=torch.int32, device="cuda")
        self.pool.block_bounds(layer, self.tables, self.lens, self.B, self.width, self.bounds, since, stream)

    def reference_bounds(self, b, j, layer):
        """(codes [Hkv][2][D] int8, steps [Hkv]) of a row's block."""
        n = min(self.bt, self.T[b] - j * self.bt)
        return bounds_of(self.hot[int(self.tab[b, j]), layer, 0, :, :n])

    # selection ----------------------------------------------------------------------
    def select(self, top, first=1, last=1, scores=True, stream=None):
        self.selected = torch.full((self.B, self.hkv, top), 12345, dtype=torch.int32, device="cuda")
        self.scores = torch.full((self.B, self.hkv, self.width), 7.0, device="cuda") if scores else None
        self.pool.select_blocks(self.layer, self.q, self.bounds, self.tables, self.lens, self.B, self.width,
                                self.selected, first=first, last=last, scores=self.scores, stream=stream)
        return self.selected

    def reference_selection(self, b, g, top, first=1, last=1):
        """(selected [top], scores [width]) of a row and head from the bounds in the buffer."""
        n = self.blocks(b)
        q = self.q[b, g * self.G:(g + 1) * self.G].double().cpu()
        q = torch.where(torch.isfinite(q), q, 0.0)
        e = max(-126, math.floor(math.log2(float(q.abs().max())))) if float(q.abs().max()) else -126
        # (a subnormal largest value has the exponent of the smallest normal one)
        c = torch.round(q * 2.0 ** (10 - e)).long()
        qp, qn = c.clamp(min=0).sum(0), c.clamp(max=0).sum(0)
        blk = torch.from_numpy(self.tab[b, :n].astype(np.int64)).cuda()
        codes, steps = (x[self.layer, g, blk].cpu() for x in (self.codes, self.steps))
        whole = (qp * codes[:, 0].long() + qn * codes[:, 1].long()).sum(1)
        x = whole.float() * steps.float()
        x[torch.isinf(steps)] = math.inf
        rank = torch.zeros(n)
        for part in (slice(0, first), slice(max(0, n - last), n)):
            x[part], rank[part] = math.inf, 1
        order = sorted(range(n), key=lambda j: (-float(rank[j]), -float(x[j]), j))[:top]
        scores = torch.full((self.width,), -math.inf)
        scores[:n] = x
        return sorted(order) + [-1] * (top - len(order)), scores

    def check_selection(self, top, first=1, last=1):
        self.select(top, first, last)
        assert self.pool.check_device() == 0
        for b in range(self.B):
            for g in range(self.hkv):
                want, scores = self.reference_selection(b, g, top, first, last)
                assert self.selected[b, g].tolist() == want, (b, g)
                assert torch.equal(self.scores[b, g].cpu(), scores), (b, g)

    # attention ----------------------------------------------------------------------
    def random_lists(self, top, seed=0, holes=0.2):
        """Each row and head's own blocks in any order, some entries negative."""
        r = np.random.RandomState(seed)
        out = np.full((self.B, self.hkv, top), -1, dtype=np.int32)
        for b in range(self.B):
            for g in range(self.hkv):
                n = min(top, self.blocks(b))
                at = np.sort(r.permutation(top)[:n])
                out[b, g, at] = r.permutation(self.blocks(b))[:n]
                out[b, g, r.rand(top) < holes] = -1 - r.randint(0, 5)
        self.selected = torch.from_numpy(out).cuda()
        return self.selected

    def attend(self, new=False, stream=None):
        self.pool.sparse_attention(self.layer, self.q, self.selected, self.tables, self.lens, self.B, self.width,
                                   self.scale, self.out, *((self.k, self.v) if new else (None, None)), stream)
        return self.out

    def reference(self, b, new=False):
        """(out [Hq][D], noise [Hq]) of row b; the arena as it was before the call."""
        out = torch.zeros(self.hq, D, dtype=torch.float64, device="cuda")
        noise = torch.zeros(self.hq, dtype=torch.float64, device="cuda")
        row = torch.from_numpy(self.tab[b].astype(np.int64)).cuda()
        for g in range(self.hkv):
            j = self.selected[b, g][self.selected[b, g] >= 0].long()
            pos = (j[:, None] * self.bt + torch.arange(self.bt, device="cuda")).flatten()
            pos = pos[pos < self.T[b]]
            if not len(pos):
                continue
            k, v = (self.hot[row[pos // self.bt], self.layer, w, g, pos % self.bt].double() for w in (0, 1))
            if new:
                k[pos == self.T[b] - 1], v[pos == self.T[b] - 1] = self.k[b, g].double(), self.v[b, g].double()
            h = slice(g * self.G, (g + 1) * self.G)
            w = torch.softmax(self.q[b, h].double() @ k.T * self.scale, 1)
            out[h] = w @ v
            noise[h] = torch.sqrt((w * w) @ (v * v).sum(1))
        return out, noise

    def assert_right(self, b, ref, noise):
        from turn_cases import ROW
        got = self.out[b].double()
        assert torch.isfinite(got).all(), f"row {b}: not finite"
        err, bound = (got - ref).norm(dim=1), ROW * (noise + ref.norm(dim=1))
        assert (err <= bound).all(), f"row {b} (T {self.T[b]}): error over its bound by {float((err - bound).max()):.3e}, " \
            f"heads {torch.nonzero(err > bound).flatten().tolist()}"

    def check(self, new=False):
        """Every row against the reference, the new token's slot, and nothing else written."""
        refs = [self.reference(b, new) for b in range(self.B)]
        before = self.hot.clone()
        self.attend(new)
        assert self.pool.check_device() == 0
        for b, r in enumerate(refs):
            self.assert_right(b, *r)
            if new and self.T[b] > 0:
                t = self.T[b] - 1
                blk, slot = int(self.tab[b, t // self.bt]), t % self.bt
                before[blk, self.layer, 0, :, slot], before[blk, self.layer, 1, :, slot] = self.k[b], self.v[b]
        assert torch.equal(self.hot.view(torch.int16), before.view(torch.int16)), "the arena"


def bounds_of(k):
    """(codes [..][2][D] int8, steps [..] bf16) of keys [..][n][D], in 64 bits."""
    x = k.double()
    hi, lo = x.amax(dim=-2), x.amin(dim=-2)
    top = torch.maximum(hi.abs(), lo.abs()).amax(dim=-1)
    fine = torch.isfinite(k).all(dim=-1).all(dim=-1)
    bits = torch.where(fine, top, 1.0).to(torch.bfloat16).view(torch.int16).int()
    e = (bits >> 7).clamp(min=1) + ((bits & 127) == 127).int()
    step = torch.exp2((e - 133).double())
    codes = torch.stack([torch.ceil(hi / step[..., None]), torch.floor(lo / step[..., None])], dim=-2)
    limit = torch.tensor([127.0, -127.0], dtype=torch.float64, device=k.device)[:, None]
    codes = torch.where(fine[..., None, None], codes, limit.expand_as(codes))
    assert codes.abs().max() <= 127
    return codes.to(torch.int8), torch.where(fine, step, math.inf).to(torch.bfloat16)
