"""Turns of an agent on a pool with 8-bit cold images, the way a serving engine makes its calls.

Each turn: the sessions resume from their 8-bit images; the turn's new tokens (a tool's result, a
user's message) of all sessions go through the model packed, `prefill_attention` writing their K and V
into the slots that `batch_reserve(counts=...)` set aside; then tokens are generated by verifying a
small tree of guesses per session and step with `tree_attention`, and the K and V of the accepted ones
are appended; a pause packs what is new into the images.

The model is a small random transformer (grouped-query attention with rotary positions, no
feed-forward part) and generation is greedy; the guesses are what followed the last token earlier in
the session. `drafts=False` generates one token a step with the fused append and decode instead, and
both give the same tokens, up to ties of the logits.

    python examples/agent_turn.py [--sessions 8] [--turns 3] [--context 1500] [--tokens 64] [--plain]
"""
from __future__ import annotations

import argparse
import itertools
import os
import sys
from dataclasses import dataclass, field

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))

from paper_2609_25782_gb300 import Pool  # noqa: E402

D = 128


class Model:
    """Random weights; `forward` leaves the attention to the caller."""

    def __init__(self, layers=4, num_q_heads=16, num_kv_heads=2, hidden=512, vocab=1000, seed=0, device="cuda"):
        g = torch.Generator(device="cpu").manual_seed(seed)
        self.L, self.Hq, self.Hkv, self.vocab = layers, num_q_heads, num_kv_heads, vocab

        def weight(*shape, scale):
            return (torch.randn(*shape, generator=g) * scale).to(device, torch.bfloat16)
        heads = num_q_heads + 2 * num_kv_heads
        self.embed, self.head = weight(vocab, hidden, scale=1.0), weight(hidden, vocab, scale=1.0)
        self.wqkv = [weight(hidden, heads * D, scale=1.5 * hidden ** -0.5) for _ in range(layers)]
        self.wo = [weight(num_q_heads * D, hidden, scale=2 * (num_q_heads * D) ** -0.5) for _ in range(layers)]
        self.freq = (10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float32) / D)).to(device)

    def rotate(self, x, positions):
        """Rotary positions of x [N][heads][D], in place."""
        a = positions.float()[:, None, None] * self.freq
        x0, x1 = x.float().chunk(2, -1)
        x.copy_(torch.cat([x0 * a.cos() - x1 * a.sin(), x1 * a.cos() + x0 * a.sin()], -1))

    def forward(self, tokens, positions, attend):
        """Logits [N][vocab]; `attend(l, q, k, v, out)` runs layer l's attention of the N tokens, q, k
        and v being views of one projection."""
        x = self.embed[tokens]
        for l in range(self.L):
            y = torch.nn.functional.rms_norm(x, x.shape[-1:])
            qkv = (y @ self.wqkv[l]).view(len(tokens), -1, D)
            q, k, v = qkv.split([self.Hq, self.Hkv, self.Hkv], dim=1)
            self.rotate(qkv[:, :self.Hq + self.Hkv], positions)
            out = torch.empty(len(tokens), self.Hq, D, dtype=torch.bfloat16, device=x.device)
            attend(l, q, k, v, out)
            x = x + out.view(len(tokens), -1) @ self.wo[l]
        return torch.nn.functional.rms_norm(x, x.shape[-1:]).float() @ self.head.float()


def offsets(counts) -> list[int]:
    """Where each session's rows of a packed batch begin, and the end."""
    return [0, *itertools.accumulate(counts)]


def draft_tree(history: list[int], branches: int = 2, depth: int = 4) -> tuple[list[int], list[int]]:
    """Tokens and parents of a session's draft tree. Node 0 is the last token, which is not in the cache
    yet; a branch is what followed it at one of its latest earlier places, each first token once."""
    tokens, parents, firsts = [history[-1]], [-1], set()
    for i in range(len(history) - 2, -1, -1):
        if history[i] != history[-1] or history[i + 1] in firsts:
            continue
        firsts.add(history[i + 1])
        parent = 0
        for t in history[i + 1:i + 1 + depth]:
            tokens.append(t)
            parents.append(parent)
            parent = len(tokens) - 1
        if len(firsts) == branches:
            break
    return tokens, parents


def ancestor_masks(parents: list[int]) -> list[int]:
    """Bit j of mask i: node i sees node j, its ancestors and itself (parents come before children)."""
    masks = []
    for i, p in enumerate(parents):
        masks.append((masks[p] if p >= 0 else 0) | 1 << i)
    return masks


def accepted(tokens: list[int], parents: list[int], answers: list[int], most: int) -> list[int]:
    """The path of at most `most` nodes from node 0 along which each child is its parent's answer."""
    path = [0]
    for i in range(1, len(tokens)):
        if len(path) < most and parents[i] == path[-1] and tokens[i] == answers[path[-1]]:
            path.append(i)
    return path


@dataclass
class Session:
    sid: int
    history: list[int] = field(default_factory=list)   # the last token is not in the cache yet
    cached: int = 0
    contexts: list[int] = field(default_factory=list)  # lengths of what the turns put in
    gaps: list[float] = field(default_factory=list)    # best logit over the next one, per generated token


class Agent:
    def __init__(self, pool: Pool, model: Model, sessions: int, max_tokens: int):
        self.pool, self.model, self.dev = pool, model, pool.device
        self.max_blocks = -(-max_tokens // pool.bt)
        self.tables = torch.empty(sessions, self.max_blocks, dtype=torch.int32, device=self.dev)
        self.lens = torch.empty(sessions, dtype=torch.int32, device=self.dev)
        self.sessions = [Session(pool.session_create(max_tokens)) for _ in range(sessions)]
        self.steps = self.generated = 0

    def _ints(self, values, dtype=torch.int32):
        return torch.tensor(values, dtype=dtype, device=self.dev)

    def _answers(self, logits):
        """The greedy token of each row, and how far its logit is above the next one."""
        top = logits.topk(2, dim=-1)
        return top.indices[:, 0].tolist(), (top.values[:, 0] - top.values[:, 1]).tolist()

    def prefill(self, batch, contexts):
        """The turn's new tokens, after the one that the last turn left out of the cache."""
        new = [s.history[s.cached:] + c for s, c in zip(batch, contexts)]
        counts = [len(n) for n in new]
        B, cu, args = len(batch), offsets(counts), self._ints
        self.pool.batch_reserve([s.sid for s in batch], self.tables, self.max_blocks, self.lens, counts=counts)
        cu_dev = args(cu)

        def attend(l, q, k, v, out):
            self.pool.prefill_attention(l, q, k, v, cu_dev, self.tables, self.lens, B, self.max_blocks, D ** -0.5, out)
        positions = args([s.cached + i for s, n in zip(batch, counts) for i in range(n)])
        logits = self.model.forward(args([t for n in new for t in n], torch.int64), positions, attend)
        answers, gaps = self._answers(logits[[c - 1 for c in cu[1:]]])
        for s, n, c, t, gap in zip(batch, counts, contexts, answers, gaps):
            s.cached += n
            s.history += c + [t]
            s.contexts.append(len(c))
            s.gaps.append(gap)

    def draft_step(self, batch, left):
        """One step: a draft tree per session is verified, the accepted path appended."""
        trees = [draft_tree(s.history) for s in batch]
        B, cu, args = len(batch), offsets([len(t) for t, _ in trees]), self._ints
        self.pool.batch_tables([s.sid for s in batch], self.tables, self.max_blocks, self.lens)
        masks = [ancestor_masks(p) for _, p in trees]
        masks_dev = args([m for ms in masks for m in ms], torch.int64)
        positions = args([s.cached + m.bit_count() - 1 for s, ms in zip(batch, masks) for m in ms])
        cu_dev, ks, vs = args(cu), [], []

        def attend(l, q, k, v, out):
            self.pool.tree_attention(l, q, k, v, masks_dev, cu_dev, self.tables, self.lens, B, self.max_blocks,
                                     D ** -0.5, out)
            ks.append(k)
            vs.append(v)
        logits = self.model.forward(args([t for tokens, _ in trees for t in tokens], torch.int64), positions, attend)
        answers, gaps = self._answers(logits)
        k, v = torch.stack(ks), torch.stack(vs)
        for s, lo, hi, (tokens, parents), most in zip(batch, cu, cu[1:], trees, left):
            path = accepted(tokens, parents, answers[lo:hi], most)
            rows = args([lo + i for i in path], torch.int64)
            self.pool.session_append(s.sid, k.index_select(1, rows), v.index_select(1, rows))
            s.cached += len(path)
            s.history += [answers[lo + i] for i in path]
            s.gaps += [gaps[lo + i] for i in path]

    def plain_step(self, batch):
        """One step: a token per session."""
        B, args = len(batch), self._ints
        self.pool.batch_reserve([s.sid for s in batch], self.tables, self.max_blocks, self.lens)

        def attend(l, q, k, v, out):
            self.pool.decode_append_attention(l, q.contiguous(), k.contiguous(), v.contiguous(), self.tables,
                                              self.lens, B, self.max_blocks, D ** -0.5, out)
        logits = self.model.forward(args([s.history[-1] for s in batch], torch.int64),
                                    args([s.cached for s in batch]), attend)
        answers, gaps = self._answers(logits)
        for s, t, gap in zip(batch, answers, gaps):
            s.cached += 1
            s.history.append(t)
            s.gaps.append(gap)

    def turn(self, contexts: list[list[int]], tokens: int, drafts: bool = True):
        """A turn of all sessions: contexts[i] goes into session i, which answers with `tokens` tokens."""
        for s in self.sessions:
            if s.cached:
                self.pool.session_resume(s.sid)
        self.prefill(self.sessions, contexts)
        ends = [len(s.history) - 1 + tokens for s in self.sessions]   # the prefill gave the first one
        while batch := [(s, e - len(s.history)) for s, e in zip(self.sessions, ends) if len(s.history) < e]:
            now, left = zip(*batch)
            before = sum(len(s.history) for s in now)
            self.draft_step(now, left) if drafts else self.plain_step(now)
            self.steps += len(now)
            self.generated += sum(len(s.history) for s in now) - before
        for s in self.sessions:
            self.pool.session_pause(s.sid)
        self.pool.check_device()


def run(sessions=8, turns=3, context=1500, tokens=64, drafts=True, seed=0, vocab=1000, block_tokens=16,
        cold_int8=True):
    """Runs the turns; the returned agent has the sessions, their tokens and the pool."""
    model = Model(vocab=vocab, seed=seed)
    g = torch.Generator().manual_seed(seed + 1)
    most = turns * (2 * context + tokens)
    row_bytes = D + 1 if cold_int8 else 2 * D
    pool = Pool(num_layers=model.L, num_hot_blocks=sessions * -(-most // block_tokens),
                cold_bytes=sessions * (model.L * 2 * model.Hkv * row_bytes * most + 256), num_q_heads=model.Hq, num_kv_heads=model.Hkv, block_tokens=block_tokens, max_sessions=sessions,
                max_batch=sessions, max_context=most, cold_int8=cold_int8)
    agent = Agent(pool, model, sessions, most)
    for _ in range(turns):
        lengths = torch.randint(1, 2 * context, (sessions,), generator=g).tolist()
        agent.turn([torch.randint(0, model.vocab, (n,), generator=g).tolist() for n in lengths], tokens, drafts)
    return agent


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--sessions", type=int, default=8)
    ap.add_argument("--turns", type=int, default=3)
    ap.add_argument("--context", type=int, default=1500, help="new tokens of a turn, on average")
    ap.add_argument("--tokens", type=int, default=64, help="tokens generated per turn")
    ap.add_argument("--plain", action="store_true", help="one token a step instead of a draft tree")
    a = ap.parse_args()
    agent = run(a.sessions, a.turns, a.context, a.tokens, not a.plain)
    stats = agent.pool.stats()
    print(f"{a.sessions} sessions, {a.turns} turns: {sum(s.cached for s in agent.sessions)} tokens cached, "
          f"{agent.generated / max(1, agent.steps):.2f} tokens a session and step, "
          f"{stats['bytes_packed'] / 1e6:.1f} MB packed, {stats['bytes_unpacked'] / 1e6:.1f} MB unpacked")


if __name__ == "__main__":
    main()
