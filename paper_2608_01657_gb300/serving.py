"""A small serving loop on the prefix cache and its KV pages.

Runs the pieces together as a server would, on a stack of attention layers with
random weights: a prefix-cache step over a batch of prompts decides which blocks
are cached, the uncached tokens' keys and values go to their pages, attention
reads cached and new pages alike (a shared prefix once for all its requests),
every request is forked into samples that share its pages, the samples decode
some tokens, losers are freed and the pool is compacted; or its beams search for
likely answers, their pages following the beams that they continue.

    python -m paper_2608_01657_gb300.serving
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import List, Optional, Sequence

import numpy as np
import torch

from . import beam
from . import binding as B
from . import kv


@dataclass
class Shape:
    layers: int = 2
    q_heads: int = 8
    kv_heads: int = 2
    head_dim: int = 64
    hidden: int = 256
    vocab: int = 1000
    page: int = 16
    cache_blocks: int = 64      # the prefix cache's pages
    private_pages: int = 128    # pages of running requests
    max_requests: int = 32
    max_tokens: int = 4096
    max_len: int = 512


class Layers:
    """Attention layers with random weights, in bfloat16."""

    def __init__(self, s: Shape, seed: int):
        g = torch.Generator("cuda").manual_seed(seed)
        def mat(*n): return (torch.randn(*n, generator=g, device="cuda") / n[-1] ** 0.5).bfloat16()  # noqa: E704
        width = (s.q_heads + 2 * s.kv_heads) * s.head_dim
        self.embed = mat(s.vocab, s.hidden) * 16
        self.qkv = [mat(width, s.hidden) for _ in range(s.layers)]
        self.out = [mat(s.hidden, s.q_heads * s.head_dim) for _ in range(s.layers)]
        self.q_norm = [torch.ones(s.head_dim, device="cuda").bfloat16() for _ in range(s.layers)]
        self.k_norm = [torch.ones(s.head_dim, device="cuda").bfloat16() for _ in range(s.layers)]
        inv = 10000.0 ** (-torch.arange(0, s.head_dim, 2, device="cuda", dtype=torch.float64) / s.head_dim)
        a = torch.arange(s.max_len, device="cuda", dtype=torch.float64)[:, None] * inv
        self.rope = torch.cat([a.cos(), a.sin()], 1).float()


class Server:
    """One prefix cache, one KV pool and the rows of the running requests."""

    def __init__(self, s: Shape, groups: int, seed: int = 0):
        self.s, self.layers = s, Layers(s, seed)
        self.cache = B.Cache(s.cache_blocks, s.page, groups, "prefixshield", B.Params(rho=(64.0,), beta=(256.0,)),
                             max_requests=s.max_requests, max_tokens=s.max_tokens)
        pages = s.cache_blocks + s.private_pages
        self.k, self.v = (torch.zeros(s.layers, pages, s.page, s.kv_heads, s.head_dim, device="cuda").bfloat16() for _ in range(2))
        width = -(-s.max_len // s.page)
        self.pool = kv.KVPool(self.k, self.v, num_q_heads=s.q_heads, first_page=s.cache_blocks, max_requests=s.max_requests,
                              max_tokens=s.max_tokens, max_row_pages=width)
        i32 = dict(dtype=torch.int32, device="cuda")
        self.tables = torch.zeros(s.max_requests, width, **i32)
        self.lens, self.held = torch.zeros(s.max_requests, **i32), torch.zeros(s.max_requests, **i32)
        self.refs = torch.zeros(s.private_pages, **i32)
        self.running = set()  # rows that hold pages
        self.tick = 0

    # -- one pass over all layers ------------------------------------------------
    def forward(self, rows: torch.Tensor, start: torch.Tensor, tokens: torch.Tensor, counts: Sequence[int],
                groups: Optional[Sequence[int]] = None, write: Optional[torch.Tensor] = None,
                written: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Hidden states of ``counts[i]`` new tokens of each row, from position ``start[i]`` on.

        ``groups``: first rows of the runs that may share a prefix, and the number of rows (None: those
        that their pages show).  Keys and values are written but for tokens where ``write`` [tokens] is False,
        and for those below ``written`` [rows], how many of a row's tokens have theirs."""
        s, w = self.s, self.layers
        T = int(sum(counts))
        at = self.pool.layout(rows.int().contiguous(), self.tables, self.lens, self.held, T,
                              counts=torch.tensor(counts, dtype=torch.int32, device="cuda"), starts=start.int().contiguous(), written=written)
        slots = at.slots if write is None else torch.where(write, at.slots, -1)
        bounds = at.group_offsets if groups is None else torch.tensor(groups, dtype=torch.int32, device="cuda")
        self.pool.plan(at.q_offsets, at.kv_lens, at.tables, T, group_offsets=bounds)
        x = w.embed[tokens.long()]
        a, b = s.q_heads * s.head_dim, (s.q_heads + s.kv_heads) * s.head_dim
        for layer in range(s.layers):
            qkv = x @ w.qkv[layer].T
            q, k, v = (t.unflatten(1, (-1, s.head_dim)) for t in (qkv[:, :a], qkv[:, a:b], qkv[:, b:]))
            q = self.pool.append(layer, q, k, v, slots, positions=at.positions, rope=w.rope, q_weight=w.q_norm[layer],
                                 k_weight=w.k_norm[layer])
            o = self.pool.attention(layer, q, s.head_dim ** -0.5)
            x = x + o.flatten(1) @ w.out[layer].T
        self.pool.check()
        return x

    # -- prompts -------------------------------------------------------------------
    def admit(self, groups: Sequence[int], prompts: List[np.ndarray], room: int) -> dict:
        """Rows 0.. for a batch of prompts, with room for ``room`` more tokens each.

        Returns the hidden state of each prompt's last token and how many tokens were cached.
        No row may be running: nothing holds the cached pages of a running row, so that a
        step could evict them and give them to a prompt of the new batch."""
        s, R = self.s, len(prompts)
        if self.running:
            raise RuntimeError(f"rows {sorted(self.running)} are running: finish them before the next batch")
        lens = [len(p) for p in prompts]
        flat = torch.from_numpy(np.concatenate(prompts).astype(np.int32)).cuda()
        offs = np.concatenate([[0], np.cumsum(lens)])
        g = torch.tensor(groups, dtype=torch.int32, device="cuda")
        self.tick += 1
        rc = self.cache.step(self.tick, g, torch.from_numpy(offs).cuda(), flat)
        if rc != B.PS_OK:
            raise RuntimeError(f"the step was refused ({rc})")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        blocks = self.cache.step_blocks(g, self.tables, status=status)[:R]
        if int(status):
            raise RuntimeError(f"the step failed ({int(status)})")
        self.running = set(range(R))
        # the cache's blocks first, then private pages for the rest of the prompt and the answer
        self.held[:R], self.lens[:R] = blocks, blocks * s.page
        rows = torch.arange(R, dtype=torch.int32, device="cuda")
        total = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.pool.fork(rows, rows, total + room, self.tables, self.lens, self.held, self.refs)
        self.lens[:R] = total
        hits = torch.minimum(self.cache.out["hit_blocks"][:R], blocks) * s.page
        start = torch.minimum(hits, total - 1)                       # at least the last token is computed
        host = start.tolist()
        counts = [n - a for n, a in zip(lens, host)]
        new = torch.cat([flat[offs[i] + host[i]:offs[i + 1]] for i in range(R)])
        # a fully cached prompt's last token has its keys and values already
        x = self.forward(rows, start, new, counts, written=hits.int())
        last = torch.tensor(np.cumsum(counts) - 1, device="cuda")
        return {"hidden": x[last], "cached": int(hits.sum())}

    # -- samples -------------------------------------------------------------------
    def sample(self, requests: int, samples: int, steps: np.ndarray) -> torch.Tensor:
        """Forks every request into ``samples`` rows and decodes steps[t, request, sample] on them.

        Returns the hidden states [t, request * samples, hidden]; the sampled rows stay."""
        n, T = requests * samples, steps.shape[0]
        rows = range(requests, requests + n)
        if self.running.intersection(rows):
            raise RuntimeError("the samples' rows are running: finish them first")
        dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
        parents = dev(np.repeat(np.arange(requests), samples))
        children = dev(np.asarray(rows))
        self.running.update(rows)
        self.pool.fork(parents, children, self.lens[parents.long()] + T, self.tables, self.lens, self.held, self.refs)
        out = []
        for t in range(T):
            start = self.lens[children.long()]
            out.append(self.forward(children, start, torch.from_numpy(steps[t].reshape(-1)).cuda(), [1] * n))
            self.lens[children.long()] += 1
        return torch.stack(out)

    # -- beams -----------------------------------------------------------------------
    def beam_search(self, hidden: torch.Tensor, beams: int, steps: int, end: Sequence[int] = ()) -> dict:
        """Likely answers of up to ``steps`` tokens to the admitted prompts.

        ``hidden``: the states that ``admit`` gave.  Returns the ``beams`` answers of each request with the
        highest mean log-probability a token: ``sequences`` [requests, beams, steps] (-1 past their ends),
        their ``lengths`` and ``scores`` (sums of log-probabilities, an end token's among them; -infinity
        where there are fewer).  The beams' rows, len(hidden) .. len(hidden) * (beams + 1), stay."""
        s, R = self.s, hidden.shape[0]
        n = R * beams
        names = range(R, R + n)
        if R + n > s.max_requests:
            raise ValueError(f"prompts and beams need {R + n} rows of {s.max_requests}")
        if steps < 1:
            raise ValueError("there must be a step")
        if beams > s.vocab - len(end):
            raise ValueError("there must be as many tokens that end nothing as beams")
        if self.running.intersection(names):
            raise RuntimeError("the beams' rows are running: finish them first")
        search = beam.BeamSearch(R, beams, s.vocab, torch.bfloat16, end)
        i32 = dict(dtype=torch.int32, device="cuda")
        children = torch.tensor(list(names), **i32)
        rows = children.view(R, beams)
        parents = torch.arange(R, **i32).repeat_interleave(beams)
        self.running.update(names)
        self.pool.fork(parents, children, self.lens[parents.long()] + 1, self.tables, self.lens, self.held, self.refs)
        whole = lambda dtype: torch.empty(steps, R, beams, dtype=dtype, device="cuda")  # noqa: E731
        all_ = beam.Selection(*(whole(t) for t in (torch.int32, torch.int32, torch.float32) * 2))
        # a prompt has one beam at first
        scores = torch.full((R, beams), -torch.inf, device="cuda")
        scores[:, 0] = 0
        logits = (hidden @ self.layers.embed.T)[:, None].expand(R, beams, s.vocab)
        for t in range(steps):
            at = search.select(logits, scores, out=beam.Selection(*(x[t] for x in all_)))
            scores = at.scores
            if t + 1 == steps:
                break
            if t > 0:  # (after the first step all rows are alike)
                self.pool.reorder(rows, at.parents, self.tables, self.lens, self.held, self.refs, grow=1)
            x = self.forward(children, self.lens[children.long()], at.tokens.view(-1), [1] * n)
            self.lens[children.long()] += 1
            logits = (x @ self.layers.embed.T).view(R, beams, s.vocab)
        self.pool.check()
        search.check()
        # the beams of the last step, and those that ended on the way: at step t with parent p, in p's row of step t - 1
        step = torch.arange(steps, device="cuda")[:, None, None].expand(steps, R, beams)
        score = torch.cat([all_.scores[-1:], all_.ended_scores]).movedim(0, 1).flatten(1)
        last = torch.cat([torch.arange(beams, **i32).expand(1, R, beams), all_.ended_parents]).movedim(0, 1).flatten(1)
        length = torch.cat([torch.full((1, R, beams), steps, device="cuda"), step]).movedim(0, 1).flatten(1)
        tokens = torch.cat([length[:, :beams], length[:, beams:] + 1], 1)  # with the end token
        best = (score / tokens).topk(beams, 1).indices
        score, last, length = (x.gather(1, best) for x in (score, last, length))
        last = torch.where(torch.isinf(score), -1, last).int().contiguous()
        sequences = search.trace(all_.tokens, all_.parents, last, lengths=length.int().contiguous())
        search.check()
        return {"sequences": sequences, "lengths": length, "scores": score}

    def finish(self, rows: Sequence[int]):
        """Frees rows and moves the pages in use together; returns (in use, moved)."""
        self.pool.release(torch.tensor(rows, dtype=torch.int32, device="cuda"), self.tables, self.lens, self.held, self.refs)
        self.running.difference_update(rows)
        counts = self.pool.compact(self.tables, self.held, self.refs)
        self.pool.check()
        return tuple(counts.tolist())


def prompts_of(groups: Sequence[int], shape: Shape, seed: int) -> List[np.ndarray]:
    """A system prompt for each group and a question of its own for each request."""
    r = np.random.RandomState(seed)
    system = {g: r.randint(0, shape.vocab, 128 + 16 * g) for g in sorted(set(groups))}
    return [np.concatenate([system[g], r.randint(0, shape.vocab, r.randint(1, 40))]) for g in groups]


def main():
    s = Shape()
    server = Server(s, groups=2)
    groups = [0, 0, 0, 1, 1]
    first = server.admit(groups, prompts_of(groups, s, 1), room=0)
    print("first batch: cached tokens", first["cached"])
    server.finish(range(len(groups)))
    again = server.admit(groups, prompts_of(groups, s, 1), room=0)
    print("the same prompts again: cached tokens", again["cached"])
    print("largest change of the last hidden states", float((again["hidden"] - first["hidden"]).abs().max()))
    steps = np.random.RandomState(2).randint(0, s.vocab, (4, len(groups), 3)).astype(np.int32)
    out = server.sample(len(groups), 3, steps)
    print("sampled hidden states", tuple(out.shape))
    print("after freeing every second sample: pages in use, moved", server.finish(range(len(groups), len(groups) * 4, 2)))
    server.finish(list(range(len(groups))) + list(range(len(groups) + 1, len(groups) * 4, 2)))
    third = server.admit(groups, prompts_of(groups, s, 2), room=0)
    found = server.beam_search(third["hidden"], beams=4, steps=6, end=[7])
    print("likeliest answers", found["sequences"][:, 0].tolist())
    tokens = found["lengths"][:, 0] + (found["lengths"][:, 0] < 6)  # with the end's
    print("their mean log-probabilities", [round(float(x), 3) for x in found["scores"][:, 0] / tokens])


if __name__ == "__main__":
    main()
