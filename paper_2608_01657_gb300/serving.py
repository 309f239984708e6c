"""A small serving loop on the prefix cache and its KV pages.

Runs the pieces together as a server would, on a stack of attention layers with
random weights: a prefix-cache step over a batch of prompts decides which blocks
are cached, the uncached tokens' keys and values go to their pages, attention
reads cached and new pages alike (a shared prefix once for all its requests),
every request is forked into samples that share its pages, the samples decode
some tokens, losers are freed and the pool is compacted.

    python -m paper_2608_01657_gb300.serving
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import List, Sequence

import numpy as np
import torch

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
                groups: Sequence[int], write=None) -> torch.Tensor:
        """Hidden states of ``counts[i]`` new tokens of each row, from position ``start[i]`` on.

        ``groups``: first rows of the runs that may share a prefix, and the number of rows."""
        s, w = self.s, self.layers
        n = torch.tensor(counts, device="cuda")
        offsets = torch.zeros(len(counts) + 1, dtype=torch.int64, device="cuda")
        offsets[1:] = n.cumsum(0)
        of = torch.repeat_interleave(torch.arange(len(counts), device="cuda"), n)
        pos = (start.long()[of] + torch.arange(len(of), device="cuda") - offsets[of])
        tables = self.tables[rows.long()].contiguous()
        slots = tables.long()[of, pos // s.page] * s.page + pos % s.page
        if write is not None:
            slots = torch.where(write, slots, -1)
        pos = pos.int()
        self.pool.plan(offsets.int(), (start.long() + n).int(), tables, len(of),
                       group_offsets=torch.tensor(groups, dtype=torch.int32, device="cuda"))
        x = w.embed[tokens.long()]
        a, b = s.q_heads * s.head_dim, (s.q_heads + s.kv_heads) * s.head_dim
        for layer in range(s.layers):
            qkv = x @ w.qkv[layer].T
            q, k, v = (t.unflatten(1, (-1, s.head_dim)) for t in (qkv[:, :a], qkv[:, a:b], qkv[:, b:]))
            q = self.pool.append(layer, q, k, v, slots, positions=pos, rope=w.rope, q_weight=w.q_norm[layer],
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
        write = torch.cat([torch.full((c,), int(h) <= a, device="cuda") for c, h, a in zip(counts, hits.tolist(), host)])
        bounds = [0] + [i for i in range(1, R) if groups[i] != groups[i - 1]] + [R]
        x = self.forward(rows, start, new, counts, bounds, write)
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
        bounds = list(range(0, n + 1, samples))  # a request's samples share its pages
        out = []
        for t in range(T):
            start = self.lens[children.long()]
            out.append(self.forward(children, start, torch.from_numpy(steps[t].reshape(-1)).cuda(), [1] * n, bounds))
            self.lens[children.long()] += 1
        return torch.stack(out)

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


if __name__ == "__main__":
    main()
