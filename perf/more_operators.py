"""Measured cases of the operators between two attention steps on KV pages.

Four operators, as a decoding loop with beam search calls them in turn:

- layout: where the new tokens of a batch of requests go (offsets, lengths,
  page tables, positions, slots, groups), from the requests' rows and counts;
- select: the best continuations of a request's beams over beams and vocabulary;
- reorder: the beams' pages follow the beams that they continue;
- trace: the sequences of tokens, back through the parents of every step.

``own`` chooses between the framework's calls and a plain form in elementary
torch operations.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}

# Neighbouring requests form a group, whose common prefix attention reads once, where
# the tokens before their new ones have so many in common and none has more query rows.
SHARE_TOKENS, SHARE_ROWS = 128, 64


# ---------------------------------------------------------------------------
# the cases
def listed():
    return [
        # one token for each of a server's running requests: the smallest batch layout, latency counts
        dict(name="layout-decode", kind="layout", requests=256, new=1, most=4096, width=256, page=16, ratio=4, spare=0,
             shape=1),
        # the uncached tokens of a batch of prompts; some prompts are cached whole
        dict(name="layout-prompts", kind="layout", requests=64, new=2048, most=4096, width=400, page=16, ratio=4, spare=0,
             shape=2),
        # drafted tokens of a ragged batch, padded to a fixed number of tokens, as a captured graph wants it
        dict(name="layout-drafts-odd", kind="layout", requests=333, new=7, most=1500, width=201, page=8, ratio=3, spare=99,
             shape=3),
        # one sequence's likeliest token, a small vocabulary: the smallest selection
        dict(name="select-greedy", kind="select", requests=1, beams=1, vocab=1000, end=0, dtype="bf16", spread=2.0,
             masked=0.0, absent=0.0),
        # a few requests' beams
        dict(name="select-few", kind="select", requests=8, beams=4, vocab=65536, end=1, dtype="bf16", spread=3.0,
             masked=0.0, absent=0.0),
        # a batch of beam searches over a large vocabulary: the largest case, bound by reading the logits
        dict(name="select-batch", kind="select", requests=128, beams=8, vocab=131072, end=1, dtype="bf16", spread=3.0,
             masked=0.0, absent=0.0),
        # logits in 32 bits, an odd vocabulary of which a grammar allows a part, beams that have ended
        dict(name="select-odd-f32", kind="select", requests=37, beams=5, vocab=50001, end=2, dtype="f32", spread=2.5,
             masked=0.6, absent=0.15),
        # one request's four beams
        dict(name="reorder-one", kind="reorder", requests=1, beams=4, tokens=1000, layers=4, kv_heads=4, dim=64, page=16,
             cached=512, dead=0.0, dtype="bf16"),
        # a batch of eight beams each over 2048 tokens
        dict(name="reorder-batch", kind="reorder", requests=64, beams=8, tokens=2048, layers=8, kv_heads=4, dim=64,
             page=16, cached=4096, dead=0.0, dtype="bf16"),
        # odd heads and beams, small pages, beams that ended
        dict(name="reorder-odd-f16", kind="reorder", requests=33, beams=5, tokens=701, layers=3, kv_heads=3, dim=80,
             page=8, cached=100, dead=0.2, dtype="f16"),
        # a short answer's beams
        dict(name="trace-short", kind="trace", requests=4, beams=4, steps=64, hyps=4, ragged=False),
        # a batch of long answers, with the hypotheses that ended on the way
        dict(name="trace-long", kind="trace", requests=128, beams=8, steps=2047, hyps=13, ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {k: max(c["work"][k] for c in _LISTED_WORK) for k in ("bytes", "flops")}
    while True:
        kind = rng.choice(["layout", "select", "select", "reorder", "trace"])
        if kind == "layout":
            page = rng.choice([8, 16, 16, 32, 64])
            before, new = _log(rng, 1, 20000), rng.choice([1, 1, rng.randint(2, 9), _log(rng, 10, 4000)])
            c = dict(kind=kind, requests=_log(rng, 1, 3000), new=new, most=before,
                     width=-(-(before + new) // page) + rng.randint(0, 50), page=page, ratio=rng.choice([1, 2, 3, 4, 8]),
                     spare=rng.choice([0, 0, rng.randint(1, 500)]), shape=rng.randint(10, 10**6))
            if c["requests"] * max(c["new"], c["width"]) > 4e6:
                continue
        elif kind == "select":
            c = dict(kind=kind, requests=_log(rng, 1, 400), beams=rng.choice([1, 2, 3, 4, 5, 8, 12, 16, 32]),
                     vocab=_log(rng, 100, 260000), end=rng.choice([0, 1, 1, 2, 5]), dtype=rng.choice(["bf16", "bf16", "f16", "f32"]),
                     spread=rng.choice([1.0, 2.0, 3.0, 4.0]), masked=rng.choice([0.0, 0.0, 0.5, 0.99]),
                     absent=rng.choice([0.0, 0.0, 0.2]))
        elif kind == "reorder":
            c = dict(kind=kind, requests=_log(rng, 1, 150), beams=rng.choice([1, 2, 3, 4, 5, 8, 16]), tokens=_log(rng, 8, 8192),
                     layers=rng.randint(1, 9), kv_heads=rng.choice([1, 2, 4, 5, 8]), dim=rng.choice([64, 80, 96, 128]),
                     page=rng.choice([8, 16, 16, 32, 64]), cached=_log(rng, 1, 5000), dead=rng.choice([0.0, 0.0, 0.1]),
                     dtype=rng.choice(["bf16", "f16"]))
            if 4 * c["layers"] * _num_pages(c) * c["page"] * c["kv_heads"] * c["dim"] > 8e9:
                continue
        else:
            beams = rng.choice([1, 2, 3, 4, 5, 8, 16, 32])
            c = dict(kind=kind, requests=_log(rng, 1, 300), beams=beams, steps=_log(rng, 1, 4000),
                     hyps=rng.choice([1, beams, 2 * beams + 1]), ragged=rng.random() < 0.6)
            if c["requests"] * c["steps"] * max(c["beams"], c["hyps"]) > 6e6:
                continue
        w = work(c)
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"]:
            return c


# ---------------------------------------------------------------------------
# what a pass cannot do without
def work(c):
    if c["kind"] == "layout":
        start, new, _ = _lengths(c)
        pages = int((-(-(start + new) // c["page"])).sum())
        tokens, n = int(new.sum()) + c["spare"], c["requests"]
        # rows, lengths, counts and held ids in; offsets, lengths, the whole tables, groups, positions and slots out
        return {"bytes": 4 * (4 * n + pages) + 4 * (3 * n + n * c["width"]) + 12 * tokens, "flops": 4 * tokens}
    if c["kind"] == "select":
        n = c["requests"] * c["beams"] * c["vocab"]
        # logits once; scale, exponential, sum and comparison of each
        return {"bytes": n * (4 if c["dtype"] == "f32" else 2) + 28 * c["requests"] * c["beams"], "flops": 4 * n}
    if c["kind"] == "reorder":
        s = _page_state(c, 0)
        children = _children(s["parents"])
        part = s["lens"] % c["page"]
        copied = int((part * np.maximum(children - 1, 0)).sum()) * 4 * c["layers"] * c["kv_heads"] * c["dim"]
        held = int(s["held"].sum())
        # every id read, those of the rows that continue another one written, the references of a row without
        # or with several children changed, the partly filled pages copied
        moved = int(s["held"][(s["parents"] != np.arange(c["beams"])) & (s["parents"] >= 0)].sum())
        return {"bytes": 2 * copied + 4 * held + 4 * moved + 8 * int(s["held"][children != 1].sum()) + 20 * s["held"].size,
                "flops": 0}
    n = c["requests"] * c["steps"]
    return {"bytes": 8 * n * c["beams"] + 4 * n * c["hyps"], "flops": n * c["hyps"]}


# ---------------------------------------------------------------------------
# the inputs
def _dev(a, dtype=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(device="cuda", dtype=dtype)


def _lengths(c):
    """Tokens before the new ones, new ones, and tokens whose keys and values are there, of each request."""
    r = np.random.RandomState(c["shape"])
    n = c["requests"]
    before = r.randint(0, c["most"] + 1, n)
    if c["new"] == 1:  # a token each
        return before, np.ones(n, np.int64), before
    if c["new"] < 10:  # drafted tokens, some requests pause
        return before, r.randint(0, c["new"] + 1, n), before
    new = r.randint(1, c["new"] + 1, n)  # prompts after what was cached of them, in whole pages
    before = before // c["page"] * c["page"]
    written = before.copy()
    whole = (r.rand(n) < 0.1) & (before > 0)  # cached whole: the last token is computed again, and not written
    before[whole] -= 1
    new[whole] = 1
    return before, new, written


def _layout_inputs(c, seed):
    r = np.random.RandomState(seed % (1 << 31))
    start, new, written = _lengths(c)
    n, ps, width = c["requests"], c["page"], c["width"]
    rows = r.permutation(n + 3)[:n]
    held = np.zeros(n + 3, np.int64)
    held[rows] = np.minimum(-(-(start + new) // ps) + r.randint(0, 3, n), width)
    lens = np.zeros(n + 3, np.int64)
    lens[rows] = start
    pages = int(held.sum()) + 10
    tables = r.randint(0, pages, (n + 3, width))
    for i in range(1, n):  # conversations of a tenant begin with its system prompt
        if r.rand() < 0.8:
            k = min(SHARE_TOKENS // ps + r.randint(0, 20), width)
            tables[rows[i], :k] = tables[rows[i - 1], :k]
    decode = c["new"] < 10
    return dict(case=c, rows=_dev(rows), tables=_dev(tables), lens=_dev(lens), held=_dev(held), pages=pages,
                counts=None if c["new"] == 1 else _dev(new), starts=None if decode else _dev(start),
                written=None if decode else _dev(written), num_tokens=int(new.sum()) + c["spare"])


def _normal(g, *shape, dtype, spread=1.0):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).mul_(spread).to(dtype)


def _end_tokens(c):
    return [(2 + 7 * i) % c["vocab"] for i in range(c["end"])]


def _select_inputs(c, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    R, B, V = c["requests"], c["beams"], c["vocab"]
    logits = _normal(g, R, B, V, dtype=DTYPES[c["dtype"]], spread=c["spread"])
    if c["masked"]:  # tokens that a grammar forbids, others for each beam; here and there all of them
        for b in range(B):
            logits[:, b].masked_fill_(torch.rand(R, V, generator=g, device="cuda") < c["masked"], -math.inf)
        logits[torch.rand(R, B, generator=g, device="cuda") < 0.05] = -math.inf
    # an end token is as likely as the best others
    for e in _end_tokens(c):
        logits[:, :, e] += 4 * c["spread"]
    scores = -20 * torch.rand(R, 1, generator=g, device="cuda") - 5 * torch.rand(R, B, generator=g, device="cuda")
    if c["absent"]:
        scores[torch.rand(R, B, generator=g, device="cuda") < c["absent"]] = -math.inf
    return dict(case=c, logits=logits, scores=scores, end_tokens=_end_tokens(c))


def _num_pages(c):
    each = -(-c["tokens"] // c["page"]) + 2
    return c["cached"] + c["requests"] * (c["beams"] + 2) * each


def _children(parents):
    """How many beams of its request continue each beam."""
    R, B = parents.shape
    return (parents[:, None, :] == np.arange(B)[None, :, None]).sum(-1)


def _page_state(c, seed):
    """Rows of beam searches under way: a request's beams share their prompt's pages, pairs of them some more."""
    r = np.random.RandomState(2000 + seed % (1 << 31))
    R, B, ps, first = c["requests"], c["beams"], c["page"], c["cached"]
    width = -(-c["tokens"] // ps) + 3
    lens = np.repeat(r.randint(1, c["tokens"] + 1, R)[:, None], B, 1)
    held = -(-lens // ps)
    full = lens // ps
    shared = np.minimum((full * r.uniform(0.3, 1, R)[:, None]).astype(np.int64), full)  # by all beams
    paired = np.minimum(shared + r.randint(0, 8, (R, 1)), full)                          # by beams 2 j and 2 j + 1
    cached = np.minimum(r.randint(0, 9, (R, 1)), shared)
    col = np.arange(width)
    perm = r.permutation(_num_pages(c) - first)
    ids = (np.arange(R * B).reshape(R, B, 1) * width + col)   # a number of each place, taken over from the beam that it is shared with
    pair, lead = ids[:, (np.arange(B) // 2 * 2)], ids[:, :1]
    ids = np.where(col < shared[..., None], lead, np.where(col < paired[..., None], pair, ids))
    live = (col < held[..., None]) & (col >= cached[..., None])
    names, back = np.unique(ids[live], return_inverse=True)
    tables = np.full((R, B, width), -1, np.int64)
    tables[live] = first + perm[back]
    blocks = r.randint(0, first, (R, 1, width))
    tables = np.where(col < cached[..., None], blocks, tables)
    refs = np.bincount(tables[tables >= first] - first, minlength=_num_pages(c) - first)
    parents = np.sort(r.randint(0, B, (R, B)), 1)
    parents = np.where(r.rand(R, 1) < 0.2, np.take_along_axis(parents, r.rand(R, B).argsort(1), 1), parents)
    parents = np.where(r.rand(R, 1) < 0.1, np.arange(B), parents)   # every beam goes on
    parents = np.where(r.rand(R, B) < c["dead"], -1, parents)
    return dict(tables=tables.reshape(R * B, width), lens=lens, held=held, refs=refs, parents=parents)


def _reorder_inputs(c, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    R, B = c["requests"], c["beams"]
    s = {k: _dev(a) for k, a in _page_state(c, seed).items()}
    shape = (c["layers"], _num_pages(c), c["page"], c["kv_heads"], c["dim"])
    k, v = (_normal(g, *shape, dtype=DTYPES[c["dtype"]]) for _ in range(2))
    rows = torch.arange(R * B, dtype=torch.int32, device="cuda").view(R, B)
    return dict(s, case=c, k=k, v=v, rows=rows, lens=s["lens"].view(-1), held=s["held"].view(-1))


def _trace_inputs(c, seed):
    r = np.random.RandomState(seed % (1 << 31))
    T, R, B, N = c["steps"], c["requests"], c["beams"], c["hyps"]
    parents = np.sort(r.randint(0, B, (T, R, B)).astype(np.int32), -1)
    beams = r.randint(0, B, (R, N))
    lengths = None
    if c["ragged"]:
        lengths = _dev(r.randint(0, T + 1, (R, N)))
        beams[r.rand(R, N) < 0.1] = -1
    return dict(case=c, tokens=_dev(r.randint(0, 131072, (T, R, B)).astype(np.int32)), parents=_dev(parents),
                beams=_dev(beams), lengths=lengths)


def _inputs(c, seed):
    return {"layout": _layout_inputs, "select": _select_inputs, "reorder": _reorder_inputs, "trace": _trace_inputs}[c["kind"]](c, seed)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:  # the handles that a serving program keeps
        from paper_2608_01657_gb300 import beam, kv
        c = case
        if c["kind"] == "layout":
            k = torch.zeros(1, s["pages"], c["page"], 1, 8, device="cuda", dtype=torch.bfloat16)
            s["pool"] = kv.KVPool(k, torch.zeros_like(k), num_q_heads=c["ratio"], max_requests=c["requests"] + 1,
                                  max_tokens=max(1, s["num_tokens"]), max_row_pages=c["width"])
        elif c["kind"] == "reorder":
            s["pool"] = kv.KVPool(s["k"], s["v"], num_q_heads=c["kv_heads"], first_page=c["cached"],
                                  max_requests=c["requests"] * c["beams"], max_row_pages=s["tables"].shape[1])
        else:
            s["search"] = beam.BeamSearch(max_requests=c["requests"], beams=c["beams"], vocab=c.get("vocab", 131072),
                                          dtype=DTYPES[c.get("dtype", "bf16")], end_tokens=s.get("end_tokens", ()))
    return s


# ---------------------------------------------------------------------------
# one pass
def run(s):
    return {"layout": _layout, "select": _select, "reorder": _reorder, "trace": _trace}[s["case"]["kind"]](s)


def _layout(s):
    c = s["case"]
    if own:
        s["out"] = s["pool"].layout(s["rows"], s["tables"], s["lens"], s["held"], s["num_tokens"], counts=s["counts"],
                                    starts=s["starts"], written=s["written"], pad=c["spare"] > 0, out=s.get("out"))
        o = s["out"]
        return {"q_offsets": o.q_offsets, "kv_lens": o.kv_lens, "tables": o.tables, "positions": o.positions,
                "slots": o.slots, "group_offsets": o.group_offsets}
    return _layout_plain(s)


def _layout_plain(s):
    c, ps, T = s["case"], s["case"]["page"], s["num_tokens"]
    n, rows, dev = c["requests"], s["rows"].long(), "cuda"
    start = (s["lens"][rows] if s["starts"] is None else s["starts"]).long()
    new = torch.ones(n, dtype=torch.int64, device=dev) if s["counts"] is None else s["counts"].long()
    written = start if s["written"] is None else s["written"].long()
    kv = start + new
    off = torch.cat([torch.zeros(1, dtype=torch.int64, device=dev), new.cumsum(0)])
    t = torch.arange(T, device=dev)
    req = torch.searchsorted(off[1:], t, right=True)
    live = req < n
    req = req.clamp(max=n - 1)
    pos = torch.where(live, start[req] + t - off[req], 0)
    slot = s["tables"][rows[req], pos // ps].long() * ps + pos % ps
    slot = torch.where(live & (pos >= written[req]), slot, -1)
    col = torch.arange(c["width"], device=dev)
    tables = torch.where(col < ((kv + ps - 1) // ps)[:, None], s["tables"][rows], -1)
    lead = -(-SHARE_TOKENS // ps)
    fit = (start >= SHARE_TOKENS) & (new * c["ratio"] <= SHARE_ROWS)
    same = (tables[1:, :lead] == tables[:-1, :lead]).all(1) & fit[1:] & fit[:-1]
    begins = torch.cat([torch.ones(1, dtype=torch.bool, device=dev), ~same])
    if c["spare"]:  # the padding is a request without keys, in a group of its own
        off, kv = torch.cat([off, off.new_full((1,), T)]), torch.cat([kv, kv.new_zeros(1)])
        tables = torch.cat([tables, tables.new_full((1, c["width"]), -1)])
        begins = torch.cat([begins, begins.new_ones(1)])
        n += 1
    i = torch.arange(n, device=dev)
    groups = torch.full((n + 1,), n, dtype=torch.int64, device=dev)
    groups.scatter_reduce_(0, begins.long().cumsum(0) - 1, i, "amin")
    return {"q_offsets": off.int(), "kv_lens": kv.int(), "tables": tables, "positions": pos.int(), "slots": slot,
            "group_offsets": groups.int()}


def _select(s):
    if own:
        s["out"] = s["search"].select(s["logits"], s["scores"], out=s.get("out"))
        o = s["out"]
        return {"tokens": o.tokens, "parents": o.parents, "scores": o.scores, "ended_tokens": o.ended_tokens,
                "ended_parents": o.ended_parents, "ended_scores": o.ended_scores}
    return _select_plain(s)


def _order(score, *ties):
    """Places in order of falling score, equal ones in order of the ties, the first tie deciding first."""
    at = torch.arange(score.shape[-1], device=score.device).expand(score.shape)
    for t in ties[::-1]:
        at = at.gather(-1, t.gather(-1, at).sort(dim=-1, stable=True).indices)
    return at.gather(-1, score.gather(-1, at).sort(dim=-1, descending=True, stable=True).indices)


def _select_plain(s):
    c, end = s["case"], s["end_tokens"]
    R, B, V, E = c["requests"], c["beams"], c["vocab"], len(end)
    x, before = s["logits"].float() + 0.0, s["scores"]  # (-0 and 0 are equal)
    # sums and scores in 64 bits: neighbours in the order may be nearer than 32 bits tell
    top = x.amax(-1).clamp(min=-3e38)
    lse = (x - top[..., None]).double().exp_().sum(-1).log() + top
    base = torch.where(lse == -math.inf, -math.inf, before.double() - lse)
    # each beam's best tokens that end nothing, equal ones by token: value and token make one whole number
    bits = x.view(torch.int32)
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * (1 << 32) + (V - 1 - torch.arange(V, device="cuda"))
    if E:
        key[..., end] = -(1 << 63)
    K = min(B, V - E)
    token = V - 1 - (key.topk(K, -1).values & 0xFFFFFFFF)
    score = x.gather(-1, token).double() + base[..., None]
    beam = torch.arange(B, device="cuda")[:, None]
    flat = score.flatten(1)
    at = _order(flat)[:, :B]
    out = {"scores": flat.gather(1, at), "parents": beam.expand(R, B, K).flatten(1).gather(1, at), "tokens": token.flatten(1).gather(1, at)}
    # all candidates in order: an end token among the first B ends its beam
    last = torch.tensor(end, dtype=torch.int64, device="cuda").expand(R, B, E)
    score = torch.cat([score, x.gather(-1, last).double() + base[..., None]], -1).flatten(1)
    token = torch.cat([token, last], -1).flatten(1)
    beam = beam.expand(R, B, K + E).flatten(1)
    at = _order(score, beam, token)[:, :B]
    ends = (torch.arange(K + E, device="cuda") >= K).expand(R, B, K + E).flatten(1).gather(1, at)
    ended = torch.where(ends, score.gather(1, at), -math.inf)
    to = torch.argsort((ended == -math.inf).int(), dim=1, stable=True)
    out |= {"ended_scores": ended.gather(1, to), "ended_parents": beam.gather(1, at).gather(1, to), "ended_tokens": token.gather(1, at).gather(1, to)}
    out = {k: torch.cat([v, v.new_zeros(R, B - v.shape[1])], 1) if v.shape[1] < B else v for k, v in out.items()}
    width = torch.arange(B, device="cuda")
    for name, n in (("", min(B, B * K)), ("ended_", min(B, B * (K + E)))):
        out[name + "scores"] = torch.where(width < n, out[name + "scores"], -math.inf)
        none = out[name + "scores"] == -math.inf
        for k in ("parents", "tokens"):
            out[name + k] = torch.where(none, -1, out[name + k]).int()
        out[name + "scores"] = out[name + "scores"].float()
    return out


def _reorder(s):
    c = s["case"]
    if own:
        s["pool"].reorder(s["rows"], s["parents"], s["tables"], s["lens"], s["held"], s["refs"], grow=1)
    else:
        _reorder_plain(s)
    return {k: s[k] for k in ("k", "v", "tables", "lens", "held", "refs")}


def _reorder_plain(s):
    c, ps, first = s["case"], s["case"]["page"], s["case"]["cached"]
    R, B = c["requests"], c["beams"]
    local = s["parents"].long().view(-1)
    alive, item = local >= 0, torch.arange(R * B, device="cuda")
    src = torch.where(alive, item // B * B + local.clamp(min=0), item)
    row = s["rows"].view(-1).long()
    table, length, held = s["tables"][row].long(), s["lens"][row].long(), s["held"][row].long()
    # the first child of each row takes its last page over
    child = torch.full((R * B,), R * B, device="cuda").scatter_reduce_(0, src[alive], item[alive], "amin")
    count = torch.zeros(R * B, dtype=torch.int64, device="cuda").index_add_(0, src[alive], torch.ones_like(src[alive]))
    heir = alive & (child[src] == item)
    col = torch.arange(table.shape[1], device="cuda")
    size = torch.where(alive, length[src], 0)
    have = torch.where(heir, held[src], size // ps)
    total = torch.where(alive, torch.maximum((size + 1 + ps - 1) // ps, have), 0)
    have = torch.minimum(have, total)
    # references: every holder's go, every heir's and sharer's come
    private = (col < held[:, None]) & (table >= first)
    full = col < (length // ps)[:, None]
    change = torch.where(full, count[:, None], (count > 0).long()[:, None]) - 1
    s["refs"].index_add_(0, table[private] - first, change[private].int())
    free = (s["refs"] == 0).nonzero()[:, 0]
    need = total - have
    begin = need.cumsum(0) - need
    source = table[src]
    new = (col >= have[:, None]) & (col < total[:, None])
    fresh = free[(begin[:, None] + col - have[:, None]).clamp(0, free.shape[0] - 1)] + first
    ids = torch.where(col < have[:, None], source, torch.where(new, fresh, table))
    s["refs"][ids[new] - first] = 1
    s["tables"][row] = ids.int()
    s["lens"][row] = size.int()
    s["held"][row] = total.int()
    # the others copy it
    copies = alive & ~heir & (size % ps > 0)
    at = (size // ps)[copies]
    a, b = source[copies, at], ids[copies, at]
    tok = (torch.arange(ps, device="cuda") < (size % ps)[copies, None])[None, :, :, None, None]
    s["k"][:, b] = torch.where(tok, s["k"][:, a], s["k"][:, b])
    s["v"][:, b] = torch.where(tok, s["v"][:, a], s["v"][:, b])


def _trace(s):
    if own:
        s["out"] = s["search"].trace(s["tokens"], s["parents"], s["beams"], lengths=s["lengths"], out=s.get("out"))
        return s["out"]
    return _trace_plain(s)


def _trace_plain(s):
    T, R, B = s["tokens"].shape
    beam = s["beams"].long()
    end = torch.full_like(beam, T) if s["lengths"] is None else s["lengths"].long()
    end = torch.where(beam >= 0, end, 0)
    t = torch.arange(T, device="cuda")
    back = end[..., None] - 1 - t            # steps from the hypothesis' last token to step t
    live = back >= 0
    left, at = back.clamp(min=0), (end - 1).clamp(min=0)[..., None].expand(back.shape)
    cur = beam.clamp(min=0)[..., None].expand(back.shape)
    jump = s["parents"].long().transpose(0, 1)  # [R, T, B]: a beam of step t -> its ancestor 2^k steps before
    step, r = 1, torch.arange(R, device="cuda")[:, None, None]
    while step < T:
        some = (left & step) > 0
        cur = torch.where(some, jump[r, at, cur], cur)
        at = torch.where(some, at - step, at)
        before = torch.cat([jump[:, :1].expand(R, step, B), jump[:, :-step]], 1)
        jump = before.gather(2, jump)
        step *= 2
    return torch.where(live, s["tokens"].transpose(0, 1)[r, t, cur], -1)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
def exact(case, seed):
    if case["kind"] != "select":  # whole numbers and moved values: nothing is computed
        return None
    s = _inputs(case, seed)
    R, B, V = case["requests"], case["beams"], case["vocab"]
    out = {k: torch.full((R, B), -1, dtype=torch.int32, device="cuda") for k in ("tokens", "parents", "ended_tokens", "ended_parents")}
    out |= {k: torch.full((R, B), -math.inf, dtype=torch.float64, device="cuda") for k in ("scores", "ended_scores")}
    ends = torch.zeros(V, dtype=torch.bool, device="cuda")
    ends[s["end_tokens"]] = True
    for r in range(R):
        x = s["logits"][r].double()
        p = s["scores"][r].double()[:, None] + (x - torch.logsumexp(x, -1, keepdim=True))
        p = torch.where(torch.isnan(p), -math.inf, p).flatten()
        best, at = p.sort(dim=0, descending=True, stable=True)
        best, at = best[:B * (len(s["end_tokens"]) + 1)], at[:B * (len(s["end_tokens"]) + 1)]
        last = ends[at % V]
        for name, keep in (("", ~last), ("ended_", last & (torch.arange(len(at), device="cuda") < B))):
            keep = (keep & (best > -math.inf)).nonzero()[:B, 0]
            out[name + "scores"][r, :len(keep)] = best[keep]
            out[name + "tokens"][r, :len(keep)] = (at[keep] % V).int()
            out[name + "parents"][r, :len(keep)] = (at[keep] // V).int()
    return out


_LISTED_WORK = [dict(work=work(c)) for c in listed()]
