"""Measured cases of the operators on the KV pages that the prefix cache hands out block ids for.

Three operators, each over one paged pool of keys and values
[layers, pages, page_size, kv_heads, head_dim]:

- append: the norm of queries and keys for each head, the position rotation,
  and the write of keys and values into the pool's pages, in one pass;
- attention: queries over the pages of their requests, the prefix that a group
  of requests shares read once for all of them;
- pages: forking, copying, freeing and compacting pages.

``own`` chooses between the framework's calls and a plain form in elementary
torch operations, in 32 bits and rounded once at the end.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


# ---------------------------------------------------------------------------
# the cases
def listed():
    return [
        # one decode batch's new tokens: the smallest call, latency counts
        dict(name="append-decode", kind="append", tokens=64, decode=True, kv_heads=8, ratio=4, dim=128, page=16,
             rope=128, interleaved=False, norm=True, dtype="bf16", layout="token"),
        # the uncached part of a step's prompts, written at once
        dict(name="append-prompts", kind="append", tokens=8191, decode=False, kv_heads=8, ratio=4, dim=128, page=16,
             rope=128, interleaved=False, norm=True, dtype="bf16", layout="token"),
        # odd heads, a partial rotation in pairs, no norm, a head-major pool
        dict(name="append-odd-f16", kind="append", tokens=777, decode=False, kv_heads=5, ratio=3, dim=80, page=8,
             rope=32, interleaved=True, norm=False, dtype="f16", layout="head"),
        # one request answering: a token against a short context
        dict(name="attend-one", kind="attention", requests=1, groups=1, prefix=512, tail=256, new=1, kv_heads=8,
             ratio=4, dim=128, page=16, dtype="bf16", layout="token", shape=1),
        # many requests over one long shared document, one token each
        dict(name="attend-shared-decode", kind="attention", requests=128, groups=1, prefix=16384, tail=1024, new=1,
             kv_heads=8, ratio=4, dim=128, page=16, dtype="bf16", layout="token", shape=2),
        # chat tenants: system prompts of up to 1024 tokens, conversations of up to 4096
        dict(name="attend-tenants-decode", kind="attention", requests=256, groups=32, prefix=1024, tail=4096, new=1,
             kv_heads=8, ratio=4, dim=128, page=16, dtype="bf16", layout="token", shape=3),
        # prompts whose first 4096 tokens are cached: the uncached ones attend to both
        dict(name="attend-prompts", kind="attention", requests=8, groups=2, prefix=4096, tail=64, new=2048,
             kv_heads=8, ratio=4, dim=128, page=16, dtype="bf16", layout="token", shape=4),
        # a few drafted tokens for each request, odd sizes, one key head a query head
        dict(name="attend-odd-f16", kind="attention", requests=33, groups=5, prefix=1000, tail=301, new=7,
             kv_heads=7, ratio=1, dim=80, page=8, dtype="f16", layout="head", shape=5),
        # parallel sampling of a few requests
        dict(name="fork-few", kind="pages", op="fork", layers=4, rows=4, items=7, tokens=1000, kv_heads=4, dim=64,
             page=16, cached=512, dtype="bf16"),
        # a beam step over a whole batch: fork the survivors, then free their rows again
        dict(name="fork-release-many", kind="pages", op="turnover", layers=8, rows=128, items=512, tokens=2048,
             kv_heads=4, dim=64, page=16, cached=4096, dtype="bf16"),
        # defragmentation of a half-empty pool
        dict(name="compact-pool", kind="pages", op="compact", layers=4, rows=256, items=0, tokens=2048, kv_heads=4,
             dim=64, page=16, cached=1024, dtype="bf16"),
        # pages brought in from elsewhere in the pool
        dict(name="copy-pages", kind="pages", op="copy", layers=8, rows=0, items=1025, tokens=0, kv_heads=8, dim=128,
             page=16, cached=0, dtype="f16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    return dict(kv_heads=rng.choice([1, 2, 4, 5, 8]), ratio=rng.choice([1, 2, 3, 4, 7, 8]),
                dim=rng.choice([64, 64, 80, 96, 128, 128, 128]), page=rng.choice([8, 16, 16, 32, 64]),
                dtype=rng.choice(["bf16", "bf16", "f16"]), layout=rng.choice(["token", "head"]))


def draw(rng):
    most = {k: max(c["work"][k] for c in _LISTED_WORK) for k in ("bytes", "flops")}
    while True:
        kind = rng.choice(["append", "attention", "attention", "pages"])
        if kind == "append":
            c = dict(kind=kind, tokens=_log(rng, 1, 12000), decode=rng.random() < 0.4, interleaved=rng.random() < 0.4,
                     norm=rng.random() < 0.6, **_heads(rng))
            c["rope"] = rng.choice([c["dim"], c["dim"], c["dim"] // 2, 0])
        elif kind == "attention":
            new = rng.choice([1, 1, rng.randint(2, 9), _log(rng, 10, 2500)])
            r = _log(rng, 1, 300)
            c = dict(kind=kind, requests=r, groups=min(r, _log(rng, 1, 40)), prefix=_log(rng, 8, 40000),
                     tail=_log(rng, 1, 5000), new=new, shape=rng.randint(10, 10**6), **_heads(rng))
        else:
            c = dict(kind=kind, op=rng.choice(["fork", "turnover", "compact", "copy"]), layers=rng.randint(1, 9),
                     rows=_log(rng, 1, 300), items=_log(rng, 1, 800), tokens=_log(rng, 8, 8192), cached=_log(rng, 1, 5000),
                     **_heads(rng))
            del c["ratio"], c["layout"]
        if _footprint(c) > 4e9:
            continue
        w = work(c)
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"]:
            return c


def _footprint(c):
    """Values that the plain form holds at once."""
    if c["kind"] == "append":
        return 8 * c["tokens"] * c["kv_heads"] * c["dim"] * (2 + c["ratio"])
    if c["kind"] == "attention":
        _, kv, _, _ = _lengths(c)
        return c["requests"] * int(kv.max()) * c["kv_heads"] * max(c["dim"], c["ratio"] * c["new"])
    return 2 * c["layers"] * _num_pages(c) * c["page"] * c["kv_heads"] * c["dim"]


# ---------------------------------------------------------------------------
# what a pass cannot do without
def work(c):
    e, d, ps = 2, c["dim"], c["page"]
    if c["kind"] == "append":
        hq, hk, t = c["kv_heads"] * c["ratio"], c["kv_heads"], c["tokens"]
        values = t * (hq + 2 * hk) * d
        return {"bytes": 2 * e * values + t * (12 + 4 * c["rope"]), "flops": 8 * t * (hq + hk) * d}
    if c["kind"] == "attention":
        new, kv, go, prefix = _lengths(c)
        hq, hk = c["kv_heads"] * c["ratio"], c["kv_heads"]
        keys = int(prefix.sum()) + int((kv - np.repeat(prefix, np.diff(go))).sum())
        seen = int((new * (kv - new) + new * (new + 1) // 2).sum())
        return {"bytes": e * d * (2 * hk * keys + 2 * hq * int(new.sum())) + 4 * (keys // ps), "flops": 4 * d * hq * seen}
    page = 2 * c["layers"] * ps * c["kv_heads"] * d * e  # bytes of one page, keys and values
    if c["op"] == "copy":
        return {"bytes": 2 * page * c["items"] + 8 * c["items"], "flops": 0}
    s = _page_state(c, 0)
    if c["op"] == "compact":
        live = int((s["refs"] > 0).sum())
        moved = int((s["refs"][live:] > 0).sum())
        return {"bytes": 2 * page * moved + 8 * int(s["held"].sum()) + 8 * s["refs"].size, "flops": 0}
    p = s["parents"]
    length = np.where(p >= 0, s["lens"][np.maximum(p, 0)], 0)
    total = -(-np.maximum(length, s["room"]) // ps)
    copied = int((length % ps).sum()) * page // ps
    refs = (8 if c["op"] == "fork" else 16) * int(total.sum())
    return {"bytes": 2 * copied + 8 * int(total.sum()) + refs, "flops": 0}


# ---------------------------------------------------------------------------
# the inputs
def _lengths(c):
    """New tokens and whole lengths of the requests, the groups' first requests, the groups' shared tokens."""
    r = np.random.RandomState(c["shape"])
    R, G, ps = c["requests"], c["groups"], c["page"]
    cut = np.sort(r.choice(R - 1, G - 1, replace=False)) + 1 if G > 1 else np.zeros(0, np.int64)
    go = np.concatenate([[0], cut, [R]]).astype(np.int64)
    prefix = r.randint(c["prefix"] // 2, c["prefix"] + 1, G) // ps * ps
    if G == 1:
        prefix[:] = c["prefix"] // ps * ps
    own_tokens = r.randint(0, c["tail"] + 1, R)
    new = r.randint(1, c["new"] + 1, R)
    return new, np.repeat(prefix, np.diff(go)) + own_tokens + new, go, prefix


def _normal(g, *shape, dtype, spread=1.0, shift=0.0):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).mul_(spread).add_(shift).to(dtype)


def _kv_pool(c, g, pages, layers=1):
    """Keys and values of a pool in use, seen as [layers, pages, page_size, kv_heads, head_dim]."""
    dt, out = DTYPES[c["dtype"]], []
    for _ in range(2):
        if c.get("layout") == "head":
            out.append(_normal(g, layers, pages, c["kv_heads"], c["page"], c["dim"], dtype=dt).transpose(2, 3))
        else:
            out.append(_normal(g, layers, pages, c["page"], c["kv_heads"], c["dim"], dtype=dt))
    return out


def _dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a)).to(device="cuda", dtype=dtype)


def _append_inputs(c, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    r = np.random.RandomState(seed % (1 << 31))
    T, hk, hq, d, ps, dt = c["tokens"], c["kv_heads"], c["kv_heads"] * c["ratio"], c["dim"], c["page"], DTYPES[c["dtype"]]
    pages = 4 * (-(-T // ps)) + 8 if not c["decode"] else max(2 * T, 16)
    k, v = _kv_pool(c, g, pages)
    perm = r.permutation(pages)
    t = np.arange(T)
    if c["decode"]:  # one token at the end of each of T requests
        pos = r.randint(0, 32768, T)
        slots = perm[t].astype(np.int64) * ps + pos % ps
    else:  # consecutive tokens of one prompt after what was cached of it
        start = int(r.randint(0, 16)) * ps
        pos = start + t
        slots = perm[t // ps].astype(np.int64) * ps + pos % ps
    if T > 16:
        slots[-3:] = -1  # a padded batch
    rows = 32768
    qkv = _normal(g, T, (hq + 2 * hk) * d, dtype=dt, spread=1.5)
    s = dict(case=c, k=k, v=v, qkv=qkv, q=qkv[:, :hq * d].view(T, hq, d), new_k=qkv[:, hq * d:(hq + hk) * d].view(T, hk, d),
             new_v=qkv[:, (hq + hk) * d:].view(T, hk, d), slots=_dev(slots, torch.int64), positions=_dev(pos, torch.int32),
             rope=None, q_weight=None, k_weight=None, q_out=torch.empty(T, hq, d, device="cuda", dtype=dt))
    if c["rope"]:
        inv = 10000.0 ** (-torch.arange(0, c["rope"], 2, device="cuda", dtype=torch.float64) / c["rope"])
        a = torch.arange(rows, device="cuda", dtype=torch.float64)[:, None] * inv
        s["rope"] = torch.cat([a.cos(), a.sin()], 1).float()
    if c["norm"]:
        s["q_weight"], s["k_weight"] = (_normal(g, d, dtype=dt, spread=0.2, shift=1.0) for _ in range(2))
    return s


def _attention_inputs(c, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    r = np.random.RandomState(seed % (1 << 31))
    new, kv, go, prefix = _lengths(c)
    R, ps, hk, hq, d = c["requests"], c["page"], c["kv_heads"], c["kv_heads"] * c["ratio"], c["dim"]
    count = -(-kv // ps)
    shared = np.repeat(prefix, np.diff(go)) // ps
    group = np.repeat(np.arange(len(prefix)), np.diff(go))
    first_shared = np.concatenate([[0], np.cumsum(prefix // ps)])
    first_own = first_shared[-1] + np.concatenate([[0], np.cumsum(count - shared)])
    pages = int(first_own[-1]) + 5
    perm = r.permutation(pages)
    col = np.arange(int(count.max()) + 3)[None]
    at = np.where(col < shared[:, None], first_shared[group][:, None] + col, first_own[:-1][:, None] + col - shared[:, None])
    tables = np.where(col < count[:, None], perm[np.minimum(at, pages - 1)], -1)
    k, v = _kv_pool(c, g, pages)
    T, dt = int(new.sum()), DTYPES[c["dtype"]]
    # scores of a few units' spread, as trained queries and keys have them
    q = _normal(g, T, hq, d, dtype=dt, spread=1.5)
    return dict(case=c, k=k, v=v, q=q, tables=_dev(tables, torch.int32), kv_lens=_dev(kv, torch.int32), pages=pages,
                q_offsets=_dev(np.concatenate([[0], np.cumsum(new)]), torch.int32), group_offsets=_dev(go, torch.int32),
                scale=d ** -0.5, longest=int(kv.max()), most=int(new.max()), out=torch.empty(T, hq, d, device="cuda", dtype=dt))


def _num_pages(c):
    if c["op"] == "copy":
        return 2 * c["items"] + 8
    each = -(-c["tokens"] // c["page"]) + 1
    if c["op"] == "compact":
        return c["cached"] + 2 * c["rows"] * each
    return c["cached"] + c["rows"] * each + c["items"] * 6 + 2 * each


def _page_state(c, seed):
    """Page tables in use: each row has a cached prefix (ids below ``cached``) and private pages, some held twice."""
    r = np.random.RandomState(1000 + seed % (1 << 31))
    ps, first, pages = c["page"], c["cached"], _num_pages(c)
    rows, items = c["rows"], c["items"]
    total_rows = rows + (items if c["op"] != "compact" else 0)
    width = -(-c["tokens"] // ps) + 4
    lens = np.zeros(total_rows, np.int64)
    lens[:rows] = r.randint(1, c["tokens"] + 1, rows)
    held = -(-lens // ps)
    cached = np.minimum(r.randint(0, 9, total_rows), held - 1).clip(0)
    col = np.arange(width)[None]
    starts = np.concatenate([[0], np.cumsum(held - cached)])
    perm = r.permutation(pages - first)
    at = np.minimum(starts[:-1][:, None] + col - cached[:, None], pages - first - 1)
    tables = np.where(col < cached[:, None], r.randint(0, first, (total_rows, width)), first + perm[np.maximum(at, 0)])
    tables = np.where(col < held[:, None], tables, -1)
    if rows > 1:  # rows forked earlier: they share their first private pages
        twin = np.arange(1, rows, 2)
        n = np.minimum(lens[twin] // ps, lens[twin - 1] // ps)
        tables[twin] = np.where(col < n[:, None], tables[twin - 1], tables[twin])
    private = tables[tables >= first] - first
    refs = np.bincount(private, minlength=pages - first).astype(np.int64)
    s = dict(tables=tables, lens=lens, held=held, refs=refs)
    if c["op"] in ("fork", "turnover"):
        parents = r.randint(0, rows, items)
        parents[7::8] = -1  # new requests
        s["parents"], s["children"] = parents, rows + np.arange(items)
        s["room"] = np.where(parents >= 0, lens[np.maximum(parents, 0)], 0) + r.randint(1, 2 * ps, items)
    return s


def _page_inputs(c, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    pages = _num_pages(c)
    k, v = _kv_pool(c, g, pages, c["layers"])
    s = dict(case=c, k=k, v=v, pages=pages)
    if c["op"] == "copy":
        perm = np.random.RandomState(seed % (1 << 31)).permutation(pages)[:2 * c["items"]]
        return dict(s, src=_dev(perm[::2], torch.int32), dst=_dev(perm[1::2], torch.int32))
    for name, a in _page_state(c, seed).items():
        s[name] = _dev(a, torch.int32)
    s["refs_out"], s["tables_out"] = torch.empty_like(s["refs"]), torch.empty_like(s["tables"])
    return s


def _inputs(c, seed):
    return {"append": _append_inputs, "attention": _attention_inputs, "pages": _page_inputs}[c["kind"]](c, seed)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:  # the handle on the pool that a serving program keeps, and a step's plan, which serves all its layers
        from paper_2608_01657_gb300 import kv
        c = case
        if c["kind"] == "append":
            s["pool"] = kv.KVPool(s["k"], s["v"], num_q_heads=c["kv_heads"] * c["ratio"])
        elif c["kind"] == "attention":
            s["pool"] = kv.KVPool(s["k"], s["v"], num_q_heads=c["kv_heads"] * c["ratio"], max_requests=c["requests"],
                                  max_tokens=s["q"].shape[0], max_row_pages=s["tables"].shape[1])
            s["pool"].plan(s["q_offsets"], s["kv_lens"], s["tables"], num_tokens=s["q"].shape[0],
                           group_offsets=s["group_offsets"])
        else:
            s["pool"] = kv.KVPool(s["k"], s["v"], num_q_heads=c["kv_heads"], first_page=c["cached"],
                                  max_requests=max(1, c["rows"] + c["items"]),
                                  max_row_pages=s["tables"].shape[1] if "tables" in s else 1)
    return s


# ---------------------------------------------------------------------------
# one pass
def run(s):
    c = s["case"]
    if c["kind"] == "append":
        return _append_own(s) if own else _append_plain(s)
    if c["kind"] == "attention":
        return s["pool"].attention(0, s["q"], scale=s["scale"], out=s["out"]) if own else _attention_plain(s)
    return {"copy": _copy, "fork": _fork, "turnover": _turnover, "compact": _compact}[c["op"]](s)


def _append_own(s):
    c = s["case"]
    s["pool"].append(0, s["q"], s["new_k"], s["new_v"], s["slots"], positions=s["positions"], rope=s["rope"],
                     interleaved=c["interleaved"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=1e-6, q_out=s["q_out"])
    return {"q": s["q_out"], "k": s["k"], "v": s["v"]}


def _norm_rotate(x, weight, rope, positions, interleaved):
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * weight.float()
    if rope is not None:
        rd = rope.shape[1]
        a = rope[positions.long()][:, None]
        cos, sin = a[..., :rd // 2], a[..., rd // 2:]
        rot, rest = x[..., :rd], x[..., rd:]
        if interleaved:
            x1, x2 = rot[..., 0::2], rot[..., 1::2]
            rot = torch.stack([x1 * cos - x2 * sin, x2 * cos + x1 * sin], -1).flatten(-2)
        else:
            x1, x2 = rot[..., :rd // 2], rot[..., rd // 2:]
            rot = torch.cat([x1 * cos - x2 * sin, x2 * cos + x1 * sin], -1)
        x = torch.cat([rot, rest], -1)
    return x


def _append_plain(s):
    c, ps = s["case"], s["case"]["page"]
    q = _norm_rotate(s["q"], s["q_weight"], s["rope"], s["positions"], c["interleaved"]).to(s["q"].dtype)
    k = _norm_rotate(s["new_k"], s["k_weight"], s["rope"], s["positions"], c["interleaved"]).to(s["k"].dtype)
    ok = s["slots"] >= 0
    at = s["slots"][ok]
    s["k"][0][at // ps, at % ps] = k[ok]
    s["v"][0][at // ps, at % ps] = s["new_v"][ok]
    return {"q": q, "k": s["k"], "v": s["v"]}


def _attention_plain(s):
    c = s["case"]
    R, ps, hk, n, g, d = c["requests"], c["page"], c["kv_heads"], c["ratio"], s["most"], c["dim"]
    L = -(-s["longest"] // ps) * ps
    ids = s["tables"][:, :L // ps].long().clamp(min=0)
    kv, first = s["kv_lens"].long(), s["q_offsets"][:-1].long()
    new = s["q_offsets"][1:].long() - first
    j = torch.arange(L, device="cuda")
    i = torch.arange(g, device="cuda")
    live = i < new[:, None]                                                         # [R, g]
    at = (first[:, None] + i).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][at].float().view(R, g, hk, n, d).permute(0, 2, 3, 1, 4).reshape(R, hk, n * g, d)
    seen = j < (kv - new)[:, None, None] + i[:, None] + 1                            # [R, g, L]
    k = s["k"][0][ids].reshape(R, L, hk, d).permute(0, 2, 3, 1).float()
    score = torch.matmul(q, k).mul_(s["scale"]).view(R, hk, n, g, L)
    del k
    score.masked_fill_(~seen[:, None, None], -math.inf)
    p = score.sub_(score.amax(-1, keepdim=True)).exp_()
    total = p.sum(-1)
    v = s["v"][0][ids].reshape(R, L, hk, d).float()
    v = torch.where((j < kv[:, None])[:, :, None, None], v, 0.0).transpose(1, 2)
    out = torch.matmul(p.view(R, hk, n * g, L), v).view(R, hk, n, g, d) / total[..., None]
    return out.permute(0, 3, 1, 2, 4).reshape(R, g, hk * n, d)[live].to(s["q"].dtype)


def _copy(s):
    if own:
        s["pool"].copy(s["src"], s["dst"])
    else:
        s["k"][:, s["dst"].long()] = s["k"][:, s["src"].long()]
        s["v"][:, s["dst"].long()] = s["v"][:, s["src"].long()]
    return {"k": s["k"], "v": s["v"]}


def _fork(s, refs_out=None):
    refs_out = s["refs_out"] if refs_out is None else refs_out
    if own:
        s["pool"].fork(s["parents"], s["children"], s["room"], s["tables"], s["lens"], s["held"], s["refs"], refs_out=refs_out)
    else:
        _fork_plain(s, refs_out)
    return {k: s[k] for k in ("k", "v", "tables", "lens", "held")} | {"refs": refs_out}


def _fork_plain(s, refs_out):
    ps, first = s["case"]["page"], s["case"]["cached"]
    parent, child = s["parents"].long(), s["children"].long()
    p = parent.clamp(min=0)
    length = torch.where(parent >= 0, s["lens"][p].long(), 0)
    full, part = length // ps, length % ps
    total = (torch.maximum(length, s["room"].long()) + ps - 1) // ps
    need = total - full
    start = need.cumsum(0) - need
    free = (s["refs"] == 0).nonzero()[:, 0] + first
    col = torch.arange(s["tables"].shape[1], device="cuda")[None]
    fresh = free[(start[:, None] + col - full[:, None]).clamp(0, free.shape[0] - 1)]
    source = s["tables"][p].long()
    keep, new = col < full[:, None], (col >= full[:, None]) & (col < total[:, None])
    row = torch.where(keep, source, torch.where(new, fresh, s["tables"][child].long()))
    s["tables"][child] = row.int()
    s["lens"][child] = length.int()
    s["held"][child] = total.int()
    refs_out.copy_(s["refs"])
    shared = source[keep & (source >= first)] - first
    refs_out.index_add_(0, shared, torch.ones_like(shared, dtype=torch.int32))
    refs_out[fresh[new] - first] = 1
    at = full.clamp(max=row.shape[1] - 1)[:, None]
    src, dst = source.gather(1, at)[:, 0].clamp(min=0), row.gather(1, at)[:, 0]
    some = part > 0
    tok = (torch.arange(ps, device="cuda") < part[some][:, None])[None, :, :, None, None]
    s["k"][:, dst[some]] = torch.where(tok, s["k"][:, src[some]], s["k"][:, dst[some]])
    s["v"][:, dst[some]] = torch.where(tok, s["v"][:, src[some]], s["v"][:, dst[some]])


def _turnover(s):
    """A step's forks, and the rows freed again."""
    out = _fork(s)
    refs = out["refs"]
    if own:
        s["pool"].release(s["children"], s["tables"], s["lens"], s["held"], refs)
    else:
        first, child = s["case"]["cached"], s["children"].long()
        rows = s["tables"][child].long()
        col = torch.arange(rows.shape[1], device="cuda")[None]
        gone = rows[(col < s["held"][child][:, None]) & (rows >= first)] - first
        refs.index_add_(0, gone, torch.full_like(gone, -1, dtype=torch.int32))
        s["held"][child] = 0
        s["lens"][child] = 0
    return out


def _compact(s):
    if own:
        s["counts"] = s["pool"].compact(s["tables"], s["held"], s["refs"], tables_out=s["tables_out"], refs_out=s["refs_out"],
                                        counts=s.get("counts"))
        return {k: s[k] for k in ("k", "v", "counts")} | {"tables": s["tables_out"], "refs": s["refs_out"]}
    first, refs = s["case"]["cached"], s["refs"]
    live = (refs > 0).sum()
    idx = torch.arange(refs.shape[0], device="cuda")
    holes = ((refs == 0) & (idx < live)).nonzero()[:, 0]
    movers = ((refs > 0) & (idx >= live)).nonzero()[:, 0].flip(0)  # the highest page fills the lowest hole
    to = idx.clone()
    to[movers] = holes
    s["k"][:, holes + first] = s["k"][:, movers + first]
    s["v"][:, holes + first] = s["v"][:, movers + first]
    refs_out = torch.where(idx < live, refs, 0)
    refs_out[holes] = refs[movers]
    t = s["tables"].long()
    private = (torch.arange(t.shape[1], device="cuda")[None] < s["held"][:, None]) & (t >= first)
    tables = torch.where(private, to[(t - first).clamp(min=0)] + first, t).int()
    counts = torch.stack([live, torch.tensor(holes.shape[0], device="cuda")]).int()
    return {"k": s["k"], "v": s["v"], "counts": counts, "tables": tables, "refs": refs_out}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
def exact(case, seed):
    if case["kind"] == "pages":  # whole numbers and moved values: nothing is computed
        return None
    s = _inputs(case, seed)
    return _append_exact(s) if case["kind"] == "append" else _attention_exact(s)


def _append_exact(s):
    c, d, ps = s["case"], s["case"]["dim"], s["case"]["page"]
    pos = s["positions"].double()
    half = c["rope"] // 2
    done = []
    for x, w in ((s["q"], s["q_weight"]), (s["new_k"], s["k_weight"])):
        x = x.double().clone()
        if w is not None:
            x = x / ((x ** 2).sum(-1, keepdim=True) / d + 1e-6).sqrt() * w.double()
        y = x.clone()
        for m in range(half):  # the pair m turns by position / 10000^(2m / rope)
            a, b = (2 * m, 2 * m + 1) if c["interleaved"] else (m, m + half)
            turn = (pos * 10000.0 ** (-2.0 * m / c["rope"]))[:, None]
            z = torch.complex(x[..., a], x[..., b]) * torch.polar(torch.ones_like(turn), turn)
            y[..., a], y[..., b] = z.real, z.imag
        done.append(y)
    k, v = s["k"].double(), s["v"].double()
    for t, at in enumerate(s["slots"].tolist()):
        if at >= 0:
            k[0, at // ps, at % ps] = done[1][t]
            v[0, at // ps, at % ps] = s["new_v"][t].double()
    return {"q": done[0], "k": k, "v": v}


def _attention_exact(s):
    c, d = s["case"], s["case"]["dim"]
    hk, n = c["kv_heads"], c["ratio"]
    qo, kv = s["q_offsets"].tolist(), s["kv_lens"].tolist()
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    for r in range(c["requests"]):
        a, b, L = qo[r], qo[r + 1], kv[r]
        ids = s["tables"][r, :-(-L // c["page"])].long()
        k = s["k"][0][ids].flatten(0, 1)[:L].double()
        v = s["v"][0][ids].flatten(0, 1)[:L].double()
        q = s["q"][a:b].double().view(b - a, hk, n, d)
        last = torch.arange(L - (b - a), L, device="cuda")
        hidden = torch.arange(L, device="cuda")[None] > last[:, None]
        for h in range(hk):
            score = torch.einsum("tnd,ld->ntl", q[:, h], k[:, h]) * s["scale"]
            weight = torch.softmax(score.masked_fill(hidden, -math.inf), -1)
            out[a:b, h * n:(h + 1) * n] = torch.einsum("ntl,ld->tnd", weight, v[:, h])
    return out


_LISTED_WORK = [dict(work=work(c)) for c in listed()]
