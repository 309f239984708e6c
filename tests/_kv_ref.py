"""Plain 64-bit statements of the operators on KV pages, for the tests.

Written from the operators' definitions, one request, token, row or page at a
time; nothing here is shared with the library."""
import math

import numpy as np
import torch

UNIT = {t: torch.finfo(t).eps / 2 for t in (torch.bfloat16, torch.float16)}   # half the spacing of values, relative


def make_pool(layers, pages, page_size, heads, dim, dtype, layout="token", seed=0, fill=None):
    """Keys and values [layers, pages, page_size, heads, dim], seen through the layout's strides."""
    g = torch.Generator("cuda").manual_seed(seed)
    out = []
    for _ in range(2):
        shape = (layers, pages, page_size, heads, dim) if layout != "head" else (layers, pages, heads, page_size, dim)
        if layout == "both":  # one tensor holds both, keys and values of a page side by side
            shape = (layers, pages, 2, page_size, heads, dim)
        t = torch.randn(shape, generator=g, device="cuda").to(dtype) if fill is None else torch.full(shape, fill, device="cuda", dtype=dtype)
        out.append(t)
        if layout == "both":
            return t[:, :, 0], t[:, :, 1]
    return tuple(t.transpose(2, 3) if layout == "head" else t for t in out)


def attention(q, k, v, q_offsets, kv_lens, tables, scale, causal):
    """Output, log-sum-exp and the error bound's parts in 64 bits.

    A = sum_j p_j |v_j| and S = max_j scale sum_e |q_e k_je| over the visible
    keys, for each query row."""
    T, hq, d = q.shape
    hk, ps = k.shape[2], k.shape[1]
    ratio = hq // hk
    out = torch.zeros(T, hq, d, dtype=torch.float64, device=q.device)
    spread = torch.zeros_like(out)
    lse = torch.full((T, hq), -math.inf, dtype=torch.float64, device=q.device)
    size = torch.zeros(T, hq, dtype=torch.float64, device=q.device)
    for r in range(len(kv_lens)):
        a, b, L = q_offsets[r], q_offsets[r + 1], kv_lens[r]
        if L == 0 or a == b:
            continue
        ids = tables[r, : -(-L // ps)].long()
        kk = k[ids].reshape(-1, hk, d)[:L].double().repeat_interleave(ratio, 1)
        vv = v[ids].reshape(-1, hk, d)[:L].double().repeat_interleave(ratio, 1)
        for t in range(a, b):
            seen = L - (b - a) + (t - a) + 1 if causal else L
            if seen <= 0:
                continue
            x = q[t].double()
            s = scale * torch.einsum("hd,lhd->hl", x, kk[:seen])
            p = torch.softmax(s, -1)
            out[t] = torch.einsum("hl,lhd->hd", p, vv[:seen])
            spread[t] = torch.einsum("hl,lhd->hd", p, vv[:seen].abs())
            lse[t] = torch.logsumexp(s, -1)
            size[t] = abs(scale) * torch.einsum("hd,lhd->hl", x.abs(), kk[:seen].abs()).amax(-1)
    return out, lse, spread, size


def attention_bound(out, spread, size, dtype, dim, longest, vmax):
    """How far a 16-bit output may be from the exact one.

    The result's own rounding (u |o|) and each weight's rounding to the pool's
    type (u A, since sum p |v| = A); scores of ``dim`` products summed in 32
    bits (an error of dim 2^-22 S each, twice in a normalized weight, with a
    few 2^-22 for the exponential and the sums); in f16, weights below 2^-14
    of the largest round to multiples of 2^-24.  A tenth more for the products
    of these."""
    u = UNIT[dtype]
    e = 2 * (dim * 2.0 ** -22 * size[..., None] + 2.0 ** -19)
    b = u * out.abs() + (u + e) * spread + 1e-30
    if dtype == torch.float16:
        b = b + longest * 2.0 ** -25 * vmax + 2.0 ** -25
    return 1.1 * b


def norm_rotate(x, weight, eps, rope, positions, interleaved):
    """x [T, H, D] in 64 bits; rope [rows, rope_dim]."""
    x = x.double().clone()
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    if rope is None:
        return x
    half = rope.shape[1] // 2
    y = x.clone()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        c, s = rope[positions.long(), i].double()[:, None], rope[positions.long(), half + i].double()[:, None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


class Pages:
    """The page calls on host arrays, one item at a time."""

    def __init__(self, tables, lens, held, refs, first, page_size):
        self.tables, self.lens, self.held, self.refs = (np.array(x) for x in (tables, lens, held, refs))
        self.first, self.ps = first, page_size

    def fork(self, parents, children, room):
        """Returns the (source page, new page, tokens) copies."""
        free = [int(i) for i in np.nonzero(self.refs == 0)[0]]
        copies, at = [], 0
        old_t, old_l, old_h = self.tables.copy(), self.lens.copy(), self.held.copy()
        for p, c, m in zip(parents, children, room):
            n = int(old_l[p]) if p >= 0 else 0
            total = -(-max(n, int(m)) // self.ps)
            if p == c:
                full, total = int(old_h[p]), max(total, int(old_h[p]))
            else:
                full = n // self.ps
                for k in range(full):
                    self.tables[c, k] = old_t[p, k]
                    if old_t[p, k] >= self.first:
                        self.refs[old_t[p, k] - self.first] += 1
            for k in range(full, total):
                page = free[at]
                at += 1
                self.refs[page] = 1
                self.tables[c, k] = self.first + page
            if p != c and n % self.ps:
                copies.append((int(old_t[p, full]), int(self.tables[c, full]), n % self.ps))
            self.lens[c], self.held[c] = n, total
        return copies

    def release(self, rows):
        for r in rows:
            for k in range(self.held[r]):
                if self.tables[r, k] >= self.first:
                    self.refs[self.tables[r, k] - self.first] -= 1
            self.held[r] = self.lens[r] = 0

    def compact(self):
        """Returns the (from, to) page ids of the moves."""
        live = int((self.refs > 0).sum())
        holes = [i for i in range(live) if self.refs[i] == 0]
        movers = [i for i in range(len(self.refs) - 1, live - 1, -1) if self.refs[i] > 0]
        moves = dict(zip(movers, holes))
        for a, b in moves.items():
            self.refs[b], self.refs[a] = self.refs[a], 0
        for r in range(self.tables.shape[0]):
            for k in range(self.held[r]):
                i = int(self.tables[r, k]) - self.first
                if i in moves:
                    self.tables[r, k] = self.first + moves[i]
        return [(self.first + a, self.first + b) for a, b in moves.items()], live
