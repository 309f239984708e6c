"""Appending to KV pages, and copying, forking, freeing and compacting them,
against plain statements."""
import numpy as np
import pytest
import torch

from _kv_ref import UNIT, Pages, make_pool, norm_rotate

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def dev(a, dtype=torch.int32):
    return torch.tensor(np.asarray(a), dtype=dtype, device="cuda")


def rope_table(rows, dim):
    inv = 10000.0 ** (-torch.arange(0, dim, 2, device="cuda", dtype=torch.float64) / dim)
    a = torch.arange(rows, device="cuda", dtype=torch.float64)[:, None] * inv
    return torch.cat([a.cos(), a.sin()], 1).float()


def check_append(T, heads, ratio, dim, ps, dtype, rope_dim=0, interleaved=False, qn=True, kn=True, layout="token",
                 skip=(), inplace=False, seed=0):
    from paper_2608_01657_gb300 import kv as KV
    pages = -(-T // ps) + 3
    k, v = make_pool(2, pages, ps, heads, dim, dtype, layout, seed)
    before_k, before_v = k.clone(), v.clone()
    g = torch.Generator("cuda").manual_seed(seed + 1)
    hq = heads * ratio
    qkv = torch.randn(T, (hq + 2 * heads) * dim, generator=g, device="cuda").mul_(2).to(dtype)
    q, nk, nv = (x.unflatten(1, (-1, dim)) for x in qkv.split([hq * dim, heads * dim, heads * dim], 1))
    r = np.random.RandomState(seed)
    slots = r.permutation(pages * ps)[:T].astype(np.int64)
    slots[list(skip)] = -1 - r.randint(0, 5, len(skip))
    pos = dev(r.randint(0, 500, T))
    rope = rope_table(500, rope_dim) if rope_dim else None
    w = [torch.randn(dim, generator=g, device="cuda").to(dtype) for _ in range(2)]
    qw, kw = w[0] if qn else None, w[1] if kn else None
    raw_q = q.clone()
    pool = KV.KVPool(k, v, num_q_heads=hq)
    got = pool.append(1, q, nk, nv, dev(slots, torch.int64), positions=pos if rope_dim else None, rope=rope,
                      interleaved=interleaved, q_weight=qw, k_weight=kw, eps=1e-5, q_out=q if inplace else None)
    pool.check()
    u = UNIT[dtype]
    for have, x, weight, where in ((got, raw_q, qw, None), (k[1], nk, kw, slots)):
        want = norm_rotate(x, weight, 1e-5, rope, pos, interleaved)
        plain = weight is None and rope is None
        # one rounding of the result, and 32-bit steps of the pair that made it: below 16 of their units
        size = norm_rotate(x, weight, 1e-5, None, None, False).abs()
        if rope is not None:
            half = rope_dim // 2
            pair = torch.arange(dim, device="cuda")
            head = pair < rope_dim
            pair[head] = pair[head] ^ 1 if interleaved else (pair[head] + half) % rope_dim
            size = size + size[..., pair]
        bound = 0.0 if plain else u * want.abs() + 16 * 2.0 ** -24 * size * (1 + dim / 16) + (2.0 ** -25 if dtype == HF else 1e-38)
        if where is None:
            assert ((have.double() - want).abs() <= bound).all()
        else:
            for t, s in enumerate(where):
                if s >= 0:
                    b = bound if plain else bound[t]
                    assert ((have[s // ps, s % ps].double() - want[t]).abs() <= b).all()
    untouched = torch.ones(pages, ps, dtype=torch.bool, device="cuda")
    for t, s in enumerate(slots):
        if s >= 0:
            untouched[s // ps, s % ps] = False
            assert torch.equal(v[1, s // ps, s % ps], nv[t])
    assert torch.equal(k[1][untouched], before_k[1][untouched]) and torch.equal(v[1][untouched], before_v[1][untouched])
    assert torch.equal(k[0], before_k[0]) and torch.equal(v[0], before_v[0])


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [8, 16, 40, 64, 72, 80, 120, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_head_sizes(dim, interleaved, dtype):
    check_append(5, 2, 3, dim, 16, dtype, rope_dim=dim // 16 * 16, interleaved=interleaved, seed=dim)


@pytest.mark.parametrize("T", [1, 2, 63, 700])
@pytest.mark.parametrize("layout", ["token", "head", "both"])
def test_append_lengths_and_layouts(T, layout):
    check_append(T, 3, 2, 64, 8, BF, rope_dim=64, layout=layout, skip=(0,) if T > 2 else (), seed=T)


@pytest.mark.parametrize("qn,kn,rope_dim", [(False, False, 0), (True, False, 0), (False, True, 32), (False, False, 64),
                                            (True, True, 0), (True, True, 16)])
def test_append_parts(qn, kn, rope_dim):
    check_append(9, 2, 2, 64, 16, BF, rope_dim=rope_dim, qn=qn, kn=kn, seed=3)
    check_append(9, 1, 1, 96, 2, HF, rope_dim=rope_dim, interleaved=True, qn=qn, kn=kn, inplace=True, seed=4)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rope_dim", [(80, 40), (64, 8), (64, 24), (128, 120), (8, 8), (72, 72)])
def test_append_odd_rotations(dim, rope_dim, interleaved):
    """Rotated parts whose halves end inside a 16-byte word."""
    check_append(6, 2, 2, dim, 16, BF, rope_dim=rope_dim, interleaved=interleaved, seed=rope_dim)


def test_append_many_heads():
    check_append(3, 40, 2, 128, 16, BF, rope_dim=128, seed=6)
    check_append(600, 1, 1, 64, 64, BF, rope_dim=64, skip=(5, 599), seed=7)


def test_append_leaves_out_bad_tokens_and_reports_them():
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 4, 16, 1, 64, BF)
    before = k.clone()
    pool = KV.KVPool(k, v, num_q_heads=1)
    x = torch.ones(4, 1, 64, device="cuda", dtype=BF)
    rope = rope_table(10, 64)
    for slots, pos in (([0, 64, 1, 2], [0, 1, 2, 3]), ([0, 5, 1, 2], [0, 10, 2, 3]), ([0, 5, 1, 2], [0, -1, 2, 3])):
        out = torch.full_like(x, 9.0)
        k.copy_(before)
        pool.append(0, x, x, x, dev(slots, torch.int64), positions=dev(pos), rope=rope, q_out=out)
        with pytest.raises(RuntimeError):
            pool.check()
        assert (out[1] == 9.0).all() and not (out[[0, 2, 3]] == 9.0).all(-1).any()
        assert torch.equal(k[0, 0, 5], before[0, 0, 5]) and not torch.equal(k[0, 0, :3], before[0, 0, :3])


@pytest.mark.parametrize("dtype,dim,rope_dim", [(BF, 128, 128), (HF, 64, 0), (BF, 40, 24), (HF, 8, 8)])
def test_queries_that_append_left_out_are_nan(dtype, dim, rope_dim):
    """In an output that the call made; the other tokens' queries are what they are."""
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 4, 16, 3, dim, dtype)
    pool = KV.KVPool(k, v, num_q_heads=9)
    q, kv = torch.randn(6, 9, dim, device="cuda").to(dtype), torch.randn(6, 3, dim, device="cuda").to(dtype)
    extra = dict(positions=dev(range(6)), rope=rope_table(10, rope_dim)) if rope_dim else {}
    want = pool.append(0, q, kv, kv, dev([0, 5, 1, 2, 3, -1], torch.int64), **extra)
    pool.check()
    del_me = torch.full_like(q, 7.0)
    del del_me
    got = pool.append(0, q, kv, kv, dev([64, 5, 1, 1 << 40, 3, -1], torch.int64), **extra)
    with pytest.raises(RuntimeError):
        pool.check()
    assert torch.isnan(got[[0, 3]]).all() and torch.equal(got[[1, 2, 4, 5]], want[[1, 2, 4, 5]])


def test_append_zero_heads_of_zeros():
    """A head of zeros stays zero under the norm."""
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 2, 16, 1, 64, BF)
    pool = KV.KVPool(k, v, num_q_heads=1)
    x = torch.zeros(1, 1, 64, device="cuda", dtype=BF)
    w = torch.ones(64, device="cuda", dtype=BF)
    out = pool.append(0, x, x, x, dev([3], torch.int64), q_weight=w, k_weight=w)
    assert not out.any() and not k[0, 0, 3].any()
    empty = torch.zeros(0, 1, 64, device="cuda", dtype=BF)
    assert pool.append(0, empty, empty, empty, dev([], torch.int64)).shape[0] == 0


def test_append_refusals():
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 2, 16, 2, 64, BF)
    pool = KV.KVPool(k, v, num_q_heads=2)
    x = torch.zeros(3, 2, 64, device="cuda", dtype=BF)
    s, pos = dev([0, 1, 2], torch.int64), dev([0, 1, 2])
    bad = [dict(slots=s.int()), dict(slots=s[:2]), dict(k=x[:2]), dict(q=x.half()), dict(rope=rope_table(4, 64)),
           dict(q_weight=torch.ones(32, device="cuda", dtype=BF)), dict(k_weight=torch.ones(64, device="cuda"))]
    for b in bad:
        args = dict(q=x, k=x, v=x, slots=s) | b
        with pytest.raises(ValueError):
            pool.append(0, **args)
    for b in (dict(rope=rope_table(4, 20)), dict(rope=rope_table(4, 80)), dict(q_weight=torch.ones(64, device="cuda", dtype=BF), eps=0.0)):
        with pytest.raises(RuntimeError):
            pool.append(0, x, x, x, s, positions=pos, **b)
    with pytest.raises(RuntimeError):
        pool.append(1, x, x, x, s)


def test_append_refuses_queries_that_lie_on_its_inputs():
    """q_out is q itself or shares no element with q, k or v."""
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 4, 16, 2, 64, BF)
    pool = KV.KVPool(k, v, num_q_heads=4)
    qkv = torch.randn(22, 12, 64, device="cuda").to(BF)  # four spare heads
    q, nk, nv, s = qkv[:21, :4], qkv[:21, 4:6], qkv[:21, 6:8], dev(range(21), torch.int64)
    weight = dict(q_weight=torch.ones(64, device="cuda", dtype=BF))
    before, want = qkv.clone(), pool.append(0, q.clone(), nk.clone(), nv.clone(), s, **weight)
    for bad in (qkv[1:, :4], qkv[:21, 1:5], qkv[:21, 2:6], qkv[:21, 5:9], torch.as_strided(qkv, (21, 4, 64), (768, 64, 1), 16),
                torch.as_strided(qkv, (21, 4, 64), (256, 64, 1), 0), qkv[:1, 8:].expand(21, 4, 64)):
        with pytest.raises(RuntimeError, match="invalid"):
            pool.append(0, q, nk, nv, s, q_out=bad, **weight)
    assert torch.equal(qkv, before)
    assert torch.equal(pool.append(0, q, nk, nv, s, q_out=qkv[1:, 8:], **weight), want)
    assert torch.equal(pool.append(0, q, nk, nv, s, q_out=q, **weight), want)
    pool.check()


# ---- pages ------------------------------------------------------------------------
def rows_in_use(rows, spare, most, ps, first, pages, seed):
    """Rows of up to ``most`` tokens with cached and private pages, some held by two rows."""
    r = np.random.RandomState(seed)
    width = -(-most // ps) + 3
    tables = np.full((rows + spare, width), -1, np.int64)
    lens, held = np.zeros(rows + spare, np.int64), np.zeros(rows + spare, np.int64)
    refs = np.zeros(pages - first, np.int64)
    ids = iter(r.permutation(pages - first))
    for i in range(rows):
        lens[i] = r.randint(0, most + 1)
        held[i] = -(-lens[i] // ps) + r.randint(0, 2)
        same = r.randint(0, lens[i - 1] // ps + 1) if i and r.rand() < 0.5 else 0
        for j in range(held[i]):
            if j < same and j < lens[i] // ps:
                tables[i, j] = tables[i - 1, j]
            elif first and j < 3:
                tables[i, j] = r.randint(0, first)
            else:
                tables[i, j] = first + next(ids)
            if tables[i, j] >= first:
                refs[tables[i, j] - first] += 1
    return tables, lens, held, refs


class Both:
    """The same page calls on the GPU and in plain form."""

    def __init__(self, rows, spare, most, ps=16, first=20, pages=400, layers=3, heads=2, dim=64, dtype=BF, layout="token",
                 seed=0):
        from paper_2608_01657_gb300 import kv as KV
        t, l, h, r = rows_in_use(rows, spare, most, ps, first, pages, seed)
        self.ref = Pages(t, l, h, r, first, ps)
        self.k, self.v = make_pool(layers, pages, ps, heads, dim, dtype, layout, seed)
        self.rk, self.rv = self.k.clone(), self.v.clone()
        self.t, self.l, self.h, self.r = dev(t), dev(l), dev(h), dev(r)
        self.pool = KV.KVPool(self.k, self.v, num_q_heads=heads, first_page=first, max_requests=600,
                              max_row_pages=t.shape[1])

    def fork(self, parents, children, room, out_of_place=False):
        refs_out = torch.full_like(self.r, 77) if out_of_place else None
        before = self.r.clone()
        self.pool.fork(dev(parents), dev(children), dev(room), self.t, self.l, self.h, self.r, refs_out=refs_out)
        self.pool.check()
        if out_of_place:
            assert torch.equal(self.r, before)
            self.r = refs_out
        for a, b, n in self.ref.fork(parents, children, room):
            self.rk[:, b, :n] = self.rk[:, a, :n]
            self.rv[:, b, :n] = self.rv[:, a, :n]
        self.same()

    def release(self, rows):
        self.pool.release(dev(rows), self.t, self.l, self.h, self.r)
        self.pool.check()
        self.ref.release(rows)
        self.same()

    def compact(self, out_of_place=False):
        to, ro = (torch.full_like(self.t, 77), torch.full_like(self.r, 77)) if out_of_place else (None, None)
        counts = self.pool.compact(self.t, self.h, self.r, tables_out=to, refs_out=ro)
        self.pool.check()
        if out_of_place:
            self.t, self.r = to, ro
        moves, live = self.ref.compact()
        assert counts.tolist() == [live, len(moves)]
        for a, b in moves:
            self.rk[:, b], self.rv[:, b] = self.rk[:, a], self.rv[:, a]
        self.same()

    def same(self):
        assert np.array_equal(self.r.cpu().numpy(), self.ref.refs)
        assert np.array_equal(self.h.cpu().numpy(), self.ref.held)
        assert np.array_equal(self.l.cpu().numpy(), self.ref.lens)
        assert np.array_equal(self.t.cpu().numpy(), self.ref.tables)
        assert torch.equal(self.k, self.rk) and torch.equal(self.v, self.rv)


@pytest.mark.parametrize("ps,layout,dtype,dim", [(16, "token", BF, 64), (2, "head", HF, 8), (64, "both", BF, 40), (8, "head", BF, 128)])
def test_a_life_of_pages(ps, layout, dtype, dim):
    """Forks, growth, new rows, releases and compactions, each compared whole."""
    b = Both(6, 10, 150, ps=ps, pages=1500 if ps == 2 else 400, layout=layout, dtype=dtype, dim=dim, seed=ps)
    room = lambda rows, more: [int(b.ref.lens[p]) + m if p >= 0 else m for p, m in zip(rows, more)]  # noqa: E731
    b.fork([0, 0, -1, 3, 2], [6, 7, 8, 9, 2], room([0, 0, -1, 3, 2], [1, 2 * ps, ps + 1, 0, 5]))
    b.release([0, 7])
    b.compact(out_of_place=True)
    b.fork([-1, 9, 6], [0, 7, 10], room([-1, 9, 6], [0, 3, 1]), out_of_place=True)
    b.release([6, 3, 2, 8])
    b.compact()
    b.compact()  # nothing left to move
    b.release(list(range(16)))
    b.compact()  # nothing in use


@pytest.mark.parametrize("out_of_place", [False, True])
def test_compaction_of_rows_wider_than_the_handles(out_of_place):
    """Every held page is renamed and every other column copied, whatever max_row_pages is."""
    from paper_2608_01657_gb300 import kv as KV
    t, l, h, r = rows_in_use(6, 3, 150, 16, 20, 400, 4)
    refs = Pages(t, l, h, r, 20, 16)
    k, v = make_pool(2, 400, 16, 2, 64, BF, seed=4)
    rk, rv = k.clone(), v.clone()
    tables, held, before = dev(t), dev(h), dev(r)
    assert (h > 2).any() and t.shape[1] > h.max()
    pool = KV.KVPool(k, v, num_q_heads=2, first_page=20, max_row_pages=2)
    to, ro = (torch.full_like(tables, 77), torch.full_like(before, 77)) if out_of_place else (None, None)
    counts = pool.compact(tables, held, before, tables_out=to, refs_out=ro)
    pool.check()
    moves, live = refs.compact()
    assert counts.tolist() == [live, len(moves)] and moves
    for a, b in moves:
        rk[:, b], rv[:, b] = rk[:, a], rv[:, a]
    assert np.array_equal((to if out_of_place else tables).cpu().numpy(), refs.tables)
    assert np.array_equal((ro if out_of_place else before).cpu().numpy(), refs.refs)
    assert torch.equal(k, rk) and torch.equal(v, rv)


@pytest.mark.parametrize("out_of_place", [False, True])
def test_compaction_reports_rows_of_impossible_lengths(out_of_place):
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 10, 16, 1, 64, BF)
    pool = KV.KVPool(k, v, num_q_heads=1)
    for held, renamed in ((4, True), (-1, False)):
        t, r = dev([[9, 8, 1]]), dev([0] * 8 + [1, 1])  # nothing moves from the third
        to = torch.full_like(t, 77) if out_of_place else None
        counts = pool.compact(t, dev([held]), r, tables_out=to)
        with pytest.raises(RuntimeError, match="invalid"):
            pool.check()
        assert counts.tolist() == [2, 2]
        assert (to if out_of_place else t).tolist() == [[0, 1, 1] if renamed else [9, 8, 1]]


def test_fork_takes_all_free_pages_or_none():
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 12, 16, 1, 64, BF)
    pool = KV.KVPool(k, v, num_q_heads=1, first_page=2, max_requests=4, max_row_pages=8)
    t, l, h, r = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((4, 8), 4, 4, 10))
    pool.fork(dev([-1, -1]), dev([0, 1]), dev([128, 32]), t, l, h, r)  # all ten
    pool.check()
    assert (r == 1).all() and h.tolist() == [8, 2, 0, 0]
    state = [x.clone() for x in (t, l, h, r, k)]
    out = torch.full_like(r, 5)
    pool.fork(dev([-1]), dev([2]), dev([1]), t, l, h, r, refs_out=out)
    with pytest.raises(RuntimeError, match="capacity"):
        pool.check()
    assert all(torch.equal(a, b) for a, b in zip(state, (t, l, h, r, k))) and torch.equal(out, r)
    pool.fork(dev([-1]), dev([2]), dev([0]), t, l, h, r)  # an empty row needs none
    pool.check()
    pool.fork(dev([]), dev([]), dev([]), t, l, h, r)
    pool.check()


def test_fork_needs_past_32_bits():
    """256 new rows whose needs add up to 2^31 pages of a pool of 30: refused, nothing changes."""
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 30, 2, 1, 8, BF)
    rows, width = 256, 1 << 23
    pool = KV.KVPool(k, v, num_q_heads=1, max_requests=rows, max_row_pages=width)
    t = torch.empty(rows, width, dtype=torch.int32, device="cuda")
    t[:, :4] = -3
    l, h, r = torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.zeros(rows, dtype=torch.int32, device="cuda"), dev([0] * 30)
    pool.fork(dev([-1] * rows), dev(range(rows)), dev([2 * width] * rows), t, l, h, r)
    with pytest.raises(RuntimeError, match="capacity"):
        pool.check()
    assert not r.any() and not l.any() and not h.any() and (t[:, :4] == -3).all()


@pytest.mark.parametrize("parents,children,room", [
    ([4], [1], [1]), ([-2], [1], [1]), ([0], [4], [1]), ([0], [-1], [1]), ([0], [1], [-1]), ([0], [1], [129]),
    ([0, 0], [1, 1], [40, 40]), ([0, 1], [1, 2], [40, 40]), ([0, 0], [0, 1], [60, 40]), ([3], [2], [1])])
def test_bad_forks_change_nothing(parents, children, room):
    """Ranges, doubled children, a child that is a parent, a parent with a page out of range."""
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 40, 16, 1, 64, BF)
    pool = KV.KVPool(k, v, num_q_heads=1, max_requests=4, max_row_pages=8)
    t = dev([[0, 1, 2, -1, -1, -1, -1, -1]] * 3 + [[40, 1, 2, -1, -1, -1, -1, -1]])
    l, h, r = dev([40, 0, 0, 40]), dev([3, 0, 0, 3]), dev([2, 2, 2] + [0] * 37)
    state = [x.clone() for x in (t, l, h, r, k)]
    pool.fork(dev(parents), dev(children), dev(room), t, l, h, r)
    with pytest.raises(RuntimeError, match="invalid"):
        pool.check()
    assert all(torch.equal(a, b) for a, b in zip(state, (t, l, h, r, k)))


def test_bad_releases_are_reported():
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 10, 16, 1, 64, BF)
    pool = KV.KVPool(k, v, num_q_heads=1, max_requests=4, max_row_pages=3)
    for rows, table, refs, after in (([2], [0, 1, 2], [1, 1, 1], [1, 1, 1]), ([0], [0, 10, 2], [1, 1, 1], [0, 1, 0]),
                                     ([0], [0, 1, 2], [1, 0, 1], [0, 0, 0])):
        r = dev(refs + [0] * 7)
        pool.release(dev(rows), dev([table, table]), dev([40, 40]), dev([3, 3]), r)
        with pytest.raises(RuntimeError):
            pool.check()
        assert r[:3].tolist() == after


def test_page_calls_on_a_pool_without_private_pages():
    """The references are an empty array: cached pages are shared, released and left where they are."""
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 8, 16, 1, 64, BF)
    before = k.clone()
    pool = KV.KVPool(k, v, num_q_heads=1, first_page=8, max_requests=4, max_row_pages=4)
    t, l, h, r = dev([[5, 2, 7, -1], [-1] * 4, [-1] * 4]), dev([48, 0, 0]), dev([3, 0, 0]), dev([])
    pool.fork(dev([0, -1]), dev([1, 2]), dev([48, 0]), t, l, h, r)
    pool.check()
    assert t.tolist() == [[5, 2, 7, -1], [5, 2, 7, -1], [-1] * 4] and l.tolist() == [48, 48, 0] and h.tolist() == [3, 3, 0]
    to = torch.full_like(t, 77)
    assert pool.compact(t, h, r, tables_out=to).tolist() == [0, 0] and torch.equal(to, t)
    pool.release(dev([0]), t, l, h, r)
    pool.check()
    assert h.tolist() == [0, 3, 0] and torch.equal(k, before)
    pool.fork(dev([1]), dev([1]), dev([49]), t, l, h, r)  # there is no page to grow into
    with pytest.raises(RuntimeError, match="capacity"):
        pool.check()
    assert h.tolist() == [0, 3, 0]


def test_many_forks_of_one_row_and_a_large_pool():
    """More chunks of the reference array than one, more items than CTAs at once."""
    b = Both(3, 500, 400, pages=9000, first=1, layers=1, heads=1, dim=8, seed=8)
    b.fork([i % 3 for i in range(500)], list(range(3, 503)), [int(b.ref.lens[i % 3]) + 1 + i % 40 for i in range(500)])
    b.release(list(range(0, 503, 2)))
    b.compact()


@pytest.mark.parametrize("layout", ["token", "head", "both"])
def test_copy(layout):
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(3, 90, 16, 3, 40, HF, layout)
    want_k, want_v = k.clone(), v.clone()
    perm = np.random.RandomState(1).permutation(90)
    src, dst = perm[:40], perm[40:80]
    want_k[:, dst], want_v[:, dst] = want_k[:, src], want_v[:, src]
    pool = KV.KVPool(k, v, num_q_heads=3)
    pool.copy(dev(src), dev(dst))
    pool.check()
    assert torch.equal(k, want_k) and torch.equal(v, want_v)
    pool.copy(dev([]), dev([]))
    pool.copy(dev([src[0], 90]), dev([dst[1], 0]))
    with pytest.raises(RuntimeError):
        pool.check()
    want_k[:, dst[1]] = want_k[:, src[0]]
    assert torch.equal(k, want_k)


def test_page_refusals():
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 10, 16, 1, 64, BF)
    pool = KV.KVPool(k, v, num_q_heads=1, first_page=4, max_requests=2, max_row_pages=3)
    t, l, h, r = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((2, 3), 2, 2, 6))
    one = dev([0])
    for bad in (dict(refs=torch.zeros(10, dtype=torch.int32, device="cuda")), dict(lens=l.long()), dict(held=h[:1]),
                dict(tables=t.t()), dict(room=dev([1, 2]))):
        args = dict(parents=one, children=one, room=one, tables=t, lens=l, held=h, refs=r) | bad
        with pytest.raises(ValueError):
            pool.fork(**args)
    with pytest.raises(RuntimeError):
        pool.fork(dev([0, 0, 0]), dev([0, 1, 0]), dev([0, 0, 0]), t, l, h, r)  # over max_requests
    with pytest.raises(ValueError):
        pool.copy(dev([0]), dev([0, 1]))
    with pytest.raises(ValueError):
        pool.compact(t, h, r, tables_out=t[:1])


def test_shifted_outputs_of_page_calls_are_refused():
    """References and tables go to their own place or to another one, not to one that overlaps it."""
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 10, 16, 1, 64, BF)
    pool = KV.KVPool(k, v, num_q_heads=1, first_page=4, max_requests=2, max_row_pages=3)
    t, h, l = torch.zeros(4, 3, dtype=torch.int32, device="cuda"), dev([0, 0]), dev([0, 0])
    both, one = dev([0] * 13), dev([0])
    refs = both[:6]
    for shift in (1, 5):
        with pytest.raises(RuntimeError, match="invalid"):
            pool.fork(one, one, one, t[:2], l, h, refs, refs_out=both[shift:shift + 6])
        with pytest.raises(RuntimeError, match="invalid"):
            pool.compact(t[:2], h, refs, refs_out=both[shift:shift + 6])
    with pytest.raises(RuntimeError, match="invalid"):
        pool.compact(t[:2], h, refs, tables_out=t[1:3])
    with pytest.raises(RuntimeError, match="invalid"):
        pool.compact(t[1:3], h, refs, tables_out=t[:2])
    pool.fork(one, one, dev([17]), t[:2], l, h, refs, refs_out=both[6:12])
    pool.compact(t[:2], h, both[6:12], tables_out=t[2:])
    pool.check()
    assert t.tolist() == [[4, 5, 0], [0, 0, 0]] * 2


# ---- the step's blocks ---------------------------------------------------------------
@pytest.mark.parametrize("policy", ["lru", "s3fifo", "prefixshield", "staticquota"])
def test_step_blocks_against_the_pool_state(policy):
    """Row i lists, for each leading resident block of request i, the block whose (group, key) is the position's."""
    import oracle as O
    from paper_2608_01657_gb300 import binding as B
    from paper_2608_01657_gb300 import workloads as W
    wl = W.make_workload(0, seed=11)
    sp = wl.spec
    c = B.Cache(sp.capacity_blocks, sp.block_size, sp.num_groups, policy, B.Params(rho=sp.rho, beta=sp.beta),
                max_requests=sp.requests_per_step, max_tokens=32768)
    for st in wl.steps(8):
        groups = torch.from_numpy(st.groups).cuda()
        assert c.step(st.now, groups, torch.from_numpy(st.offsets).cuda(), torch.from_numpy(st.tokens).cuda()) == 0
        R = st.num_requests
        width = int(np.max(np.diff(st.offsets)) // sp.block_size) + 1
        tables = torch.full((R, width), -5, dtype=torch.int32, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        counts = c.step_blocks(groups, tables, status=status).cpu().numpy()
        assert int(status) == 0
        e = c.export()
        where = {(int(g), int(k)): b for b, (r, g, k) in enumerate(zip(e["resident"], e["group"], e["key"])) if r}
        res = c.fetch(R)
        t = tables.cpu().numpy()
        for i in range(R):
            keys = O.chain_keys(c.params.hash_seed, int(st.groups[i]), sp.block_size, st.tokens[st.offsets[i]:st.offsets[i + 1]])
            want = []
            for key in keys:
                b = where.get((int(st.groups[i]), int(key)))
                if b is None:
                    break
                want.append(b)
            assert counts[i] == len(want) and t[i, :len(want)].tolist() == want
            assert (t[i, len(want):] == -5).all()
            mine = res["admitted_ids"][res["admitted_offsets"][i]:res["admitted_offsets"][i + 1]]
            assert set(mine.tolist()) <= set(want) or len(want) < len(keys)
        narrow = torch.full((R, 1), -5, dtype=torch.int32, device="cuda")
        short = c.step_blocks(groups, narrow, status=status).cpu().numpy()
        assert np.array_equal(short, np.minimum(counts, 1))
        assert (int(status) == B.PS_ERR_CAPACITY) == bool((counts > 1).any())


def test_step_blocks_after_a_failed_step():
    from paper_2608_01657_gb300 import binding as B
    c = B.Cache(64, 16, 2, "lru", B.Params(), max_requests=4, max_tokens=1024)
    offs = torch.tensor([0, 64], device="cuda")
    toks = torch.arange(64, dtype=torch.int32, device="cuda")
    g = dev([5])  # no such group
    assert c.step(1, g, offs, toks) == 0
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    tables = torch.zeros(1, 4, dtype=torch.int32, device="cuda")
    assert c.step_blocks(g, tables, status=status).tolist() == [0] and int(status) == B.PS_ERR_INVALID_ARG
    with pytest.raises(RuntimeError):
        c.step_blocks(dev([0] * 5), torch.zeros(5, 4, dtype=torch.int32, device="cuda"))


def test_step_blocks_needs_a_step_of_so_many_requests():
    """What no step wrote is not read: refused on the host."""
    from paper_2608_01657_gb300 import binding as B
    c = B.Cache(64, 16, 2, "lru", B.Params(), max_requests=8, max_tokens=1024)
    toks = torch.arange(64, dtype=torch.int32, device="cuda")
    offs = torch.tensor([0, 32, 64], device="cuda")
    groups, tables = dev([0, 1, 0]), torch.zeros(3, 4, dtype=torch.int32, device="cuda")

    def refused(n):
        with pytest.raises(RuntimeError):
            c.step_blocks(groups[:n], tables[:n])

    refused(1)  # no step yet
    assert c.step_blocks(groups[:0], tables[:0]) is not None
    assert c.step(1, groups[:2], offs, toks) == 0
    refused(3)  # the step had two requests
    assert c.step_blocks(groups[:2], tables[:2]).tolist() == [2, 2]
    assert c.step_blocks(groups[:1], tables[:1]).tolist() == [2]
    c.cached_prefix(groups[:2], offs, toks)
    refused(1)  # the probe's scratch is the step's
    assert c.step(2, groups[:2], offs, toks) == 0
    assert c.step_blocks(groups[:2], tables[:2]).tolist() == [2, 2]
    assert c.reset() == 0
    refused(1)


def test_step_blocks_refuses_wrong_arrays():
    """An array that is too short, or of another type or place, is not handed to the kernel."""
    from paper_2608_01657_gb300 import binding as B
    c = B.Cache(64, 16, 2, "lru", B.Params(), max_requests=8, max_tokens=1024)
    toks = torch.arange(64, dtype=torch.int32, device="cuda")
    offs = torch.tensor([0, 32, 64], device="cuda")
    groups, tables = dev([0, 1]), torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    assert c.step(1, groups, offs, toks) == 0
    for bad in (dict(counts=dev([0])), dict(counts=dev([0, 0], torch.int64)), dict(counts=dev([0] * 4)[::2]),
                dict(groups=groups.long()), dict(groups=groups.cpu()), dict(groups=dev([[0], [1]])),
                dict(status=dev([])), dict(status=dev([0], torch.int64)), dict(counts=torch.zeros(2, dtype=torch.int32)),
                dict(tables=tables[:1]), dict(tables=tables.long())):
        with pytest.raises(ValueError):
            c.step_blocks(**(dict(groups=groups, tables=tables) | bad))
    assert c.step_blocks(groups, tables, counts=dev([7, 7, 7])).tolist() == [2, 2, 7]
