"""The beam step on rows of pages, against a plain statement: all rows let go of
their pages, then each takes those that it continues, one row at a time."""
import numpy as np
import pytest
import torch

from _kv_ref import make_pool

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def dev(a, dtype=torch.int32):
    return torch.tensor(np.array(a), dtype=dtype, device="cuda")


class Search:
    """A pool on the GPU and its plain twin."""

    def __init__(self, requests, beams, most, ps=16, pages=600, first=5, layers=2, heads=2, dim=64, dtype=BF, layout="token",
                 spare=2, seed=0, equal=False):
        from paper_2608_01657_gb300 import kv as KV
        r = np.random.RandomState(seed)
        self.r, self.ps, self.first, self.B = r, ps, first, beams
        n = requests * beams + spare
        self.width = -(-most // ps) + 4
        self.rows = r.permutation(n)[:requests * beams].reshape(requests, beams)
        self.lens, self.held = np.zeros(n, np.int64), np.zeros(n, np.int64)
        self.tables = r.randint(0, pages, (n, self.width))  # what is past the pages held stays
        free = list(first + r.permutation(pages - first))
        for beam_rows in self.rows:
            length = r.randint(1, most + 1)
            full, cached = length // ps, r.randint(0, 4)
            share = r.randint(0, full + 1)
            lead = [int(r.randint(0, first)) if k < cached else free.pop() for k in range(share)]
            for row in beam_rows:
                own = length if equal else r.randint(share * ps, length + 1)
                self.lens[row] = own
                self.held[row] = min(-(-own // ps) + r.randint(0, 2), self.width)
                self.tables[row, :self.held[row]] = lead + [free.pop() for _ in range(self.held[row] - share)]
        self.refs = np.zeros(pages - first, np.int64)
        for i in range(n):
            for p in self.tables[i, :self.held[i]]:
                if p >= first:
                    self.refs[p - first] += 1
        self.refs[free[0] - first] = 3   # a page that something else holds
        self.k, self.v = make_pool(layers, pages, ps, heads, dim, dtype, layout, seed)
        self.rk, self.rv = self.k.clone(), self.v.clone()
        self.pool = KV.KVPool(self.k, self.v, num_q_heads=heads, first_page=first, max_requests=requests * beams, max_row_pages=self.width)
        self.t, self.l, self.h, self.f = dev(self.tables), dev(self.lens), dev(self.held), dev(self.refs)

    def plain(self, parents, grow):
        t, lens, held = self.tables.copy(), self.lens.copy(), self.held.copy()
        for row in self.rows.ravel():
            for p in t[row, :held[row]]:
                if p >= self.first:
                    self.refs[p - self.first] -= 1
        made = []
        for rows, par in zip(self.rows, parents):
            taken = set()
            for j, (row, q) in enumerate(zip(rows, par)):
                if q < 0:
                    self.lens[row] = self.held[row] = 0
                    continue
                src = rows[q]
                n = lens[src]
                have = n // self.ps if q in taken else held[src]
                total = max(have, -(-(n + grow) // self.ps))
                self.tables[row, :have] = t[src, :have]
                for p in t[src, :have]:
                    if p >= self.first:
                        self.refs[p - self.first] += 1
                part = n % self.ps if q in taken else 0
                made.append((row, have, total, t[src, have] if part else 0, part))
                taken.add(q)
                self.lens[row], self.held[row] = n, total
        free = [int(i) for i in np.nonzero(self.refs == 0)[0]][::-1]
        for row, have, total, src, part in made:
            for k in range(have, total):
                page = free.pop()
                self.refs[page] = 1
                self.tables[row, k] = self.first + page
            if part:
                dst = self.tables[row, have]
                self.rk[:, dst, :part], self.rv[:, dst, :part] = self.rk[:, src, :part], self.rv[:, src, :part]

    def step(self, parents, grow=1, out_of_place=False):
        out = torch.full_like(self.f, 77) if out_of_place else None
        self.pool.reorder(dev(self.rows), dev(parents), self.t, self.l, self.h, self.f, grow=grow, refs_out=out)
        self.pool.check()
        if out_of_place:
            self.f = out
        self.plain(np.asarray(parents), grow)
        self.same()

    def same(self):
        assert np.array_equal(self.h.cpu().numpy(), self.held) and np.array_equal(self.l.cpu().numpy(), self.lens)
        assert np.array_equal(self.f.cpu().numpy(), self.refs)
        assert np.array_equal(self.t.cpu().numpy(), self.tables)
        assert torch.equal(self.k, self.rk) and torch.equal(self.v, self.rv)

    def random_parents(self, dead=0.0):
        p = self.r.randint(0, self.B, self.rows.shape)
        return np.where(self.r.rand(*p.shape) < dead, -1, p)


@pytest.mark.parametrize("requests,beams,most,ps,layout,dtype,dim", [
    (1, 1, 40, 16, "token", BF, 64), (1, 4, 100, 16, "token", BF, 64), (3, 5, 60, 8, "head", HF, 80), (7, 2, 90, 2, "both", BF, 8),
    (2, 32, 70, 16, "token", HF, 128), (5, 8, 300, 64, "head", BF, 40)])
@pytest.mark.parametrize("large", [True, False])
def test_beam_steps(requests, beams, most, ps, layout, dtype, dim, large):
    """Steps in a row: identity, permutations, one winner, random, ends, and none left; references of one chunk and of more."""
    s = Search(requests, beams, most, ps, pages=(7000 if ps == 2 else 2500) if large else 2000, layout=layout, dtype=dtype, dim=dim,
               seed=beams)
    every = np.tile(np.arange(beams), (requests, 1))
    s.step(every, grow=0)
    s.step(every[:, ::-1], out_of_place=True)
    s.step(np.full((requests, beams), beams - 1), grow=ps + 1)
    s.step(s.random_parents())
    s.step(s.random_parents(0.4), grow=2 * ps, out_of_place=True)
    s.step(s.random_parents(0.2), grow=0)    # an empty beam may be continued
    s.step(np.full((requests, beams), -1))
    assert not s.held[s.rows].any()
    s.step(every, grow=3)


def test_rows_of_many_columns_and_a_large_pool():
    """More columns than a CTA takes at a time, more chunks of references than one."""
    s = Search(3, 4, 1400, ps=2, pages=9000, first=1, layers=1, heads=1, dim=8, seed=3)
    for grow in (1, 7, 0):
        s.step(s.random_parents(0.1), grow=grow)


def test_many_requests():
    s = Search(300, 3, 30, ps=8, pages=9000, layers=1, heads=1, dim=8, seed=5)
    for _ in range(3):
        s.step(s.random_parents(0.05))


def test_pages_that_a_call_frees_serve_it():
    """A pool with no free page at all: the losers' pages become the winners' copies."""
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 6, 16, 1, 64, BF)
    pool = KV.KVPool(k, v, num_q_heads=1, max_requests=2, max_row_pages=3)
    t, l, h, r = dev([[0, 1, 2], [3, 4, 5]]), dev([40, 41]), dev([3, 3]), dev([1] * 6)
    want = k[0, 5, :9].clone()
    pool.reorder(dev([[0, 1]]), dev([[1, 1]]), t, l, h, r)
    pool.check()
    assert t.tolist() == [[3, 4, 5], [3, 4, 0]] and r.tolist() == [1, 0, 0, 2, 2, 1] and l.tolist() == [41, 41] and h.tolist() == [3, 3]
    assert torch.equal(k[0, 0, :9], want)


def small():
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 12, 16, 1, 64, BF)
    pool = KV.KVPool(k, v, num_q_heads=1, first_page=2, max_requests=4, max_row_pages=4)
    return pool, k, [dev([[2, 3, 4, 0], [2, 3, 5, 0], [6, 7, 0, 0], [0, 1, 8, 0]]), dev([40, 42, 20, 33]), dev([3, 3, 2, 3]),
                     dev([2, 2, 1, 1, 1, 1, 1, 0, 0, 0])]


@pytest.mark.parametrize("out_of_place", [False, True])
@pytest.mark.parametrize("what", ["row", "row below", "twice", "twice elsewhere", "parent", "parent below", "len", "held", "held most",
                                  "id", "id below", "no reference", "wide", "capacity", "references below zero"])
def test_bad_steps_change_nothing(what, out_of_place):
    pool, k, (t, l, h, r) = small()
    rows, parents, grow = [[0, 1], [2, 3]], [[0, 0], [1, 0]], 1
    if what == "row": rows[1][0] = 4                    # noqa: E701
    elif what == "row below": rows[0][1] = -1           # noqa: E701
    elif what == "twice": rows[0][1] = 0                # noqa: E701
    elif what == "twice elsewhere": rows[1][1] = 0      # noqa: E701
    elif what == "parent": parents[0][1] = 2            # noqa: E701
    elif what == "parent below": parents[0][1] = -2     # noqa: E701
    elif what == "len": l[1] = 49                       # noqa: E701
    elif what == "held": h[2] = -1                      # noqa: E701
    elif what == "held most": h[2] = 5                  # noqa: E701
    elif what == "id": t[3, 1] = 12                     # noqa: E701
    elif what == "id below": t[3, 0] = -1               # noqa: E701
    elif what == "no reference": r[4] = 0               # noqa: E701
    elif what == "wide": grow = 30                      # noqa: E701
    elif what == "references below zero":
        r[0], parents = 1, [[-1, -1], [1, 0]]
    else:
        r[7:] = 1
    state = [x.clone() for x in (t, l, h, r, k)]
    if what == "capacity":
        parents = [[0, 1], [0, 0]]   # two new pages, and one of row 3 is freed
        grow = 16
    out = torch.full_like(r, 9) if out_of_place else None
    pool.reorder(dev(rows), dev(parents), t, l, h, r, grow=grow, refs_out=out)
    with pytest.raises(RuntimeError, match="capacity" if what == "capacity" else "invalid"):
        pool.check()
    assert all(torch.equal(a, b) for a, b in zip(state, (t, l, h, r, k)))
    assert out is None or torch.equal(out, r)
    # the handle's own counts are as before: a good step works
    pool, k, (t, l, h, r) = (pool, k, small()[2])
    pool.reorder(dev([[0, 1], [2, 3]]), dev([[0, 0], [1, 0]]), t, l, h, r)
    pool.check()
    assert t.tolist() == [[2, 3, 4, 0], [2, 3, 5, 0], [0, 1, 8, 0], [6, 7, 8, 0]] and l.tolist() == [40, 40, 33, 20]
    assert r.tolist() == [2, 2, 1, 1, 1, 1, 1, 0, 0, 0]


def test_reorder_refusals():
    pool, k, (t, l, h, r) = small()
    rows, parents = dev([[0, 1], [2, 3]]), dev([[0, 0], [1, 0]])
    for bad in (dict(grow=-1), dict(rows=dev([[0, 1, 2, 3, 3]]), parents=dev([[0] * 5])),
                dict(rows=torch.zeros(0, 33, dtype=torch.int32, device="cuda"), parents=torch.zeros(0, 33, dtype=torch.int32, device="cuda")),
                dict(refs_out=t.view(-1)[:10]), dict(lens=t[0], tables=t), dict(held=l), dict(parents=t.view(-1)[2:6].view(2, 2))):
        with pytest.raises(RuntimeError):
            pool.reorder(**(dict(rows=rows, parents=parents, tables=t, lens=l, held=h, refs=r) | bad))
    for bad in (dict(rows=dev([0, 1])), dict(parents=dev([[0, 0]])), dict(rows=dev([[0, 1], [2, 3]], torch.int64)), dict(refs=r[:5]),
                dict(parents=parents.t()), dict(refs_out=dev([0] * 3)), dict(lens=dev([1]))):
        with pytest.raises(ValueError):
            pool.reorder(**(dict(rows=rows, parents=parents, tables=t, lens=l, held=h, refs=r) | bad))
    none = torch.zeros(0, 4, dtype=torch.int32, device="cuda")
    out = torch.zeros_like(r)
    pool.reorder(none, none, t, l, h, r, refs_out=out)
    pool.check()
    assert torch.equal(out, r)


def test_calls_without_requests_lie_between_others():
    """They pass the references on that the call right before them wrote."""
    s = Search(8, 4, 300, pages=4000, seed=13)
    rows, none = dev(s.rows), torch.zeros(0, 4, dtype=torch.int32, device="cuda")
    steps = [s.random_parents() for _ in range(6)]
    parents = [dev(p) for p in steps]
    mid, last = torch.empty_like(s.f), s.f
    for p in parents:
        s.pool.reorder(rows, p, s.t, s.l, s.h, last, refs_out=mid)
        last = torch.empty_like(mid)
        s.pool.reorder(none, none, s.t, s.l, s.h, mid, refs_out=last)
    s.pool.check()
    for p in steps:
        s.plain(p, 1)
    s.f = last
    s.same()


def test_a_pool_without_private_pages():
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 8, 16, 1, 64, BF)
    pool = KV.KVPool(k, v, num_q_heads=1, first_page=8, max_requests=2, max_row_pages=4)
    t, l, h, r = dev([[5, 2, 7, -1], [1, 6, -1, -1]]), dev([48, 32]), dev([3, 2]), dev([])
    pool.reorder(dev([[0, 1]]), dev([[1, 0]]), t, l, h, r, grow=0)
    pool.check()
    assert t.tolist() == [[1, 6, 7, -1], [5, 2, 7, -1]] and l.tolist() == [32, 48] and h.tolist() == [2, 3]
    pool.reorder(dev([[0, 1]]), dev([[1, 0]]), t, l, h, r, grow=1)
    with pytest.raises(RuntimeError, match="capacity"):
        pool.check()
    assert l.tolist() == [32, 48]


def test_reorder_is_captured_and_replayed():
    s = Search(4, 4, 100, seed=9)
    rows, parents = dev(s.rows), dev(s.random_parents())
    s.pool.reorder(rows, parents, s.t, s.l, s.h, s.f)
    s.plain(parents.cpu().numpy(), 1)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.pool.reorder(rows, parents, s.t, s.l, s.h, s.f)
    s.same()
    for _ in range(3):
        p = s.random_parents(0.1)
        parents.copy_(dev(p))
        g.replay()
        s.pool.check()
        s.plain(p, 1)
        s.same()


def test_reorder_on_another_stream():
    s = Search(2, 3, 50, seed=11)
    st = torch.cuda.Stream()
    p = s.random_parents()
    rows, parents = dev(s.rows), dev(p)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        torch.cuda._sleep(100_000_000)
    s.pool.reorder(rows, parents, s.t, s.l, s.h, s.f, stream=st)
    where = parents.data_ptr()
    del parents
    assert not st.query() and dev(p).data_ptr() != where
    s.pool.check()
    s.plain(p, 1)
    s.same()


@pytest.mark.parametrize("name", [-1, -2, 12])
@pytest.mark.parametrize("where", ["first beam", "second beam", "all beams", "after another", "one beam"])
def test_impossible_ids_change_nothing(where, name):
    """In whole pages' columns, whose ids no copy uses; -1, the usual filler of tables, among them."""
    pool, k, (t, l, h, r) = small()
    rows, parents = ([[0], [1], [2], [3]], [[0]] * 4) if where == "one beam" else ([[0, 1], [2, 3]], [[0, 0], [1, 0]])
    at = {"first beam": (0, 0), "second beam": (1, 0), "all beams": (slice(0, 2), 1), "after another": (slice(2, 4), 0), "one beam": (3, 1)}[where]
    t[at] = name
    if where == "after another":   # the beams' ids differ, so that each is looked at
        t[2, 0] = -1 if name != -1 else 13
    state = [x.clone() for x in (t, l, h, r, k)]
    out = torch.full_like(r, 9)
    pool.reorder(dev(rows), dev(parents), t, l, h, r, refs_out=out)
    with pytest.raises(RuntimeError, match="invalid"):
        pool.check()
    assert all(torch.equal(a, b) for a, b in zip(state, (t, l, h, r, k))) and torch.equal(out, r)
    # and the changes that were found by then are forgotten
    t, l, h, r = small()[2]
    pool.reorder(dev([[0, 1], [2, 3]]), dev([[0, 0], [1, 0]]), t, l, h, r)
    pool.check()
    assert r.tolist() == [2, 2, 1, 1, 1, 1, 1, 0, 0, 0]


def test_an_impossible_id_of_a_partly_filled_page_is_not_copied():
    """A row that claims a page more than it has: the id past its own is the filler."""
    pool, k, (t, l, h, r) = small()
    t[:, 3], l[0], h[0] = -1, 50, 4
    state = [x.clone() for x in (t, l, h, r, k)]
    pool.reorder(dev([[0, 1], [2, 3]]), dev([[0, 0], [1, 0]]), t, l, h, r)
    with pytest.raises(RuntimeError, match="invalid"):
        pool.check()
    assert all(torch.equal(a, b) for a, b in zip(state, (t, l, h, r, k)))
