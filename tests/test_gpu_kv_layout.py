"""Batches laid out on the GPU, against plain loops: whole numbers, so every value is compared."""
import numpy as np
import pytest
import torch

from _kv_ref import attention, attention_bound, make_pool

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
SHARE_TOKENS, SHARE_ROWS = 128, 64


def dev(a, dtype=torch.int32):
    return torch.tensor(np.asarray(a), dtype=dtype, device="cuda")


def plain(rows, tables, lens, held, T, counts, starts, written, pad, ps, ratio):
    """One request and one token at a time."""
    n, width = len(rows), tables.shape[1]
    start = [int(lens[r]) for r in rows] if starts is None else [int(x) for x in starts]
    count = [1] * n if counts is None else [int(x) for x in counts]
    off, out, pos, slots = [0], np.full((n + pad, width), -1, np.int64), np.zeros(T, np.int64), np.full(T, -1, np.int64)
    for i, r in enumerate(rows):
        kv = start[i] + count[i]
        for k in range(-(-kv // ps)):
            out[i, k] = tables[r, k]
        for j in range(count[i]):
            p = start[i] + j
            pos[off[-1] + j] = p
            if written is None or p >= written[i]:
                slots[off[-1] + j] = int(tables[r, p // ps]) * ps + p % ps
        off.append(off[-1] + count[i])
    lead, groups = -(-SHARE_TOKENS // ps), []
    for i, r in enumerate(rows):
        fit = [start[j] >= SHARE_TOKENS and count[j] * ratio <= SHARE_ROWS for j in (i - 1, i)] if i else [False]
        if not (all(fit) and (tables[r, :lead] == tables[rows[i - 1], :lead]).all()):
            groups.append(i)
    kv = [a + b for a, b in zip(start, count)]
    if pad:
        off, kv, groups = off + [T], kv + [0], groups + [n]
    groups += [n + pad] * (n + pad + 1 - len(groups))
    return off, kv, out, pos, slots, groups


def equal(got, want):
    for a, b in zip(got, want):
        assert a.shape == np.asarray(b).shape and (a.cpu().numpy() == np.asarray(b)).all()


def pool_of(ps, width, requests, tokens, ratio=2, pages=400):
    from paper_2608_01657_gb300 import kv as KV
    k = torch.zeros(1, pages, ps, 2, 8, device="cuda", dtype=BF)
    return KV.KVPool(k, torch.zeros_like(k), num_q_heads=2 * ratio, max_requests=requests, max_tokens=max(1, tokens),
                     max_row_pages=width)


def batch(n, most_before, most_new, ps, seed, spare_rows=2, alike=0.7, pages=400):
    r = np.random.RandomState(seed)
    rows = r.permutation(n + spare_rows)[:n]
    start, count = r.randint(0, most_before + 1, n), r.randint(0, most_new + 1, n)
    width = -(-(most_before + most_new) // ps) + 2
    held, lens = np.zeros(n + spare_rows, np.int64), np.zeros(n + spare_rows, np.int64)
    held[rows] = np.minimum(-(-(start + count) // ps) + r.randint(0, 2, n), width)
    lens[rows] = start
    tables = r.randint(0, pages, (n + spare_rows, width))
    for i in range(1, n):
        if r.rand() < alike:
            k = r.randint(0, width + 1)
            tables[rows[i], :k] = tables[rows[i - 1], :k]
    return rows, tables, lens, held, count, start


@pytest.mark.parametrize("pad,spare", [(False, 0), (False, 5), (True, 0), (True, 131)])
@pytest.mark.parametrize("n,before,new,ps,ratio", [(1, 0, 1, 16, 1), (1, 700, 300, 2, 4), (3, 40, 1, 64, 2), (7, 300, 9, 8, 4),
                                                   (33, 500, 40, 16, 2), (1023, 300, 2, 32, 8), (1024, 200, 3, 16, 1)])
def test_layout(n, before, new, ps, ratio, pad, spare):
    rows, tables, lens, held, count, start = batch(n, before, new, ps, seed=n + ps)
    T = int(count.sum()) + spare
    pool = pool_of(ps, tables.shape[1], n + 1, T, ratio)
    t, ln, h = dev(tables), dev(lens), dev(held)
    got = pool.layout(dev(rows), t, ln, h, T, counts=dev(count), pad=pad)
    pool.check()
    equal(got, plain(rows, tables, lens, held, T, count, None, None, int(pad), ps, ratio))
    # other starts, and tokens that are written already; into the same arrays
    r = np.random.RandomState(n)
    start = np.maximum(start - r.randint(0, 30, n), 0)
    written = start + r.randint(-3, 5, n)
    again = pool.layout(dev(rows), t, ln, h, T, counts=dev(count), starts=dev(start), written=dev(written), pad=pad, out=got)
    pool.check()
    assert again is got
    equal(got, plain(rows, tables, lens, held, T, count, start, written, int(pad), ps, ratio))


@pytest.mark.parametrize("n", [1025, 2048, 5000, 9001])
@pytest.mark.parametrize("pad", [False, True])
def test_layout_of_many_requests(n, pad):
    """More than one CTA scans at once."""
    rows, tables, lens, held, count, start = batch(n, 150, 3, 16, seed=n, alike=0.9)
    T = int(count.sum()) + 7
    pool = pool_of(16, tables.shape[1], n + 1, T, 4)
    for _ in range(2):
        got = pool.layout(dev(rows), dev(tables), dev(lens), dev(held), T, counts=dev(count), pad=pad)
    pool.check()
    equal(got, plain(rows, tables, lens, held, T, count, None, None, int(pad), 16, 4))
    assert got.group_offsets[1:].diff().gt(1).any()  # some groups of several
    off = torch.arange(n + 1 + pad, dtype=torch.int32, device="cuda")
    ones = np.minimum(count, 0) + 1
    held[rows] = np.maximum(held[rows], -(-(start + 1) // 16))
    got = pool.layout(dev(rows), dev(tables), dev(lens), dev(held), n, pad=pad, groups=False)
    pool.check()
    assert got.group_offsets is None
    want = plain(rows, tables, lens, held, n, ones, None, None, int(pad), 16, 4)
    equal(got[:5], want[:5])
    assert pad or torch.equal(got.q_offsets, off)


def test_layout_without_rows_counts_or_requests():
    rows, tables, lens, held, count, start = batch(9, 100, 1, 8, seed=4, spare_rows=0)
    order = np.arange(9)
    held = -(-(lens + 1) // 8)
    pool = pool_of(8, tables.shape[1], 9, 20)
    got = pool.layout(None, dev(tables), dev(lens), dev(held), 9)
    pool.check()
    equal(got, plain(order, tables, lens, held, 9, None, None, None, 0, 8, 2))
    none = dev([], torch.int32)
    for pad, T in ((False, 0), (False, 3), (True, 0), (True, 20)):
        got = pool.layout(none, dev(tables), dev(lens), dev(held), T, pad=pad)
        pool.check()
        equal(got, plain([], tables, lens, held, T, None, None, None, int(pad), 8, 2))
    # requests without tokens
    got = pool.layout(dev(order), dev(tables), dev(lens), dev(held), 0, counts=dev([0] * 9))
    pool.check()
    equal(got, plain(order, tables, lens, held, 0, [0] * 9, None, None, 0, 8, 2))


@pytest.mark.parametrize("n", [5, 1500])
@pytest.mark.parametrize("pad", [False, True])
@pytest.mark.parametrize("what", ["row", "row below", "count", "start", "held", "pages", "tokens", "huge"])
def test_a_batch_out_of_range_is_left_out_whole(what, pad, n):
    rows, tables, lens, held, count, start = batch(n, 60, 3, 16, seed=2)
    T = int(count.sum())
    pool = pool_of(16, tables.shape[1], n + 1, T)
    i = n // 2
    if what == "row": rows[i] = n + 2                   # noqa: E701
    elif what == "row below": rows[i] = -1              # noqa: E701
    elif what == "count": count[i] = -1                 # noqa: E701
    elif what == "start": start[i] = -1                 # noqa: E701
    elif what == "held": held[rows[i]] = tables.shape[1] + 1  # noqa: E701
    elif what == "pages": start[i] = held[rows[i]] * 16 - count[i] + 1  # noqa: E701
    elif what == "huge": count[i] = start[i] = 2 ** 31 - 1  # noqa: E701
    else: T -= 1                                        # noqa: E701
    got = pool.layout(dev(rows), dev(tables), dev(lens), dev(held), T, counts=dev(count), starts=dev(start), pad=pad)
    with pytest.raises(RuntimeError, match="capacity" if what == "tokens" else "invalid"):
        pool.check()
    assert not got.q_offsets.any() and not got.kv_lens.any() and not got.positions.any()
    assert (got.tables == -1).all() and (got.slots == -1).all()
    assert torch.equal(got.group_offsets, torch.arange(n + 1 + pad, dtype=torch.int32, device="cuda"))
    pool.plan(got.q_offsets, got.kv_lens, got.tables, T, group_offsets=got.group_offsets)
    with pytest.raises(RuntimeError, match="invalid"):
        pool.check()


def test_page_ids_out_of_range_are_reported():
    tables = np.array([[3, 400, 5], [1, 2, -1]])
    pool = pool_of(16, 3, 2, 80)
    got = pool.layout(dev([0, 1]), dev(tables), dev([0, 0]), dev([3, 3]), 68, counts=dev([20, 48]))
    with pytest.raises(RuntimeError, match="invalid"):
        pool.check()
    want = plain([0, 1], tables, [0, 0], [3, 3], 68, [20, 48], None, None, 0, 16, 2)
    slots = np.array(want[4])
    slots[16:20] = slots[20 + 32:] = -1
    equal([got.slots, got.positions], [slots, want[3]])


def test_layout_refuses_what_the_host_sees():
    pool = pool_of(16, 4, 4, 10)
    t, ln, h, rows = dev(np.zeros((4, 4))), dev([0] * 4), dev([1] * 4), dev([0, 1])
    good = pool.layout(rows, t, ln, h, 2)
    for bad in (dict(num_tokens=11), dict(rows=dev([0] * 5), num_tokens=5), dict(rows=dev([0] * 4), num_tokens=4, pad=True),
                dict(num_tokens=-1)):
        with pytest.raises((ValueError, RuntimeError)):
            pool.layout(**(dict(rows=rows, tables=t, lens=ln, held=h, num_tokens=2) | bad))
    for bad in (dict(counts=dev([1])), dict(starts=dev([1, 1], torch.int64)), dict(written=dev([1])), dict(held=dev([1])),
                dict(lens=dev([1])), dict(tables=t.t()), dict(rows=dev([0, 1, 2])), dict(pad=True), dict(num_tokens=3)):
        with pytest.raises(ValueError):
            pool.layout(**(dict(rows=rows, tables=t, lens=ln, held=h, num_tokens=2, out=good) | bad))
    # outputs on inputs or on one another
    for bad in (good._replace(tables=t[:2]), good._replace(kv_lens=rows), good._replace(kv_lens=good.positions),
                good._replace(q_offsets=good.tables.view(-1)[:3])):
        with pytest.raises(RuntimeError):
            pool.layout(rows, t, ln, h, 2, out=bad)
    pool.check()


def test_a_padded_layout_is_replayed_planned_and_attended():
    """layout -> append -> plan -> attention in one graph, with counts that change from replay to replay."""
    from paper_2608_01657_gb300 import kv as KV
    ps, heads, ratio, d, n, T = 16, 2, 4, 64, 6, 40
    k, v = make_pool(1, 100, ps, heads, d, BF, seed=3)
    pool = KV.KVPool(k, v, num_q_heads=heads * ratio, max_requests=n + 1, max_tokens=T, max_row_pages=14)
    r = np.random.RandomState(1)
    tables = r.permutation(100)[:n * 14].reshape(n, 14)
    tables[1:4, :9] = tables[0, :9]       # a shared prefix of 144 tokens
    t, lens, held = dev(tables), dev([0] * n), dev([14] * n)
    counts, rows = dev([1] * n), dev(range(n))
    q = torch.randn(T, heads * ratio, d, device="cuda").to(BF)
    nk, nv = (torch.randn(T, heads, d, device="cuda").to(BF) for _ in range(2))
    out = torch.empty_like(q)
    made = pool.layout(rows, t, lens, held, T, counts=counts, pad=True)

    def step():
        pool.layout(rows, t, lens, held, T, counts=counts, pad=True, out=made)
        pool.append(0, q, nk, nv, made.slots, q_out=out)
        pool.plan(made.q_offsets, made.kv_lens, made.tables, T, group_offsets=made.group_offsets)
        pool.attention(0, q, 0.125, out=out)

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for new, before in (([1] * n, [200, 150, 170, 180, 0, 31]), ([0, 7, 3, 1, 20, 9], [144, 150, 160, 144, 3, 47]), ([0] * n, [160] * n)):
        counts.copy_(dev(new))
        lens.copy_(dev(before))
        g.replay()
        pool.check()
        total = sum(new)
        kv = [a + b for a, b in zip(new, before)]
        bounds = np.concatenate([[0], np.cumsum(new)])
        want, _, spread, size = attention(q[:total], k[0], v[0], bounds, kv, t, 0.125, True)
        err = (out[:total].double() - want).abs()
        assert (err <= attention_bound(want, spread, size, BF, d, 230, 6.0)).all()
        assert not out[total:].any()   # the padding sees no key
        for i in range(n):
            for j in range(new[i]):
                p = before[i] + j
                last = [m for m in range(n) for x in range(new[m]) if tables[m, (before[m] + x) // ps] == tables[i, p // ps]
                        and (before[m] + x) % ps == p % ps and (m, x) != (i, j)]
                if not last:
                    assert torch.equal(k[0, tables[i, p // ps], p % ps], nk[bounds[i] + j])


def test_layouts_whose_memory_has_changed():
    """An earlier layout is written where its memory is now, and refused if that no longer fits."""
    pool = pool_of(16, 4, 4, 10)
    args = dev([2, 0]), dev(np.arange(16).reshape(4, 4)), dev([5, 20, 40, 0]), dev([4] * 4), 2
    want, out = pool.layout(*args), pool.layout(*args)
    old = out.slots.data_ptr()
    out.slots.set_(torch.full((2,), -7, dtype=torch.int64, device="cuda"))
    assert out.slots.data_ptr() != old
    assert pool.layout(*args, out=out) is out
    pool.check()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    out.tables.set_(torch.zeros(1, 4, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        pool.layout(*args, out=out)


def test_layout_on_another_stream():
    pool = pool_of(16, 4, 4, 10)
    t, ln, h = dev(np.arange(16).reshape(4, 4)), dev([5, 20, 40, 0]), dev([4] * 4)
    want = pool.layout(dev([2, 0]), t, ln, h, 2)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    block = torch.empty(2, dtype=torch.int32, device="cuda")
    torch.cuda._sleep(100_000_000)
    block.fill_(7)
    where = block.data_ptr()
    del block
    rows = dev([2, 0])
    s.wait_stream(torch.cuda.current_stream())
    got = pool.layout(rows, t, ln, h, 2, stream=s)
    assert where not in [x.data_ptr() for x in got]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
