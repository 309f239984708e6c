"""Attention over KV pages against a plain 64-bit statement of it."""
import math

import numpy as np
import pytest
import torch

from _kv_ref import attention, attention_bound, make_pool

pytestmark = pytest.mark.gpu
BF, HF = torch.bfloat16, torch.float16


def batch(new, kv, prefix, groups, page_size, seed=0, extra_pages=3):
    """Tables of a batch; the requests of a group share its prefix's full pages.

    ``groups``: first requests of the groups; ``prefix``: each group's shared tokens."""
    R = len(new)
    r = np.random.RandomState(seed)
    width = max(1, max(-(-n // page_size) for n in kv)) + 2
    need = R * width + sum(prefix) // page_size + extra_pages
    ids = iter(r.permutation(need))
    tables = np.full((R, width), -7, np.int64)   # never a page
    bounds = list(groups) + [R]
    for g in range(len(groups)):
        shared = [next(ids) for _ in range(prefix[g] // page_size)]
        for i in range(bounds[g], bounds[g + 1]):
            n = -(-kv[i] // page_size)
            row = (shared + [next(ids) for _ in range(n)])[:n]
            tables[i, :n] = row
    return tables, need, bounds


def run(new, kv, heads, ratio, dim, page_size, dtype, prefix=None, groups=None, layout="token", causal=True, seed=0,
        scale=None, shared=True, poison=True, stream=None):
    from paper_2608_01657_gb300 import kv as KV
    groups = [0] if groups is None else groups
    prefix = [0] * len(groups) if prefix is None else prefix
    tables, pages, bounds = batch(new, kv, prefix, groups, page_size, seed)
    k, v = make_pool(1, pages, page_size, heads, dim, dtype, layout, seed + 1)
    qo = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = int(qo[-1])
    if poison:  # what no request holds: NaN, and the unwritten end of each last page
        held = torch.zeros(pages, page_size, dtype=torch.bool, device="cuda")
        for i, n in enumerate(kv):
            for t in range(n):
                held[tables[i, t // page_size], t % page_size] = True
        k[0][~held] = float("nan")
        v[0][~held] = float("nan")
    g = torch.Generator("cuda").manual_seed(seed + 2)
    q = torch.randn(T, heads * ratio, dim, generator=g, device="cuda").mul_(1.5).to(dtype)
    scale = dim ** -0.5 if scale is None else scale
    dev = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
    t_dev = dev(tables)
    pool = KV.KVPool(k, v, num_q_heads=heads * ratio, max_requests=len(new), max_tokens=max(1, T),
                     max_row_pages=tables.shape[1])
    out = torch.full((T, heads * ratio, dim), 7.0, dtype=dtype, device="cuda")
    lse = torch.full((T, heads * ratio), 7.0, device="cuda")
    pool.plan(dev(qo), dev(kv), t_dev, T, group_offsets=dev(bounds) if shared else None, causal=causal, stream=stream)
    pool.attention(0, q, scale, out=out, lse=lse, stream=stream)
    pool.check()
    want, want_lse, spread, size = attention(q, k[0], v[0], qo.tolist(), list(kv), t_dev, scale, causal)
    assert torch.isfinite(out.double()).all()
    if T:
        vmax = max([1.0] + [float(v[0][t_dev[i, :-(-n // page_size)].long()].reshape(-1, heads, dim)[:n].abs().max())
                            for i, n in enumerate(kv) if n])
        bound = attention_bound(want, spread, size, dtype, dim, max(max(kv), 1), vmax)
        err = (out.double() - want).abs()
        assert (err <= bound).all(), float((err / bound).max())
        empty = torch.isinf(want_lse)
        assert torch.equal(torch.isinf(lse) & (lse < 0), empty)
        # scores' error, and the sum's: up to the longest row's additions in 32 bits
        lb = dim * 2.0 ** -22 * size + max(max(kv), 1) * 2.0 ** -23 + 2.0 ** -20 * want_lse.abs().nan_to_num(0, 0, 0) + 2.0 ** -19
        assert ((lse.double() - want_lse).abs() <= lb)[~empty].all()
    return pool, q, out, lse


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [8, 40, 64, 72, 80, 96, 104, 128])
def test_head_sizes(dim, dtype):
    run([1, 3, 1, 40], [70, 3, 1, 129], 2, 2, dim, 16, dtype, seed=dim)


@pytest.mark.parametrize("page_size", [2, 4, 8, 16, 32, 64])
@pytest.mark.parametrize("layout", ["token", "head", "both"])
def test_page_sizes_and_layouts(page_size, layout):
    ps = page_size
    run([1, 1, 2, 33], [ps, ps + 1, 5 * ps - 1, 130], 3, 2, 64, ps, BF, layout=layout, seed=ps)


@pytest.mark.parametrize("heads,ratio", [(1, 1), (7, 1), (2, 3), (1, 16), (1, 17), (3, 5), (2, 64)])
def test_head_groups(heads, ratio):
    run([1, 2, 1, 9], [50, 200, 16, 33], heads, ratio, 64, 16, BF, seed=heads * ratio)


@pytest.mark.parametrize("new,kv", [
    ([1], [1]), ([1], [63]), ([1], [64]), ([1], [65]), ([1], [1000]), ([128], [128]), ([129], [129]), ([257], [300]),
    ([1, 0, 1], [5, 9, 0]), ([0], [0]), ([0, 0, 2], [0, 40, 2]), ([4, 4], [0, 0]), ([5, 3], [2, 1]), ([300], [17]),
    ([31, 32, 33, 127], [31, 512, 100, 127]),
])
@pytest.mark.parametrize("causal", [True, False])
def test_lengths_and_empty_rows(new, kv, causal):
    """Rows that see nothing (no keys, or more new tokens than keys) give 0."""
    run(new, kv, 2, 4, 64, 16, BF, causal=causal, seed=len(new))


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("ratio,new", [(1, 1), (4, 1), (8, 1), (4, 5), (4, 16), (4, 17)])
def test_shared_prefix(ratio, new, dtype):
    r = np.random.RandomState(ratio * 100 + new)
    groups, R = [0, 1, 6, 7, 20], 24
    prefix = [256, 640, 1024, 128, 336]
    bounds = groups + [R]
    n = r.randint(1, new + 1, R)
    kv = [prefix[g] + int(r.randint(0, 150)) + int(n[i]) for g in range(5) for i in range(bounds[g], bounds[g + 1])]
    run(n, kv, 2, ratio, 128, 16, dtype, prefix=prefix, groups=groups, seed=new)


def test_shared_prefix_equals_unshared():
    """The grouping changes what is read, not what is computed (within the outputs' own bounds)."""
    args = ([1] * 20, [700 + 13 * i for i in range(20)], 2, 4, 64, 16, BF)
    kw = dict(prefix=[640], groups=[0], seed=4)
    _, _, a, la = run(*args, **kw)
    _, _, b, lb = run(*args, shared=False, **kw)
    assert (a.double() - b.double()).abs().max() <= 2 * 2.0 ** -8 * b.double().abs().max()
    assert (la - lb).abs().max() < 1e-4


def test_groups_that_share_less_than_their_lengths():
    """Tables part ways inside the shorter rows, a member has no queries, another's prefix is all it has."""
    run([1, 0, 1, 1, 2], [400, 320, 321, 1000, 323], 2, 4, 64, 16, BF, prefix=[320], groups=[0], seed=9)
    run([1, 1, 1], [300, 301, 302], 2, 4, 64, 16, BF, prefix=[0], groups=[0], seed=10)
    run([1, 1, 60], [600, 601, 662], 1, 4, 64, 16, BF, prefix=[592], groups=[0], seed=11)
    run([1, 1, 1], [512, 512, 512], 1, 4, 64, 16, BF, prefix=[512], groups=[0], seed=12, causal=False)


@pytest.mark.parametrize("kv", [4097, 20000])
def test_long_rows_are_split(kv):
    run([1, 1], [kv, 3], 1, 8, 128, 16, BF, seed=kv)
    run([200], [kv], 1, 2, 128, 16, BF, seed=kv + 1)


def test_prompts_after_a_cached_prefix():
    run([500, 130, 1, 64], [900, 130, 301, 464], 2, 4, 128, 16, BF, seed=21)
    run([513, 200], [1025, 640], 1, 3, 96, 32, HF, seed=22, layout="head")


@pytest.mark.parametrize("scale", [0.0, -0.3, 4.0])
def test_scales(scale):
    """A scale of 0 averages the values; large scores underflow all weights but a few."""
    run([1, 70], [300, 100], 2, 2, 64, 16, BF, scale=scale, seed=31)


def test_strided_queries_and_outputs():
    from paper_2608_01657_gb300 import kv as KV
    pool, q, out, _ = run([3, 1], [40, 17], 2, 2, 64, 16, BF, seed=41)
    wide = torch.randn(4, 6, 80, device="cuda").to(BF)
    wide[:, 1:5, 8:72] = q
    got = torch.zeros(4, 4, 3, 64, device="cuda", dtype=BF)
    pool.attention(0, wide[:, 1:5, 8:72], 64 ** -0.5, out=got[:, :, 1])
    assert torch.equal(got[:, :, 1], out)
    assert not got[:, :, 0].any() and not got[:, :, 2].any()
    assert KV is not None


def test_same_bits_again_and_on_another_stream():
    args, kw = ([1] * 9 + [70], [2000 + 31 * i for i in range(9)] + [900], 2, 4, 64, 16, BF), dict(prefix=[800], groups=[0], seed=51)
    _, _, a, la = run(*args[:1], args[1], *args[2:], **kw)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        _, _, b, lb = run(*args[:1], args[1], *args[2:], stream=s, **kw)
    s.synchronize()
    assert torch.equal(a, b) and torch.equal(la, lb)


@pytest.mark.parametrize("new", [1, 5])
def test_same_bits_many_times_under_memory_traffic(new):
    """Many short prefixes beside many long rows: loads land in any order, results do not change."""
    from paper_2608_01657_gb300 import kv as KV
    r = np.random.RandomState(3)
    groups, per, ps = 24, 8, 16
    prefix = [ps * int(r.randint(10, 70)) for _ in range(groups)]
    n = [new] * (groups * per)
    kv = [prefix[i // per] + int(r.randint(1, 3000)) + new for i in range(groups * per)]
    tables, pages, bounds = batch(n, kv, prefix, [g * per for g in range(groups)], ps)
    k, v = make_pool(1, pages, ps, 4, 128, BF)
    q = torch.randn(sum(n), 16, 128, device="cuda").to(BF)
    dev = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
    pool = KV.KVPool(k, v, num_q_heads=16, max_requests=len(n), max_tokens=sum(n), max_row_pages=tables.shape[1])
    pool.plan(dev(np.concatenate([[0], np.cumsum(n)])), dev(kv), dev(tables), sum(n), group_offsets=dev(bounds))
    first = pool.attention(0, q, 0.09).clone()
    for _ in range(60):
        outs = [pool.attention(0, q, 0.09) for _ in range(3)]
        assert all(torch.equal(o, first) for o in outs)
    pool.check()


def test_non_finite_values_stay_with_their_rows():
    """A NaN key or value reaches the rows that see it and no others."""
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 40, 16, 1, 64, BF, seed=61)
    tables = torch.arange(40, device="cuda", dtype=torch.int32).view(4, 10)
    kv = torch.tensor([100, 100, 100, 100], dtype=torch.int32, device="cuda")
    qo = torch.arange(5, dtype=torch.int32, device="cuda")
    q = torch.randn(4, 4, 64, device="cuda").to(BF)
    pool = KV.KVPool(k, v, num_q_heads=4, max_requests=4, max_tokens=4, max_row_pages=10)
    k[0, 3, 2] = float("nan")        # a key of request 0
    v[0, 14, 1, 0, 5] = float("inf")  # a value of request 1
    pool.plan(qo, kv, tables, 4)
    out = pool.attention(0, q, 0.125)
    pool.check()
    assert torch.isnan(out[0]).all()
    assert not torch.isfinite(out[1, :, 5]).any() and torch.isfinite(out[1, :, :5]).all()
    assert torch.isfinite(out[2:]).all()


def test_offsets_past_32_bits():
    """Pages beyond 2^31 elements of the pool."""
    from paper_2608_01657_gb300 import kv as KV
    pages = (1 << 31) // (16 * 2 * 64) + 300
    k = torch.empty(1, pages, 16, 2, 64, dtype=BF, device="cuda")
    v = torch.empty_like(k)
    ids = torch.arange(pages - 7, pages, device="cuda")
    g = torch.Generator("cuda").manual_seed(5)
    k[0, ids] = torch.randn(7, 16, 2, 64, generator=g, device="cuda").to(BF)
    v[0, ids] = torch.randn(7, 16, 2, 64, generator=g, device="cuda").to(BF)
    q = torch.randn(33, 4, 64, generator=g, device="cuda").to(BF)
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    for new in (1, 33):
        tables = ids.int().view(1, 7).contiguous()
        pool = KV.KVPool(k, v, num_q_heads=4, max_requests=1, max_tokens=33, max_row_pages=7)
        pool.plan(dev([0, new]), dev([110]), tables, new)
        out = pool.attention(0, q[:new], 0.125)
        pool.check()
        want, _, spread, size = attention(q[:new], k[0], v[0], [0, new], [110], tables, 0.125, True)
        assert ((out.double() - want).abs() <= attention_bound(want, spread, size, BF, 64, 110, 1.0)).all()


@pytest.mark.parametrize("what", ["offset", "last", "length", "page", "negative", "group"])
def test_bad_batches_are_reported_and_write_nothing(what):
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 20, 16, 1, 64, BF)
    pool = KV.KVPool(k, v, num_q_heads=2, max_requests=3, max_tokens=8, max_row_pages=4)
    qo, kv, go = [0, 1, 3, 4], [20, 30, 64], [0, 2, 3]
    tables = np.arange(12).reshape(3, 4)
    if what == "offset":
        qo = [0, 3, 1, 4]
    elif what == "last":
        qo = [0, 1, 3, 5]
    elif what == "length":
        kv = [20, 65, 64]
    elif what == "page":
        tables[2, 3] = 20
    elif what == "negative":
        tables[0, 0] = -1
    else:
        go = [0, 3, 2]
    dev = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
    out = torch.full((4, 2, 64), 3.0, dtype=BF, device="cuda")
    q = torch.randn(4, 2, 64, device="cuda").to(BF)
    pool.plan(dev(qo), dev(kv), dev(tables), 4, group_offsets=dev(go))
    pool.attention(0, q, 0.125, out=out)
    with pytest.raises(RuntimeError, match="invalid argument"):
        pool.check()
    assert (out == 3.0).all()
    # the handle goes on
    pool.plan(dev([0, 1, 3, 4]), dev([20, 30, 64]), dev(np.arange(12).reshape(3, 4)), 4)
    pool.attention(0, q, 0.125, out=out)
    pool.check()
    assert not (out == 3.0).any()


def test_refusals():
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 8, 16, 2, 64, BF)
    pool = KV.KVPool(k, v, num_q_heads=4, max_requests=2, max_tokens=4, max_row_pages=4)
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    q = torch.zeros(4, 4, 64, dtype=BF, device="cuda")
    with pytest.raises(ValueError):
        pool.attention(0, q, 1.0)                                       # no plan
    with pytest.raises(RuntimeError):
        pool.plan(dev([0, 1, 2, 3]), dev([1, 1, 1]), torch.zeros(3, 4, dtype=torch.int32, device="cuda"), 3)  # requests
    with pytest.raises(RuntimeError):
        pool.plan(dev([0, 5]), dev([5]), torch.zeros(1, 4, dtype=torch.int32, device="cuda"), 5)             # tokens
    pool.plan(dev([0, 4]), dev([4]), torch.zeros(1, 4, dtype=torch.int32, device="cuda"), 4)
    for bad in (q.half(), q[:3], torch.zeros(4, 2, 64, dtype=BF, device="cuda"), q.cpu(),
                torch.zeros(4, 4, 68, dtype=BF, device="cuda")[..., 4:]):
        with pytest.raises(ValueError):
            pool.attention(0, bad, 1.0)
    for bad in (math.inf, math.nan):
        with pytest.raises(RuntimeError):
            pool.attention(0, q, bad)
    with pytest.raises(RuntimeError):
        pool.attention(1, q, 1.0)                                       # layer
    for kw in (dict(num_q_heads=3), dict(num_q_heads=4, first_page=-1), dict(num_q_heads=4, max_tokens=0)):
        with pytest.raises(ValueError):
            KV.KVPool(k, v, **kw)
    with pytest.raises(ValueError):
        KV.KVPool(k.float(), v.float(), num_q_heads=4)
    with pytest.raises(ValueError):
        KV.KVPool(*make_pool(1, 8, 16, 2, 136, BF), num_q_heads=4)       # head size
    with pytest.raises(ValueError):
        KV.KVPool(*make_pool(1, 8, 12, 2, 64, BF), num_q_heads=4)        # page size


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("new,kv,ratio,shared", [
    ([3], [40], 4, 0), ([3, 1], [3000, 17], 4, 0),      # narrow tiles, whole and split
    ([20], [70], 4, 0), ([20, 2], [5000, 30], 4, 0),    # wide tiles of one row block
    ([60], [60], 4, 0), ([60], [4000], 4, 0), ([200, 7], [333, 7], 2, 0),  # of two, several
    ([10], [4], 4, 0), ([70], [20], 4, 0),              # rows that see nothing
    ([5, 4, 1], [270, 300, 257], 4, 256),               # after a shared prefix
])
def test_non_finite_values_of_later_tokens(new, kv, ratio, shared, dtype):
    """What a causal row does not see does not reach it: NaN and infinities in later tokens' keys and values."""
    from paper_2608_01657_gb300 import kv as KV
    heads, dim, ps = 2, 72, 16
    tables, pages, bounds = batch(new, kv, [shared], [0], ps, seed=len(new))
    k, v = make_pool(1, pages, ps, heads, dim, dtype, "token", sum(kv))
    r = np.random.RandomState(sum(new))
    for i, n in enumerate(new):  # some of the new tokens
        for j, pos in enumerate(r.permutation(np.arange(max(kv[i] - n, shared), kv[i]))[:3]):
            page, at = int(tables[i, pos // ps]), int(pos % ps)
            v[0, page, at, j % heads, int(r.randint(dim))] = [float("nan"), float("inf"), -float("inf")][j]
            v[0, page, at, j % heads, 71] = float("inf")
            if j == 0:
                k[0, page, at, 1, 5] = float("inf")
    qo = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = int(qo[-1])
    g = torch.Generator("cuda").manual_seed(3)
    q = torch.randn(T, heads * ratio, dim, generator=g, device="cuda").to(dtype)
    dev = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
    pool = KV.KVPool(k, v, num_q_heads=heads * ratio, max_requests=len(new), max_tokens=T, max_row_pages=tables.shape[1])
    pool.plan(dev(qo), dev(kv), dev(tables), T, group_offsets=dev(bounds) if shared else None)
    lse = torch.empty(T, heads * ratio, device="cuda")
    outs = [pool.attention(0, q, 0.1, lse=lse) for _ in range(3)]
    pool.check()
    for o in outs[1:]:
        assert torch.equal(o.view(torch.int16), outs[0].view(torch.int16))
    want, _, spread, size = attention(q, k[0], v[0], qo.tolist(), kv, dev(tables), 0.1, True)
    finite = torch.isfinite(want)
    assert not finite.all() and finite.any()
    assert torch.equal(torch.isfinite(outs[0]), finite)
    bound = attention_bound(want, spread, size, dtype, dim, max(kv), 8.0)
    assert ((outs[0].double() - want).abs() <= bound)[finite].all()


def test_graph_replay_gives_the_same_bits():
    """Append, plan and attention captured in one graph and replayed on new inputs in the same places."""
    from paper_2608_01657_gb300 import kv as KV
    new, kv, heads, ratio, dim, ps = [1, 40, 1, 3], [300, 400, 17, 3], 2, 4, 128, 16
    tables, pages, bounds = batch(new, kv, [256], [0], ps, seed=2)
    T = sum(new)
    qo = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    dev = lambda a, t=torch.int32: torch.tensor(np.asarray(a), dtype=t, device="cuda")  # noqa: E731
    pos = np.concatenate([np.arange(L - n, L) for n, L in zip(new, kv)])
    slots = np.concatenate([[tables[i, p // ps] * ps + p % ps for p in range(L - n, L)] for i, (n, L) in enumerate(zip(new, kv))])
    args = dict(slots=dev(slots, torch.int64), positions=dev(pos), rope=torch.randn(512, dim, device="cuda"))
    where = (dev(qo), dev(kv), dev(tables), dev(bounds))
    k, v = make_pool(1, pages, ps, heads, dim, BF, seed=3)
    pool = KV.KVPool(k, v, num_q_heads=heads * ratio, max_requests=len(new), max_tokens=T, max_row_pages=tables.shape[1])
    g = torch.Generator("cuda").manual_seed(9)
    inputs = [torch.randn(T, h, dim, generator=g, device="cuda").to(BF) for h in (heads * ratio, heads, heads)]
    q2, out = torch.empty_like(inputs[0]), torch.empty_like(inputs[0])

    def call():
        pool.plan(*where[:3], T, group_offsets=where[3])
        pool.append(0, *inputs, q_out=q2, **args)
        pool.attention(0, q2, 0.1, out=out)

    call()  # the kernels are loaded before the capture
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        call()
    for seed in (10, 11):
        g.manual_seed(seed)
        for t in inputs:
            t.copy_(torch.randn(t.shape, generator=g, device="cuda").to(BF))
        graph.replay()
        torch.cuda.synchronize()
        first = out.clone()
        out.zero_()
        call()
        torch.cuda.synchronize()
        assert torch.equal(first, out) and out.float().abs().max() > 0
    pool.check()


def test_attention_before_its_captured_plan_has_run_writes_nothing():
    """A plan that was only captured has divided nothing yet."""
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 12, 16, 2, 64, BF, seed=5)
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    where = dev([0, 1, 21]), dev([40, 60]), torch.arange(8, device="cuda", dtype=torch.int32).view(2, 4)
    q = torch.randn(21, 8, 64, device="cuda").to(BF)
    make = lambda: KV.KVPool(k, v, num_q_heads=8, max_requests=2, max_tokens=21, max_row_pages=4)  # noqa: E731
    first = make()  # the kernels are loaded before the capture
    first.plan(*where, 21)
    want = first.attention(0, q, 0.125)
    pool, out = make(), torch.full_like(want, 7.0)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        pool.plan(*where, 21)
    pool.attention(0, q, 0.125, out=out)
    assert (out == 7.0).all()
    graph.replay()
    pool.attention(0, q, 0.125, out=out)
    pool.check()
    assert torch.equal(out, want)


def test_outputs_on_their_queries_are_refused():
    """An output shares no element with the queries, nor with itself; among them it may lie."""
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 12, 16, 2, 64, BF, seed=5)
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    pool = KV.KVPool(k, v, num_q_heads=4, max_requests=2, max_tokens=21, max_row_pages=4)
    pool.plan(dev([0, 1, 21]), dev([40, 60]), torch.arange(8, device="cuda", dtype=torch.int32).view(2, 4), 21)
    both = torch.randn(23, 8, 64, device="cuda").to(BF)
    q = both[:21, :4]
    want = pool.attention(0, q.clone(), 0.125)
    flat = both.view(-1)
    shifted = torch.as_strided(both, (21, 4, 64), (512, 64, 1), 8)
    steps = torch.as_strided(both, (21, 4, 64), (256, 64, 1), 0)
    before = both.clone()
    for bad in (q, shifted, both[1:22, :4], both[:21, 3:7], steps, flat[:64].expand(21, 4, 64), both[2:3, 4:].expand(21, 4, 64)):
        with pytest.raises(RuntimeError, match="invalid"):
            pool.attention(0, q, 0.125, out=bad)
    assert torch.equal(both, before)
    for good in (both[:21, 4:], both[2:, 4:]):
        assert torch.equal(pool.attention(0, q, 0.125, out=good), want)
    pool.check()


def test_outputs_that_nothing_wrote_are_nan():
    """After a bad plan an output that the call made holds NaN, not what the memory held before."""
    from paper_2608_01657_gb300 import kv as KV
    for dtype, dim, T in ((BF, 128, 300), (HF, 72, 3), (BF, 8, 1)):
        k, v = make_pool(1, 20, 16, 2, dim, dtype)
        dev = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
        pool = KV.KVPool(k, v, num_q_heads=6, max_requests=1, max_tokens=T, max_row_pages=20)
        q = torch.randn(T, 6, dim, device="cuda").to(dtype)
        tables = torch.arange(20, device="cuda", dtype=torch.int32).view(1, 20)
        pool.plan(dev([0, T]), dev([321]), tables, T)
        for stream in (None, torch.cuda.Stream()):
            torch.cuda.synchronize()
            with torch.cuda.stream(stream or torch.cuda.current_stream()):
                del_me = torch.full_like(q, 7.0)
                del del_me
            assert torch.isnan(pool.attention(0, q, 0.1, stream=stream)).all()
        with pytest.raises(RuntimeError):
            pool.check()
        pool.plan(dev([0, T]), dev([320]), tables, T)
        assert torch.isfinite(pool.attention(0, q, 0.1)).all()
        pool.check()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [72, 80])
@pytest.mark.parametrize("new", [20, 70])
def test_finite_rows_are_not_looked_at_again(new, dim, dtype):
    """Tiles that write their own outputs leave no mark in the workspace: none of their numbers is
    taken for one that is not finite, whatever earlier calls left on the SMs."""
    from paper_2608_01657_gb300 import kv as KV
    R, heads, ratio, ps = 40, 8, 3, 16
    dev = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
    tables = torch.arange(R * 8, device="cuda", dtype=torch.int32).view(R, 8)
    offsets, lens = dev(np.arange(R + 1) * new), dev([new + i for i in range(R)])
    for d, fill in ((128, math.nan), (dim, None)):
        k, v = make_pool(1, R * 8, ps, heads, d, dtype, seed=d)
        if fill is not None:
            v.fill_(fill)
        q = torch.randn(R * new, heads * ratio, d, device="cuda").to(dtype)
        pool = KV.KVPool(k, v, num_q_heads=heads * ratio, max_requests=R, max_tokens=R * new, max_row_pages=8)
        pool.workspace.zero_()
        pool.plan(offsets, lens, tables, R * new)
        before = pool.workspace.clone()
        out = pool.attention(0, q, 0.1)
        pool.check()
        assert torch.isnan(out).all() if fill is not None else torch.isfinite(out).all()
    assert torch.equal(pool.workspace, before)


@pytest.mark.parametrize("groups", [None, [0], [0, 0]])
def test_a_batch_of_no_requests(groups):
    """A step in which nobody has anything to say, grouped or not."""
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 8, 16, 2, 64, BF)
    pool = KV.KVPool(k, v, num_q_heads=4, max_requests=2, max_tokens=4, max_row_pages=4)
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    none = torch.zeros(0, 4, dtype=torch.int32, device="cuda")
    pool.plan(dev([0]), dev([]), none, 0, group_offsets=None if groups is None else dev(groups))
    assert pool.attention(0, torch.zeros(0, 4, 64, device="cuda", dtype=BF), 0.125).shape == (0, 4, 64)
    pool.check()
    with pytest.raises(RuntimeError):
        pool.plan(dev([0, 1]), dev([1]), torch.zeros(1, 4, dtype=torch.int32, device="cuda"), 1, group_offsets=dev([0]))
    with pytest.raises(RuntimeError):
        pool.plan(dev([0, 1]), dev([1]), torch.zeros(1, 4, dtype=torch.int32, device="cuda"), 1, group_offsets=dev([0, 0, 1]))


def test_tokens_without_requests_are_refused():
    """On the host: attention of such a batch would run nothing at all."""
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 8, 16, 2, 64, BF)
    pool = KV.KVPool(k, v, num_q_heads=4, max_requests=2, max_tokens=4, max_row_pages=4)
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731
    with pytest.raises(RuntimeError, match="ps_kv_plan"):
        pool.plan(dev([0]), dev([]), torch.zeros(0, 4, dtype=torch.int32, device="cuda"), 3)
    with pytest.raises(ValueError):
        pool.attention(0, torch.zeros(3, 4, 64, device="cuda", dtype=BF), 0.125)
    pool.check()


@pytest.mark.parametrize("new,dim", [(1, 64), (20, 128)])
def test_a_layer_that_is_not_finite_leaves_the_later_ones_alone(new, dim):
    """Its tiles' marks stay until the next plan, but the later calls do not follow them: the plan's
    header is as the plan left it after one finite call."""
    from paper_2608_01657_gb300 import kv as KV
    R, heads, ps = 6, 2, 16
    dev = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
    tables = torch.arange(R * 2, device="cuda", dtype=torch.int32).view(R, 2)
    k, v = make_pool(2, R * 2, ps, heads, dim, BF, seed=dim)
    v[0].fill_(math.nan)
    q = torch.randn(R * new, heads, dim, device="cuda").to(BF)
    pool = KV.KVPool(k, v, num_q_heads=heads, max_requests=R, max_tokens=R * new, max_row_pages=2)
    pool.workspace.zero_()
    pool.plan(dev(np.arange(R + 1) * new), dev([new] * R), tables, R * new)
    before = pool.workspace.clone()
    for finite_calls in (1, 2, 1):
        for layer in [0] + [1] * finite_calls:
            out = pool.attention(layer, q, 0.1)
            assert torch.isfinite(out).all() == (layer == 1) and torch.isnan(out).all() == (layer == 0)
        # a byte for each tile and head
        assert int((pool.workspace != before).sum()) == R * heads
    pool.check()
