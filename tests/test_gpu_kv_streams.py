"""The pool's calls on streams other than the current one."""
import gc

import pytest
import torch

from _kv_ref import make_pool

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


def dev(a, dtype=torch.int32):
    return torch.tensor(a, dtype=dtype, device="cuda")


def busy_block(shape, dtype):
    """Frees a block of memory on which the current stream is still at work; returns its address."""
    t = torch.empty(shape, dtype=dtype, device="cuda")
    torch.cuda._sleep(200_000_000)  # a tenth of a second
    t.fill_(3)
    return t.data_ptr()


def small(first_page=0, **kw):
    from paper_2608_01657_gb300 import kv as KV
    k, v = make_pool(1, 12, 16, 2, 64, BF, seed=5)
    return KV.KVPool(k, v, num_q_heads=8, first_page=first_page, **(dict(max_requests=2, max_tokens=300, max_row_pages=4) | kw))


WHERE = ([0, 1, 21], [40, 60], [[0, 1, 2, 3], [4, 5, 6, 7]])


@pytest.fixture(scope="module", autouse=True)
def kernels_are_loaded():
    """So that no first launch holds a test up while a stream is kept busy."""
    pool = small()
    pool.plan(*(dev(a) for a in WHERE), 21)
    x = torch.zeros(21, 8, 64, device="cuda", dtype=BF)
    pool.append(0, x, x[:, :2], x[:, :2], dev([-1] * 21, torch.int64))
    pool.attention(0, x, 1.0)
    pool.copy(dev([0]), dev([1]))
    pool.check()


@pytest.mark.parametrize("raw", [False, True])
def test_outputs_are_not_memory_that_the_current_stream_still_writes(raw):
    """What a call on another stream makes is that stream's memory."""
    pool = small()
    offsets, lens, tables = (dev(a) for a in WHERE)
    q, kv = torch.randn(21, 8, 64, device="cuda").to(BF), torch.randn(21, 2, 64, device="cuda").to(BF)
    slots = dev(range(150, 171), torch.int64)
    pool.plan(offsets, lens, tables, 21)
    want_q, want = pool.append(0, q, kv, kv, slots), pool.attention(0, q, 0.125)
    held, refs = dev([4, 4]), dev([1] * 8 + [0] * 4)
    s = torch.cuda.Stream()
    on = s.cuda_stream if raw else s
    torch.cuda.synchronize()
    calls = ((want_q, lambda: pool.append(0, q, kv, kv, slots, stream=on)), (want, lambda: pool.attention(0, q, 0.125, stream=on)),
             (dev([8, 0]), lambda: pool.compact(tables, held, refs, stream=on)))
    for right, call in calls:
        torch.cuda.synchronize()
        block = busy_block(right.shape, right.dtype)
        got = call()
        assert got.data_ptr() != block
        torch.cuda.synchronize()
        assert torch.equal(got, right)


def test_workspace_and_status_are_the_streams_own():
    nbytes = small().workspace.numel()
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    blocks = {busy_block(nbytes, torch.uint8), busy_block(1, torch.int32)}
    pool = small(stream=s)
    assert not blocks & {pool.workspace.data_ptr(), pool.status.data_ptr()}
    torch.cuda.synchronize()
    assert int(pool.status) == 0


def test_step_blocks_counts_on_another_stream():
    from paper_2608_01657_gb300 import binding as B
    c = B.Cache(64, 16, 2, "lru", B.Params(), max_requests=8, max_tokens=1024)
    toks = torch.arange(64, dtype=torch.int32, device="cuda")
    groups, tables = dev([0, 1]), torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    assert c.step(1, groups, torch.tensor([0, 32, 64], device="cuda"), toks) == 0
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    block = busy_block(2, torch.int32)
    counts = c.step_blocks(groups, tables, stream=s)
    assert counts.data_ptr() != block
    torch.cuda.synchronize()
    assert counts.tolist() == [2, 2]


@pytest.mark.parametrize("named", [True, False])
def test_a_plans_tensors_outlive_its_attention(named):
    """Temporaries given to a plan stay until the work on its streams is done, the next plan made or not."""
    pool = small(max_row_pages=600)
    q = torch.randn(21, 8, 64, device="cuda").to(BF)
    table = torch.zeros(2, 600, dtype=torch.int32, device="cuda")
    s, other = torch.cuda.Stream(), torch.cuda.Stream()
    for planned_on, run_on in ((s, s), (other, s)):
        torch.cuda.synchronize()
        big = table.clone()
        with torch.cuda.stream(torch.cuda.current_stream() if named else planned_on):
            pool.plan(dev(WHERE[0]), dev(WHERE[1]), big, 21, stream=planned_on if named else None)
        planned_on.synchronize()
        with torch.cuda.stream(run_on):
            torch.cuda._sleep(400_000_000)
        with torch.cuda.stream(torch.cuda.current_stream() if named else run_on):
            pool.attention(0, q, 0.125, stream=run_on if named else None)
        where = big.data_ptr()
        del big
        pool.plan(dev(WHERE[0]), dev(WHERE[1]), table, 21, stream=run_on)
        assert not run_on.query()
        again = torch.empty(2, 600, dtype=torch.int32, device="cuda")
        assert again.data_ptr() != where


def test_a_pool_outlives_its_calls():
    pool = small()
    offsets, lens, tables = (dev(a) for a in WHERE)
    q, s = torch.randn(21, 8, 64, device="cuda").to(BF), torch.cuda.Stream()
    nbytes, where = pool.workspace.numel(), {t.data_ptr() for t in (pool.workspace, pool.status, pool.k, pool.v)}
    shape = pool.k.shape
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        torch.cuda._sleep(400_000_000)
        pool.plan(offsets, lens, tables, 21)
        pool.attention(0, q, 0.125)
    del pool
    gc.collect()
    assert not s.query()
    new = [torch.empty(nbytes, dtype=torch.uint8, device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")]
    new += [torch.empty(shape, dtype=BF, device="cuda") for _ in range(2)]
    assert not where & {t.data_ptr() for t in new}


def test_arguments_of_a_call_that_names_its_stream_outlive_it():
    pool = small()
    offsets, lens, tables = (dev(a) for a in WHERE)
    kv, slots = torch.randn(21, 2, 64, device="cuda").to(BF), dev(range(150, 171), torch.int64)
    s = torch.cuda.Stream()
    pool.plan(offsets, lens, tables, 21)
    calls = (lambda q: pool.append(0, q, kv, kv, slots, stream=s), lambda q: pool.attention(0, q, 0.125, stream=s),
             lambda q: pool.attention(0, kv.repeat_interleave(4, 1), 0.125, out=q, stream=s.cuda_stream))
    for call in calls:
        torch.cuda.synchronize()
        q = torch.zeros(21, 8, 64, device="cuda", dtype=BF)
        where = q.data_ptr()
        with torch.cuda.stream(s):
            torch.cuda._sleep(400_000_000)
        call(q)
        del q
        assert not s.query()
        assert torch.empty(21, 8, 64, device="cuda", dtype=BF).data_ptr() != where
    torch.cuda.synchronize()
    src = dev(range(6))
    where = src.data_ptr()
    with torch.cuda.stream(s):
        torch.cuda._sleep(400_000_000)
    pool.copy(src, dev(range(6, 12)), stream=s)
    del src
    assert not s.query()
    assert dev(range(6)).data_ptr() != where
    torch.cuda.synchronize()
    pool.check()


@pytest.mark.parametrize("named", [True, False])
def test_check_sees_errors_of_calls_on_other_streams(named):
    pool = small()
    x = torch.zeros(1, 8, 64, device="cuda", dtype=BF)
    good, bad = dev([0], torch.int64), dev([12 * 16], torch.int64)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    pool.append(0, x, x[:, :2], x[:, :2], good)
    for _ in range(2):
        with torch.cuda.stream(s):
            torch.cuda._sleep(200_000_000)
            if not named:
                pool.append(0, x, x[:, :2], x[:, :2], bad)
        if named:
            pool.append(0, x, x[:, :2], x[:, :2], bad, stream=s)
        with pytest.raises(RuntimeError, match="invalid argument"):
            pool.check()
        pool.check()
        pool.append(0, x, x[:, :2], x[:, :2], good, stream=s)
        pool.check()
