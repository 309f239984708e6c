"""The pool's calls on streams other than the current one."""
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
