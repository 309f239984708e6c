"""The largest calls: vocabularies and rows at their limits, rows of pages past a grid's columns, misaligned steps."""
import math

import numpy as np
import pytest
import torch

from test_gpu_beam import BF, F32, bound, dev, make, search, trace_plain
from test_gpu_beam_far import strict
from test_gpu_kv_reorder import Search

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [1 << 24, (1 << 24) - 2049])
def test_the_largest_vocabulary(V, dtype):
    x, s = make(2, 2, V, dtype, seed=V)
    x[0, 0, -1], x[1, 1, -3] = 40, 35
    got = search(2, 2, V, dtype, [V - 1]).select(x, s)
    strict(x, s, [V - 1], got)
    # sums of as many equal terms: 2^24 of 1, and of the greatest that there are below the border and past it
    for value in (0.0, 2.0 ** 21, -(2.0 ** 21), 1e9, -1e9):
        x.fill_(value)
        h = search(2, 2, V, dtype)
        got = h.select(x, s)
        h.check()
        first = s.argmax(1)
        assert (got.tokens == torch.arange(2, device="cuda")).all() and (got.parents == first[:, None]).all()
        want = s.amax(1, keepdim=True).double() - math.log(V)
        assert ((got.scores - want).abs() <= bound(want, V)).all(), value


@pytest.mark.parametrize("R,B,V", [(1 << 20, 1, 3), (1 << 15, 32, 40), (300000, 3, 9), (20000, 2, 50001)])
def test_the_most_rows(R, B, V):
    """More parts than 32-bit products of shares have room for."""
    g = torch.Generator("cuda").manual_seed(V)
    x = torch.randn(R, B, V, generator=g, device="cuda", dtype=BF)
    at = torch.randint(0, V, (R, B), generator=g, device="cuda")
    x.scatter_(2, at[..., None], 60.0)   # the others have no weight beside it
    s = -torch.rand(R, B, generator=g, device="cuda")
    s[torch.rand(R, B, generator=g, device="cuda") < 0.2] = -math.inf
    h = search(R, B, V, BF)
    got = h.select(x, s)
    h.check()
    best, parent = s.max(1)
    gone = best == -math.inf
    token = torch.where(gone, -1, at.gather(1, parent[:, None])[:, 0])
    assert torch.equal(got.tokens[:, 0], token.int()) and torch.equal(got.parents[:, 0], torch.where(gone, -1, parent).int())
    assert torch.equal(gone, got.scores[:, 0] == -math.inf)
    assert (got.scores[:, 0] - best)[~gone].abs().max() <= float(bound(best.new_ones(()).double(), V))
    rows = [0, 1, R // 2, R - 1]
    strict(x[rows], s[rows], (), type(got)(*(t[rows] for t in got)))


@pytest.mark.parametrize("requests,beams,most,ps", [(1, 3, 40000, 2), (2, 2, 36000, 2)])
def test_rows_of_more_columns_than_a_grid_takes_at_once(requests, beams, most, ps):
    s = Search(requests, beams, most, ps=ps, pages=requests * beams * (most // ps + 8) + 100, first=4, layers=1, heads=1, dim=8, seed=most)
    # (rows whose lengths are drawn: one is the longest)
    assert s.width > 64 * 256
    for grow in (1, 5):
        s.step(s.random_parents(0.1), grow=grow)
    every = np.tile(np.arange(beams), (requests, 1))
    s.step(every[:, ::-1], grow=0)


@pytest.mark.parametrize("off", [1, 2, 3])
def test_steps_that_begin_off_a_word(off):
    T, R, B, N = 700, 2, 4, 5
    r = np.random.RandomState(off)
    tokens, parents = r.randint(0, 1 << 30, (T, R, B)), r.randint(0, B, (T, R, B))
    beams, lengths = r.randint(-1, B, (R, N)), r.randint(0, T + 1, (R, N))
    place = lambda a: torch.cat([dev(np.zeros(off)), dev(a.ravel())])[off:].view(a.shape)  # noqa: E731
    h = search(R, B, 100)
    for t, p in ((place(tokens), dev(parents)), (dev(tokens), place(parents)), (place(tokens), place(parents))):
        got = h.trace(t, p, dev(beams), lengths=dev(lengths))
        h.check()
        assert (got.cpu().numpy() == trace_plain(tokens, parents, beams, lengths)).all()


def test_traces_of_many_requests():
    T, R, B, N = 3, 70001, 2, 3
    r = np.random.RandomState(1)
    tokens, parents = r.randint(0, 1 << 30, (T, R, B)), r.randint(0, B, (T, R, B))
    beams = r.randint(0, B, (R, N))
    got = search(R, B, 100).trace(dev(tokens), dev(parents), dev(beams)).cpu().numpy()
    at, cur = np.arange(R)[:, None], beams
    for t in range(T - 1, -1, -1):
        assert (got[:, :, t] == tokens[t, at, cur]).all()
        cur = parents[t, at, cur]
