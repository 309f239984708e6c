"""Beam search's selection over logits far from 0, against the definition in 64 bits: masks of finite values, rows
of nothing else, and outliers.  Every candidate has a tolerance of its own score's size, as one of -1e30 says nothing
about the others."""
import math

import pytest
import torch

from test_gpu_beam import BF, F32, HF, all_scores, bound, make, search

pytestmark = pytest.mark.gpu


def strict(logits, scores, end, got, exact_order=False):
    """Every value of every output, what lies past the candidates included.

    exact_order: no two candidates of different scores are nearer than the scores' errors."""
    R, B, V = logits.shape
    p = all_scores(logits, scores)
    last = torch.zeros(V, dtype=torch.bool, device="cuda")
    last[list(end)] = True
    for r in range(R):
        flat = p[r].flatten()
        best, at = flat.sort(descending=True, stable=True)
        some = int((best > -math.inf).sum())
        best, at = best[:some], at[:some]
        ends = last[at % V]
        tol = bound(best, V)

        def same(tok, par, sc, want, places, n):
            assert (tok[n:] == -1).all() and (par[n:] == -1).all() and (sc[n:] == -math.inf).all()
            tok, par, sc, want, places = (x[:n] for x in (tok, par, sc, want, places))
            assert ((tok >= 0) & (tok < V) & (par >= 0) & (par < B)).all()
            if exact_order:
                assert tok.tolist() == (places % V).tolist() and par.tolist() == (places // V).tolist()
            i = par.long() * V + tok
            near = bound(want, V)
            assert len(set(i.tolist())) == n
            assert (sc.double() - want).abs().le(near).all()
            assert (flat[i] - want).abs().le(2 * near).all()
            return i

        go = best[~ends]
        i = same(got.tokens[r], got.parents[r], got.scores[r], go, at[~ends], min(B, len(go)))
        assert not last[i % V].any()
        if got.ended_tokens is None:
            continue
        # an end token is in if fewer than B candidates may come before it, and may be in if fewer than B surely do
        e, te = best[ends], tol[ends]
        must = sum(int((best >= s - 2 * t).sum()) - 1 < B for s, t in zip(e, te))
        may = sum(int((best > s + 2 * t).sum()) < B for s, t in zip(e, te))
        n = int((got.ended_tokens[r] >= 0).sum())
        assert n == int(ends[:B].sum()) if exact_order else must <= n <= min(may, B)
        i = same(got.ended_tokens[r], got.ended_parents[r], got.ended_scores[r], e, at[ends], n)
        assert last[i % V].all()


def select(x, s, end=()):
    R, B, V = x.shape
    h = search(R, B, V, x.dtype, end)
    got = h.select(x, s)
    h.check()
    assert all(torch.equal(a, b) for a, b in zip(got, h.select(x, s)))
    return got


def masks(B, V, seed):
    """Rows of which half or nearly all tokens are masked; blocks: the tail, and 2048 of every 4096 tokens from the
    first on, so that a reader of runs meets masked ones before others."""
    g = torch.Generator("cuda").manual_seed(seed)
    v = torch.arange(V, device="cuda")
    out = torch.stack([(torch.rand(B, V, generator=g, device="cuda") < 0.5), (torch.rand(B, V, generator=g, device="cuda") < 0.99),
                       (v >= V // 10).expand(B, V), (v // 2048 % 2 == 0).expand(B, V), (v < V - V // 20 - 1).expand(B, V)])
    out[:, :, -1] = False   # a token of every row is not masked
    return out


VALUES = [-1e8, -1e9, -1e10, -1e20, -1e30, -1e37, -2e38, -3e38]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,V", [(1, 5000), (8, 5000), (1, 131072), (8, 131072), (32, 131072), (2, 300001)])
def test_rows_with_finite_masks(B, V, dtype):
    for value in VALUES + [-1e4, -3e6, -5e6, -1e7, -1e12]:
        x, s = make(5, B, V, dtype, seed=B + V)
        x = x.masked_fill(masks(B, V, seed=V), value)
        strict(x, s, (), select(x, s))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,V", [(1, 1000), (8, 5000), (32, 5000), (3, 131072)])
def test_rows_of_one_value(B, V, dtype):
    """All logits alike: each token's log-probability is -log V, the tokens come in order, those of the best beam first."""
    for value in VALUES + [-z for z in VALUES] + [2.0 ** 21, -(2.0 ** 21), 2.0 ** 22, -(2.0 ** 22), -5e6, 1e7, 0.0]:
        x = torch.full((2, B, V), value, device="cuda").to(dtype)
        s = -0.5 * torch.arange(B, device="cuda").float().expand(2, B).contiguous()
        got = select(x, s)
        strict(x, s, (), got, exact_order=True)
        want = s.new_full((), -math.log(V))
        assert (got.scores - want).abs().max() <= float(bound(want.double(), V)), value


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,V", [(1, 1000), (8, 5000), (32, 5000), (2, 131072), (9, 131072)])
def test_outliers(B, V, dtype):
    """One logit of a row far above or below the others."""
    for value in (1e8, 1e10, 1e30, 3e38, 5e6, 3e6, 1e5):
        for sign in (1, -1):
            x, s = make(3, B, V, dtype, seed=V + B)
            x[0, :, V // 3] = sign * value
            x[1, B // 2, V - 1] = sign * value
            x[2, :, 0] = sign * value
            x[2, 0, V // 2] = -sign * value
            strict(x, s, (), select(x, s))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("B,V", [(1, 3000), (8, 70001), (12, 40001)])
def test_rows_far_from_zero(B, V, dtype):
    """Where the reference's rounding matters most, on both sides of every border; parts and lanes on either side."""
    for to in (1e5, 1e6, 2.0 ** 21, 2.0 ** 22, 2.0 ** 23, 1e9, 1e30):
        for sign in (1, -1):
            x, s = make(2, B, V, F32, seed=V)
            x = x + sign * to
            x[1, :, :V // 2] -= 40 if to < 1e9 else to / 2 ** 20
            x = x.to(dtype)
            strict(x, s, (), select(x, s))


def test_masks_of_half_precision():
    for value in (-65504.0, -6e4, -1e4):
        for B, V in ((1, 5000), (8, 131072)):
            x, s = make(5, B, V, HF, seed=V)
            x = x.masked_fill(masks(B, V, seed=B), value)
            strict(x, s, (), select(x, s))
            x[0, 0] = value
            strict(x, s, (), select(x, s))


@pytest.mark.parametrize("dtype", [BF, F32])
def test_end_tokens_among_masked_ones(dtype):
    for value in (-1e9, -1e10, -1e30):
        for B, V in ((3, 5000), (8, 131072), (17, 70000)):
            x, s = make(5, B, V, dtype, seed=V)
            x = x.masked_fill(masks(B, V, seed=B), value)
            end = [0, V // 2, V - 1]
            x[:, :, V - 1] += 9
            x[1:, :, V // 2] = value
            strict(x, s, end, select(x, s, end))
