"""Beam search's selection and traces, against their definitions in 64 bits."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
BF, HF, F32 = torch.bfloat16, torch.float16, torch.float32


def dev(a, dtype=torch.int32):
    return torch.tensor(np.array(a), dtype=dtype, device="cuda")


def search(*a, **kw):
    from paper_2608_01657_gb300 import beam
    return beam.BeamSearch(*a, **kw)


def all_scores(logits, scores):
    """[requests, beams, vocab] in 64 bits; -infinity where a token cannot follow or a beam has no candidates."""
    x, c = logits.double(), scores.double()[..., None]
    good = torch.isfinite(c) & ~(torch.isnan(x) | (x == math.inf)).any(-1, keepdim=True) & (x > -math.inf).any(-1, keepdim=True)
    far = x - torch.where(good, x, 0.0).amax(-1, keepdim=True)   # first, so that logits far from 0 lose nothing
    # (sums of columns, so that equal rows' sums are equal to the last bit: those of rows depend on where they lie)
    total = torch.where(good, far, 0.0).exp().movedim(-1, 0).contiguous().sum(0)[..., None]
    p = c + (far - total.log())
    return torch.where(good & (x > -math.inf), p, -math.inf)


def bound(scores, vocab):
    """How far a score may be off.

    Its rounding to 32 bits, 2^-24 of it.  The sum: 2^-22 a term for the exponential;
    the terms' exponents t, rounded once at 2^-24 |t| and off by 1.3e-8 |t| for the
    factor, are ln 2 (2^-24 + 2^-26) E|t| < 2^-24 E|t| of the whole, where the mean E|t|
    over the terms' shares is at most 1 + log2 of their number; the whole numbers, 2^-33
    for each of 1024 lanes' sums and 2^-32 for each of 32 parts', twice, of a sum of 1/2
    at least, 2^-22 + 2^-25; 32-bit additions, 18 of a chunk's terms and one for each of
    a lane's chunks of a part (vocab / 2^15 + 1 at most), also rescaled at 2^-22.  So
    2^-22 (2.2 + (1 + log2 vocab) / 4) + 2^-24 (18 + 5 (vocab / 2^15 + 1)), which is less
    than what is given here."""
    chunks = vocab / 2 ** 13 + 1
    return 2.0 ** -24 * scores.abs() + 2.0 ** -22 * (2 + math.log2(vocab + 1)) + 2.0 ** -24 * (36 + 6 * chunks)


def check(logits, scores, end, got, exact_order=False):
    """exact_order: no two candidates of different beams are nearer than the scores' errors."""
    R, B, V = logits.shape
    p = all_scores(logits, scores)
    tol = bound(torch.where(torch.isfinite(p), p, 0.0).amin((1, 2)), V)
    last = torch.zeros(V, dtype=torch.bool, device="cuda")
    last[list(end)] = True
    for r in range(R):
        flat = p[r].flatten()
        best, at = flat.sort(descending=True, stable=True)
        best, at = best[best > -math.inf], at[best > -math.inf]
        ends = last[at % V]
        go = best[~ends][:B], at[~ends][:B]
        stop = best[:B][ends[:B]], at[:B][ends[:B]]
        for (s, i), tok, par, sc in ((go, got.tokens, got.parents, got.scores), (stop, got.ended_tokens, got.ended_parents, got.ended_scores)):
            if tok is None:
                continue
            n = len(s)
            if exact_order or B == 1:
                assert tok[r, :n].tolist() == (i % V).tolist() and par[r, :n].tolist() == (i // V).tolist()
            elif sc is got.ended_scores:  # an end token at the border may be in or out
                n2 = int((tok[r] >= 0).sum())
                near = best[B - 1] if len(best) >= B else -math.inf
                assert abs(n2 - n) <= int(((best - near).abs() <= 2 * tol[r])[ends].sum())
                n = min(n, n2)
                s = s[:n]
            assert (tok[r, n:] == -1).all() or sc is got.ended_scores
            assert (sc[r, :n].double() - s).abs().le(tol[r]).all()
            flat_at = par[r, :n].long() * V + tok[r, :n]
            assert len(set(flat_at.tolist())) == n and (last[tok[r, :n].long()] == (sc is got.ended_scores)).all()
            assert (flat[flat_at] - s).abs().le(2 * tol[r]).all()
            if sc is got.scores:
                assert (par[r, n:] == -1).all() and (sc[r, n:] == -math.inf).all()


def make(R, B, V, dtype, seed, spread=3.0, masked=0.0):
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn(R, B, V, generator=g, device="cuda") * spread
    if masked:
        x[torch.rand(R, B, V, generator=g, device="cuda") < masked] = -math.inf
    s = -10 * torch.rand(R, B, generator=g, device="cuda")
    return x.to(dtype), s


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("R,B,V", [(1, 1, 1), (2, 1, 7), (1, 3, 2), (3, 4, 31), (2, 32, 33), (5, 5, 1000), (1, 8, 2048), (3, 2, 2049),
                                   (2, 16, 4097), (1, 32, 16384), (2, 7, 16411), (1, 4, 50001), (3, 8, 131072), (1, 1, 300001), (2, 9, 5000), (3, 12, 40001), (1, 17, 3001), (1, 31, 131072),
                                   (2, 32, 70867), (40, 24, 700)])
def test_select(R, B, V, dtype):
    end = sorted({0, V // 2, V - 1} if V > 3 else set())
    x, s = make(R, B, V, dtype, seed=V + B)
    for e in end:
        x[:, :, e] += 9
    h = search(R + 1, B, V, dtype, end)
    got = h.select(x, s)
    h.check()
    check(x, s, end, got)
    again = h.select(x, s)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    # no end tokens: everything goes on, nothing ends
    h = search(R, B, V, dtype)
    got = h.select(x, s, ended=False)
    assert got.ended_tokens is None
    check(x, s, (), got)
    got = h.select(x, s)
    h.check()
    assert (got.ended_tokens == -1).all() and (got.ended_scores == -math.inf).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("offset", [0, 1, 3, 7])
def test_rows_that_begin_anywhere(offset, dtype):
    """Strided, unaligned and expanded logits."""
    R, B, V = 3, 4, 5003
    big, s = make(R, B + 2, V + 20, dtype, seed=offset)
    x = big[:, 1:B + 1, offset:offset + V]
    h = search(R, B, V, dtype, [5])
    got = h.select(x, s[:, :B].contiguous())
    h.check()
    check(x, s[:, :B], [5], got)
    one = x[:, :1].expand(R, B, V)
    got = h.select(one, s[:, :B].contiguous())
    h.check()
    check(one, s[:, :B], [5], got)


@pytest.mark.parametrize("V", [40, 3001, 70000])
def test_equal_logits_go_to_the_lowest_token(V):
    """Few distinct values, beams of powers of two apart: ties are exact within and across beams."""
    R, B = 4, 8
    g = torch.Generator("cuda").manual_seed(V)
    x = torch.randint(0, 3, (R, 1, V), generator=g, device="cuda").float().expand(R, B, V).contiguous()
    s = -torch.randint(0, 2, (R, B), generator=g, device="cuda").float()
    s[1] = -3.0
    for dtype in (BF, F32):
        h = search(R, B, V, dtype, [V // 3, 1])
        got = h.select(x.to(dtype), s)
        h.check()
        check(x, s, [V // 3, 1], got, exact_order=True)
    x[:] = 0.0
    x[:, :, ::2] = -0.0   # equal to 0
    for dtype in (BF, F32):
        h = search(R, B, V, dtype)
        got = h.select(x.to(dtype), s)
        assert (got.tokens[1] == torch.arange(B, device="cuda")).all() and (got.parents[1] == 0).all()
        check(x, s, (), got, exact_order=True)


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("B", [9, 12, 16, 17, 31, 32])
def test_many_beams(B, dtype):
    """Ties, eight end tokens, few candidates, beams that are absent or not finite, where a beam has a warp."""
    R = 8
    for V in (B, 50, 3001, 40001):
        g = torch.Generator("cuda").manual_seed(V + B)
        x = torch.randint(0, 3, (R, 1, V), generator=g, device="cuda").to(dtype).expand(R, B, V).contiguous()
        # (no two different scores are near one another: logits are whole numbers)
        s = -0.37 * torch.randint(0, 2, (R, B), generator=g, device="cuda").float()
        s[1] = -3.0
        end = sorted({0, 1, 5, B - 1, V - 1, V // 2, V // 3, V - 2})
        s[2, 1:] = -math.inf                # a first step
        s[3] = -math.inf
        x[4] = -math.inf
        x[4, B - 1, 3] = 2                  # one candidate in all
        x[5, :, 2:] = -math.inf             # two tokens of every beam
        s[6, B - 1] = 40.0                  # one beam before all others
        h = search(R, B, V, dtype, end)
        got = h.select(x, s)
        h.check()
        check(x, s, end, got, exact_order=True)
        got = search(R, B, V, dtype).select(x, s)
        check(x, s, (), got, exact_order=True)
        x[7, B // 2, V - 1] = math.nan
        s[0, 0] = math.inf
        got = h.select(x, s)
        with pytest.raises(RuntimeError, match="invalid"):
            h.check()
        check(x, s, end, got, exact_order=True)
        assert (got.parents[7] != B // 2).all() and (got.parents[0] != 0).all()


@pytest.mark.parametrize("rising", [True, False])
def test_sorted_logits(rising):
    """Every logit greater than all before it, or less."""
    V, B = 40000, 32
    x = torch.arange(V, device="cuda").float().sub(V).mul(1e-3).expand(2, B, V).contiguous()
    if not rising:
        x = x.flip(-1).contiguous()
    s = -torch.arange(B, device="cuda").float().expand(2, B).contiguous() * 0.37
    h = search(2, B, V, F32, [V - 2, 1])
    got = h.select(x, s)
    h.check()
    check(x, s, [V - 2, 1], got)


@pytest.mark.parametrize("dtype", [BF, HF, F32])
def test_masked_rows_and_absent_beams(dtype):
    R, B, V = 8, 4, 3333
    x, s = make(R, B, V, dtype, seed=6, masked=0.99)
    x[1] = -math.inf                      # nothing may follow
    x[2, :, :] = -math.inf
    x[2, 3, 17] = -5                      # one candidate in all
    x[3, 1:] = -math.inf                  # one beam's candidates
    x[4, :, 9:] = -math.inf
    s[5, 1:] = -math.inf                  # a first step: one beam
    x[5, 2] = math.nan                    # of a beam that is not there: not read
    s[6] = -math.inf
    s[7, 0] = -1e30
    h = search(R, B, V, dtype, [17, 3])
    got = h.select(x, s)
    h.check()
    check(x, s, [17, 3], got)
    assert (got.tokens[[1, 2, 6]] == -1).all() and (got.ended_tokens[2, 0], got.ended_parents[2, 0]) == (17, 3)
    assert abs(float(got.ended_scores[2, 0]) - float(s[2, 3])) < 1e-5 and (got.parents[5] <= 0).all()


def test_extreme_logits():
    """The type's ends among the logits, and log-sums far from 0."""
    V, B = 5000, 3
    for dtype, top in ((BF, 3e38), (HF, 65504.0), (F32, 3.4e38)):
        x, s = make(4, B, V, dtype, seed=1)
        x[0, 0, 70] = top
        x[1] = -top                        # masks of the lowest value: all alike
        x[2, :, 100:] = torch.finfo(dtype).min
        x[3, 1] = x[3, 1] / 1000 + 1000
        h = search(4, B, V, dtype)
        got = h.select(x, s, ended=False)
        h.check()
        check(x, s, (), got)


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("at", [0, 1, 2500, 20010])
def test_beams_that_are_not_finite_are_reported(dtype, bad, at):
    R, B, V = 3, 2, 20011
    x, s = make(R, B, V, dtype, seed=2)
    h = search(R, B, V, dtype, [4])
    x[1, 1, at] = bad
    got = h.select(x, s)
    with pytest.raises(RuntimeError, match="beam search.*invalid"):
        h.check()
    check(x, s, [4], got)
    assert (got.parents[1] == 0).all() and (got.parents >= 0).all()
    x[1, 1, at] = 0
    s[2, 0] = bad
    got = h.select(x, s)
    with pytest.raises(RuntimeError, match="invalid"):
        h.check()
    check(x, s, [4], got)
    assert (got.parents[2] == 1).all()
    s[2, 0] = 0
    check(x, s, [4], h.select(x, s))
    h.check()


def test_a_large_batch_and_small_rows():
    """More rows than CTAs at once; a handle for more requests than a call has."""
    for R, B, V, dtype in ((3000, 4, 50, BF), (700, 8, 2500, HF), (1, 1, 100, F32)):
        x, s = make(R, B, V, dtype, seed=R)
        h = search(4000, B, V, dtype, [3])
        got = h.select(x, s)
        h.check()
        rows = list(range(0, R, max(1, R // 40)))
        check(x[rows], s[rows], [3], type(got)(*(t[rows] for t in got)))


@pytest.mark.parametrize("R", [1024, 1100])
def test_absent_beams_of_large_batches(R):
    """Up to 4096 rows, of which those that are not there are left out, and more, of which they are passed over."""
    B, V = 4, 5000
    x, s = make(R, B, V, BF, seed=R)
    g = torch.Generator("cuda").manual_seed(R)
    gone = torch.rand(R, B, generator=g, device="cuda") < 0.6
    gone[:3] = True
    gone[-2:, 1:] = True
    s[gone] = -math.inf
    x[gone] = math.nan
    h = search(R, B, V, BF, [7])
    got = h.select(x, s)
    h.check()
    assert (got.tokens[:3] == -1).all()
    rows = [0, 1, 2, R - 2, R - 1] + list(range(3, R, R // 30))
    check(x[rows], s[rows], [7], type(got)(*(t[rows] for t in got)))
    s[:] = -math.inf
    got = h.select(x, s)
    h.check()
    assert (got.tokens == -1).all() and (got.ended_parents == -1).all() and (got.scores == -math.inf).all()


@pytest.mark.parametrize("R", [31, 65, 3001, 3103, 3777, 4095])
def test_absent_rows_at_every_word_of_the_list(R):
    """Every row has a continuation of its own, so that a row that is taken for another one shows; single rows, up to
    the most of which absent ones are left out, and few of long rows."""
    V = 5000 if R > 100 else 300001
    g = torch.Generator("cuda").manual_seed(R)
    x = torch.zeros(R, 1, V, device="cuda", dtype=BF)
    at = torch.randint(0, V, (R,), generator=g, device="cuda")
    x[torch.arange(R, device="cuda"), 0, at] = 20.0
    s = -torch.rand(R, 1, generator=g, device="cuda")
    for share in (0.0, 0.3, 0.97):
        gone = torch.rand(R, generator=g, device="cuda") < share
        gone[-1] = False
        c = torch.where(gone[:, None], -math.inf, s)
        h = search(R, 1, V, BF)
        got = h.select(x, c)
        h.check()
        assert torch.equal(got.tokens[:, 0], torch.where(gone, -1, at).int()) and torch.equal(got.parents[:, 0], -gone.int())
        check(x[-3:], c[-3:], (), type(got)(*(t[-3:] for t in got)))
        assert (got.scores[gone] == -math.inf).all() and (got.ended_tokens == -1).all()
        want = s[:, 0].double() - math.log1p((V - 1) * math.exp(-20))
        assert (got.scores[:, 0].double() - want)[~gone].abs().max() <= float(bound(want, V).max())


def test_scores_in_place_and_outputs_reused():
    x, s = make(5, 4, 9000, BF, seed=8)
    h = search(5, 4, 9000, BF, [2])
    want = h.select(x, s)
    kept = s.clone()
    out = want._replace(scores=s)
    out = h.select(x, s, out=out)
    h.check()
    check(x, kept, [2], out)
    assert out.scores.data_ptr() == s.data_ptr()


def test_outputs_whose_memory_has_changed():
    """An output of an earlier call is written where its memory is now, and refused if that no longer fits."""
    x, s = make(3, 4, 500, BF, seed=9)
    h = search(3, 4, 500, BF, [2])
    want, out = h.select(x, s), h.select(x, s)
    old = out.tokens.data_ptr()
    out.tokens.set_(torch.full((3, 4), -7, dtype=torch.int32, device="cuda"))
    assert out.tokens.data_ptr() != old
    got = h.select(x, s, out=out)
    h.check()
    assert got is out and all(torch.equal(a, b) for a, b in zip(out, want))
    out.scores.set_(torch.zeros(2, 4, device="cuda"))
    with pytest.raises(ValueError):
        h.select(x, s, out=out)


def test_rows_far_apart():
    """A request's and a beam's logits past the 32-bit offsets of a buffer of 8.6 GB."""
    V, far = 3001, (1 << 31) + 8 * 5
    flat = torch.empty(2 * far + V, dtype=BF, device="cuda")
    x = flat.as_strided((2, 2, V), (far, far, 1))  # (request 0's second beam is request 1's first)
    y, s = make(2, 2, V, BF, seed=4)
    x[0, 0], x[1, 0], x[1, 1] = y[0, 0], y[1, 0], y[1, 1]
    h = search(2, 2, V, BF, [9])
    got = h.select(x, s)
    h.check()
    check(x.contiguous(), s, [9], got)


def test_select_refusals():
    x, s = make(2, 3, 100, BF, seed=1)
    h = search(2, 3, 100, BF, [1])
    good = h.select(x, s)
    for bad in (dict(logits=x.float()), dict(logits=x[:, :2]), dict(logits=x[..., :50]), dict(logits=x[..., ::1].transpose(0, 1)),
                dict(scores=s.double()), dict(scores=s[:1]), dict(scores=s.t()), dict(logits=x.cpu()), dict(logits=x.flatten(0, 1)),
                dict(out=good._replace(tokens=good.tokens.long())), dict(out=good._replace(scores=good.scores[:1]))):
        with pytest.raises(ValueError):
            h.select(**(dict(logits=x, scores=s) | bad))
    flat = x.view(-1).view(torch.int32)
    shifted = torch.empty(20, device="cuda")
    for bad in (dict(out=good._replace(tokens=good.parents)), dict(out=good._replace(ended_scores=good.scores)),
                dict(out=good._replace(ended_tokens=None)), dict(out=good._replace(tokens=flat[:6].view(2, 3))),
                dict(scores=shifted[:6].view(2, 3), out=good._replace(scores=shifted[3:9].view(2, 3)))):
        with pytest.raises(RuntimeError):
            h.select(**(dict(logits=x, scores=s) | bad))
    big, bs = make(3, 3, 100, BF, seed=1)
    with pytest.raises(RuntimeError):
        h.select(big, bs)
    none = h.select(x[:0], s[:0])
    assert none.tokens.shape == (0, 3)
    h.check()
    for bad in (dict(dtype=torch.float64), dict(beams=33), dict(end_tokens=[100]), dict(end_tokens=[1, 1]), dict(vocab=0),
                dict(end_tokens=range(9)), dict(max_requests=0)):
        with pytest.raises(ValueError):
            search(**(dict(max_requests=2, beams=3, vocab=100) | bad))


def test_select_is_captured_and_replayed():
    R, B, V = 3, 4, 20000
    x, s = make(R, B, V, BF, seed=3)
    h = search(R, B, V, BF, [7])
    out = h.select(x, s)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        h.select(x, s, out=out)
    for seed in range(4, 7):
        y, t = make(R, B, V, BF, seed=seed)
        x.copy_(y), s.copy_(t)
        g.replay()
        h.check()
        check(x, s, [7], out)


def test_select_on_another_stream():
    R, B, V = 2, 4, 3000
    x, s = make(R, B, V, BF, seed=3)
    st = torch.cuda.Stream()
    h = search(R, B, V, BF, [7])
    want = h.select(x, s)
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        torch.cuda._sleep(200_000_000)
    y = x.clone()
    torch.cuda.current_stream().synchronize()
    where = y.data_ptr()
    got = h.select(y, s, stream=st)
    del y
    assert not st.query() and torch.empty_like(x).data_ptr() != where
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    h.check()


# ---- traces ---------------------------------------------------------------------
def trace_plain(tokens, parents, beams, lengths):
    T, R, B = tokens.shape
    out = np.full((R, beams.shape[1], T), -1, np.int64)
    for r in range(R):
        for h in range(beams.shape[1]):
            b, L = beams[r, h], T if lengths is None else lengths[r, h]
            for t in range(L - 1, -1, -1):
                if b < 0:
                    break
                out[r, h, t] = tokens[t, r, b]
                b = parents[t, r, b]
                if not 0 <= b < B and t > 0:
                    break
    return out


@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 63, 500, 511, 512, 513, 1024, 1537])
@pytest.mark.parametrize("R,B,N", [(1, 1, 1), (3, 4, 4), (2, 32, 5), (2, 5, 70)])
def test_trace(T, R, B, N):
    r = np.random.RandomState(T + B)
    tokens, parents = r.randint(0, 1 << 30, (T, R, B)), r.randint(0, B, (T, R, B))
    parents[0] = r.randint(-50, 50, (R, B))  # the first step's lead nowhere
    beams, lengths = r.randint(-1, B, (R, N)), r.randint(0, T + 1, (R, N))
    h = search(R, B, 100)
    for ln in (None, lengths, np.minimum(lengths, 1)):
        got = h.trace(dev(tokens), dev(parents), dev(beams), lengths=None if ln is None else dev(ln))
        h.check()
        assert (got.cpu().numpy() == trace_plain(tokens, parents, beams, ln)).all()


@pytest.mark.parametrize("T,B,N", [(1537, 32, 64), (1537, 31, 1), (900, 4, 64), (129, 5, 7)])
def test_traces_of_every_length(T, B, N):
    """Hypotheses that end at every step, those at the borders of what fits into shared memory among them."""
    r = np.random.RandomState(T + B)
    R = T // N + 1
    tokens, parents = r.randint(0, 1 << 24, (T, R, B)), r.randint(0, B, (T, R, B))
    beams, lengths = r.randint(0, B, (R, N)), np.minimum(np.arange(R * N), T).reshape(R, N)
    h = search(R, B, 100)
    got = h.trace(dev(tokens), dev(parents), dev(beams), lengths=dev(lengths))
    h.check()
    assert (got.cpu().numpy() == trace_plain(tokens, parents, beams, lengths)).all()


def test_bad_traces_are_reported():
    T, R, B, N = 100, 2, 3, 4
    r = np.random.RandomState(1)
    tokens, parents = r.randint(0, 1000, (T, R, B)), r.randint(0, B, (T, R, B))
    beams, lengths = r.randint(0, B, (R, N)), np.full((R, N), T)
    h = search(R, B, 100)
    for what in ("beam", "beam below", "length", "length below", "parent", "parent below", "parent unused"):
        p, b, ln = parents.copy(), beams.copy(), lengths.copy()
        if what == "beam": b[1, 2] = B                   # noqa: E701
        elif what == "beam below": b[1, 2] = -2          # noqa: E701
        elif what == "length": ln[1, 2] = T + 1          # noqa: E701
        elif what == "length below": ln[1, 2] = -1       # noqa: E701
        elif what == "parent": p[70, 1] = B              # noqa: E701
        elif what == "parent below": p[70, 1] = -1       # noqa: E701
        else:
            ln[:] = 40
            p[70, 1] = -1
        want = trace_plain(tokens, p, np.where(b >= B, -1, b), np.where((ln > T) | (ln < 0), 0, ln))
        got = h.trace(dev(tokens), dev(p), dev(b), lengths=dev(ln))
        if what == "parent unused":
            h.check()
        else:
            with pytest.raises(RuntimeError, match="invalid"):
                h.check()
        assert (got.cpu().numpy() == want).all(), what


def test_traces_captured_and_on_another_stream():
    T, R, B, N = 700, 3, 5, 4
    h = search(R, B, 100)
    r = np.random.RandomState(17)
    new = lambda: [dev(r.randint(*a)) for a in ((0, 100, (T, R, B)), (0, B, (T, R, B)), (-1, B, (R, N)), (0, T + 1, (R, N)))]  # noqa: E731
    arrays = new()
    out = h.trace(*arrays)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        h.trace(*arrays, out=out)
    for _ in range(3):
        for a, b in zip(arrays, new()):
            a.copy_(b)
        g.replay()
        h.check()
        assert np.array_equal(out.cpu().numpy(), trace_plain(*(a.cpu().numpy() for a in arrays)))
    st = torch.cuda.Stream()
    copies = [a.clone() for a in arrays]
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        torch.cuda._sleep(100_000_000)
    got = h.trace(*copies, stream=st)
    where = copies[0].data_ptr()
    del copies
    assert not st.query() and torch.empty_like(arrays[0]).data_ptr() != where
    torch.cuda.synchronize()
    assert torch.equal(got, out)


def test_trace_refusals():
    h = search(2, 3, 100)
    t, b = dev(np.zeros((4, 2, 3))), dev(np.zeros((2, 5)))
    for bad in (dict(tokens=t.long()), dict(parents=t[:3]), dict(beams=b[:1]), dict(lengths=b[:, :4]), dict(tokens=t[..., :2]),
                dict(out=dev(np.zeros((2, 5, 3)))), dict(beams=b.t()), dict(beams=b[0])):
        with pytest.raises(ValueError):
            h.trace(**(dict(tokens=t, parents=t.clone(), beams=b) | bad))
    big = dev(np.zeros(100))
    with pytest.raises(RuntimeError):
        h.trace(t, big[:24].view(4, 2, 3), b, out=big[20:60].view(2, 5, 4))
    with pytest.raises(RuntimeError):
        h.trace(dev(np.zeros((4, 3, 3))), dev(np.zeros((4, 3, 3))), dev(np.zeros((3, 1))))
    for shape, n in (((0, 2, 3), 5), ((4, 2, 3), 0), ((4, 0, 3), 5)):
        z = torch.zeros(shape, dtype=torch.int32, device="cuda")
        assert h.trace(z, z.clone(), torch.zeros(shape[1], n, dtype=torch.int32, device="cuda")).shape == (shape[1], n, shape[0])
    h.check()
