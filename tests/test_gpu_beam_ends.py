"""What lies past a selection's candidates: every entry of every output, written over what was there before; and sizes past 32 bits."""
import math

import numpy as np
import pytest
import torch

from test_gpu_beam import BF, F32, HF, make, search
from test_gpu_beam_far import strict

pytestmark = pytest.mark.gpu


def over_garbage(h, x, s):
    """Outputs that were full of other values."""
    from paper_2608_01657_gb300 import beam
    shape = tuple(s.shape)
    ints = lambda: torch.full(shape, 77, dtype=torch.int32, device="cuda")  # noqa: E731
    floats = lambda: torch.full(shape, 7.5, device="cuda")  # noqa: E731
    out = beam.Selection(ints(), ints(), floats(), ints(), ints(), floats())
    got = h.select(x, s, out=out)
    assert got is out
    return out


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("B", [1, 2, 5, 8, 9, 12, 17, 31, 32])
def test_exact_ties(B, dtype):
    """Whole numbers as logits: every order is known, and so is how many end tokens there are."""
    R = 8
    for V in sorted({B, B + 1, 50, 3001, 40001}):
        g = torch.Generator("cuda").manual_seed(V + B)
        x = torch.randint(0, 3, (R, 1, V), generator=g, device="cuda").to(dtype).expand(R, B, V).contiguous()
        s = -0.37 * torch.randint(0, 2, (R, B), generator=g, device="cuda").float()
        s[1] = -3.0
        end = sorted({0, V - 1, V // 2, V // 3, min(5, V - 1)})
        s[2, 1:] = -math.inf                # a first step
        s[3] = -math.inf                    # no beam
        x[4] = -math.inf
        x[4, B - 1, V // 2] = 2             # one candidate in all, which ends
        x[5, :, 2:] = -math.inf             # two tokens of every beam
        x[6, :, 1:] = -math.inf             # an end token of every beam and nothing else
        s[7, B - 1] = 40.0                  # one beam before all others
        for ends in (end, [end[0]], []):
            h = search(R, B, V, dtype, ends)
            got = over_garbage(h, x, s)
            h.check()
            strict(x, s, ends, got, exact_order=True)


@pytest.mark.parametrize("dtype", [BF, HF, F32])
@pytest.mark.parametrize("R,B,V", [(2, 1, 7), (3, 4, 31), (2, 32, 33), (5, 5, 1000), (1, 8, 2048), (2, 16, 4097), (3, 3, 50001),
                                   (2, 9, 5000), (3, 12, 40001), (1, 31, 131072), (40, 24, 700), (64, 8, 5001)])
def test_scores_at_random(R, B, V, dtype):
    end = sorted({0, V // 2, V - 1})
    x, s = make(R, B, V, dtype, seed=V + B, masked=0.3)
    x[:, :, end] += 6
    h = search(R, B, V, dtype, end)
    got = over_garbage(h, x, s)
    h.check()
    strict(x, s, end, got)
    s[:, ::2] = -math.inf
    got = over_garbage(h, x, s)
    h.check()
    strict(x, s, end, got)


@pytest.mark.parametrize("B", [3, 11])
def test_beams_that_are_not_finite(B):
    """They are reported, have no candidates, and leave what the others found in place."""
    R, V, end = 4, 5003, [1, 7]
    x, s = make(R, B, V, BF, seed=B)
    x[:, :, end] += 12
    x[0] = math.nan
    x[1, 1:] = math.inf
    s[2, :] = math.nan
    s[3, 0] = math.inf
    h = search(R, B, V, BF, end)
    got = over_garbage(h, x, s)
    with pytest.raises(RuntimeError, match="invalid"):
        h.check()
    strict(x, s, end, got)
    none = np.array([0, 2])
    assert (got.tokens[none] == -1).all() and (got.ended_tokens[none] == -1).all()


def test_sizes_of_more_than_32_bits_are_refused():
    """The library's numbers have 32 bits: 2^32 + 7 is not token 7."""
    from paper_2608_01657_gb300 import kv
    far = 1 << 32
    for bad in (dict(end_tokens=[far + 7]), dict(end_tokens=[1, far + 1]), dict(vocab=far + 100), dict(beams=far + 3), dict(max_requests=far + 2),
                dict(end_tokens=[7 - far])):
        with pytest.raises(ValueError, match="out of range"):
            search(**(dict(max_requests=2, beams=3, vocab=100) | bad))
    h = search(2, 3, 100)
    z = lambda *n: torch.zeros(n, dtype=torch.int32, device="cuda")  # noqa: E731
    for steps, requests, hyps in ((far + 1, 0, 1), (1, 0, far + 1)):
        with pytest.raises(ValueError, match="out of range"):
            h.trace(z(steps, requests, 3), z(steps, requests, 3), z(requests, hyps))
    k = torch.zeros(1, 8, 16, 1, 8, device="cuda", dtype=BF)
    pool = kv.KVPool(k, k.clone(), num_q_heads=1, max_requests=2, max_tokens=8, max_row_pages=2)
    tables, lens, held, refs = z(2, 2), z(2), z(2), z(8)
    with pytest.raises(ValueError, match="out of range"):
        pool.layout(z(1), tables, lens, held, far + 1)
    with pytest.raises(ValueError, match="out of range"):
        pool.reorder(z(1, 1), z(1, 1), tables, lens, held, refs, grow=far)
    assert not held.any()
    pool.check()
