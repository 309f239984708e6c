"""Beam search through the server: layout, append, attention, selection, reordering and traces together."""
import numpy as np
import pytest
import torch

from test_gpu_beam import check, trace_plain
from test_gpu_kv_serving import dense, near

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("beams,end", [(1, ()), (4, (7, 500)), (5, tuple(range(100, 108)))])
def test_every_step_of_a_beam_search(beams, end, monkeypatch):
    """Selections by their definition, states against a dense recomputation, sequences and pages in the end."""
    from paper_2608_01657_gb300 import beam
    from paper_2608_01657_gb300 import serving as S
    s = S.Shape(private_pages=400)
    server = S.Server(s, groups=2, seed=3)
    groups = [0, 0, 1, 1]
    prompts = S.prompts_of(groups, s, 3)
    prompts[1] = prompts[1][:128]   # whole pages: every beam's first token needs a new one
    hidden = server.admit(groups, prompts, room=0)["hidden"]
    seen, states = [], []
    select, forward = beam.BeamSearch.select, S.Server.forward

    def watched(self, logits, scores, **kw):
        got = select(self, logits, scores, **kw)
        seen.append((logits.clone(), scores.clone(), beam.Selection(*(t.clone() for t in got))))
        return got

    def stated(self, rows, start, tokens, counts, *a, **kw):
        x = forward(self, rows, start, tokens, counts, *a, **kw)
        states.append(x)
        return x

    monkeypatch.setattr(beam.BeamSearch, "select", watched)
    monkeypatch.setattr(S.Server, "forward", stated)
    steps, R = 20, len(groups)
    found = server.beam_search(hidden, beams, steps, end)
    server.pool.check()
    assert len(seen) == steps and len(states) == steps - 1
    for logits, scores, got in seen:
        check(logits, scores, end, got)
    for a, b in zip(seen, seen[1:]):
        assert torch.equal(a[2].scores, b[1])
    tokens, parents = (np.stack([x[2][i].cpu().numpy() for x in seen]) for i in (0, 1))
    # the states of the last step's beams, each on its own pages
    whole = trace_plain(tokens[:-1], parents[:-1], np.tile(np.arange(beams), (R, 1)), None)
    for r in range(R):
        for j in range(beams):
            want = dense(server.layers, s, np.concatenate([prompts[r], whole[r, j]]))[-1]
            assert near(states[-1][r * beams + j], want)
    # the answers: among the last beams and the ended ones, by the mean of their log-probabilities
    for r in range(R):
        every = [(float(seen[-1][2].scores[r, j]) / steps, steps, j) for j in range(beams)]
        for t, (_, _, got) in enumerate(seen):
            every += [(float(got.ended_scores[r, j]) / (t + 1), t, int(got.ended_parents[r, j])) for j in range(beams)
                      if int(got.ended_tokens[r, j]) >= 0]
        every.sort(key=lambda x: -x[0])
        for j, (mean, length, last) in enumerate(every[:beams]):
            L = int(found["lengths"][r, j])
            assert abs(float(found["scores"][r, j]) / (L + (L < steps)) - mean) < 1e-5 * abs(mean)
            if j == 0 or abs(every[j - 1][0] - mean) > 1e-4 and (j + 1 == len(every) or abs(every[j + 1][0] - mean) > 1e-4):
                assert L == length
                if length:
                    assert found["sequences"][r, j, :L].tolist() == trace_plain(tokens, parents, np.array([[last]] * R), np.array([[length]] * R))[r, 0, :L].tolist()
            assert (found["sequences"][r, j, L:] == -1).all()
    # every reference is a row's
    held, tables = server.held.cpu().numpy(), server.tables.cpu().numpy()
    refs = np.zeros(s.private_pages, np.int64)
    for i in range(s.max_requests):
        for p in tables[i, :held[i]]:
            if p >= s.cache_blocks:
                refs[p - s.cache_blocks] += 1
    assert (refs == server.refs.cpu().numpy()).all()
    used, _ = server.finish(list(range(R)) + list(range(R, R + R * beams)))
    assert used == 0


def test_one_beam_is_greedy():
    from paper_2608_01657_gb300 import serving as S
    s = S.Shape()
    server = S.Server(s, groups=2, seed=5)
    groups = [0, 1]
    prompts = S.prompts_of(groups, s, 5)
    hidden = server.admit(groups, prompts, room=0)["hidden"]
    found = server.beam_search(hidden, 1, 3)
    first = (hidden @ server.layers.embed.T).float().argmax(1)
    assert found["sequences"][:, 0, 0].tolist() == first.tolist() and (found["lengths"] == 3).all()
    with pytest.raises(RuntimeError, match="running"):
        server.beam_search(hidden, 1, 3)


def test_the_example_searches(capsys):
    from paper_2608_01657_gb300 import serving as S
    S.main()
    text = capsys.readouterr().out
    assert "likeliest answers" in text and "mean log-probabilities" in text
