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


def test_searches_that_are_refused():
    """Before anything is forked: too many rows, fewer tokens that go on than beams, what BeamSearch refuses."""
    from paper_2608_01657_gb300 import serving as S
    s = S.Shape(vocab=6)
    server = S.Server(s, groups=2, seed=5)
    hidden = server.admit([0, 1], S.prompts_of([0, 1], s, 5), room=0)["hidden"]
    held, running = server.held.clone(), set(server.running)
    for bad in (dict(beams=16), dict(beams=5, end=[1, 3]), dict(beams=0), dict(beams=2, end=[6]), dict(beams=2, end=[1, 1]), dict(beams=2, steps=0)):
        with pytest.raises(ValueError):
            server.beam_search(hidden, **(dict(steps=3) | bad))
    assert torch.equal(held, server.held) and running == server.running
    found = server.beam_search(hidden, 4, 3, [1, 3])
    server.pool.check()
    assert found["sequences"].shape == (2, 4, 3)


def test_a_search_without_pages_says_so():
    from paper_2608_01657_gb300 import serving as S
    s = S.Shape()
    server = S.Server(s, groups=2, seed=5)
    hidden = server.admit([0, 1], S.prompts_of([0, 1], s, 5), room=0)["hidden"]
    free = (server.refs == 0).nonzero().flatten()
    server.refs[free[3:]] = 1
    with pytest.raises(RuntimeError, match="capacity"):
        server.beam_search(hidden, 8, 2)


def test_a_captured_step_is_the_eager_one():
    """Selection, the beam step and the layout of what follows, in one graph, step after step."""
    from paper_2608_01657_gb300 import beam
    from paper_2608_01657_gb300 import kv as KV
    R, B, V, ps, pages, width = 3, 4, 3000, 16, 200, 8
    dev = lambda a: torch.tensor(a, dtype=torch.int32, device="cuda")  # noqa: E731

    class Side:
        def __init__(self):
            self.k, self.v = (torch.zeros(1, pages, ps, 1, 64, device="cuda").bfloat16() for _ in range(2))
            self.pool = KV.KVPool(self.k, self.v, num_q_heads=1, max_requests=R * B + 1, max_tokens=64, max_row_pages=width)
            self.search = beam.BeamSearch(R, B, V, end_tokens=[5])
            # every beam with 20 tokens: a page that all beams of a request share and one of its own
            t = np.zeros((R * B, width), np.int64)
            refs = np.zeros(pages, np.int64)
            for i in range(R * B):
                t[i, 0], t[i, 1] = i // B, R + i
                refs[i // B] += 1
                refs[R + i] += 1
            self.t, self.refs = dev(t), dev(refs)
            self.l, self.h = dev([20] * (R * B)), dev([2] * (R * B))
            self.rows = dev(np.arange(R * B).reshape(R, B))
            self.x = torch.zeros(R, B, V, device="cuda").bfloat16()
            self.scores = torch.zeros(R, B, device="cuda")
            self.out, self.at = None, None

        def step(self):
            self.out = self.search.select(self.x, self.scores, out=self.out)
            self.pool.reorder(self.rows, self.out.parents, self.t, self.l, self.h, self.refs)
            self.at = self.pool.layout(self.rows.view(-1), self.t, self.l, self.h, R * B + 3, pad=True, out=self.at)
            self.l += 1
            self.scores.copy_(self.out.scores)

        def all(self):
            return [*self.out, *self.at, self.t, self.l, self.h, self.refs, self.scores]

    eager, graph = Side(), Side()
    g = torch.Generator("cuda").manual_seed(2)
    replay = None
    for i in range(40):
        eager.x.copy_(torch.randn(R, B, V, device="cuda", generator=g))
        graph.x.copy_(eager.x)
        eager.step()
        if i == 1:  # (captured, not run)
            torch.cuda.synchronize()
            replay = torch.cuda.CUDAGraph()
            with torch.cuda.graph(replay):
                graph.step()
        replay.replay() if replay else graph.step()
        for side in (eager, graph):
            side.pool.check()
            side.search.check()
        assert all(torch.equal(a, b) for a, b in zip(eager.all(), graph.all()))
        assert (eager.l == 21 + i).all() and int(eager.refs.sum()) == int(eager.h.sum())


def test_the_example_searches(capsys):
    from paper_2608_01657_gb300 import serving as S
    S.main()
    text = capsys.readouterr().out
    assert "likeliest answers" in text and "mean log-probabilities" in text
