"""The operators together: prefix-cache steps, pages, appends, attention, forks
and compaction, against a dense forward pass without any cache."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def dense(layers, s, tokens):
    """Hidden states of one sequence in 32 bits, rounded to bfloat16 where the server does."""
    x = layers.embed[torch.from_numpy(np.asarray(tokens, np.int64)).cuda()]
    n, half = len(tokens), s.head_dim // 2
    c, sn = layers.rope[:n, :half][:, None], layers.rope[:n, half:][:, None]
    for layer in range(s.layers):
        qkv = (x @ layers.qkv[layer].T).float().unflatten(1, (-1, s.head_dim))
        q, k, v = qkv.split([s.q_heads, s.kv_heads, s.kv_heads], 1)

        def turn(t):
            t = t * torch.rsqrt((t * t).mean(-1, keepdim=True) + 1e-6)
            a, b = t[..., :half], t[..., half:]
            return torch.cat([a * c - b * sn, b * c + a * sn], -1).bfloat16().float()

        q, k = turn(q), turn(k)
        rep = s.q_heads // s.kv_heads
        k, v = k.repeat_interleave(rep, 1), v.repeat_interleave(rep, 1)
        score = torch.einsum("qhd,khd->hqk", q, k) * s.head_dim ** -0.5
        score = score.masked_fill(torch.ones(n, n, device="cuda").triu(1).bool(), -torch.inf)
        o = torch.einsum("hqk,khd->qhd", score.softmax(-1), v).bfloat16()
        x = x + o.flatten(1) @ layers.out[layer].T
    return x


def near(got, want):
    """bfloat16 states after two layers: each layer adds a few roundings of 2^-9 of the values' spread."""
    got, want = got.float(), want.float()
    return float((got - want).norm() / want.norm()) < 0.02


@pytest.mark.parametrize("seed", [1, 2])
def test_serving_equals_dense_recomputation(seed):
    from paper_2608_01657_gb300 import serving as S
    s = S.Shape()
    server = S.Server(s, groups=3, seed=seed)
    groups = [0, 0, 0, 1, 1, 2]
    prompts = S.prompts_of(groups, s, seed)
    first = server.admit(groups, prompts, room=0)
    for i, p in enumerate(prompts):
        assert near(first["hidden"][i], dense(server.layers, s, p)[-1])
    server.finish(range(len(groups)))
    # the same system prompts with other questions: the systems' blocks are cached now
    r = np.random.RandomState(seed)
    prompts = [np.concatenate([p[: 128 + 16 * g], r.randint(0, s.vocab, 5 + 9 * i)]) for i, (g, p) in enumerate(zip(groups, prompts))]
    prompts[1] = prompts[1][: 128]  # one whole number of cached blocks: nothing new but the last token
    second = server.admit(groups, prompts, room=0)
    assert second["cached"] >= sum(len(p) // 16 * 16 for p in prompts) // 2
    for i, p in enumerate(prompts):
        assert near(second["hidden"][i], dense(server.layers, s, p)[-1])
    steps = r.randint(0, s.vocab, (3, len(groups), 2)).astype(np.int32)
    out = server.sample(len(groups), 2, steps)
    for i, p in enumerate(prompts):
        for j in range(2):
            want = dense(server.layers, s, np.concatenate([p, steps[:, i, j]]))[-3:]
            assert near(out[:, 2 * i + j], want)
    # free every second sample, move the pages together, decode on
    keep = [len(groups) + k for k in range(0, 12, 2)]
    used, _ = server.finish([len(groups) + k for k in range(1, 12, 2)])
    assert used == int((server.refs > 0).sum()) and bool((server.refs[:used] > 0).all())
    rows = torch.tensor(keep, dtype=torch.int32, device="cuda")
    server.pool.fork(rows, rows, server.lens[rows.long()] + 1, server.tables, server.lens, server.held, server.refs)
    last = r.randint(0, s.vocab, len(keep))
    x = server.forward(rows, server.lens[rows.long()], torch.from_numpy(last.astype(np.int32)).cuda(), [1] * len(keep), [0, len(keep)])
    for i, p in enumerate(prompts):
        assert near(x[i], dense(server.layers, s, np.concatenate([p, steps[:, i, 0], last[i:i + 1]]))[-1])


def test_the_example_runs(capsys):
    from paper_2608_01657_gb300 import serving as S
    S.main()
    text = capsys.readouterr().out
    assert "first batch" in text and "sampled hidden states (4, 15, 256)" in text


def test_no_batch_is_admitted_while_rows_name_cached_pages():
    """Nothing holds a running row's cached pages: the next batch could be given them."""
    from paper_2608_01657_gb300 import serving as S
    s = S.Shape()
    server = S.Server(s, groups=2, seed=1)
    groups = [0, 0, 1]
    prompts, others = S.prompts_of(groups, s, 1), S.prompts_of(groups, s, 2)
    steps = np.zeros((2, 3, 2), np.int32)
    server.admit(groups, prompts, room=0)
    with pytest.raises(RuntimeError, match="running"):
        server.admit(groups, others, room=0)
    before = server.sample(3, 2, steps)
    with pytest.raises(RuntimeError, match="running"):
        server.sample(3, 2, steps)          # the rows hold the first samples
    server.finish(range(3))                 # the samples go on
    with pytest.raises(RuntimeError, match="running"):
        server.admit(groups, others, room=0)
    server.finish(range(3, 9))
    assert not server.refs.any()
    server.admit(groups, others, room=0)
    server.finish(range(3))
    server.admit(groups, prompts, room=0)   # the same again
    assert near(server.sample(3, 2, steps), before)


def test_tokens_that_are_not_written():
    """A mask of tokens, after the groups, as a keyword, or as a number for each row; rows and starts of any kind."""
    from paper_2608_01657_gb300 import serving as S
    s = S.Shape()
    server = S.Server(s, groups=2, seed=4)
    groups, n = [0, 0, 1], 3
    prompts = S.prompts_of(groups, s, 4)
    server.admit(groups, prompts, room=8)
    rows = torch.arange(n, device="cuda")
    start = server.lens[:n].long().repeat_interleave(2)[::2]          # 64 bits, with strides
    counts = [2, 1, 3]
    tokens = torch.arange(sum(counts), device="cuda")
    k, v = server.k.clone(), server.v.clone()
    want = server.forward(rows, start, tokens, counts, [0, n])         # all are written
    full = server.k.clone()
    places = [(int(server.tables[i, (int(start[i]) + j) // s.page]), (int(start[i]) + j) % s.page) for i in range(n) for j in range(counts[i])]
    for at, off in places:
        assert not torch.equal(full[:, at, off], k[:, at, off])
    write = torch.tensor([True, False, True, False, False, True], device="cuda")
    for kind in ("place", "keyword", "rows", "both"):
        server.k.copy_(k), server.v.copy_(v)
        keep = write.tolist()
        if kind == "place":
            server.forward(rows, start, tokens, counts, [0, n], write)
        elif kind == "keyword":
            server.forward(rows.int(), start.int(), tokens, counts, write=write)
        else:
            written = (start + torch.tensor([1, 0, 2], device="cuda")).int()
            server.forward(rows, start, tokens, counts, [0, n], write if kind == "both" else None, written)
            keep = [False, True, True, False, False, True]
            keep = [a and b for a, b in zip(keep, write.tolist())] if kind == "both" else keep
        for (at, off), kept in zip(places, keep):
            assert torch.equal(server.k[:1, at, off], (full if kept else k)[:1, at, off]), kind
    server.k.copy_(k), server.v.copy_(v)
    assert torch.equal(server.forward(rows, start, tokens, counts, [0, n], torch.ones_like(write)), want)
