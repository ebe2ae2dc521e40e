"""Verification of drafted trees on both sides of the size from which the passes over
the vocabulary are launches of their own (16 chunks of 1024 logits), against the
definition in 64 bits."""
import numpy as np
import pytest

from test_gpu_kv import batch, dev
from test_gpu_tree import tree
from test_gpu_tree_verify import KINDS, check, eq, inputs, say  # noqa: F401 (eq: the fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("replace", [False, True])
@pytest.mark.parametrize("target,draft", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", None)])
@pytest.mark.parametrize("vocab", [15361, 16384, 16385, 17409])
def test_trees(eq, vocab, target, draft, replace):
    say("passes", vocab, target, draft, replace)
    r = np.random.default_rng(vocab)
    news = [1, 2, 0, 9, 21, 5]
    parents, t, d, tokens, u = inputs(r, news, vocab, spread=1.5)
    say(check(eq, news, parents, tokens, dev(t, KINDS[target]),
              None if draft is None else dev(d, KINDS[draft]), u, replace=replace))


@pytest.mark.parametrize("vocab", [16384, 16400])
@pytest.mark.parametrize("kind,kids", [("chain", 1), ("chain", 256), ("star", 256), ("star", 2), ("tree", 1)])
def test_shapes_and_bounds_of_children(eq, kind, kids, vocab):
    r = np.random.default_rng(5)
    news = [33, 7, 3, 1, 12]
    parents, t, d, tokens, u = inputs(r, news, vocab, kind)
    check(eq, news, parents, tokens, dev(t), dev(d), u, kids=kids)


@pytest.mark.parametrize("height", [0.97, 1.0 - 2.0 ** -24])
@pytest.mark.parametrize("vocab", [16384, 16390])
def test_many_rejections(eq, vocab, height):
    """More of them than passes are launched."""
    r = np.random.default_rng(6)
    news = [30, 12, 20, 1]
    parents, t, d, tokens, u = inputs(r, news, vocab, "star", spread=1.0, noise=1.5)
    u[:] = height
    say(check(eq, news, parents, tokens, dev(t), dev(d), u))
    u[:] = 0  # and all of them accepted
    parents = [tree(r, n, "chain") for n in news]
    assert [k for k, _ in check(eq, news, parents, tokens, dev(t), dev(d), u)] == news


@pytest.mark.parametrize("vocab", [16384, 16390])
def test_temperatures_and_damaged_rows(eq, vocab):
    """Greedy and sampled sequences together; rows behind a rejection that hold a NaN or
    nothing, and drafts that are the target."""
    r = np.random.default_rng(7)
    news, temps = [6] * 8, [1.0, 0.5, 0.0, float("nan"), 5.0, 1e-4, 0.9, 1.0]
    parents, t, d, tokens, u = inputs(r, news, vocab)
    check(eq, news, parents, tokens, dev(t), dev(d), u, temps)
    d[36:] = t[36:]
    check(eq, news, parents, tokens, dev(t), dev(d), u, temps)
    t[[1, 13, 20, 45], [5, vocab - 1, 9000, 0]] = np.nan
    d[[2, 7, 31, 44], [vocab - 1, 0, 15000, 3]] = np.nan
    t[25], d[3] = -np.inf, -np.inf
    for height in (0.0, 0.6, 0.95):
        u[:] = height
        check(eq, news, parents, tokens, dev(t), dev(d), u, temps)


@pytest.mark.parametrize("vocab", [16384, 16390])
def test_replays(eq, vocab):
    """A captured call on a workspace that others spoil, with new numbers each time."""
    r = np.random.default_rng(8)
    news = [7, 12, 0, 5]
    parents, t, d, tokens, u = inputs(r, news, vocab, "star", spread=1.0)
    b, _, _ = batch(eq, news, [n + 5 for n in news], 32, 40, n_tokens=sum(news))
    out = [torch.empty(n, dtype=torch.int32, device="cuda") for n in (sum(news), 4, 4)]
    args = [b, dev(np.concatenate(parents).astype(np.int32)), dev(tokens), dev(t), dev(d), dev(u)]
    ws, other = (eq.verify_workspace(b, vocab) for _ in range(2))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        eq.eq_tree_verify(*args, *out, ws)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        eq.eq_tree_verify(*args, *out, ws)
    for i in range(6):
        args[5].uniform_()
        args[4].copy_(args[3] + 0.7 * torch.randn_like(args[3]))
        if i % 2:
            ws.fill_(255)
        g.replay()
        want = [torch.empty_like(x) for x in out]
        eq.eq_tree_verify(*args, *want, other)
        torch.cuda.synchronize()
        for x, y in zip(out, want):
            assert torch.equal(x, y), i
