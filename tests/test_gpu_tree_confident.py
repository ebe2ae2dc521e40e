"""Verification against drafts that are sure of one token: what is left of q after its
rejection is a small part, down to nothing in 64 bits, and the next children are drawn
from that part alone.

The definition in 64 bits zeroes the rejected token and divides by the sum of the others,
so that what it leaves of q is right to 2^-50 of itself.  Where q(x) falls below 2^-900 of
the whole, the rule of the header is expected instead."""
import sys

import numpy as np
import pytest

import tree_ref
from test_gpu_kv import dev
from test_gpu_tree_verify import KINDS, check

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def eq():
    import paper_2601_22787_amd as m
    m.lib()
    assert torch.cuda.is_available()
    return m


def drawn(r, logits, temp, n):
    """n tokens, one after another without replacement."""
    return np.argsort(-(logits.astype(np.float64) / temp + r.gumbel(size=len(logits))), kind="stable")[:n]


# both forms of the passes over the vocabulary: in the walk's block, and in launches
@pytest.mark.parametrize("vocab", [6, 1027, 5003, 17001, 40003])
@pytest.mark.parametrize("temp", [1.0, 0.25])
@pytest.mark.parametrize("gap", [10, 20, 30, 40, 100, 400])
def test_tokens(eq, gap, temp, vocab):
    """A dominant logit `gap` T above the others, which the target gives little; trees of
    one node with 2 to 5 children, at many random numbers."""
    say("confident", gap, temp, vocab)
    r = np.random.default_rng(gap * vocab)
    news = [3, 6, 4, 3, 6, 5, 3, 4]
    parents = [np.array([-1] + [0] * (n - 1)) for n in news]
    rows = sum(news)
    t = r.standard_normal((rows, vocab)).astype(np.float32)
    d = (temp * r.standard_normal((rows, vocab))).astype(np.float32)
    tokens, row = np.zeros(rows, np.int32), 0
    for s, n in enumerate(news):
        top = (0, vocab - 1, vocab // 2, vocab * 3 // 4, 3, vocab - 2, 1, vocab // 3)[s]
        d[row, top] = d[row].max() + gap * temp
        t[row, top] = t[row].min()
        tokens[row + 1:row + n] = drawn(r, d[row], temp, n - 1)
        if s % 2:  # children that the target likes: accepted at some of the numbers
            t[row, tokens[row + 2]] = t[row].max() + 2
        row += n
    many = 0
    for i in range(4):
        u = r.random(rows).astype(np.float32)
        got = check(eq, news, parents, tokens, dev(t), dev(d), u, temps=[temp] * len(news))
        many += sum(k for k, _ in got) - len(news)
    say("accepted", many)


@pytest.mark.parametrize("target,draft", [("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("vocab", [3001, 20011])
def test_what_is_left_falls_child_by_child(eq, vocab, target, draft):
    """Eight children, each 2^-10 to 2^-60 of the one before, all of them rejected at
    most of the random numbers: 2^-70 to 2^-420 of q are left for the last."""
    r = np.random.default_rng(vocab)
    news = [9] * 6
    parents = [np.array([-1] + [0] * 8)] * 6
    t = r.standard_normal((54, vocab)).astype(np.float32)
    d = r.standard_normal((54, vocab)).astype(np.float32)
    tokens = np.zeros(54, np.int32)
    for s in range(6):
        # neighbours, in one chunk, and others anywhere
        x = np.arange(8) + 4 * s + 1020 if s % 2 else r.permutation(vocab)[:8]
        tokens[9 * s + 1:9 * s + 9] = x
        d[9 * s, x] = 400 - (7, 14, 21, 28, 35, 42)[s] * np.arange(8)
        t[9 * s, x[:7]] -= 3
    for i in range(5):
        u = r.random(54).astype(np.float32)
        if i < 2:
            u[np.arange(54) % 9 != 0] = (0.5, 0.9)[i]
        check(eq, news, parents, tokens, dev(t, KINDS[target]), dev(d, KINDS[draft]), u)
        check(eq, news, parents, tokens, dev(t, KINDS[target]), dev(d, KINDS[draft]), u, replace=True)


@pytest.mark.parametrize("vocab", [500, 18000])
def test_nothing_left_of_the_draft(eq, vocab):
    """With less than 2^-900 of q left the second child is not tested, and the token
    behind the path is of what is left of p."""
    r = np.random.default_rng(vocab)
    n = 12
    news = [3] * n
    t = r.standard_normal((3 * n, vocab)).astype(np.float32)
    d = np.zeros((3 * n, vocab), np.float32)
    d[::3, 7] = [650, 700, 740, 750, 800, 1000, 3000, 1e5, 1e30, 3e38, 2000, 1e10]
    d[3 * 5, 8:] = -np.inf  # and nothing at all but both children
    tokens = np.tile(np.array([0, 7, 4], np.int32), n)
    t[::3, 4] += 6  # the second child would be accepted at most random numbers
    d[::3, 4] += 2
    parents = dev(np.tile(np.array([-1, 0, 0], np.int32), n))
    b = eq.KvBatch(dev(3 * np.arange(n + 1, dtype=np.int32)), dev(np.full(n, 3, np.int32)),
                   dev(np.zeros((n, 1), np.int32)), n_tokens=3 * n, max_new=3, max_len=32)
    path = torch.empty(3 * n, dtype=torch.int32, device="cuda")
    kept, nxt = torch.empty(2, n, dtype=torch.int32, device="cuda")
    ws = eq.verify_workspace(b, vocab, draft=True)
    for i in range(6):
        u = r.random(3 * n).astype(np.float32)
        u[1::3] = 0.5
        ws.fill_(255)
        eq.eq_tree_verify(b, parents, dev(tokens), dev(t), dev(d), dev(u), path, kept, nxt, ws)
        for s in range(n):
            p, q = tree_ref.softmax(t[3 * s], 1.0), tree_ref.softmax(d[3 * s], 1.0)
            want = tree_ref.invert(np.maximum(p - q, 0), np.float64(u[3 * s]))
            assert path[3 * s:3 * s + 3].tolist() == [0, -1, -1], (i, s)
            assert int(kept[s]) == 1 and int(nxt[s]) == want, (i, s, int(nxt[s]), want)


@pytest.mark.parametrize("gap,temp", [(10, 1.0), (20, 1.0), (30, 1.0), (35, 1.0), (40, 1.0), (35, 0.25),
                                      (200, 1.0), (2000, 0.005)])
@pytest.mark.parametrize("vocab,n", [(3, 20000), (2051, 8000), (17 * 1024 + 3, 1500)])
def test_what_is_kept_is_distributed_as_the_target(eq, vocab, n, gap, temp):
    """p = (.05, .05, .9) and a draft of (b, b - gap, b - gap - 3), a tree for each of many b:
    the first token behind node 0 comes as often as the target says, within 5 standard
    deviations."""
    r = np.random.default_rng(1000 * gap + vocab)
    at = [0, vocab // 2, vocab - 1]
    one = np.full((2, vocab), -100, np.float64)  # (what is neither weighs e^-80 and less)
    one[1] -= gap
    one[0, at] = np.log([0.05, 0.05, 0.9])
    one[1, at] = [0, -gap, -3 - gap]
    one = (temp * one).astype(np.float32)
    rows = torch.empty(2, 3 * n, vocab, device="cuda")
    rows[:] = dev(one)[:, None]
    rows[1] += dev(np.repeat(temp * r.integers(-640, 640, n) / 64, 3).astype(np.float32))[:, None]
    q = one[1].astype(np.float64)[at] / temp
    tokens = np.zeros((n, 3), np.int32)
    tokens[:, 1:] = np.array(at)[np.argsort(-(q + r.gumbel(size=(n, 3))), axis=1)[:, :2]]
    b = eq.KvBatch(dev(3 * np.arange(n + 1, dtype=np.int32)), dev(np.full(n, 3, np.int32)),
                   dev(np.zeros((n, 1), np.int32)), n_tokens=3 * n, max_new=3, max_len=32)
    path = torch.empty(3 * n, dtype=torch.int32, device="cuda")
    kept, nxt = torch.empty(2, n, dtype=torch.int32, device="cuda")
    eq.eq_tree_verify(b, dev(np.tile(np.array([-1, 0, 0], np.int32), n)), dev(tokens.reshape(-1)),
                      rows[0], rows[1], dev(r.random(3 * n).astype(np.float32)), path, kept, nxt,
                      eq.verify_workspace(b, vocab, draft=True), max_children=2,
                      temperature=dev(np.full(n, temp, np.float32)))
    second = path.view(n, 3)[:, 1].cpu().numpy()
    first = np.where(second > 0, tokens[np.arange(n), np.maximum(second, 0)], nxt.cpu().numpy())
    p = tree_ref.softmax(one[0], temp)[at]
    found = np.array([(first == x).mean() for x in at])
    say(gap, temp, np.round(p, 4), np.round(found, 4), "accepted", (second > 0).mean())
    assert found.sum() == pytest.approx(1.0)
    assert (np.abs(found - p) <= 5 * np.sqrt(p * (1 - p) / n)).all()
