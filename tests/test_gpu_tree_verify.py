"""Verification of drafted trees against its definition in 64 bits, token for token:
chains and trees, drawn and given children, all types, rows at odd addresses, one
token to many, distributions without mass in places, and damaged rows."""
import sys

import numpy as np
import pytest

import tree_ref
from test_gpu_kv import batch, dev
from test_gpu_tree import tree

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

KINDS = {"f32": torch.float32, "bf16": torch.bfloat16}


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def eq():
    import paper_2601_22787_amd as m
    m.lib()
    assert torch.cuda.is_available()
    return m


def inputs(r, news, vocab, kind="tree", spread=2.5, noise=0.7):
    """Parents, logits of a target and a draft, likely tokens and random numbers."""
    rows = sum(news)
    parents = [tree(r, n, kind) for n in news]
    target = (spread * r.standard_normal((rows, vocab))).astype(np.float32)
    draft = (target + noise * r.standard_normal((rows, vocab))).astype(np.float32)
    tokens, row = np.zeros(rows, np.int32), 0
    for n, p in zip(news, parents):
        for i in range(1, n):
            rank = int((p[1:i] == p[i]).sum())
            order = np.argsort(-(draft[row + p[i]] + r.gumbel(size=vocab)), kind="stable")
            tokens[row + i] = order[rank % vocab]
        row += n
    return parents, target, draft, tokens, r.random(rows).astype(np.float32)


def check(eq, news, parents, tokens, target, draft, random, temps=None, replace=False, kids=256,
          seed=0, spoil=True):
    """target and draft: device tensors (draft: or None).  Compares all sequences."""
    vocab = target.shape[1]
    b, starts, _ = batch(eq, news, [n + 5 for n in news], 32, 400, n_tokens=sum(news))
    path = torch.full((sum(news),), 99, dtype=torch.int32, device="cuda")
    kept, nxt = torch.full((2, len(news)), 99, dtype=torch.int32, device="cuda")
    ws = eq.verify_workspace(b, vocab, draft=draft is not None)
    if spoil:
        ws.fill_(255)
    eq.eq_tree_verify(b, dev(np.concatenate(parents).astype(np.int32)), dev(tokens), target, draft,
                      dev(random), path, kept, nxt, ws,
                      temperature=None if temps is None else dev(np.array(temps, np.float32)),
                      replace=replace, max_children=kids)
    t64 = target.double().cpu().numpy()
    d64 = None if draft is None else draft.double().cpu().numpy()
    out = []
    for s, n in enumerate(news):
        at = slice(starts[s], starts[s] + n)
        if n == 0:
            assert kept[s] == 0 and nxt[s] == -1
            continue
        ref, token = tree_ref.verify(parents[s], tokens[at], t64[at], None if d64 is None else d64[at],
                                     random[at], 1.0 if temps is None else np.float32(temps[s]), replace)
        got = path[at].tolist()
        assert got == ref + [-1] * (n - len(ref)), (s, got, ref)
        assert int(kept[s]) == len(ref) and int(nxt[s]) == token, (s, int(nxt[s]), token)
        out.append((len(ref), token))
    return out


@pytest.mark.parametrize("replace", [False, True])
@pytest.mark.parametrize("target,draft", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"),
                                          ("bf16", "bf16"), ("f32", None), ("bf16", None)])
@pytest.mark.parametrize("vocab", [1, 2, 5, 1000, 1024, 1027, 5003])
def test_trees(eq, vocab, target, draft, replace):
    say("verify", vocab, target, draft, replace)
    r = np.random.default_rng(vocab)
    news = [1, 2, 0, 9, 33, 16, 5, 24]
    parents, t, d, tokens, u = inputs(r, news, vocab, spread=1.5)
    lengths = check(eq, news, parents, tokens, dev(t, KINDS[target]),
                    None if draft is None else dev(d, KINDS[draft]), u, replace=replace)
    say(lengths)


@pytest.mark.parametrize("kind,kids", [("chain", 1), ("chain", 256), ("star", 256), ("star", 2),
                                       ("tree", 1)])
def test_shapes_and_bounds_of_children(eq, kind, kids):
    """More children than the bound says: slower, and the same."""
    r = np.random.default_rng(5)
    news = [40, 7, 256, 3, 1, 64, 12]
    parents, t, d, tokens, u = inputs(r, news, 3001, kind)
    check(eq, news, parents, tokens, dev(t), dev(d), u, kids=kids)
    check(eq, news, parents, tokens, dev(t), None, u, kids=kids)


@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("height", [0.97, 1.0 - 2.0 ** -24])
def test_many_rejections(eq, height, draft):
    """Random numbers near 1: most children are rejected, and what is left of p is a
    small part of it."""
    r = np.random.default_rng(6)
    news = [30, 12, 20, 1]
    parents, t, d, tokens, u = inputs(r, news, 2500, "star", spread=1.0, noise=1.5)
    u[:] = height
    say(check(eq, news, parents, tokens, dev(t), dev(d) if draft else None, u))
    u[:] = 0  # and all of them accepted
    parents = [tree(r, n, "chain") for n in news]
    assert [k for k, _ in check(eq, news, parents, tokens, dev(t), dev(d) if draft else None, u)] == news


def test_temperatures(eq):
    r = np.random.default_rng(7)
    news = [9] * 10
    temps = [1.0, 0.5, 0.0, -1.0, float("nan"), 5.0, float("inf"), 1e-4, 1e-40, 0.9]
    for kind in ("f32", "bf16"):
        parents, t, d, tokens, u = inputs(r, news, 1500)
        # some drafted tokens are the largest logits, which in BF16 have equals
        for i in range(1, 90, 2):
            p = parents[i // 9][i % 9]
            if p >= 0:
                tokens[i] = int(np.argmax(dev(t, KINDS[kind]).float().cpu().numpy()[i // 9 * 9 + p]))
        td, dd = dev(t, KINDS[kind]), dev(d, KINDS[kind])
        check(eq, news, parents, tokens, td, dd, u, temps)
        check(eq, news, parents, tokens, td, None, u, temps)


def test_equal_logits_and_the_lowest_of_them(eq):
    news = [3, 3]
    parents = [np.array([-1, 0, 0])] * 2
    t = np.zeros((6, 4000), np.float32)
    t[0, [1500, 3999, 20]] = 3
    tokens = np.array([0, 1500, 20, 0, 3999, 1500], np.int32)
    t[3] = -np.inf
    t[3, [3999, 1500]] = -1e30
    u = np.full(6, 0.5, np.float32)
    out = check(eq, news, parents, tokens, dev(t), None, u, temps=[0, 0])
    assert out == [(2, 0), (2, 0)]


def test_masses_in_few_places(eq):
    """Logits of -infinity and far apart; a draft that is the target; a draft without
    a common token; random numbers outside [0, 1)."""
    r = np.random.default_rng(11)
    news, vocab = [4] * 8, 2100
    parents, t, d, tokens, u = inputs(r, news, vocab, "star")
    for s in range(8):
        at = slice(4 * s, 4 * s + 4)
        allowed = r.permutation(vocab)[:(1, 2, 3, 50, 1000, 3, 3, 3)[s]]
        cut = np.full(vocab, -np.inf, np.float32)
        cut[allowed] = 0
        t[at] += cut
        if s < 5:
            d[at] += cut
            tokens[at] = allowed[np.arange(4) % len(allowed)]
    d[20:24] = t[20:24]
    d[24:28, np.isfinite(t[24])] = -np.inf
    t[28:32] *= 1e30
    u[[0, 1, 2, 6, 9, 13]] = [1.0, -3.0, float("nan"), float("inf"), 2.0, -float("inf")]
    check(eq, news, parents, tokens, dev(t), dev(d), u)
    check(eq, news, parents, tokens, dev(t), None, u)


def test_rows_without_a_distribution(eq):
    """A NaN, +infinity, or nothing at all in a row that is looked at: the walk ends
    there.  In a row that is not, nothing happens."""
    r = np.random.default_rng(12)
    for greedy in (False, True):
        news, vocab = [4] * 7, 1400
        parents, t, d, tokens, u = inputs(r, news, vocab, "chain")
        u[:] = 0
        for s in range(7):
            for i in range(1, 4):
                tokens[4 * s + i] = int(np.argmax(t[4 * s + i - 1]))
        t[1, 1399] = np.nan
        t[4, 0] = np.inf
        t[10] = -np.inf
        d[13, 700] = np.nan
        d[19] = np.nan      # a leaf's
        d[20] = -np.inf
        tokens[27] = vocab  # outside, and a damaged row behind it
        t[27] = np.nan
        out = check(eq, news, parents, tokens, dev(t), dev(d), u, temps=[0.0 if greedy else 1.0] * 7)
        assert [x[0] for x in out[:3]] == [2, 1, 3] and [x[1] for x in out[:3]] == [-1] * 3
        assert greedy or (out[3] == (2, -1) and out[5] == (1, -1))
        assert out[6][0] == 3 and out[6][1] >= 0
        check(eq, news, parents, tokens, dev(t), None, u, temps=[0.0 if greedy else 1.0] * 7)


def test_tokens_and_parents_that_are_none(eq):
    r = np.random.default_rng(13)
    news = [12, 12]
    parents, t, d, tokens, u = inputs(r, news, 900, "star")
    parents = [np.array([5, 0, 0, 3, 12, 0, 1, 1, -1, -7, 1 << 30, 0]), np.array([-1] + [0] * 11)]
    tokens[[1, 14]] = [-1, 900]
    tokens[[2, 16, 17]] = [-(1 << 31), 1 << 30, tokens[15]]
    check(eq, news, parents, tokens, dev(t), dev(d), u)
    check(eq, news, parents, tokens, dev(t), None, u)
    u[:] = 1
    check(eq, news, parents, tokens, dev(t), dev(d), u, replace=True)
    check(eq, news, parents, tokens, dev(t), None, u)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_strided_rows_and_another_stream(eq, kind):
    """Logits as columns of a wider buffer, at an odd element."""
    r = np.random.default_rng(14)
    news = [6, 11]
    parents, t, d, tokens, u = inputs(r, news, 1999)
    wide = torch.zeros(17, 4101, dtype=KINDS[kind], device="cuda")
    wide[:, 1:2000], wide[:, 2001:4000] = dev(t, KINDS[kind]), dev(d, KINDS[kind])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        check(eq, news, parents, tokens, wide[:, 1:2000], wide[:, 2001:4000], u)


def test_a_large_vocabulary(eq):
    r = np.random.default_rng(15)
    news = [5, 3]
    parents, t, d, tokens, u = inputs(r, news, 300007)
    for i in range(4):
        u[:] = r.random(8)
        check(eq, news, parents, tokens, dev(t), dev(d), u)
        check(eq, news, parents, tokens, dev(t), None, u)


def test_what_is_kept_is_distributed_as_the_target(eq):
    """65536 small trees of one distribution each: the first token behind node 0 comes
    as often as the target says, within 5 standard deviations."""
    r = np.random.default_rng(16)
    for draft in (True, False):
        n, vocab = 20000, 6
        t = np.repeat((1.2 * r.standard_normal((1, vocab))).astype(np.float32), 3 * n, axis=0)
        d = np.repeat((1.2 * r.standard_normal((1, vocab))).astype(np.float32), 3 * n, axis=0)
        tokens = np.zeros((n, 3), np.int32)
        if draft:  # two children, drawn without replacement
            tokens[:, 1:] = np.argsort(-(d[:n] + r.gumbel(size=(n, vocab))), axis=1)[:, :2]
        else:
            tokens[:, 1:] = [4, 1]
        b = eq.KvBatch(dev(3 * np.arange(n + 1, dtype=np.int32)), dev(np.full(n, 3, np.int32)),
                       dev(np.zeros((n, 1), np.int32)), n_tokens=3 * n, max_new=3, max_len=32)
        path = torch.empty(3 * n, dtype=torch.int32, device="cuda")
        kept, nxt = torch.empty(2, n, dtype=torch.int32, device="cuda")
        eq.eq_tree_verify(b, dev(np.tile(np.array([-1, 0, 0], np.int32), n)), dev(tokens.reshape(-1)),
                          dev(t), dev(d) if draft else None, dev(r.random(3 * n).astype(np.float32)),
                          path, kept, nxt, eq.verify_workspace(b, vocab, draft=draft), max_children=2)
        second = path.view(n, 3)[:, 1].cpu().numpy()
        first = np.where(second > 0, tokens[np.arange(n), np.maximum(second, 0)], nxt.cpu().numpy())
        p = tree_ref.softmax(t[0], 1.0)
        found = np.bincount(first, minlength=vocab) / n
        say(draft, np.round(p, 4), np.round(found, 4), "accepted", (second > 0).mean())
        assert (np.abs(found - p) <= 5 * np.sqrt(p * (1 - p) / n)).all()


@pytest.mark.parametrize("temp", [1.0, 0.0])
@pytest.mark.parametrize("which", ["target", "draft"])
@pytest.mark.parametrize("at", [slice(0, 1024), slice(1024, 2048), slice(2048, 3000), slice(0, 3000),
                                slice(1500, 1501)])
def test_nan_wherever_it_is(eq, at, which, temp):
    """One, a whole chunk of them, and a row of nothing else; beside -infinity too."""
    r = np.random.default_rng(17)
    news = [3, 3, 3]
    parents, t, d, tokens, u = inputs(r, news, 3000, "chain")
    u[:] = 0
    for s in range(3):
        for i in range(1, 3):
            tokens[3 * s + i] = int(np.argmax(t[3 * s + i - 1]))
    x = t if which == "target" else d
    x[1, at] = np.nan
    x[4] = np.where(np.arange(3000) % 7 == 0, x[4], -np.inf)
    x[4, at] = np.nan
    x[7] = -np.inf
    x[7, at] = np.nan
    out = check(eq, news, parents, tokens, dev(t), dev(d), u, temps=[temp] * 3)
    assert temp == 0 and which == "draft" or [k for _, k in out] == [-1] * 3
    check(eq, news, parents, tokens, dev(t), None, u, temps=[temp] * 3)


def test_a_vocabulary_of_more_than_2_to_the_20(eq):
    """More chunks than a block keeps the sums of."""
    r = np.random.default_rng(18)
    news, vocab = [4, 3, 1], (1 << 20) + 77
    parents, t, d, tokens, u = inputs(r, news, vocab, "star", spread=1.0)
    for height in (0.0, 0.6, 0.9, 0.999):
        u[:] = height
        u[[0, 4, 7]] = r.random(3)
        for draft in (dev(d), None):
            check(eq, news, parents, tokens, dev(t), draft, u)


def test_two_graphs_share_a_workspace(eq):
    """Captured one after another on one workspace, replayed in turn with other numbers
    and eager calls between; every replay equals the eager call."""
    r = np.random.default_rng(19)
    news, vocab = [7, 12, 0, 5], 2200
    calls = []
    for kind in ("tree", "star"):
        parents, t, d, tokens, u = inputs(r, news, vocab, kind)
        b, _, _ = batch(eq, news, [n + 5 for n in news], 32, 40, n_tokens=sum(news))
        out = [torch.empty(n, dtype=torch.int32, device="cuda") for n in (sum(news), 4, 4)]
        calls.append((b, dev(np.concatenate(parents).astype(np.int32)), dev(tokens), dev(t), dev(d), dev(u), out))
    ws, other = (eq.verify_workspace(calls[0][0], vocab) for _ in range(2))

    def run(c, out, room):
        eq.eq_tree_verify(*c[:6], *out, room)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for c in calls:
            run(c, c[6], ws)
    torch.cuda.current_stream().wait_stream(s)
    graphs = []
    for c in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run(c, c[6], ws)
        graphs.append(g)
    for i in range(6):
        for c, g in zip(calls, graphs):
            c[5].uniform_()
            c[3].normal_()
            c[4].copy_(c[3] + 0.5 * torch.randn_like(c[3]))
            for x in c[6]:
                x.fill_(77)
            if i % 2:
                ws.fill_(255)
            g.replay()
            want = [torch.empty_like(x) for x in c[6]]
            run(c, want, other)
            torch.cuda.synchronize()
            for x, y in zip(c[6], want):
                assert torch.equal(x, y), i


def test_what_earlier_kernels_leave_behind(eq):
    """The same tokens every time, also after kernels that leave NaN in local memory."""
    from test_gpu_kv import batch as kv_batch
    import kv_ref
    r = np.random.default_rng(20)
    n = 300
    b, starts, _ = kv_batch(eq, [1] * n, [130] * n, 32, 5 * n)
    cache = eq.KvCache(torch.full((5 * n, kv_ref.page_bytes(2, 128, 32)), 255, dtype=torch.uint8, device="cuda"),
                       page_tokens=32, kv_heads=2, head_dim=128)
    q = torch.full((n, 16, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    o = torch.empty_like(q)
    news, vocab = [9, 20, 3, 33, 16], 5000
    parents, t, d, tokens, u = inputs(r, news, vocab)
    td, dd = dev(t), dev(d)
    for i in range(10):
        u[:] = r.random(sum(news))
        for draft in (dd, None):
            eq.eq_attn_kv4(cache, b, q, 0.1, o, eq.attn_workspace(cache, b, 16))
            check(eq, news, parents, tokens, td, draft, u)
    assert torch.isnan(o).all()
