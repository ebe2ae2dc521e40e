"""A sequence verified alone and among others: its statistics are grouped differently (1 to
3 chunks a wavefront), its path and token are the same, and the same call gives them
again."""
import numpy as np
import pytest

from test_gpu_kv import batch, dev
from test_gpu_tree_verify import KINDS, check, eq, inputs, say  # noqa: F401 (eq: the fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("target,draft", [("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"), ("bf16", None)])
@pytest.mark.parametrize("vocab", [15003, 30011])  # passes in the walk's block, and in launches
def test_alone_and_among_others(eq, vocab, target, draft):
    r = np.random.default_rng(vocab)
    one = [9, 5, 12]  # verified alone
    # rows x chunks x (with a draft, twice) / 3072 is how many chunks a wavefront takes
    chunks, sides = -(-vocab // 1024), 1 if draft is None else 2
    sizes = [max(1, per * 3072 // (chunks * sides) + 8) for per in (0, 2, 3)]
    parents, t, d, tokens, u = inputs(r, one + [12] * (-(-max(sizes) // 12)), vocab, spread=1.5)
    td, dd = dev(t, KINDS[target]), None if draft is None else dev(d, KINDS[draft])
    seen = []
    for size in [0] + sizes:
        n, rows = len(one), sum(one)
        while rows < size:
            n, rows = n + 1, rows + 12
        news = (one + [12] * n)[:n]
        got = check(eq, news, parents[:n], tokens[:rows], td[:rows], None if dd is None else dd[:rows], u[:rows])
        say("verified", vocab, target, draft, "rows", rows, "a wavefront's chunks",
            min(max(rows * chunks * sides // 3072, 1), 3))
        seen.append(got[:3])
        b, _, _ = batch(eq, news, [k + 5 for k in news], 32, 2000, n_tokens=rows)
        out = []
        for _ in range(2):
            res = [torch.full((k,), 9, dtype=torch.int32, device="cuda") for k in (rows, n, n)]
            eq.eq_tree_verify(b, dev(np.concatenate(parents[:n]).astype(np.int32)), dev(tokens[:rows]), td[:rows],
                              None if dd is None else dd[:rows], dev(u[:rows]), *res,
                              eq.verify_workspace(b, vocab, draft=dd is not None))
            out.append(res)
        assert all(torch.equal(x, y) for x, y in zip(*out))
    for i, k in enumerate(one):  # each of them alone
        at = slice(sum(one[:i]), sum(one[:i]) + k)
        assert check(eq, [k], [parents[i]], tokens[at], td[at], None if dd is None else dd[at], u[at])[0] == seen[0][i]
    assert all(x == seen[0] for x in seen)
