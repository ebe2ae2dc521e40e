"""How near to a border tokens of verification are exact, where rejections have left a
small part G of p, a difference of rounded numbers.

With e = 2^-38.8 for an exponential, p and q are off by d = 2 e = 2^-37.8 of themselves.  The
sum of max(p - t q, 0), or of some of its terms, is off by at most d (p + t q), summed up 2 d,
and by what t is off times the q in it, Q': t + G / Q in the place of t makes an error E of it
E (1 - Q' / Q) + 2 d / Q, at most 2 d / Q' after any number of steps, so 2 d again.  A running
sum over the whole, at which a random number passes it, is then off by at most
2 (2 d + 2 d) / G = 2^-34.8 / G.  The header says about 2^-35 over what is left."""
import numpy as np
import pytest

from test_gpu_kv import dev
from test_gpu_tree_verify import eq, say  # noqa: F401 (eq: the fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def softmax(x):
    """With 64 bits of mantissa, where the platform has them."""
    e = np.exp(x.astype(np.longdouble) - x.max())
    return e / e.sum()


@pytest.mark.parametrize("shift", [0.0, 0.37109375])
@pytest.mark.parametrize("vocab", [3001, 20003])
@pytest.mark.parametrize("kids", [1, 4, 12, 20, 24, 27, 29, 30])
def test_borders_of_what_is_left(eq, vocab, kids, shift):
    """One half of the tokens is the target's, and of the draft's with half its mass, in
    the same proportions; the children are of the other half.  Each rejection halves
    what is left."""
    r = np.random.default_rng(vocab + kids)
    half = r.permutation(vocab)[:vocab // 2]
    mine = np.zeros(vocab, bool)
    mine[half] = True
    x = np.round(256 * 1.5 * r.standard_normal(vocab)) / 256  # sums of these are exact
    t = np.where(mine, x, -60).astype(np.float32)
    d = np.where(mine, x, -60.0)
    # the other half's mass, with a largest logit of its own
    at = np.flatnonzero(~mine)[: vocab // 3]
    d[at] = np.round(256 * r.standard_normal(len(at))) / 256
    d[at] += np.round(256 * np.log(np.exp(x[mine]).sum() / np.exp(d[at]).sum())) / 256
    d[at[-1]] = max(d.max(), x.max()) + shift
    d = (d + 1.25).astype(np.float32)
    p, q = softmax(t), softmax(d)
    tokens = at[:kids]
    g, left = np.longdouble(1), p
    for c in tokens:
        assert (1 - 2.0 ** -24) * float(q[c]) > float(left[c])
        left = np.maximum(left - q, 0)
        q = q.copy()
        q[c] = 0
        q = q / q.sum()
        g *= left.sum()
        left = left / left.sum()
    assert g > 2.0 ** -31.5
    n = 400
    rows = torch.empty(2, n * (kids + 1), vocab, device="cuda")
    rows[0], rows[1] = dev(t), dev(d)
    u = np.full((n, kids + 1), 1, np.float32)  # (taken as 1 - 2^-24: rejected)
    u[:, 0] = r.random(n)
    tree = np.tile(np.array([-1] + [0] * kids, np.int32), n)
    b = eq.KvBatch(dev((kids + 1) * np.arange(n + 1, dtype=np.int32)), dev(np.full(n, kids + 1, np.int32)),
                   dev(np.zeros((n, 1), np.int32)), n_tokens=n * (kids + 1), max_new=kids + 1, max_len=32)
    path = torch.empty(n * (kids + 1), dtype=torch.int32, device="cuda")
    kept, nxt = torch.empty(2, n, dtype=torch.int32, device="cuda")
    eq.eq_tree_verify(b, dev(tree), dev(np.tile(np.concatenate(([0], tokens)).astype(np.int32), n)), rows[0],
                      rows[1], dev(u.reshape(-1)), path, kept, nxt, eq.verify_workspace(b, vocab, draft=True))
    assert (kept == 1).all()
    run = np.cumsum(left)
    run = np.concatenate(([0], run / run[-1])).astype(np.float64)
    token, v = nxt.cpu().numpy(), u[:, 0].astype(np.float64)
    assert (token >= 0).all()
    # how far outside of its token's part a random number is
    off = float(np.maximum(np.maximum(run[token] - v, v - run[token + 1]), 0).max())
    g = float(g)
    say("border", vocab, kids, shift, "left 2^%.1f, off %.3g = 2^%.1f over it" %
        (np.log2(g), off, np.log2(max(off * g, 1e-30))))
    assert off <= 2.0 ** -34.8 / g
