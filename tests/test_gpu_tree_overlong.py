"""Attention of trees where a sequence has more rows than the call takes: its first
max_new rows and the other sequences' are as if the rest were not there."""
import numpy as np
import pytest

from test_gpu_attn import filled
from test_gpu_kv import batch, dev
from test_gpu_tree import check, eq, masked, say, tree  # noqa: F401 (eq: the fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


# blocks of 128 columns whose chunks the device shares out, and blocks of 16 columns
@pytest.mark.parametrize("at", [0, 1, 2])
@pytest.mark.parametrize("hq,bound,window", [(64, 8192, 4096), (64, 8192, 0), (64, 8192, 40), (8, 0, 1024), (8, 0, 0)])
def test_more_rows_than_the_bound(eq, hq, bound, window, at):
    say("over-long", hq, bound, window, at)
    r = np.random.default_rng(window + at)
    hk, dim, page, nodes, over = 8, 64, 64, 16, 2000
    news, lens = [nodes, 11, nodes], [6000, 5200, 4400]
    news[at] = nodes  # of the longer one's rows, as many as the bound
    real = [over if i == at else n for i, n in enumerate(news)]
    have = [t + real[i] - n for i, (t, n) in enumerate(zip(lens, news))]  # with the skipped rows'
    n_pages = sum(-(-t // page) for t in have) + 1
    b, starts, _ = batch(eq, real, have, page, n_pages, seed=5, bound=max(bound, max(have)), max_new=nodes)
    cache, k, v, _ = filled(eq, r, have, page, hk, dim, n_pages, b, starts)
    parents = [tree(r, n) for n in news]
    mask, pos, seen = masked(news, lens, parents, window)
    # the call's rows among the batch's; the first of a sequence's have its masks, with a
    # bit of a skipped row
    rows = np.concatenate([starts[i] + np.arange(n) for i, n in enumerate(news)])
    all_mask = r.integers(-(1 << 31), 1 << 31, (starts[-1], 1)).astype(np.int32)
    all_mask[rows] = mask | np.where(np.repeat(np.arange(3) == at, news), 1 << 20, 0)[:, None].astype(np.int32)
    all_pos = np.full(starts[-1], 1 << 29, np.int32)
    all_pos[rows] = pos
    q = dev(r.standard_normal((starts[-1], hq, dim)).astype(np.float32), torch.bfloat16)
    out = torch.full((starts[-1], hq, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = eq.attn_tree_workspace(cache, b, hq)
    if ws is not None:
        ws.fill_(255)
    eq.eq_attn_kv4_tree(cache, b, q, dim ** -0.5, dev(all_mask), out, ws,
                        positions=dev(all_pos) if window else None, window=window)
    o, qn = out.double().cpu().numpy(), q.double().cpu().numpy()
    base = 0
    for i, (n, t) in enumerate(zip(news, lens)):
        at_rows = slice(starts[i], starts[i] + n)
        check(o[at_rows], qn[at_rows], k[base:base + t], v[base:base + t], [seen[i]], dim ** -0.5)
        base += have[i]
    others = np.ones(starts[-1], bool)
    others[rows] = False
    assert (o[others] == 7.0).all()
