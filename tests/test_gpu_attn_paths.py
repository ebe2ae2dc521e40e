"""Attention over the 4-bit cache on launch paths that need long caches, loose
bounds or many columns: codes read as streams, chunks of several query tiles,
more chunks than the join takes at a time, windows in chunks, lengths above the
host's bound.  Every case names its path and the rule has to choose it."""
import sys

import numpy as np
import pytest

import attn_rules
import kv_ref
from test_gpu_attn import check, filled, scales_of
from test_gpu_kv import batch, dev

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


def run(eq, cache, b, q, scale, window, heads):
    """The output, twice the same from a workspace of NaN."""
    out = torch.full_like(q, 7.0)
    ws = eq.attn_workspace(cache, b, heads)
    for o in (out, torch.empty_like(q)):
        if ws is not None:
            ws.fill_(255)
        eq.eq_attn_kv4(cache, b, q, scale, o, ws, window=window)
    assert torch.equal(out.view(torch.int16), o.view(torch.int16))
    return out.double().cpu().numpy()


PATHS = [
    # news, lens, hq, hk, dim, page, window, bound; prompt, pair, stream, most chunks joined
    ([1, 1], [5000, 70], 8, 8, 128, 32, 0, 98304, 0, 1, 1, 2),
    ([1, 1], [70, 4500], 8, 8, 128, 128, 0, 98304, 0, 1, 1, 2),
    ([12, 3], [4200, 100], 8, 8, 128, 64, 0, 98304, 0, 0, 1, 2),
    ([9], [300], 16, 16, 128, 128, 0, 98304, 0, 0, 1, 1),
    ([1, 0, 2, 3], [5000, 0, 40, 129], 16, 8, 64, 32, 0, 98304, 0, 1, 1, 2),
    ([2, 1, 1, 4], [4300, 1, 128, 600], 16, 8, 64, 128, 0, 98304, 0, 1, 1, 2),
    ([8, 1, 1, 5], [4300, 1, 128, 600], 16, 8, 64, 64, 0, 98304, 0, 0, 1, 2),
    ([16, 1, 1, 5], [4300, 1, 128, 600], 8, 8, 64, 256, 0, 98304, 0, 0, 1, 2),
    ([1, 1], [5000, 70], 8, 8, 128, 32, 300, 98304, 0, 1, 0, 1),
    # several tiles of 16 columns, each in several chunks
    ([5], [3000], 16, 2, 128, 64, 0, 0, 0, 0, 0, 6),
    ([7, 4], [2500, 2200], 8, 1, 64, 32, 0, 0, 0, 0, 0, 5),
    ([5], [6000], 16, 2, 128, 32, 3000, 0, 0, 0, 0, 6),
    ([61, 2], [2100, 2], 1, 1, 64, 128, 0, 4000, 0, 0, 0, 5),
    # the join's second step (33 chunks) and second round (65)
    ([1], [17000], 4, 1, 128, 64, 0, 0, 0, 1, 0, 34),
    ([2], [40000], 3, 1, 64, 128, 0, 0, 0, 1, 0, 79),
    ([3], [34000], 5, 1, 128, 32, 0, 0, 0, 0, 0, 67),
    ([20], [17000], 4, 1, 128, 64, 0, 0, 1, 0, 0, 67),
    ([40], [12500], 2, 1, 64, 32, 0, 0, 1, 0, 0, 49),
    # many columns with a window, in chunks
    ([100], [2000], 2, 1, 128, 64, 1000, 8192, 1, 0, 0, 5),
    ([90], [9000], 1, 1, 64, 32, 4000, 0, 1, 0, 0, 17),
]


@pytest.mark.parametrize("news,lens,hq,hk,dim,page,window,bound,prompt,pair,stream,chunks", PATHS)
def test_path(eq, news, lens, hq, hk, dim, page, window, bound, prompt, pair, stream, chunks):
    say("path", news, lens, hq, hk, dim, page, window, bound, "expects", prompt, pair, stream, chunks)
    group, most, max_new = hq // hk, max(max(lens), bound), max(news)
    p = attn_rules.plan(len(lens), hk, group, max_new, most, window, dim)
    joined = max(max(attn_rules.joined(p, group, n, t, most, window), default=0)
                 for n, t in zip(news, lens))
    assert (p.prompt, p.pair, p.stream, joined) == (prompt, pair, stream, chunks), (p, joined)
    r = np.random.default_rng(sum(lens) + dim)
    n_pages = sum(-(-t // page) for t in lens) + 1
    b, starts, _ = batch(eq, news, lens, page, n_pages, seed=7, bound=bound)
    w = attn_rules.plan(len(lens), hk, group, max_new, most, 0, dim)
    assert eq.eq_attn_kv4_workspace_bytes(_of(eq, page, hk, dim), b, hq) == (
        len(lens) * hk * w.q_tiles * w.chunks * w.cols * (dim + 2) * 4 if w.chunks > 1 else 0)
    cache, k, v, _ = filled(eq, r, lens, page, hk, dim, n_pages, b, starts)
    q = dev(r.standard_normal((starts[-1], hq, dim)).astype(np.float32), torch.bfloat16) * 2
    o = run(eq, cache, b, q, dim ** -0.5, window, hq)
    check(o, q.double().cpu().numpy(), k, v, news, lens, dim ** -0.5, window)


def _of(eq, page, heads, dim):
    """A cache of these sizes for host-side questions."""
    return eq.KvCache.empty(1, page_tokens=page, kv_heads=heads, head_dim=dim)


@pytest.mark.parametrize("hq,new,held,max_len", [(4, 3, 300, 200), (4, 40, 300, 200), (1, 6, 3000, 2900),
                                                 (8, 40, 8300, 8192)])
@pytest.mark.parametrize("window", [0, 150, 1])
def test_lengths_above_the_bound(eq, hq, new, held, max_len, window):
    """kv_len beyond max_len: tokens behind the bound are absent, positions stay."""
    say("above", hq, new, held, max_len, window)
    dim, page = 64, 32
    r = np.random.default_rng(held + hq)
    n_pages = -(-held // page)
    whole, _, _ = batch(eq, [new], [held], page, n_pages)
    cache, k, v, _ = filled(eq, r, [held], page, 1, dim, n_pages, whole, None)
    b = eq.KvBatch(*whole.tensors, n_tokens=new, max_new=new, max_len=max_len)
    q = dev(r.standard_normal((new, hq, dim)).astype(np.float32), torch.bfloat16)
    o = run(eq, cache, b, q, 0.125, window, hq)
    present = [np.arange(held) < max_len]
    check(o, q.double().cpu().numpy(), k, v, [new], [held], 0.125, window, present)


@pytest.mark.parametrize("hq,max_len", [(2, 200), (32, 200), (32, 8192)])
@pytest.mark.parametrize("window", [0, 100])
def test_the_longest_length(eq, hq, max_len, window):
    """kv_len of 2^31 - 1: all held tokens are seen without a window, none with one."""
    say("longest", hq, max_len, window)
    dim, page, new = 64, 32, 3
    r = np.random.default_rng(hq)
    n_pages = max_len // page + 1
    whole, _, _ = batch(eq, [new], [max_len], page, n_pages)
    cache, k, v, _ = filled(eq, r, [max_len], page, 1, dim, n_pages, whole, None)
    b = eq.KvBatch(whole.tensors[0], dev(np.array([2**31 - 1], np.int32)), whole.tensors[2],
                   n_tokens=new, max_new=new, max_len=max_len)
    q = dev(r.standard_normal((new, hq, dim)).astype(np.float32), torch.bfloat16)
    o = run(eq, cache, b, q, 0.125, window, hq)
    if window:
        assert (o == 0).all()
        return
    wt = scales_of(v)[:, 0]
    for h in range(hq):
        ref, bound = kv_ref.attention64(q[:, h].double().cpu().numpy(), k[:, 0], v[:, 0], wt, 0.125,
                                        np.ones((new, max_len), bool))
        assert (np.abs(o[:, h] - ref) <= bound).all(), h
