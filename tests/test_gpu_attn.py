"""Attention over the 4-bit cache against attention in 64 bits on the values
that the cache holds: lengths from nothing to many chunks, pages that end inside
a tile, grouped heads, windows, masked tokens that hold anything, absent pages,
other streams and captured graphs."""
import sys

import numpy as np
import pytest

import kv_ref
from test_gpu_kv import batch, dev, tables

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


def filled(eq, r, lens, page, heads, dim, n_pages, b, starts_all, tokens_of=None, size=1.0):
    """A cache whose bytes are all 0xFF (scales NaN) but for the sequences'
    tokens, written by eq_kv_append: (cache, keys, values, value scales), per
    sequence [T, heads, dim] in 64 bits as read back."""
    cache = eq.KvCache(torch.full((n_pages, kv_ref.page_bytes(heads, dim, page)), 255,
                                  dtype=torch.uint8, device="cuda"),
                       page_tokens=page, kv_heads=heads, head_dim=dim)
    total = sum(lens)
    k = r.standard_normal((total, heads, dim)) * np.exp(0.5 * r.standard_normal((1, heads, dim)))
    v = r.standard_normal((total, heads, dim)) * np.exp(size * r.standard_normal((total, heads, 1)))
    whole = eq.KvBatch(dev(np.concatenate(([0], np.cumsum(lens))).astype(np.int32)),
                       b.tensors[1], b.tensors[2], n_tokens=total, max_new=max(lens),
                       max_len=max(lens))
    kd, vd = dev(k.astype(np.float32)), dev(v.astype(np.float32))
    eq.eq_kv_append(cache, whole, kd, vd)
    ko, vo = torch.empty(2, total, heads, dim, dtype=torch.bfloat16, device="cuda")
    eq.eq_kv_read(cache, whole, ko, vo)
    return cache, ko.double().cpu().numpy(), vo.double().cpu().numpy(), whole


def scales_of(v):
    """The value scales that belong to read-back values [T, heads, dim]."""
    top = np.abs(v).max(axis=2)
    _, e = np.frexp(top)  # the largest code is 4 or 6: 0.5 or 0.75 times 2^3
    return np.where(top > 0, 2.0 ** (e - 3), 2.0 ** -103)


def check(out, q, k, v, news, lens, scale, window, present=None):
    """out [tokens, Hq, D] against the reference, sequence by sequence."""
    hq, hk = q.shape[1], k.shape[1]
    row = base = 0
    worst = 0.0
    for s, (n, t) in enumerate(zip(news, lens)):
        pos = np.arange(t - n, t)[:, None]
        j = np.arange(t)[None, :]
        seen = (j <= pos) & (pos >= 0)
        if window:
            seen &= j > pos - window
        if present is not None:
            seen &= present[s][None, :t]
        for h in range(hq):
            g = h // (hq // hk)
            vv = v[base:base + t, g]
            wt = scales_of(vv[:, None])[:, 0] if t else np.zeros(0)
            ref, bound = kv_ref.attention64(q[row:row + n, h], k[base:base + t, g], vv, wt, scale, seen)
            err = np.abs(out[row:row + n, h] - ref)
            assert (err <= bound).all(), (s, h, float((err / bound).max()))
            if n:
                worst = max(worst, float((err / bound).max()))
        row += n
        base += t
    say("largest error over its bound:", round(worst, 3))


CASES = [
    # news, lens, hq, hk, dim, page, window
    ([1], [1], 1, 1, 64, 32, 0),
    ([1], [1], 8, 8, 128, 128, 0),
    ([1, 1, 0, 1, 1, 1], [31, 32, 0, 33, 127, 128], 8, 1, 128, 32, 0),
    ([1, 1, 1], [129, 160, 257], 4, 4, 64, 64, 0),
    ([1, 1], [511, 513], 10, 2, 128, 64, 0),
    ([2, 3, 1], [2, 300, 65], 7, 1, 128, 128, 0),
    ([5, 8], [5, 400], 16, 4, 64, 32, 100),
    ([1, 4], [700, 900], 48, 2, 128, 32, 0),
    ([3, 1], [200, 130], 32, 1, 64, 256, 33),
    ([70, 9], [70, 140], 6, 2, 128, 32, 0),
    ([130], [257], 4, 1, 64, 32, 0),
    ([65, 1], [300, 1], 5, 5, 64, 4096, 64),
    ([40, 12], [200, 12], 8, 2, 128, 64, 1),
    ([1], [5000], 8, 1, 128, 128, 0),
    ([1, 1], [4200, 3], 4, 2, 64, 32, 0),
    ([3], [2600], 4, 2, 128, 64, 2300),
    ([200], [1500], 2, 1, 128, 64, 0),
    ([300], [300], 3, 3, 64, 32, 0),
    # many columns in all: 128 of them in a block
    ([40, 33, 36, 0, 38], [140, 33, 200, 0, 71], 128, 64, 128, 32, 0),
    ([66, 33, 70, 35], [66, 133, 90, 171], 128, 64, 64, 64, 50),
]


# bound 8192: columns in blocks of 128 wherever there are more than 64 of a
# sequence and head, and cached tokens in chunks
@pytest.mark.parametrize("bound", [0, 8192])
@pytest.mark.parametrize("news,lens,hq,hk,dim,page,window", CASES)
def test_attention(eq, news, lens, hq, hk, dim, page, window, bound):
    say("attn", news, lens, hq, hk, dim, page, window, bound)
    r = np.random.default_rng(sum(lens) + hq)
    n_pages = sum(-(-t // page) for t in lens) + 1
    b, starts, table = batch(eq, news, lens, page, n_pages, seed=5, bound=bound)
    cache, k, v, _ = filled(eq, r, lens, page, hk, dim, n_pages, b, starts)
    q = dev(r.standard_normal((starts[-1], hq, dim)).astype(np.float32), torch.bfloat16) * 2
    out = torch.full((starts[-1], hq, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    scale = dim ** -0.5
    ws = eq.attn_workspace(cache, b, hq)
    if ws is not None:
        ws.fill_(255)  # NaN: nothing may be read before it is written
    eq.eq_attn_kv4(cache, b, q, scale, out, ws, window=window)
    check(out.double().cpu().numpy(), q.double().cpu().numpy(), k, v, news, lens, scale, window)
    again = torch.empty_like(out)
    eq.eq_attn_kv4(cache, b, q, scale, again, ws, window=window)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))


@pytest.mark.parametrize("hq,bound", [(2, 0), (32, 8192)])
def test_rows_before_the_first_token_are_zero(eq, hq, bound):
    """More new rows than tokens: the rows that have no position see nothing."""
    r = np.random.default_rng(2)
    b, starts, table = batch(eq, [5], [3], 32, 2, bound=bound)
    full, _, _ = batch(eq, [3], [3], 32, 2)
    cache, k, v, _ = filled(eq, r, [3], 32, 1, 64, 2, full, None)
    q = dev(r.standard_normal((5, hq, 64)).astype(np.float32), torch.bfloat16)
    out = torch.full((5, hq, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    eq.eq_attn_kv4(cache, b, q, 0.125, out, eq.attn_workspace(cache, b, hq))
    o = out.double().cpu().numpy()
    assert (o[:2] == 0).all()
    check(o[2:], q.double().cpu().numpy()[2:], k, v, [3], [3], 0.125, 0)


@pytest.mark.parametrize("bound", [0, 8192])
def test_absent_pages_are_absent_tokens(eq, bound):
    r = np.random.default_rng(4)
    lens, news, page, hk, dim = [300, 90], [2, 90], 32, 2, 128
    b, starts, table = batch(eq, news, lens, page, 14, bound=bound)
    cache, k, v, _ = filled(eq, r, lens, page, hk, dim, 14, b, starts)
    gone = table.copy()
    gone[0, [0, 5]], gone[1, :2] = [-1, 14], [-3, 1 << 30]
    present = [np.ones(300, bool), np.ones(90, bool)]
    present[0][0:32] = present[0][160:192] = present[1][0:64] = False
    b2 = eq.KvBatch(b.tensors[0], b.tensors[1], dev(gone), n_tokens=92, max_new=90,
                    max_len=max(300, bound))
    q = dev(r.standard_normal((92, 4, dim)).astype(np.float32), torch.bfloat16)
    out = torch.full((92, 4, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    eq.eq_attn_kv4(cache, b2, q, dim ** -0.5, out, eq.attn_workspace(cache, b2, 4))
    o = out.double().cpu().numpy()
    check(o, q.double().cpu().numpy(), k, v, news, lens, dim ** -0.5, 0, present)
    assert (o[2:66] == 0).all()  # rows that see absent pages alone


@pytest.mark.parametrize("dim,new,bound", [(64, 1, 0), (128, 1, 0), (128, 24, 0), (128, 24, 8192),
                                           (64, 150, 0), (64, 150, 8192)])
def test_sharp_scores_and_values_of_unlike_size(eq, dim, new, bound):
    """Scores up to hundreds (P from 1 to an underflow), values that differ by
    2^40 between the tokens of a tile, zero queries, zero values."""
    r = np.random.default_rng(dim + new)
    lens, page = [290], 64
    b, starts, _ = batch(eq, [new], lens, page, 5, bound=bound)
    cache, k, v, whole = filled(eq, r, lens, page, 1, dim, 5, b, starts)
    kd = dev(r.standard_normal((290, 1, dim)).astype(np.float32))
    vd = dev(r.standard_normal((290, 1, dim)).astype(np.float32))
    vd *= torch.exp2(torch.randint(-20, 20, (290, 1, 1), device="cuda").float())
    vd[100] = 0
    kd[7] *= 1e-20
    eq.eq_kv_append(cache, whole, kd, vd)
    ko, vo = torch.empty(2, 290, 1, dim, dtype=torch.bfloat16, device="cuda")
    eq.eq_kv_read(cache, whole, ko, vo)
    q = r.standard_normal((new, 4, dim)) * np.array([0, 1, 12, 60])[None, :, None]
    q = dev(q.astype(np.float32), torch.bfloat16)
    out = torch.empty_like(q)
    eq.eq_attn_kv4(cache, b, q, dim ** -0.5, out, eq.attn_workspace(cache, b, 4))
    check(out.double().cpu().numpy(), q.double().cpu().numpy(), ko.double().cpu().numpy(),
          vo.double().cpu().numpy(), [new], lens, dim ** -0.5, 0)


@pytest.mark.parametrize("bound", [0, 8192])
@pytest.mark.parametrize("dim,new,heads", [(128, 40, 2), (64, 40, 2), (128, 150, 4)])
def test_nan_reaches_those_that_see_it(eq, dim, new, heads, bound):
    r = np.random.default_rng(6)
    lens, page, news = [new + 160], 32, [new]
    t = lens[0]
    b, starts, _ = batch(eq, news, lens, page, t // 32 + 1, bound=bound)
    cache, _, _, whole = filled(eq, r, lens, page, 1, dim, t // 32 + 1, b, starts)
    for which in ("k", "v", "q"):
        kd, vd = torch.randn(2, t, 1, dim, device="cuda")
        q = torch.randn(new, heads, dim, device="cuda").to(torch.bfloat16)
        eq.eq_kv_append(cache, whole, kd, vd)
        clean = torch.empty_like(q)
        ws = eq.attn_workspace(cache, b, heads)
        eq.eq_attn_kv4(cache, b, q, 0.1, clean, ws)
        bad = torch.zeros(new, heads, dtype=torch.bool, device="cuda")
        if which == "q":
            q[13, 1, dim - 1], q[20, 0, 3] = float("nan"), float("inf")
            bad[13, 1] = bad[20, 0] = True
        else:
            x = kd if which == "k" else vd
            x[t - new + 17, 0, 40] = float("nan")  # a new token: rows 17 on see it
            bad[17:] = True
            eq.eq_kv_append(cache, whole, kd, vd)
        out = torch.empty_like(q)
        eq.eq_attn_kv4(cache, b, q, 0.1, out, ws)
        assert torch.isnan(out[bad]).all(), which
        assert torch.equal(out[~bad].view(torch.int16), clean[~bad].view(torch.int16)), which


def test_strided_queries_and_another_stream(eq):
    r = np.random.default_rng(8)
    lens, news = [100, 37], [3, 2]
    b, starts, _ = batch(eq, news, lens, 32, 7)
    cache, k, v, _ = filled(eq, r, lens, 32, 2, 64, 7, b, starts)
    wide = torch.randn(5, 8 * 64, device="cuda").to(torch.bfloat16)
    q = wide[:, 128:384].unflatten(1, (4, 64))
    out, ref = torch.empty(2, 5, 4, 64, dtype=torch.bfloat16, device="cuda")
    eq.eq_attn_kv4(cache, b, q.contiguous(), 0.125, ref, eq.attn_workspace(cache, b, 4))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    eq.eq_attn_kv4(cache, b, q, 0.125, out, eq.attn_workspace(cache, b, 4), stream=s)
    s.synchronize()
    assert torch.equal(out.view(torch.int16), ref.view(torch.int16))
    check(out.double().cpu().numpy(), q.double().cpu().numpy(), k, v, news, lens, 0.125, 0)


@pytest.mark.parametrize("max_len", [1280, 5120])  # one chunk a sequence, several
def test_graph_of_a_generation_step(eq, max_len):
    """Norm and rotation, append and attention captured once, at the sizes that
    bound the run, and replayed as the sequences grow, with eager work between;
    every replay equals the eager calls bit for bit."""
    hq, hk, dim, page, n = 8, 2, 128, 32, 3
    start_lens, wide = [30, max_len - 80, 0], max_len // 32
    table = dev(np.random.default_rng(0).permutation(3 * wide).reshape(3, wide).astype(np.int32))
    lens = torch.tensor(start_lens, dtype=torch.int32, device="cuda")
    pos = torch.empty(3, dtype=torch.int32, device="cuda")
    starts = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    cos, sin = tables(max_len, dim // 2)
    rope = eq.Rope(dev(cos), dev(sin))
    w = torch.randn(dim, device="cuda").to(torch.bfloat16)
    b = eq.KvBatch(starts, lens, table, n_tokens=n, max_new=1, max_len=max_len)
    xq, xk, xv = (torch.randn(n, h, dim, device="cuda") for h in (hq, hk, hk))

    def state():
        g = torch.Generator(device="cuda")
        g.manual_seed(1)
        c = eq.KvCache.empty(3 * wide, page_tokens=page, kv_heads=hk, head_dim=dim)
        c.pages.copy_(torch.randint(0, 120, c.pages.shape, device="cuda", generator=g))
        return c, [torch.empty(n, h, dim, dtype=torch.bfloat16, device="cuda") for h in (hq, hk, hq)]

    def step(c, o, ws):
        eq.eq_qk_norm_rope(xq, xk, o[0], o[1], q_weight=w, k_weight=w, rope=rope, positions=pos)
        eq.eq_kv_append(c, b, o[1], xv)
        eq.eq_attn_kv4(c, b, o[0], dim ** -0.5, o[2], ws)

    ca, oa = state()
    cb, ob = state()
    wsa, wsb = eq.attn_workspace(ca, b, hq), eq.attn_workspace(cb, b, hq)
    assert (wsa is not None) == (max_len == 5120)
    pos.copy_(lens)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step(ca, oa, wsa)
    torch.cuda.current_stream().wait_stream(s)
    ca.pages.copy_(cb.pages)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(ca, oa, wsa)
    for i in range(5):
        pos.copy_(lens)
        lens.add_(1)
        xq.normal_(), xk.normal_(), xv.normal_()
        for o in oa:
            o.fill_(float("nan"))
        if wsa is not None:
            wsa.fill_(255)
        g.replay()
        step(cb, ob, wsb)
        torch.cuda.synchronize()
        for x, y in zip(oa, ob):
            assert torch.equal(x.view(torch.int16), y.view(torch.int16)), i
        assert torch.equal(ca.pages, cb.pages), i
        assert torch.isfinite(ob[2]).all(), i
