"""Norm and rotation of query and key heads, appending to the 4-bit cache and
reading it back, against a plain implementation: the cache byte for byte
(codes, scales, and every byte that must not change)."""
import sys

import numpy as np
import pytest

import kv_ref

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


def dev(x, kind=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if kind is None else t.to(kind)


def tables(rows, half, seed=0):
    a = np.arange(rows)[:, None] * 10000.0 ** (-np.arange(half) / max(half, 1))
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def batch(eq, news, lens, page, n_pages, seed=0, bound=0, **over):
    """A batch over a shuffled pool: (KvBatch, starts, page table).  bound: the
    most tokens that the page table has room for, where that is more."""
    r = np.random.default_rng(seed)
    starts = np.concatenate(([0], np.cumsum(news))).astype(np.int32)
    width = max(1, -(-max(max(lens), bound) // page))
    free = r.permutation(n_pages).astype(np.int32)
    table = np.full((len(lens), width), -1, dtype=np.int32)
    at = 0
    for i, t in enumerate(lens):
        n = -(-t // page)
        table[i, :n] = free[at:at + n]
        at += n
    a = dict(n_tokens=int(starts[-1]), max_new=max(news), max_len=max(max(lens), bound))
    a.update(over)
    b = eq.KvBatch(dev(starts), dev(np.array(lens, dtype=np.int32)), dev(table), **a)
    return b, starts, table


@pytest.mark.parametrize("tokens,hq,hk,dim,rot,pairs,norm,dtype,strided", [
    (1, 1, 1, 16, 16, False, True, "f32", False),
    (1, 64, 8, 128, 128, False, True, "f32", False),
    (5, 3, 0, 64, 32, False, True, "bf16", False),
    (37, 5, 2, 80, 32, False, True, "bf16", True),
    (33, 4, 4, 96, 96, True, True, "f32", True),
    (9, 2, 1, 256, 256, False, True, "bf16", False),
    (9, 2, 1, 256, 48, False, False, "f32", True),
    (130, 8, 1, 128, 64, True, False, "bf16", True),
    (3, 2, 2, 48, 0, False, True, "f32", False),
    (3, 7, 3, 112, 112, False, True, "bf16", "odd"),
])
def test_norm_rope(eq, tokens, hq, hk, dim, rot, pairs, norm, dtype, strided):
    """BF16 rounding (2^-8), a mean of up to 256 squares, a reciprocal square
    root and four more roundings in fp32 (2^-20 of the two rotated terms)."""
    say("norm", tokens, hq, hk, dim, rot, pairs, norm, dtype, strided)
    r = np.random.default_rng(tokens + dim)
    kind = torch.float32 if dtype == "f32" else torch.bfloat16
    pad = 1 if strided == "odd" else 8 if strided else 0
    x = dev(r.standard_normal((tokens, (hq + hk) * dim + pad)).astype(np.float32), kind) * 3
    x[0, :dim] = 0                      # a head of zeros
    q = x[:, pad:pad + hq * dim].unflatten(1, (hq, dim))
    k = x[:, pad + hq * dim:].unflatten(1, (hk, dim)) if hk else None
    if strided == "odd":                # rows that no 16-byte load can take
        assert q.data_ptr() % 16 and q.stride(0) % 8
    if not strided:
        q, k = q.contiguous(), None if k is None else k.contiguous()
    w = [dev(r.standard_normal(dim).astype(np.float32), torch.bfloat16) if norm else None
         for _ in range(2)]
    pos = r.integers(-2, 40, tokens).astype(np.int32)  # some outside the table of 37 rows
    cos, sin = tables(37, rot // 2)
    rope = eq.Rope(dev(cos), dev(sin), pairs=pairs) if rot else None
    out = [torch.full((tokens, h, dim), 7.0, dtype=torch.bfloat16, device="cuda") for h in (hq, hk)]
    eq.eq_qk_norm_rope(q, k, out[0], out[1] if hk else None, q_weight=w[0],
                       k_weight=w[1] if hk else None, eps=1e-5, rope=rope, positions=dev(pos))
    c, s = cos[np.clip(pos, 0, 36)][:, None], sin[np.clip(pos, 0, 36)][:, None]
    for y, a, wt in ((out[0], q, w[0]), (out[1], k, w[1])):
        if a is None:
            continue
        n = kv_ref.norm64(a.double().cpu().numpy(), None if wt is None else wt.double().cpu().numpy(),
                          1e-5)
        ref = kv_ref.rotate64(n, c, s, pairs) if rot else n
        size = kv_ref.rotate64(np.abs(n), np.abs(c), -np.abs(s), pairs) if rot else np.abs(n)
        if rot:  # both halves' sums of magnitudes
            size = np.maximum(np.abs(size), kv_ref.rotate64(np.abs(n), np.abs(c), np.abs(s), pairs))
        err = np.abs(y.double().cpu().numpy() - ref)
        assert (err <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -18 * np.abs(size) + 1e-30).all()


def test_norm_rope_in_place_stream_and_nan(eq):
    x = torch.randn(19, 6, 128, device="cuda").to(torch.bfloat16)
    k = torch.randn(19, 2, 128, device="cuda").to(torch.bfloat16)
    k[4, 1, 100] = float("nan")
    k[5, 0, 3] = float("inf")
    w = torch.randn(128, device="cuda").to(torch.bfloat16)
    cos, sin = tables(64, 64)
    rope, pos = eq.Rope(dev(cos), dev(sin)), torch.arange(19, dtype=torch.int32, device="cuda")
    a, b = torch.empty_like(x), torch.empty_like(k)
    eq.eq_qk_norm_rope(x, k, a, b, q_weight=w, k_weight=w, rope=rope, positions=pos)
    assert torch.isnan(b[4, 1]).all() and torch.isfinite(b[4, 0]).all()
    assert not torch.isfinite(b[5, 0]).all() and torch.isfinite(b[5, 1]).all()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    eq.eq_qk_norm_rope(x, k, x, k, q_weight=w, k_weight=w, rope=rope, positions=pos, stream=s)
    s.synchronize()
    assert torch.equal(x.view(torch.int16), a.view(torch.int16))
    assert torch.equal(torch.nan_to_num(k, 9.0), torch.nan_to_num(b, 9.0))


APPEND = [
    # news, lens, heads, dim, page, rot, pairs, dtype, layout
    ([1], [1], 1, 64, 32, 0, False, "f32", "plain"),
    ([1, 0, 1, 1], [33, 0, 64, 130], 2, 128, 32, 128, False, "f32", "plain"),
    ([7, 9, 1], [7, 40, 9], 3, 64, 64, 64, True, "bf16", "plain"),
    ([50, 3], [61, 3], 2, 128, 32, 96, False, "bf16", "fused"),
    ([23, 1, 8], [150, 129, 8], 1, 128, 128, 16, False, "f32", "odd"),
    ([40], [90], 2, 64, 4096, 48, True, "bf16", "odd"),
    ([33, 5], [70, 6], 2, 64, 32, 16, False, "f32", "fused"),
    ([3, 20], [30, 20], 2, 128, 64, 128, False, "bf16 f32", "plain"),
    ([9], [19], 1, 64, 32, 32, True, "f32 bf16", "plain"),
]


def _rows(r, tokens, heads, dim, dtype, layout):
    if " " in dtype:  # keys and values of two types
        return tuple(_rows(r, tokens, heads, dim, d, layout)[i] for i, d in enumerate(dtype.split()))
    kind = torch.float32 if dtype == "f32" else torch.bfloat16
    x = r.standard_normal((tokens, 2 * heads * dim + 8)) * np.exp(r.standard_normal((tokens, 1)) * 2)
    x = dev(x.astype(np.float32), kind)
    off = 1 if layout == "odd" else 8 if layout == "fused" else 0
    k = x[:, off:off + heads * dim].unflatten(1, (heads, dim))
    v = x[:, off + heads * dim:off + 2 * heads * dim].unflatten(1, (heads, dim))
    return (k.contiguous(), v.contiguous()) if layout == "plain" else (k, v)


@pytest.mark.parametrize("news,lens,heads,dim,page,rot,pairs,dtype,layout", APPEND)
@pytest.mark.parametrize("given", [False, True])
def test_append_and_read(eq, news, lens, heads, dim, page, rot, pairs, dtype, layout, given):
    """The pool's bytes are exactly the plain ones, those of other tokens
    included, and reading gives the codes' values."""
    say("append", news, lens, heads, dim, page, rot, pairs, dtype, layout, given)
    r = np.random.default_rng(sum(lens) + dim)
    n_pages = sum(-(-t // page) for t in lens) + 2
    pool = kv_ref.Pool(n_pages, page, heads, dim)
    pool.raw[:] = r.integers(0, 256, pool.raw.shape)  # earlier tokens and stale ones
    cache = eq.KvCache(dev(pool.raw), page_tokens=page, kv_heads=heads, head_dim=dim)
    b, starts, table = batch(eq, news, lens, page, n_pages, seed=3)
    k, v = _rows(r, starts[-1], heads, dim, dtype, layout)
    rope = pos = None
    if rot:
        cos, sin = tables(200, rot // 2)
        rope = eq.Rope(dev(cos), dev(sin), pairs=pairs)
        pos = r.integers(0, 200, starts[-1]).astype(np.int32) if given else None
    eq.eq_kv_append(cache, b, k, v, rope=rope, positions=None if pos is None else dev(pos))
    kn, vn = k.float().cpu().numpy(), v.float().cpu().numpy()
    place = np.concatenate([np.arange(t - n, t) for n, t in zip(news, lens)])
    if rot:
        at = place if pos is None else pos
        kn = kv_ref.rotate32(kn, cos[at][:, None], sin[at][:, None], pairs)
    want = np.empty((2, starts[-1], heads, dim))
    for s in range(len(lens)):
        for row in range(starts[s], starts[s + 1]):
            p = int(place[row])
            for h in range(heads):
                pool.put(table[s, p // page], p % page, h, kn[row, h], vn[row, h])
                want[0, row, h], want[1, row, h] = pool.get(table[s, p // page], p % page, h)
    got = cache.pages.cpu().numpy()
    assert np.array_equal(got, pool.raw), np.argwhere(got != pool.raw)[:5]
    ko = torch.full((starts[-1], heads, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    vo = ko.clone()
    eq.eq_kv_read(cache, b, ko, vo)
    assert np.array_equal(ko.double().cpu().numpy(), want[0])
    assert np.array_equal(vo.double().cpu().numpy(), want[1])


def test_append_rounds_to_even_and_keeps_its_range(eq):
    """Every tie between two codes, both signs, magnitudes from denormal to the
    largest, a group at the edge where its scale steps, zeros."""
    dim, page = 64, 32
    x = np.zeros((32, 1, dim), dtype=np.float32)
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=np.float32)
    for t in range(32):
        x[t, 0, :8] = np.concatenate((ties, [6.0])) * (-1) ** t
        x[t, 0, 8:16] = np.nextafter(np.concatenate((ties, [6.0])), np.float32(0))
        x[t, 0, 32:40] = np.concatenate((ties, [6.9]))
        x[t] *= np.float32(2.0) ** (t - 16)
    x[0], x[1] = 0, -0.0
    x[2, 0, 5], x[2, 0, 40] = 1e-42, -1e-30
    x[3, 0, 5], x[3, 0, 40] = 3.4e38, -3e38
    x[4, 0, 0] = np.float32(1.75)
    x[4, 0, 32] = np.nextafter(np.float32(1.75), np.float32(0))
    pool = kv_ref.Pool(1, page, 1, dim)
    cache = eq.KvCache(dev(pool.raw), page_tokens=page, kv_heads=1, head_dim=dim)
    b, _, _ = batch(eq, [32], [32], page, 1)
    eq.eq_kv_append(cache, b, dev(x), dev(x[:, :, ::-1].copy()))
    for t in range(32):
        pool.put(0, t, 0, x[t, 0], x[t, 0, ::-1])
    assert np.array_equal(cache.pages.cpu().numpy(), pool.raw)


def test_append_non_finite_groups_read_as_nan(eq):
    dim, page = 128, 32
    cache = eq.KvCache.empty(2, page_tokens=page, kv_heads=2, head_dim=dim)
    b, _, _ = batch(eq, [5], [37], page, 2)
    k, v = torch.randn(2, 5, 2, dim, device="cuda")
    k[1, 0, 40], k[2, 1, 0], v[3, 1, 127] = float("nan"), float("inf"), float("-inf")
    eq.eq_kv_append(cache, b, k, v)
    ko, vo = torch.empty(2, 5, 2, dim, dtype=torch.bfloat16, device="cuda")
    eq.eq_kv_read(cache, b, ko, vo)
    bad = torch.zeros(5, 2, dim, dtype=torch.bool, device="cuda")
    bad[1, 0, 32:64] = bad[2, 1, :32] = True
    assert torch.equal(torch.isnan(ko), bad)
    bad = torch.zeros(5, 2, dim, dtype=torch.bool, device="cuda")
    bad[3, 1] = True
    assert torch.equal(torch.isnan(vo), bad)


def test_rows_and_pages_outside_the_bounds_are_skipped(eq):
    """Page numbers that are not there, more rows or tokens than the host's
    bounds: nothing outside is written, the rest is."""
    dim, page, heads = 64, 32, 1
    lens, news = [70, 20], [40, 20]
    base = np.random.default_rng(1).integers(0, 256, (4, kv_ref.page_bytes(heads, dim, page)),
                                             dtype=np.uint8)
    k, v = torch.randn(2, 60, heads, dim, device="cuda")
    starts, table = np.array([0, 40, 60], np.int32), np.array([[0, 9, 2], [-5, -1, -1]], np.int32)

    def run(**over):
        cache = eq.KvCache(dev(base), page_tokens=page, kv_heads=heads, head_dim=dim)
        a = dict(n_tokens=60, max_new=40, max_len=96)
        a.update(over)
        b = eq.KvBatch(dev(starts), dev(np.array(lens, np.int32)), dev(table), **a)
        eq.eq_kv_append(cache, b, k, v)
        o = torch.full((2, 60, heads, dim), 7.0, dtype=torch.bfloat16, device="cuda")
        eq.eq_kv_read(cache, b, o[0], o[1])
        return cache.pages.cpu().numpy(), o

    def expect(rows):
        pool = kv_ref.Pool(4, page, heads, dim)
        pool.raw[:] = base
        for i in rows:
            p = 30 + i
            pool.put(table[0, p // page], p % page, 0, k[i, 0].cpu().numpy(), v[i, 0].cpu().numpy())
        return pool.raw

    there = [i for i in range(40) if (30 + i) // page != 1]   # page 9 does not exist
    for over, rows in (({}, there), ({"max_new": 1}, [0]), ({"n_tokens": 3, "max_new": 3}, [0, 1]),
                       ({"max_len": 66}, [i for i in there if i < 36])):
        got, o = run(**over)
        assert np.array_equal(got, expect(rows)), over
        left = torch.ones(60, dtype=torch.bool)
        left[[r for r in rows]] = False
        if "n_tokens" not in over:
            assert (o[:, left.cuda()] == 7.0).all(), over
        assert (o[:, ~left.cuda()] != 7.0).any(), over


@pytest.mark.parametrize("length", [97, 2**30 + 5, 2**31 - 1])
def test_rows_behind_the_longest_length_are_left_out(eq, length):
    """One row a sequence, at the end of a length above the host's bound: the
    cache and the outputs stay as they are."""
    dim, page, heads = 64, 32, 2
    base = np.random.default_rng(2).integers(0, 256, (3, kv_ref.page_bytes(heads, dim, page)),
                                             dtype=np.uint8)
    cache = eq.KvCache(dev(base), page_tokens=page, kv_heads=heads, head_dim=dim)
    b = eq.KvBatch(dev(np.array([0, 1, 2], np.int32)), dev(np.array([length] * 2, np.int32)),
                   dev(np.array([[0, 1, 2]] * 2, np.int32)), n_tokens=64, max_new=64, max_len=96)
    k, v = torch.randn(2, 64, heads, dim, device="cuda")
    eq.eq_kv_append(cache, b, k, v)
    o = torch.full((2, 64, heads, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    eq.eq_kv_read(cache, b, o[0], o[1])
    assert np.array_equal(cache.pages.cpu().numpy(), base)
    assert (o == 7.0).all()


def test_pool_beyond_32_bits(eq):
    """The last page of a pool of more than 4 GiB."""
    dim, page, heads = 128, 128, 8
    nbytes = kv_ref.page_bytes(heads, dim, page)
    n = (5 << 30) // nbytes
    cache = eq.KvCache.empty(n, page_tokens=page, kv_heads=heads, head_dim=dim)
    cache.pages[0] = 0
    lens = dev(np.array([9], np.int32))
    table = dev(np.array([[n - 1]], np.int32))
    b = eq.KvBatch(dev(np.array([0, 9], np.int32)), lens, table, n_tokens=9, max_new=9, max_len=9)
    k, v = torch.randn(2, 9, heads, dim, device="cuda")
    eq.eq_kv_append(cache, b, k, v)
    o = torch.empty(2, 9, heads, dim, dtype=torch.bfloat16, device="cuda")
    eq.eq_kv_read(cache, b, o[0], o[1])
    assert not cache.pages[0].any()
    # E2M1 is within a quarter of the value (0.25 to 0.5 apart: half of 2^-1) or
    # of the smallest step of the group (a quarter of 2^(b-127) <= top / 14)
    for x, y in ((k, o[0]), (v, o[1])):
        top = x.abs().amax(dim=-1, keepdim=True)
        assert ((x - y.float()).abs() <= torch.maximum(x.abs() / 4, top / 14)).all()
    # queries whose scores are flat average the values that were read
    q = torch.zeros(9, heads, dim, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(q)
    eq.eq_attn_kv4(cache, b, q, 1.0, out, eq.attn_workspace(cache, b, heads))
    ref = o[1].double().cumsum(0) / torch.arange(1, 10, device="cuda")[:, None, None]
    assert ((out.double() - ref).abs() <= 2.0 ** -7 * o[1].double().abs().amax()).all()
