"""Drafted trees: masks and positions, attention of their nodes over the 4-bit cache
against attention in 64 bits, and a whole step of speculative decoding in a graph."""
import sys

import numpy as np
import pytest

import kv_ref
import tree_ref
from test_gpu_attn import filled, scales_of
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


def tree(r, n, kind="tree"):
    """Parents of n nodes."""
    if kind == "chain":
        return np.arange(-1, n - 1)
    if kind == "star":
        return np.array([-1] + [0] * (n - 1))[:n]
    if kind == "roots":  # several under the cached tokens
        return np.array([r.integers(-1, i) if i else -1 for i in range(n)])
    return np.array([r.integers(max(0, i - 9), i) if i else -1 for i in range(n)])


def masked(news, lens, parents, window=0):
    """(mask words, positions, per sequence what each node sees [n, T])."""
    words = max(1, -(-max(news) // 32))
    mask, pos, seen = [], [], []
    for n, t, p in zip(news, lens, parents):
        own, at = tree_ref.masks(p, t - n, window)
        mask.append(tree_ref.words(own, words))
        pos.append(at)
        j = np.arange(t)[None, :]
        old = (j < t - n) & own.any(axis=1)[:, None]
        if window:
            old &= j > np.maximum(at, t - n)[:, None] - window
        s = np.broadcast_to(old, (n, t)).copy()
        for k in range(max(0, n - t), n):
            s[:, t - n + k] = own[:, k]
        s[:max(0, n - t)] = False
        seen.append(s)
    return (np.concatenate(mask).astype(np.int32), np.concatenate(pos).astype(np.int32), seen)


def check(out, q, k, v, seen, scale):
    """out [tokens, Hq, D] against the reference; seen: per sequence [n, T]."""
    hq, hk = q.shape[1], k.shape[1]
    row = base = 0
    worst = 0.0
    for s, m in enumerate(seen):
        n, t = m.shape
        for h in range(hq):
            g = h // (hq // hk)
            vv = v[base:base + t, g]
            wt = scales_of(vv[:, None])[:, 0] if t else np.zeros(0)
            ref, bound = kv_ref.attention64(q[row:row + n, h], k[base:base + t, g], vv, wt, scale, m)
            err = np.abs(out[row:row + n, h] - ref)
            assert (err <= bound).all(), (s, h, float((err / bound).max()))
            if n:
                worst = max(worst, float((err / bound).max()))
        row += n
        base += t
    say("largest error over its bound:", round(worst, 3))


# ---------------------------------------------------------------------- masks
@pytest.mark.parametrize("window", [0, 1, 3, 300])
@pytest.mark.parametrize("news", [[1], [2, 0, 33], [64, 1, 31, 0, 32], [256, 255, 5], [65]])
def test_masks_and_positions(eq, news, window):
    say("mask", news, window)
    r = np.random.default_rng(sum(news) + window)
    lens = [n + int(r.integers(0, 500)) for n in news]
    lens[0] = max(0, news[0] - 1)  # fewer tokens than rows
    kinds = ["chain", "tree", "star", "roots"]
    parents = [tree(r, n, kinds[(i + window) % 4]) for i, n in enumerate(news)]
    flat = np.concatenate(parents).astype(np.int32)
    b, starts, _ = batch(eq, news, [max(t, 1) for t in lens], 32, 100, n_tokens=sum(news) + 3,
                         max_new=max(news))
    b.tensors[1].copy_(dev(np.array(lens, dtype=np.int32)))
    words = -(-max(news) // 32)
    mask = torch.full((sum(news) + 3, words), 77, dtype=torch.int32, device="cuda")
    pos = torch.full((sum(news) + 3,), 77, dtype=torch.int32, device="cuda")
    eq.eq_tree_mask(b, dev(np.concatenate((flat, [0, 0, 0])).astype(np.int32)), mask, pos, window=window)
    ref = [tree_ref.masks(p, t - n, window) for p, t, n in zip(parents, lens, news)]
    assert np.array_equal(mask.cpu().numpy()[:-3],
                          np.concatenate([tree_ref.words(m, words) for m, _ in ref]))
    assert np.array_equal(pos.cpu().numpy()[:-3], np.concatenate([p for _, p in ref]))
    assert (mask[-3:] == 77).all() and (pos[-3:] == 77).all()  # rows of no sequence


def test_nodes_that_hang_on_nothing_are_left_out(eq):
    parents = np.array([-1, 0, 5, 2, -2, 4, 1, 7, 1 << 30, -(1 << 31), 8], dtype=np.int32)
    b, _, _ = batch(eq, [11], [40], 32, 2)
    mask, pos = eq.tree_buffers(b)
    eq.eq_tree_mask(b, dev(parents), mask, pos)
    own, at = tree_ref.masks(parents, 29)
    assert np.array_equal(mask.cpu().numpy(), tree_ref.words(own, 1))
    assert pos.tolist() == at.tolist() == [29, 30, -1, -1, -1, -1, 31, -1, -1, -1, -1]


# ------------------------------------------------------------------ attention
CASES = [
    # news, lens, hq, hk, dim, page, window
    ([1], [1], 1, 1, 64, 32, 0),
    ([1], [1], 8, 8, 128, 128, 0),
    ([8], [8], 1, 1, 128, 64, 0),
    ([8], [130], 1, 1, 64, 32, 0),
    ([4, 1, 0, 3], [31, 33, 0, 260], 4, 2, 128, 32, 0),
    ([7, 2], [127, 129], 8, 1, 64, 64, 0),
    ([33, 64, 31], [160, 64, 700], 4, 2, 128, 64, 0),
    ([13, 9, 0, 12, 5], [700, 90, 0, 12, 555], 16, 4, 64, 32, 100),
    ([20], [300], 2, 1, 128, 4096, 7),
    ([256, 200], [900, 200], 2, 2, 64, 32, 0),
    ([256], [256], 8, 4, 128, 64, 0),
    ([70, 256], [400, 300], 2, 1, 128, 32, 150),
    ([16, 3], [4200, 2100], 8, 1, 128, 128, 0),
    ([40, 33, 36, 0, 38], [140, 33, 200, 0, 71], 128, 64, 128, 32, 0),
    ([66, 33, 70, 35], [66, 133, 90, 171], 128, 64, 64, 64, 50),
]


# bound 8192: columns in blocks of 128 wherever there are more than 64 of a
# sequence and head, and cached tokens in chunks
@pytest.mark.parametrize("bound", [0, 8192])
@pytest.mark.parametrize("news,lens,hq,hk,dim,page,window", CASES)
def test_attention(eq, news, lens, hq, hk, dim, page, window, bound):
    say("tree attn", news, lens, hq, hk, dim, page, window, bound)
    r = np.random.default_rng(sum(lens) + hq)
    n_pages = sum(-(-t // page) for t in lens) + 1
    b, starts, _ = batch(eq, news, lens, page, n_pages, seed=5, bound=bound)
    cache, k, v, _ = filled(eq, r, lens, page, hk, dim, n_pages, b, starts)
    parents = [tree(r, n, ["tree", "chain", "roots", "star"][i % 4]) for i, n in enumerate(news)]
    for p in parents:
        if len(p) > 6:
            p[5] = 6  # no node, nor what is behind it
    mask, pos, seen = masked(news, lens, parents, window)
    q = dev(r.standard_normal((starts[-1], hq, dim)).astype(np.float32), torch.bfloat16) * 2
    out = torch.full((starts[-1], hq, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    scale = dim ** -0.5
    ws = eq.attn_tree_workspace(cache, b, hq)
    if ws is not None:
        ws.fill_(255)  # NaN: nothing may be read before it is written
    eq.eq_attn_kv4_tree(cache, b, q, scale, dev(mask), out, ws, positions=dev(pos) if window else None,
                        window=window)
    check(out.double().cpu().numpy(), q.double().cpu().numpy(), k, v, seen, scale)
    again = torch.empty_like(out)
    eq.eq_attn_kv4_tree(cache, b, q, scale, dev(mask), again, ws, positions=dev(pos), window=window)
    assert torch.equal(out.view(torch.int16), again.view(torch.int16))


# more columns than the card runs at once: chunks by the lengths of all (65 sequences: none)
MANY = [
    ([130, 70, 129], [5000, 300, 2500], 64, 64, 64, 128, 0),
    ([130, 0, 129], [3100, 0, 130], 64, 64, 64, 32, 0),
    ([130, 70, 129], [5000, 300, 2500], 64, 64, 64, 64, 4000),
    ([9] * 32, [9, 4200] + [40] * 30, 64, 8, 128, 64, 0),
    ([66] + [1] * 64, [2300] + [3] * 64, 4, 4, 64, 32, 0),
]


@pytest.mark.parametrize("news,lens,hq,hk,dim,page,window", MANY)
def test_attention_of_many(eq, news, lens, hq, hk, dim, page, window):
    test_attention(eq, news, lens, hq, hk, dim, page, window, 8192)


@pytest.mark.parametrize("bound", [0, 8192])
@pytest.mark.parametrize("news,lens,hq,hk,dim,page", [c[:6] for c in CASES])
def test_a_chain_is_causal_attention(eq, news, lens, hq, hk, dim, page, bound):
    """Bit for bit: the same tiles, the same sums."""
    r = np.random.default_rng(3)
    n_pages = sum(-(-t // page) for t in lens) + 1
    b, starts, _ = batch(eq, news, lens, page, n_pages, seed=5, bound=bound)
    cache, _, _, _ = filled(eq, r, lens, page, hk, dim, n_pages, b, starts)
    mask, pos = eq.tree_buffers(b)
    eq.eq_tree_mask(b, dev(np.concatenate([tree(r, n, "chain") for n in news]).astype(np.int32)), mask, pos)
    q = dev(r.standard_normal((starts[-1], hq, dim)).astype(np.float32), torch.bfloat16)
    out, ref = torch.empty(2, starts[-1], hq, dim, dtype=torch.bfloat16, device="cuda")
    eq.eq_attn_kv4_tree(cache, b, q, 0.1, mask, out, eq.attn_tree_workspace(cache, b, hq))
    eq.eq_attn_kv4(cache, b, q, 0.1, ref, eq.attn_workspace(cache, b, hq))
    assert torch.equal(out.view(torch.int16), ref.view(torch.int16))


@pytest.mark.parametrize("bound,hq", [(0, 2), (0, 8), (8192, 8)])
def test_any_mask(eq, bound, hq):
    """Bits that are no tree's: later tokens, not oneself, bits beyond the rows, and
    rows without any, which see nothing of the cached tokens either."""
    r = np.random.default_rng(9)
    news, lens, page, hk, dim = [12, 4], [150, 40], 32, 2, 128
    news[0] = 40 if bound else 12
    b, starts, _ = batch(eq, news, lens, page, 8, bound=bound)
    cache, k, v, _ = filled(eq, r, lens, page, hk, dim, 8, b, starts)
    mask = r.integers(-(1 << 31), 1 << 31, (sum(news), b.mask_words)).astype(np.int32)
    mask[3] = mask[news[0] + 1] = 0
    seen, row = [], 0
    for n, t in zip(news, lens):
        bits = (mask[row:row + n, :, None].view(np.uint32) >> np.arange(32, dtype=np.uint32) & 1)
        bits = bits.reshape(n, -1).astype(bool)
        s = np.zeros((n, t), bool)
        s[:, :t - n] = bits.any(axis=1)[:, None]  # a bit beyond the rows makes a node all the same
        s[:, t - n:] = bits[:, :n]
        seen.append(s)
        row += n
    q = dev(r.standard_normal((sum(news), hq, dim)).astype(np.float32), torch.bfloat16)
    out = torch.full((sum(news), hq, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    eq.eq_attn_kv4_tree(cache, b, q, 0.1, dev(mask), out, eq.attn_tree_workspace(cache, b, hq))
    o = out.double().cpu().numpy()
    check(o, q.double().cpu().numpy(), k, v, seen, 0.1)
    assert (o[3] == 0).all() and (o[news[0] + 1] == 0).all()


@pytest.mark.parametrize("hq,bound", [(2, 0), (32, 8192)])
def test_rows_before_the_first_token_are_zero(eq, hq, bound):
    """More rows than tokens: the first rows have no place, and see nothing."""
    r = np.random.default_rng(2)
    b, starts, _ = batch(eq, [5], [3], 32, 2, bound=bound)
    full, _, _ = batch(eq, [3], [3], 32, 2)
    cache, k, v, _ = filled(eq, r, [3], 32, 1, 64, 2, full, None)
    mask, pos, seen = masked([5], [3], [tree(r, 5, "star")])
    q = dev(r.standard_normal((5, hq, 64)).astype(np.float32), torch.bfloat16)
    out = torch.full((5, hq, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    eq.eq_attn_kv4_tree(cache, b, q, 0.125, dev(mask), out, eq.attn_tree_workspace(cache, b, hq))
    o = out.double().cpu().numpy()
    assert (o[:2] == 0).all() and (o[2:] != 0).any()
    check(o, q.double().cpu().numpy(), k, v, seen, 0.125)


@pytest.mark.parametrize("bound", [0, 8192])
def test_absent_pages_and_nodes_that_are_not_seen(eq, bound):
    """A page that is not there is no tokens; NaN reaches the nodes that see it alone."""
    r = np.random.default_rng(4)
    lens, news, page, hk, hq, dim = [300], [40], 32, 1, 4, 128
    b, starts, table = batch(eq, news, lens, page, 11, bound=bound)
    cache, k, v, whole = filled(eq, r, lens, page, hk, dim, 11, b, starts)
    mask, pos, seen = masked(news, lens, [tree(r, 40, "star")])
    q = dev(r.standard_normal((40, hq, dim)).astype(np.float32), torch.bfloat16)
    out = torch.empty_like(q)
    gone = table.copy()
    gone[0, [1, 8]] = [-1, 1 << 30]
    b2 = eq.KvBatch(b.tensors[0], b.tensors[1], dev(gone), n_tokens=40, max_new=40,
                    max_len=max(300, bound))
    ws = eq.attn_tree_workspace(cache, b, hq)
    eq.eq_attn_kv4_tree(cache, b2, q, 0.1, dev(mask), out, ws)
    there = seen[0].copy()
    there[:, 32:64] = there[:, 256:288] = False
    check(out.double().cpu().numpy(), q.double().cpu().numpy(), k, v, [there], 0.1)
    clean = torch.empty_like(q)
    eq.eq_attn_kv4_tree(cache, b, q, 0.1, dev(mask), clean, ws)
    for which in (0, 1):
        kv = [dev(k.astype(np.float32)), dev(v.astype(np.float32))]
        kv[which][260 + 17, 0, 40] = float("nan")  # node 17, a leaf
        eq.eq_kv_append(cache, whole, *kv)
        eq.eq_attn_kv4_tree(cache, b, q, 0.1, dev(mask), out, ws)
        bad = torch.zeros(40, dtype=torch.bool, device="cuda")
        bad[17] = True
        assert torch.isnan(out[bad]).all()
        assert torch.equal(out[~bad].view(torch.int16), clean[~bad].view(torch.int16))


def test_strided_queries_and_another_stream(eq):
    r = np.random.default_rng(8)
    lens, news = [100, 37], [3, 2]
    b, starts, _ = batch(eq, news, lens, 32, 7)
    cache, k, v, _ = filled(eq, r, lens, 32, 2, 64, 7, b, starts)
    mask, pos, seen = masked(news, lens, [tree(r, 3, "star"), tree(r, 2)])
    wide = torch.randn(5, 8 * 64, device="cuda").to(torch.bfloat16)
    q = wide[:, 128:384].unflatten(1, (4, 64))
    out = torch.empty(5, 4, 64, dtype=torch.bfloat16, device="cuda")
    md = dev(mask)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    eq.eq_attn_kv4_tree(cache, b, q, 0.125, md, out, eq.attn_tree_workspace(cache, b, 4), stream=s)
    s.synchronize()
    check(out.double().cpu().numpy(), q.double().cpu().numpy(), k, v, seen, 0.125)


@pytest.mark.parametrize("n", [64, 66])
def test_batches_of_many_ragged_trees(eq, n):
    """Up to 64 sequences share chunks of one length that their lengths set; more have the
    host's."""
    r = np.random.default_rng(n)
    news = [int(x) for x in r.integers(0, 24, n)]
    news[5] = 40
    lens = [k + int(x) if k else 0 for k, x in zip(news, r.integers(0, 90, n))]
    lens[7] = news[7] + 2500
    n_pages = sum(-(-t // 64) for t in lens) + 1
    b, starts, _ = batch(eq, news, lens, 64, n_pages, seed=5, bound=8192)
    cache, k, v, _ = filled(eq, r, lens, 64, 1, 64, n_pages, b, starts)
    mask, pos, seen = masked(news, lens, [tree(r, k) for k in news])
    q = dev(r.standard_normal((starts[-1], 2, 64)).astype(np.float32), torch.bfloat16)
    out = torch.full((starts[-1], 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = eq.attn_tree_workspace(cache, b, 2)
    ws.fill_(255)
    eq.eq_attn_kv4_tree(cache, b, q, 0.125, dev(mask), out, ws)
    check(out.double().cpu().numpy(), q.double().cpu().numpy(), k, v, seen, 0.125)
