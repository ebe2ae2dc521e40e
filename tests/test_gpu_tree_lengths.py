"""Lengths after a path was kept, of sequences with more rows than tokens: their first
rows have no place in the cache, and count for nothing in what is left."""
import numpy as np
import pytest

import kv_ref
from test_gpu_kv import dev
from test_gpu_tree_keep import eq, move, say  # noqa: F401 (eq: the fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_lengths_end_at_the_last_kept_place(eq):
    #        base  -2 -2 -2 -2 -2 -9 -6  0   3   -1   no rows
    lens = np.array([4, 4, 4, 4, 4, 0, 2, 6, 9, 255, 7], np.int32)
    news = np.array([6, 6, 6, 6, 6, 9, 8, 6, 6, 256, 0], np.int32)
    kept = np.array([5, 6, 2, 1, -3, 9, 7, 4, 6, 256, 3], np.int32)
    starts = np.concatenate(([0], np.cumsum(news))).astype(np.int32)
    n, page, heads, dim = len(lens), 32, 2, 64
    table = np.random.default_rng(0).permutation(9 * n).reshape(n, 9).astype(np.int32)
    b = eq.KvBatch(dev(starts), dev(lens), dev(table), n_tokens=int(starts[-1]), max_new=256, max_len=288)
    path = np.full(starts[-1], -1, np.int32)
    for s in range(n):  # every node, or with one left out
        m = max(0, min(kept[s], news[s]))
        path[starts[s]:starts[s] + m] = np.arange(m) + (np.arange(m) > 0) * (m < news[s])
    raw = np.random.default_rng(1).integers(0, 256, (9 * n, kv_ref.page_bytes(heads, dim, page)), dtype=np.uint8)
    pages = dev(raw)
    new_len = torch.full((n,), 99, dtype=torch.int32, device="cuda")
    eq.eq_kv_keep(eq.KvCache(pages, page_tokens=page, kv_heads=heads, head_dim=dim), b, dev(path),
                  dev(kept), new_len)
    m = np.where(news > 0, np.clip(kept, 0, news), news)
    want = np.maximum(lens - (news - m), 0)
    say("lengths", new_len.tolist(), want.tolist())
    assert new_len.tolist() == want.tolist()
    assert (new_len.cpu().numpy() <= lens).all()
    ref = raw.copy()
    for s in range(n):
        move(ref, raw, table[s], page, heads, dim, lens[s] - news[s], path[starts[s]:starts[s + 1]],
             int(kept[s]), int(news[s]))
    assert np.array_equal(pages.cpu().numpy(), ref)


def test_paths_that_are_none_and_lengths(eq):
    """Entries before their place or behind the rows, counts outside the rows, pages that
    are not there; a sequence of 6 rows and 4 tokens of which 5 are kept ends at place 3."""
    r = np.random.default_rng(1)
    news, lens, heads, dim, page = [9, 9, 9, 9, 6], [40, 9, 100, 64, 4], 2, 128, 32
    starts = np.concatenate(([0], np.cumsum(news))).astype(np.int32)
    table = np.full((5, 4), -1, np.int32)
    for s, (first, pages_of) in enumerate(((0, 2), (2, 1), (3, 4), (7, 2), (9, 1))):
        table[s, :pages_of] = first + np.arange(pages_of)
    table[2, 2], table[3, 1] = -1, 12
    b = eq.KvBatch(dev(starts), dev(np.array(lens, np.int32)), dev(table), n_tokens=42, max_new=9, max_len=100)
    raw = r.integers(0, 256, (12, kv_ref.page_bytes(heads, dim, page)), dtype=np.uint8)
    path = np.array([0, 0, 9, 5, 3, -7, 1 << 30, 8, -(1 << 31)] + [0, 2, 3, 4, 5, 6, 7, 8, 8] +
                    [0, 3, 4, 6, 7, 8, -1, -1, -1] + [0, 2, 5, 8, -1, -1, -1, -1, -1] +
                    [0, 1, 4, 4, 5, -1], np.int32)
    kept = np.array([9, 1 << 30, 6, 4, 5], np.int32)
    pages = dev(raw)
    cache = eq.KvCache(pages, page_tokens=page, kv_heads=heads, head_dim=dim)
    new_len = torch.empty(5, dtype=torch.int32, device="cuda")
    eq.eq_kv_keep(cache, b, dev(path), dev(kept), new_len)
    ref = raw.copy()
    for s, n in enumerate(news):
        move(ref, raw, table[s], page, heads, dim, lens[s] - n, path[starts[s]:starts[s] + n],
             int(kept[s]), n)
    assert np.array_equal(pages.cpu().numpy(), ref)
    assert new_len.tolist() == [40, 9, 97, 59, 3]
    # nothing kept: nothing moves; and no lengths asked for
    before = pages.clone()
    eq.eq_kv_keep([cache], b, dev(path), dev(np.array([0, -5, 0, 0, 0], np.int32)))
    assert torch.equal(pages, before)
