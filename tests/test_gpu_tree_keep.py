"""Keeping an accepted path in the cache, byte for byte, and a whole step of
speculative decoding in a captured graph."""
import sys

import numpy as np
import pytest

import kv_ref
import tree_ref
from test_gpu_kv import batch, dev, tables
from test_gpu_tree import tree

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


def move(pool, old, table, page, heads, dim, base, path, kept, n):
    """Token k of the new ones becomes token path[k] of the pool as it was."""
    a = kv_ref.Pool(1, page, heads, dim)
    for k in range(min(max(kept, 0), n)):
        if not k < path[k] < n:
            continue
        src, dst = base + path[k], base + k
        if src < 0 or dst < 0:
            continue
        ps, pd = table[src // page], table[dst // page]
        if not (0 <= ps < len(pool) and 0 <= pd < len(pool)):
            continue
        ts, td = src % page, dst % page
        for h in range(heads):
            at = h * a.hb
            pool[pd, at + td * (dim // 2):at + (td + 1) * (dim // 2)] = \
                old[ps, at + ts * (dim // 2):at + (ts + 1) * (dim // 2)]
            for g in range(dim // 32):
                pool[pd, a._key_scale(h, td, g)] = old[ps, a._key_scale(h, ts, g)]
            pool[pd, a._value_scale(h, td)] = old[ps, a._value_scale(h, ts)]
            code = old[ps, a._value_bytes(h, ts)] >> (4 * (ts % 2)) & 15
            v = pool[pd, a._value_bytes(h, td)]
            pool[pd, a._value_bytes(h, td)] = (v & 15) | code << 4 if td % 2 else (v & 240) | code


@pytest.mark.parametrize("layers", [1, 3, 128])
@pytest.mark.parametrize("news,lens,heads,dim,page", [
    ([1], [1], 1, 64, 32),
    ([5], [5], 1, 128, 32),
    ([8, 0, 33], [31, 0, 70], 3, 64, 32),
    ([40, 17, 3, 64], [100, 17, 66, 300], 5, 128, 64),
    ([256, 100], [300, 131], 2, 128, 128),
    ([9, 9, 9], [4100, 41, 73], 8, 64, 4096),
])
def test_kept_bytes(eq, news, lens, heads, dim, page, layers):
    if layers > 3 and heads > 3:
        layers = 7
    say("keep", news, lens, heads, dim, page, layers)
    r = np.random.default_rng(sum(lens))
    n_pages = sum(-(-t // page) for t in lens) + 1
    b, starts, table = batch(eq, news, lens, page, n_pages, n_tokens=sum(news) + 2)
    raw = r.integers(0, 256, (layers, n_pages, kv_ref.page_bytes(heads, dim, page)), dtype=np.uint8)
    pages = dev(raw)
    path = np.full(sum(news) + 2, -1, np.int32)
    kept = np.zeros(len(news), np.int32)
    for s, n in enumerate(news):
        m = int(r.integers(1, n + 1)) if n else 0
        kept[s] = m
        path[starts[s]:starts[s] + m] = np.sort(r.permutation(n)[:m]) if n else 0
    new_len = torch.full((len(news),), 99, dtype=torch.int32, device="cuda")
    caches = eq.KvCaches([eq.KvCache(p, page_tokens=page, kv_heads=heads, head_dim=dim) for p in pages])
    eq.eq_kv_keep(caches, b, dev(path), dev(kept), new_len)
    ref = raw.copy()
    for x, old in zip(ref, raw):
        for s, n in enumerate(news):
            move(x, old, table[s], page, heads, dim, lens[s] - n, path[starts[s]:starts[s] + n],
                 int(kept[s]), n)
    assert np.array_equal(pages.cpu().numpy(), ref)
    assert new_len.tolist() == [t - n + k for t, n, k in zip(lens, news, kept)]


def test_paths_and_counts_that_are_none(eq):
    """Entries before their place or behind the rows, counts outside the rows, pages
    that are not there: left out, and nothing else is touched."""
    r = np.random.default_rng(1)
    news, lens, heads, dim, page = [9, 9, 9, 9, 6], [40, 9, 100, 64, 4], 2, 128, 32
    b, starts, table = batch(eq, news, lens, page, 12)
    gone = table.copy()
    gone[2, 2], gone[3, 1] = -1, 12  # new places 91 .. 95 and 55 .. 63
    b = eq.KvBatch(b.tensors[0], b.tensors[1], dev(gone), n_tokens=42, max_new=9, max_len=100)
    raw = r.integers(0, 256, (12, kv_ref.page_bytes(heads, dim, page)), dtype=np.uint8)
    path = np.array([0, 0, 9, 5, 3, -7, 1 << 30, 8, -(1 << 31)] + [0, 2, 3, 4, 5, 6, 7, 8, 8] +
                    [0, 3, 4, 6, 7, 8, -1, -1, -1] + [0, 2, 5, 8, -1, -1, -1, -1, -1] +
                    [0, 1, 4, 4, 5, -1], np.int32)
    kept = np.array([9, 1 << 30, 6, 4, 5], np.int32)
    pages = dev(raw)
    new_len = torch.empty(5, dtype=torch.int32, device="cuda")
    eq.eq_kv_keep(eq.KvCache(pages, page_tokens=page, kv_heads=heads, head_dim=dim), b, dev(path),
                  dev(kept), new_len)
    ref = raw.copy()
    for s, n in enumerate(news):
        move(ref, raw, gone[s], page, heads, dim, lens[s] - n, path[starts[s]:starts[s] + n],
             int(kept[s]), n)
    assert np.array_equal(pages.cpu().numpy(), ref)
    assert new_len.tolist() == [40, 9, 97, 59, 5]
    # nothing kept: nothing moves; and no lengths asked for
    before = pages.clone()
    eq.eq_kv_keep([eq.KvCache(pages, page_tokens=page, kv_heads=heads, head_dim=dim)], b, dev(path),
                  dev(np.array([0, -5, 0, 0, 0], np.int32)))
    assert torch.equal(pages, before)


def test_a_step_in_a_graph(eq):
    """Masks, norm and rotation, append, attention, verification and keeping, captured
    once and replayed with other logits, trees and growing lengths, with eager work
    between: every replay equals the eager calls bit for bit, and the cache holds what
    appending the kept tokens in order would have left."""
    hq, hk, dim, page, n, nodes, vocab, layers = 8, 2, 128, 32, 3, 9, 1203, 2
    wide = 12
    table = dev(np.random.default_rng(0).permutation(n * wide).reshape(n, wide).astype(np.int32))
    starts = dev(np.array([0, 9, 14, 23], np.int32))
    rows = [9, 5, 9]
    cos, sin = tables(wide * page, dim // 2)
    rope = eq.Rope(dev(cos), dev(sin))
    g = torch.Generator(device="cuda")
    g.manual_seed(2)

    def normal(*shape, kind=torch.float32):
        return torch.randn(*shape, device="cuda", generator=g).to(kind)

    weight = normal(dim, kind=torch.bfloat16)
    x = [[normal(23, h, dim) for h in (hq, hk, hk)] for _ in range(layers)]
    target, draft = normal(23, vocab), normal(23, vocab)
    parents = torch.zeros(23, dtype=torch.int32, device="cuda")
    tokens = torch.zeros(23, dtype=torch.int32, device="cuda")
    u = torch.rand(23, device="cuda", generator=g)
    temps = torch.tensor([1.0, 0.0, 0.7], device="cuda")

    class State:
        def __init__(self):
            self.lens = torch.tensor([30, 64, 0], dtype=torch.int32, device="cuda")
            self.len_now = torch.empty_like(self.lens)
            self.batch = eq.KvBatch(starts, self.len_now, table, n_tokens=23, max_new=nodes,
                                    max_len=wide * page)
            self.pages = torch.zeros(layers, n * wide, kv_ref.page_bytes(hk, dim, page),
                                     dtype=torch.uint8, device="cuda")
            self.caches = eq.KvCaches([eq.KvCache(p, page_tokens=page, kv_heads=hk, head_dim=dim)
                                       for p in self.pages])
            self.mask, self.pos = eq.tree_buffers(self.batch)
            self.o = [[torch.empty(23, h, dim, dtype=torch.bfloat16, device="cuda") for h in (hq, hk, hq)]
                      for _ in range(layers)]
            self.aws = eq.attn_tree_workspace(self.caches.caches[0], self.batch, hq)
            self.path = torch.empty(23, dtype=torch.int32, device="cuda")
            self.kept, self.next, self.new = torch.empty(3, n, dtype=torch.int32, device="cuda")
            self.vws = eq.verify_workspace(self.batch, vocab)

        def step(self):
            torch.add(self.lens, starts[1:] - starts[:-1], out=self.len_now)
            eq.eq_tree_mask(self.batch, parents, self.mask, self.pos)
            for cache, o, (q, k, v) in zip(self.caches.caches, self.o, x):
                eq.eq_qk_norm_rope(q, k, o[0], o[1], q_weight=weight, k_weight=weight, rope=rope,
                                   positions=self.pos)
                eq.eq_kv_append(cache, self.batch, o[1], v)
                eq.eq_attn_kv4_tree(cache, self.batch, o[0], dim ** -0.5, self.mask, o[2], self.aws)
            eq.eq_tree_verify(self.batch, parents, tokens, target, draft, u, self.path, self.kept,
                              self.next, self.vws, temperature=temps, max_children=8)
            eq.eq_kv_keep(self.caches, self.batch, self.path, self.kept, self.new)
            self.lens.copy_(self.new)

    a, b = State(), State()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        a.step()
    torch.cuda.current_stream().wait_stream(s)
    a.lens.copy_(b.lens)
    a.pages.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.step()
    r = np.random.default_rng(3)
    straight = State()  # the kept tokens, appended one after another
    for i in range(6):
        trees = [tree(r, k, ("tree", "star", "chain")[(i + j) % 3]) for j, k in enumerate(rows)]
        parents.copy_(dev(np.concatenate(trees).astype(np.int32)))
        for row in x:
            for y in row:
                y.normal_(generator=g)
        target.normal_(generator=g)
        draft.copy_(target + 0.3 * normal(23, vocab))
        best = (target + 0.2 * normal(23, vocab)).argmax(dim=1).cpu().numpy()
        at = np.concatenate([starts[j].item() + np.maximum(p, 0) for j, p in enumerate(trees)])
        tokens.copy_(dev(best[at].astype(np.int32)))
        u.uniform_(generator=g)
        u.mul_(0.05)
        before = b.lens.tolist()
        for t in (a.path, a.kept, a.next, a.new):
            t.fill_(77)
        a.vws.fill_(255)
        graph.replay()
        b.step()
        torch.cuda.synchronize()
        for y, z in ((a.path, b.path), (a.kept, b.kept), (a.next, b.next), (a.lens, b.lens),
                     (a.pages, b.pages), (a.mask, b.mask), (a.pos, b.pos)):
            assert torch.equal(y, z), i
        for p, q in zip(a.o, b.o):
            assert torch.equal(p[2].view(torch.int16), q[2].view(torch.int16)), i
        say(i, "kept", b.kept.tolist(), "next", b.next.tolist())
        for j in range(n):
            lo, hi = starts[j].item(), starts[j + 1].item()
            ref, token = tree_ref.verify(trees[j], tokens[lo:hi].cpu().numpy(),
                                         target[lo:hi].double().cpu().numpy(),
                                         draft[lo:hi].double().cpu().numpy(), u[lo:hi].cpu().numpy(),
                                         temps[j].item())
            assert b.path[lo:lo + len(ref)].tolist() == ref and b.next[j].item() == token
        # the same tokens without a tree
        kept = b.kept.tolist()
        pick = torch.tensor([starts[j].item() + k for j in range(n)
                             for k in b.path[starts[j]:starts[j] + kept[j]].tolist()], device="cuda")
        flat = eq.KvBatch(dev(np.concatenate(([0], np.cumsum(kept))).astype(np.int32)), b.lens, table,
                          n_tokens=sum(kept), max_new=max(kept), max_len=wide * page)
        whole = eq.KvBatch(dev(np.concatenate(([0], np.cumsum(b.lens.tolist()))).astype(np.int32)), b.lens,
                           table, n_tokens=sum(b.lens.tolist()), max_new=max(b.lens.tolist()),
                           max_len=wide * page)
        for c, other, o, row in zip(straight.caches.caches, b.caches.caches, b.o, x):
            eq.eq_kv_append(c, flat, o[1][pick].contiguous(), row[2][pick].contiguous())
            got, want = (torch.empty(2, whole.n_tokens, hk, dim, dtype=torch.bfloat16, device="cuda")
                         for _ in range(2))
            eq.eq_kv_read(c, whole, want[0], want[1])
            eq.eq_kv_read(other, whole, got[0], got[1])
            assert torch.equal(got.view(torch.int16), want.view(torch.int16)), i
        assert b.lens.tolist() == [t + k for t, k in zip(before, kept)]
