"""What the drafted trees' entry points refuse, on the host and before any launch
(the pointers here are never followed), and the closed form that the kernels use."""
import ctypes

import numpy as np
import pytest

import paper_2601_22787_amd as eq
import tree_ref
from test_kv_abi import P, batch, cache, ref
from test_kv_limits import OnDevice


def mask(b, parents=P, out=P, pos=P, window=0):
    return eq.lib().eq_tree_mask(ref(b), parents, window, out, pos, None)


def attn(c, b, q=P, qs=512, heads=4, scale=1.0, window=0, m=P, pos=P, out=P, ws=P, nbytes=1 << 40):
    return eq.lib().eq_attn_kv4_tree(ref(c), ref(b), q, qs, heads, scale, window, m, pos, out, ws,
                                     nbytes, None)


def verify(b, parents=P, tokens=P, target=P, ts=100, tk=0, draft=P, ds=100, dk=1, vocab=100, temp=None,
           random=P, kids=1, path=P, kept=P, nxt=P, ws=P, nbytes=1 << 40):
    return eq.lib().eq_tree_verify(ref(b), parents, tokens, target, ts, tk, draft, ds, dk, vocab, temp,
                                   random, 0, kids, path, kept, nxt, ws, nbytes, None)


def keep(caches, b, path=P, kept=P, new_len=None, n=None):
    array = (ctypes.c_void_p * max(1, len(caches)))(*(ref(c) for c in caches))
    return eq.lib().eq_kv_keep(array, len(caches) if n is None else n, ref(b), path, kept, new_len, None)


BAD = [dict(seq_start=None), dict(n_seqs=65536), dict(max_new=5), dict(n_tokens=(1 << 30) + 1),
       dict(n_tokens=300, max_new=257)]


@pytest.mark.parametrize("call", [mask, verify, lambda b: attn(cache(), b), lambda b: keep([cache()], b)])
def test_batches_that_are_refused(call):
    for over in BAD:
        assert call(batch(**over)) == eq.EQ_EINVAL, over
    assert call(None) == eq.EQ_EINVAL
    assert call(batch(n_seqs=0)) == eq.EQ_OK


def test_masks_refused():
    for over in (dict(parents=None), dict(out=None), dict(pos=None)):
        assert mask(batch(), **over) == eq.EQ_EINVAL, over
    assert mask(batch(kv_len=None)) == eq.EQ_EINVAL
    assert mask(batch(max_new=0), parents=None, out=None, pos=None) == eq.EQ_OK


def test_attention_refused():
    for over in (dict(m=None), dict(window=5, pos=None), dict(q=None), dict(q=P + 2), dict(out=None),
                 dict(out=P + 8), dict(qs=508), dict(qs=256), dict(heads=3), dict(heads=0),
                 dict(scale=0.0), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert attn(cache(), batch(), **over) == eq.EQ_EINVAL, over
    c, long, wide = cache(), batch(max_pages=200, max_len=12000), batch(n_tokens=300, max_new=257)
    need = eq.lib().eq_attn_kv4_tree_workspace_bytes(ref(c), ref(long), 4)
    assert need > 0
    for over in (dict(ws=None), dict(nbytes=need - 1), dict(ws=P + 4)):
        assert attn(c, long, **over) == eq.EQ_EINVAL, over
    assert eq.lib().eq_attn_kv4_tree_workspace_bytes(ref(c), ref(wide), 4) == 0


def test_verification_refused():
    for over in (dict(parents=None), dict(tokens=None), dict(target=None), dict(random=None),
                 dict(path=None), dict(kept=None), dict(nxt=None), dict(ws=None), dict(ws=P + 8),
                 dict(ts=99), dict(ds=99), dict(tk=2), dict(dk=2), dict(vocab=0),
                 dict(vocab=(1 << 24) + 1, ts=1 << 25, ds=1 << 25), dict(kids=0),
                 dict(target=P + 2), dict(target=P + 1, tk=1), dict(draft=P + 1)):
        assert verify(batch(), **over) == eq.EQ_EINVAL, over
    b, wide = batch(), batch(max_new=257, n_tokens=300)

    def size(b, vocab, draft):
        return eq.lib().eq_tree_verify_workspace_bytes(ref(b), vocab, draft)

    assert verify(b, nbytes=size(b, 100, 1) - 1) == eq.EQ_EINVAL
    assert verify(b, draft=None, nbytes=size(b, 100, 0) - 1) == eq.EQ_EINVAL
    assert 0 < size(b, 100, 0) < size(b, 100, 1)
    assert size(b, 0, 0) == size(b, (1 << 24) + 1, 0) == size(wide, 100, 0) == size(None, 100, 0) == 0


def test_keeping_refused():
    a, size = cache(), eq.eq_kv_page_bytes(2, 128, 64) * 3
    b = cache(pages=P + (size + 127) // 128 * 128)
    for other in (cache(), cache(pages=P + 128), cache(pages=P + size - 128),
                  cache(pages=P + 8 * size, page_tokens=32), cache(pages=P + 8 * size, kv_heads=4),
                  cache(pages=P + 8 * size, head_dim=64), cache(pages=P + 8 * size, n_pages=4),
                  cache(pages=P + 8 * size + 64)):
        assert keep([a, other], batch()) == eq.EQ_EINVAL
    assert keep([], batch()) == eq.EQ_EINVAL
    assert keep([a], batch(), n=129) == eq.EQ_EINVAL
    for over in (dict(path=None), dict(kept=None), dict(new_len=P)):
        assert keep([a, b], batch(), **over) == eq.EQ_EINVAL, over
    assert keep([a, b], batch(n_seqs=0)) == eq.EQ_OK


def test_lengths_after_keeping_are_refused_where_the_call_reads():
    """new_len on kv_len, kept, path or seq_start, or on a part of them."""
    a, far = cache(), P + (1 << 20)
    b = batch(n_seqs=4, n_tokens=40, max_new=4, seq_start=far, kv_len=far + 4096)
    path, kept = far + 8192, far + 12288
    for new_len in (far, far + 4 * 4, far + 4096, far + 4096 + 12, far + 4096 - 12, path, path + 4 * 39,
                    path - 12, kept, kept - 4, kept + 12):
        assert keep([a], b, path, kept, new_len) == eq.EQ_EINVAL, hex(new_len - far)


def _call(which, at):
    """One call with every part on cuda:0 but for what `at` names."""
    torch = pytest.importorskip("torch")
    bf, i32, f32, u8 = torch.bfloat16, torch.int32, torch.float32, torch.uint8

    class Rows(OnDevice):
        def stride(self, i=None):
            s = OnDevice.stride(self)
            return s if i is None else s[i]

    def t(name, shape, dtype=i32):
        return Rows(shape, dtype, at.get(name, at.get("all", 0)))

    class Stream:
        cuda_stream, device_index = 0, at.get("stream", at.get("all", 0))

    stream = Stream if "stream" in at else None
    batch = eq.KvBatch(t("batch", (2,)), t("batch", (1,)), t("batch", (1, 3)), n_tokens=4, max_new=4,
                       max_len=100)
    cache = eq.KvCache(t("cache", (3, eq.eq_kv_page_bytes(2, 64, 64)), u8), page_tokens=64, kv_heads=2,
                       head_dim=64)
    if which == "mask":
        return eq.eq_tree_mask(batch, t("parents", (4,)), t("mask", (4, 1)), t("positions", (4,)),
                               stream=stream)
    if which == "attn":
        return eq.eq_attn_kv4_tree(cache, batch, t("q", (4, 4, 64), bf), 0.1, t("mask", (4, 1)),
                                   t("out", (4, 4, 64), bf), t("ws", (1 << 20,), u8),
                                   positions=t("positions", (4,)), stream=stream)
    if which == "verify":
        return eq.eq_tree_verify(batch, t("parents", (4,)), t("tokens", (4,)), t("target", (4, 50), f32),
                                 t("draft", (4, 50), bf), t("random", (4,), f32), t("path", (4,)),
                                 t("kept", (1,)), t("next", (1,)), t("ws", (1 << 20,), u8),
                                 temperature=t("temperature", (1,), f32), stream=stream)
    return eq.eq_kv_keep(cache, batch, t("path", (4,)), t("kept", (1,)), t("new_len", (1,)),
                         stream=stream)


PARTS = {"mask": ("batch", "parents", "mask", "positions"),
         "attn": ("cache", "batch", "q", "mask", "out", "ws", "positions"),
         "verify": ("batch", "parents", "tokens", "target", "draft", "random", "path", "kept", "next",
                    "ws", "temperature"),
         "keep": ("cache", "batch", "path", "kept", "new_len")}


@pytest.mark.parametrize("which,part", [(w, p) for w, parts in PARTS.items()
                                        for p in parts + ("stream", "all")])
def test_tensors_that_are_not_on_the_current_device_are_refused(which, part, monkeypatch):
    """A kernel would follow another device's addresses."""
    pytest.importorskip("torch")
    eq._kinds()
    monkeypatch.setattr(eq, "_current", lambda: 0)
    monkeypatch.setattr(eq, "_raw_stream", lambda device: 0)
    called, real = [], eq.lib()

    class Lib:
        def __getattr__(self, name):
            return getattr(real, name) if name == "eq_kv_page_bytes" else lambda *a: called.append(name) or 0

    monkeypatch.setattr(eq, "_lib", Lib())
    _call(which, {})
    assert len(called) == 1
    with pytest.raises(ValueError, match="device"):
        _call(which, {part: 1})
    assert len(called) == 1


def test_the_binding_refuses_types_and_sizes(monkeypatch):
    torch = pytest.importorskip("torch")
    eq._kinds()
    monkeypatch.setattr(eq, "_current", lambda: 0)
    for over in (dict(shape=(3, 50)), dict(shape=(4, 49)), dict(dtype=torch.float16)):
        a = dict(shape=(4, 50), dtype=torch.float32)
        a.update(over)
        x = OnDevice(a["shape"], a["dtype"], 0)
        with pytest.raises(ValueError, match="draft"):
            eq._logit_rows(x, type("B", (), {"n_tokens": 4}), 50, "draft", 0)
    with pytest.raises(ValueError, match="kept"):
        eq._ints(OnDevice((3,), torch.int64, 0), 3, "kept", 0)
    with pytest.raises(ValueError, match="kept"):
        eq._ints(OnDevice((2,), torch.int32, 0), 3, "kept", 0)
    for kids in (0, -1, 1 << 32):
        with pytest.raises(ValueError, match="max_children"):
            eq.eq_tree_verify(None, None, None, None, None, None, None, None, None, None,
                              max_children=kids)
    for window in (-1, 1 << 32):
        with pytest.raises(ValueError, match="window"):
            eq.eq_tree_mask(None, None, None, None, window=window)
        with pytest.raises(ValueError, match="window"):
            eq.eq_attn_kv4_tree(None, None, None, 1.0, None, None, window=window)
    with pytest.raises(ValueError, match="no caches"):
        eq.KvCaches([])


@pytest.mark.parametrize("replace", [False, True])
def test_one_family_holds_every_rejection(replace):
    """What is left of p after rejections is max(p - t q, 0) over its sum G(t), with t
    + G / Q in the place of t each time, and the next child's chance is as defined."""
    r = np.random.default_rng(2)
    for _ in range(50):
        v = int(r.integers(3, 40))
        p, q0 = tree_ref.softmax(2 * r.standard_normal(v), 1), tree_ref.softmax(2 * r.standard_normal(v), 1)
        rest, q, t, left, live = p, q0.copy(), 0.0, 1.0, np.ones(v, bool)
        for _ in range(6):
            g = np.maximum(p - t * q0, 0).sum()
            if g < 1e-9 or not live.any():
                break
            # any child that may be rejected
            able = np.flatnonzero((rest < q) & live & (q > 0))
            x = int(r.choice(able)) if len(able) else int(r.choice(np.flatnonzero(live)))
            if q[x] > 0:
                mine = max(p[x] - t * q0[x], 0) * left / (g * q0[x])
                assert abs(mine - rest[x] / q[x]) <= 1e-9 * max(1, mine)
            if not rest[x] < q[x]:
                break  # never rejected
            rest = np.maximum(rest - q, 0)
            if not replace:
                q[x] = 0
                live[x] = False
                q = q / q.sum() if q.sum() > 0 else q
            if rest.sum() <= 0:
                break
            rest = rest / rest.sum()
            t += g / left
            left -= 0 if replace else q0[x]
            if left < 1e-9:
                break
            w = np.maximum(p - t * q0, 0)
            assert np.abs(w / w.sum() - rest).max() <= 1e-9 / g
