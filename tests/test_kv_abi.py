"""What the cache's and attention's entry points refuse, on the host and before
any launch (the pointers here are never followed)."""
import ctypes

import numpy as np
import pytest

import kv_ref
import paper_2601_22787_amd as eq

FAKE = np.zeros(4096, dtype=np.uint8)
P = (FAKE.ctypes.data + 255) // 256 * 256


def cache(**over):
    a = dict(pages=P, n_pages=3, page_tokens=64, kv_heads=2, head_dim=128)
    a.update(over)
    return eq.eq_kv_cache(**a)


def batch(**over):
    a = dict(seq_start=P, kv_len=P, page_table=P, n_seqs=2, max_pages=3, n_tokens=4, max_new=2,
             max_len=100)
    a.update(over)
    return eq.eq_kv_batch(**a)


def rope(**over):
    a = dict(cos=P, sin=P, rows=10, dims=128, pairs=0)
    a.update(over)
    return eq.eq_rope(**a)


def ref(x):
    return None if x is None else ctypes.addressof(x)


def append(c, b, k=P, ks=256, kk=0, v=P, vs=256, kv=1, r=None):
    return eq.lib().eq_kv_append(ref(c), ref(b), k, ks, kk, v, vs, kv, None, ref(r), None)


def read(c, b, k=P, v=P):
    return eq.lib().eq_kv_read(ref(c), ref(b), k, v, None)


def attn(c, b, q=P, qs=512, heads=4, scale=1.0, out=P, ws=P, nbytes=1 << 40):
    return eq.lib().eq_attn_kv4(ref(c), ref(b), q, qs, heads, scale, 0, out, ws, nbytes, None)


def norm(q=P, qs=256, hq=2, qo=P, k=P, ks=128, hk=1, ko=P, kind=0, tokens=3, dim=128, eps=1e-5,
         pos=P, r=None):
    return eq.lib().eq_qk_norm_rope(q, qs, hq, None, qo, k, ks, hk, None, ko, kind, tokens, dim, eps,
                                    pos, ref(r), None)


@pytest.mark.parametrize("heads,dim,page", [(1, 64, 32), (8, 128, 32), (8, 128, 64), (2, 64, 4096),
                                            (1024, 128, 128)])
def test_page_bytes(heads, dim, page):
    assert eq.eq_kv_page_bytes(heads, dim, page) == kv_ref.page_bytes(heads, dim, page)


def test_page_bytes_of_unsupported_sizes():
    for a in ((0, 128, 64), (1025, 128, 64), (8, 96, 64), (8, 256, 64), (8, 128, 16), (8, 128, 48),
              (8, 128, 8192), (8, 128, 0)):
        assert eq.eq_kv_page_bytes(*a) == 0, a


BAD_CACHE = [dict(pages=None), dict(pages=P + 64), dict(n_pages=0), dict(n_pages=1 << 31),
             dict(page_tokens=48), dict(kv_heads=0), dict(head_dim=80)]
BAD_BATCH = [dict(seq_start=None), dict(kv_len=None), dict(page_table=None), dict(n_seqs=65536),
             dict(max_new=5), dict(max_len=193), dict(n_tokens=(1 << 30) + 1, max_new=1),
             dict(max_pages=0)]


@pytest.mark.parametrize("call", [append, read, attn])
def test_caches_and_batches_that_are_refused(call):
    for over in BAD_CACHE:
        assert call(cache(**over), batch()) == eq.EQ_EINVAL, over
    for over in BAD_BATCH:
        assert call(cache(), batch(**over)) == eq.EQ_EINVAL, over
    assert call(None, batch()) == eq.EQ_EINVAL
    assert call(cache(), None) == eq.EQ_EINVAL


@pytest.mark.parametrize("call", [append, read, attn])
def test_nothing_to_do(call):
    assert call(cache(), batch(n_seqs=0)) == eq.EQ_OK
    assert call(cache(), batch(max_new=0)) == eq.EQ_OK


def test_append_refusals():
    for a in (dict(k=None), dict(v=None), dict(ks=255), dict(vs=255), dict(kk=2), dict(kv=2)):
        assert append(cache(), batch(), **a) == eq.EQ_EINVAL, a
    for a in (dict(cos=None), dict(sin=P + 8), dict(rows=0), dict(dims=0), dict(dims=24),
              dict(dims=144)):
        assert append(cache(), batch(), r=rope(**a)) == eq.EQ_EINVAL, a


def test_read_refusals():
    for a in (dict(k=None), dict(v=None), dict(k=P + 8), dict(v=P + 2)):
        assert read(cache(), batch(), **a) == eq.EQ_EINVAL, a


def test_attention_refusals():
    for a in (dict(q=None), dict(out=None), dict(q=P + 8), dict(out=P + 4), dict(qs=511),
              dict(qs=508), dict(heads=0), dict(heads=3), dict(heads=1 << 17), dict(scale=0.0),
              dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert attn(cache(), batch(), **a) == eq.EQ_EINVAL, a
    c, b = cache(page_tokens=4096), batch(max_len=12000)
    need = eq.lib().eq_attn_kv4_workspace_bytes(ref(c), ref(b), 4)
    assert need > 0
    for a in (dict(ws=None), dict(nbytes=need - 1), dict(ws=P + 4)):
        assert attn(c, b, **a) == eq.EQ_EINVAL, a
    assert eq.lib().eq_attn_kv4_workspace_bytes(ref(c), ref(b), 3) == 0
    assert eq.lib().eq_attn_kv4_workspace_bytes(ref(cache(head_dim=96)), ref(b), 4) == 0


def test_norm_refusals():
    for a in (dict(q=None), dict(qo=None), dict(qo=P + 8), dict(k=None), dict(ko=P + 2), dict(qs=255),
              dict(ks=127), dict(kind=2), dict(dim=72), dict(dim=272), dict(dim=0),
              dict(eps=-1.0), dict(eps=float("nan")), dict(hq=5000), dict(pos=None, r=rope()),
              dict(r=rope(dims=144))):
        assert norm(**a) == eq.EQ_EINVAL, a
    assert norm(tokens=0) == eq.EQ_OK


def test_binding_refusals():
    torch = pytest.importorskip("torch")
    t = torch.zeros(4, 2, 128)
    with pytest.raises(ValueError):  # host tensors
        eq.KvCache(torch.zeros(1 << 20, dtype=torch.uint8), page_tokens=64, kv_heads=2, head_dim=128)
    with pytest.raises(ValueError):
        eq.Rope(t[0], t[1])
    with pytest.raises(ValueError):
        eq.eq_qk_norm_rope(t, None, t, None)
    i = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        eq.KvBatch(i, i[:2], i.view(1, 3), n_tokens=1, max_new=1, max_len=1)
