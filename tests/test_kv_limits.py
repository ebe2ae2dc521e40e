"""Calls at the ends of the cache operators' ranges, on the host: of no tokens,
of more than a launch or an argument can count, on several devices."""
import ctypes

import numpy as np
import pytest

import paper_2601_22787_amd as eq

FAKE = np.zeros(4096, dtype=np.uint8)
P = (FAKE.ctypes.data + 255) // 256 * 256


@pytest.mark.parametrize("rope", [False, True])
def test_norm_of_no_tokens(rope):
    """What torch gives for an empty tensor's address is 0."""
    r = eq.eq_rope(P, P, 10, 128, 0)
    at = ctypes.addressof(r) if rope else None
    for tokens, hq, hk, rc in ((0, 64, 8, eq.EQ_OK), (3, 0, 0, eq.EQ_OK), (1, 64, 0, eq.EQ_EINVAL)):
        assert eq.lib().eq_qk_norm_rope(None, hq * 128, hq, P, None, None, hk * 128, hk, P, None, 0,
                                        tokens, 128, 1e-5, None, at, None) == rc
    # what is no size of a head stays refused
    assert eq.lib().eq_qk_norm_rope(None, 8, 64, None, None, None, 8, 8, None, None, 0, 0, 72, 1e-5,
                                    None, None, None) == eq.EQ_EINVAL


def _bounds(heads, max_new):
    c = eq.eq_kv_cache(P, 3, 64, heads, 128)
    b = eq.eq_kv_batch(P, P, P, 1, 3, max_new, max_new, 100)
    return c, b, heads * 128


def test_bounds_beyond_one_launch_are_refused():
    """2^32 threads along x and more: refused by the call, not by the launch."""
    lib, at = eq.lib(), ctypes.addressof
    for heads, max_new in ((8, 1 << 26), (1024, 1 << 19)):
        c, b, width = _bounds(heads, max_new)
        assert lib.eq_kv_append(at(c), at(b), P, width, 0, P, width, 0, None, None, None) == eq.EQ_EINVAL
    c, b, width = _bounds(1024, 1 << 21)
    assert lib.eq_kv_read(at(c), at(b), P, P, None) == eq.EQ_EINVAL
    for heads, q_heads, max_new in ((1024, 1024, (1 << 21) - 1), (8, 64, 1 << 25), (1, 65535, 1 << 20)):
        c, b, _ = _bounds(heads, max_new)
        assert lib.eq_attn_kv4_workspace_bytes(at(c), at(b), q_heads) == 0
        assert lib.eq_attn_kv4(at(c), at(b), P, q_heads * 128, q_heads, 1.0, 0, P, P, 1 << 60,
                               None) == eq.EQ_EINVAL


@pytest.mark.parametrize("window", [-1, -(1 << 31), 1 << 32, (1 << 32) + 5])
def test_windows_that_are_not_32_bits_are_refused(window):
    torch = pytest.importorskip("torch")
    q = torch.zeros(1, 1, 64)
    with pytest.raises(ValueError, match="window"):
        eq.eq_attn_kv4(None, None, q, 1.0, q, window=window)


@pytest.mark.parametrize("over", [dict(n_tokens=(1 << 32) + 4), dict(max_new=1 << 32),
                                  dict(max_len=(1 << 33) + 64), dict(max_len=-1)])
def test_batch_bounds_that_are_not_32_bits_are_refused(over):
    torch = pytest.importorskip("torch")
    i = torch.zeros(3, dtype=torch.int32)
    a = dict(n_tokens=4, max_new=2, max_len=64)
    a.update(over)
    with pytest.raises(ValueError, match="32 bits"):
        eq.KvBatch(i, i[:2], i[:2].view(2, 1), **a)


def test_sizes_that_are_not_32_bits_have_no_page_or_workspace():
    for a in ((8 + (1 << 32), 128, 64), (8, 128 + (1 << 32), 64), (8, 128, 64 - (1 << 32))):
        assert eq.eq_kv_page_bytes(*a) == 0, a

    class Handle:
        def __init__(self, raw):
            self.raw, self.ptr = raw, ctypes.addressof(raw)

    c = Handle(eq.eq_kv_cache(P, 3, 4096, 2, 128))
    b = Handle(eq.eq_kv_batch(P, P, P, 2, 3, 4, 2, 12000))
    assert eq.eq_attn_kv4_workspace_bytes(c, b, 4) > 0
    assert eq.eq_attn_kv4_workspace_bytes(c, b, 4 + (1 << 32)) == 0


def test_norm_of_more_tokens_than_32_bits_is_refused():
    torch = pytest.importorskip("torch")
    q = torch.zeros(1, 1, 16).expand((1 << 32) + 1, 1, 16)
    with pytest.raises(ValueError, match="tokens"):
        eq.eq_qk_norm_rope(q, None, q, None)


class OnDevice:
    """What the binding looks at of a contiguous tensor on cuda:`index`."""
    is_cuda = True

    def __init__(self, shape, dtype, index):
        torch = pytest.importorskip("torch")
        self.shape, self.dtype, self.device = tuple(shape), dtype, torch.device("cuda", index)

    def get_device(self):
        return self.device.index

    def data_ptr(self):
        return P

    def is_contiguous(self):
        return True

    def dim(self):
        return len(self.shape)

    def numel(self):
        return int(np.prod(self.shape))

    def element_size(self):
        return self.dtype.itemsize

    def stride(self):
        return tuple(int(np.prod(self.shape[i + 1:])) for i in range(len(self.shape)))


def _call(which, at):
    """One call with every part on cuda:0 but for what `at` names."""
    torch = pytest.importorskip("torch")
    bf, i32, f32, u8 = torch.bfloat16, torch.int32, torch.float32, torch.uint8

    def t(name, shape, dtype=bf):
        return OnDevice(shape, dtype, at.get(name, at.get("all", 0)))

    def rope():
        return eq.Rope(t("rope", (9, 32), f32), t("rope", (9, 32), f32))

    class Stream:
        cuda_stream, device_index = 0, at.get("stream", at.get("all", 0))

    stream = Stream if "stream" in at else None
    if which == "norm":
        return eq.eq_qk_norm_rope(t("q", (4, 4, 64)), t("k", (4, 2, 64)), t("q_out", (4, 4, 64)),
                                  t("k_out", (4, 2, 64)), q_weight=t("q_weight", (64,)),
                                  k_weight=t("k_weight", (64,)), rope=rope(),
                                  positions=t("positions", (4,), i32), stream=stream)
    cache = eq.KvCache(t("cache", (3, eq.eq_kv_page_bytes(2, 64, 64)), u8), page_tokens=64, kv_heads=2,
                       head_dim=64)
    batch = eq.KvBatch(t("batch", (2,), i32), t("batch", (1,), i32), t("batch", (1, 3), i32),
                       n_tokens=4, max_new=4, max_len=100)
    if which == "append":
        return eq.eq_kv_append(cache, batch, t("k", (4, 2, 64)), t("v", (4, 2, 64), f32), rope=rope(),
                               positions=t("positions", (4,), i32), stream=stream)
    if which == "read":
        return eq.eq_kv_read(cache, batch, t("k", (4, 2, 64)), t("v", (4, 2, 64)), stream=stream)
    return eq.eq_attn_kv4(cache, batch, t("q", (4, 4, 64)), 0.125, t("out", (4, 4, 64)),
                          t("ws", (1 << 20,), u8), stream=stream)


@pytest.mark.parametrize("which,part", [("norm", p) for p in (
    "q", "k", "q_out", "k_out", "q_weight", "k_weight", "rope", "positions", "stream", "all")] + [
    ("append", p) for p in ("cache", "batch", "k", "v", "rope", "positions", "stream", "all")] + [
    ("read", p) for p in ("cache", "batch", "k", "v", "stream", "all")] + [
    ("attn", p) for p in ("cache", "batch", "q", "out", "ws", "stream", "all")])
def test_tensors_that_are_not_on_the_current_device_are_refused(which, part, monkeypatch):
    """A kernel would follow another device's addresses."""
    torch = pytest.importorskip("torch")
    eq._kinds()
    monkeypatch.setattr(eq, "_current", lambda: 0)
    monkeypatch.setattr(eq, "_raw_stream", lambda device: 0)
    called = []

    class Lib:
        def __getattr__(self, name):
            return getattr(real, name) if name == "eq_kv_page_bytes" else lambda *a: called.append(name) or 0

    real = eq.lib()
    monkeypatch.setattr(eq, "_lib", Lib())
    _call(which, {})
    assert len(called) == 1
    with pytest.raises(ValueError, match="device"):
        _call(which, {part: 1})
    assert len(called) == 1


def test_tables_on_two_devices_are_refused():
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError, match="device"):
        eq.Rope(OnDevice((9, 32), torch.float32, 0), OnDevice((9, 32), torch.float32, 1))
