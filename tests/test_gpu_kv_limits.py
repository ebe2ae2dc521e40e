"""Calls at the ends of the cache operators' ranges, on the device."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def eq():
    import paper_2601_22787_amd as m
    m.lib()
    assert torch.cuda.is_available()
    return m


def test_norm_of_no_tokens(eq):
    def empty(heads):
        return torch.empty(0, heads, 128, dtype=torch.bfloat16, device="cuda")

    w = torch.ones(128, dtype=torch.bfloat16, device="cuda")
    table = torch.ones(4, 64, device="cuda")
    eq.eq_qk_norm_rope(empty(8), empty(2), empty(8), empty(2), q_weight=w, k_weight=w,
                       rope=eq.Rope(table, table),
                       positions=torch.empty(0, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()


def test_norm_of_more_tokens_than_a_launch_counts(eq):
    """2^24 + 300 rows of one head of each: every row is a copy of one of 1024,
    so the whole output is the small call's over and over, bit for bit."""
    tokens, period, dim = (1 << 24) + 300, 1024, 16
    x = torch.randn(period, 3, dim, device="cuda").to(torch.bfloat16)
    w = torch.randn(dim, device="cuda").to(torch.bfloat16)
    angle = torch.rand(period, dim // 2, device="cuda")
    rope = eq.Rope(angle.cos(), angle.sin())
    at = torch.randperm(period, device="cuda").int()
    few = [torch.empty(period, h, dim, dtype=torch.bfloat16, device="cuda") for h in (2, 1)]
    eq.eq_qk_norm_rope(x[:, :2], x[:, 2:], few[0], few[1], q_weight=w, k_weight=w, rope=rope,
                       positions=at)
    times = -(-tokens // period)
    rows = x.repeat(times, 1, 1)[:tokens]
    many = [torch.full((tokens, h, dim), 7.0, dtype=torch.bfloat16, device="cuda") for h in (2, 1)]
    eq.eq_qk_norm_rope(rows[:, :2], rows[:, 2:], many[0], many[1], q_weight=w, k_weight=w, rope=rope,
                       positions=at.repeat(times)[:tokens].contiguous())
    for y, ref in zip(many, few):
        whole = y[:tokens // period * period].view(-1, period, *ref.shape[1:])
        assert torch.equal(whole.view(torch.int16), ref.view(torch.int16).expand_as(whole))
        assert torch.equal(y[tokens // period * period:], ref[:tokens % period])


@pytest.mark.parametrize("dim,new,bound", [(128, 6, 0), (64, 6, 0), (128, 40, 0), (64, 40, 0),
                                           (128, 80, 8192), (64, 80, 8192)])
def test_small_query_channels_enter_exactly(eq, dim, new, bound):
    """Query channels of 2^-14 of the largest of their 32, with all 8 bits: against
    a key that takes nothing else they are scores of -16 to -32, so that a lost bit
    (2^-8 at least) would change P by 6% at least.  P times a value's scale and the
    output are rounded to 8 bits, 2^-8 each, and the rest is in fp32."""
    length, page = new + 1, 32
    width = max(bound, length + page - 1) // page
    table = torch.arange(width, dtype=torch.int32, device="cuda").view(1, -1)
    cache = eq.KvCache.empty(width, page_tokens=page, kv_heads=1, head_dim=dim)

    def of(rows):
        return eq.KvBatch(torch.tensor([0, rows], dtype=torch.int32, device="cuda"),
                          torch.tensor([length], dtype=torch.int32, device="cuda"), table,
                          n_tokens=rows, max_new=rows, max_len=max(length, bound))

    # the first token: even channels and a value; the others have neither
    k, v = torch.zeros(2, length, 1, dim, device="cuda")
    k[0, 0, ::2], v[0] = -(2.0 ** 21), 1
    eq.eq_kv_append(cache, of(length), k, v)
    i = torch.arange(new, device="cuda")
    x = (128 + i * 37 % 128).double() * 2.0 ** -21
    q = torch.zeros(new, 1, dim, dtype=torch.bfloat16, device="cuda")
    at = 2 * (i * 11 % (dim // 2))
    q[i, 0, at], q[i, 0, at + 1] = x.to(torch.bfloat16), 1
    assert torch.equal(q[i, 0, at].double(), x)
    out = torch.empty_like(q)
    b = of(new)
    eq.eq_attn_kv4(cache, b, q, 0.125, out, eq.attn_workspace(cache, b, 1))
    p = torch.exp(-(2.0 ** 18) * x)
    ref = p / (p + (i + 1))  # a row sees the first token, the ones between and itself
    err = (out[:, 0].double() - ref[:, None]).abs() / ref[:, None]
    assert (err <= 2.0 ** -7 + 2.0 ** -12).all(), float(err.max())


@pytest.mark.parametrize("dim,new,bound", [(128, 6, 0), (64, 6, 0), (128, 40, 0), (64, 40, 0),
                                           (128, 80, 8192), (64, 80, 8192)])
def test_small_weights_keep_their_bits(eq, dim, new, bound):
    """Two tokens with values in other channels: the second's P times its scale is
    2^-13.2 to 2^-13.98 of the first's, and its channels are as exact as 8 bits of it
    and of the output are (2^-8 each)."""
    length, page = new + 2, 32
    width = max(bound, length + page - 1) // page
    table = torch.arange(width, dtype=torch.int32, device="cuda").view(1, -1)
    cache = eq.KvCache.empty(width, page_tokens=page, kv_heads=1, head_dim=dim)

    def of(rows):
        return eq.KvBatch(torch.tensor([0, rows], dtype=torch.int32, device="cuda"),
                          torch.tensor([length], dtype=torch.int32, device="cuda"), table,
                          n_tokens=rows, max_new=rows, max_len=max(length, bound))

    k, v = torch.zeros(2, length, 1, dim, device="cuda")
    k[1, 0, 0], v[0, 0, ::2], v[1, 0, 1::2] = -1, 1, 2.0 ** -6
    eq.eq_kv_append(cache, of(length), k, v)
    i = torch.arange(new, device="cuda")
    score = 40 + (i * 5 % 18).double() / 4  # 8 times it
    q = torch.zeros(new, 1, dim, dtype=torch.bfloat16, device="cuda")
    q[:, 0, 0] = score.to(torch.bfloat16)
    assert torch.equal(q[:, 0, 0].double(), score)
    out = torch.empty_like(q)
    b = of(new)
    eq.eq_attn_kv4(cache, b, q, 0.125, out, eq.attn_workspace(cache, b, 1))
    p = torch.exp(-score / 8)
    total = 1 + p + (i + 1)  # and the tokens without a key up to the row's own
    for first, ref in ((0, 1 / total), (1, p * 2.0 ** -6 / total)):
        err = (out[:, 0, first::2].double() - ref[:, None]).abs() / ref[:, None]
        assert (err <= 2.0 ** -7 + 2.0 ** -12).all(), (first, float(err.max()))
