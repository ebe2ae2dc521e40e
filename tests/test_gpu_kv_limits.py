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
