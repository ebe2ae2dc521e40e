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
