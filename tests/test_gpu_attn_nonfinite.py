"""Attention of inputs that are not finite, or too large for 16 bits on the way: rows that do
not see them are as the formulas have them, whatever the tensor cores made of them first."""
import pytest

from test_gpu_attn import Call

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2609_06086_gb300 as P
    return P


def test_rows_beside_a_nan_hold_their_second_result(P):
    """Values of one token in a tile are NaN: the rows before it in that tile are first
    written as NaN and then as they are, in this order, every time."""
    n, t = 250, 230
    at = torch.arange(n, device="cuda")
    c = Call(P, [n], 64, 8, 128, "bf16", starts=False)
    c.x[2][t] = float("nan")
    want = None
    for _ in range(20):
        c.o.fill_(77)
        c.forward()
        if want is None:
            want = c.o.clone()
        assert torch.isfinite(c.o[:t].double()).all() and c.o[t:].isnan().all()
        assert torch.equal(c.o[:t], want[:t])
    c.without_what_is_not_finite()
    c.check_forward(at < t)
