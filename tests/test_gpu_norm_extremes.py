"""The norm of rows whose squares vanish or pass 32 bits."""
import numpy as np
import pytest

from test_gpu_norm import Call

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2609_06086_gb300 as P
    return P


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [40, 700, 5000, 20001])
def test_no_eps_and_squares_that_vanish(P, dtype, cols):
    """r is infinite, and y = h r w by the formula in 32 bits: an infinity with h's and w's sign,
    NaN where h is 0; the rows beside are as they are."""
    rows = 5
    x = np.random.default_rng(cols).standard_normal((rows, cols))
    x[1] = np.where(np.arange(cols) % 3, np.where(np.arange(cols) % 2, 1e-30, -1e-30), 0)
    x[3] = 0
    c = Call(P, rows, cols, dtype, dtype, "int8", add=False, x=x)
    c.n.eps = 0.0
    c.forward()
    h, w = c.h.float(), c.w
    r = torch.tensor(float("inf"), device="cuda")
    assert (c.rstd[[1, 3]] == float("inf")).all()
    want = (h * r * w).to(c.y.dtype)
    assert torch.equal(c.y[1].isnan(), h[1] == 0) and c.y[3].isnan().all()
    assert torch.equal(c.y[1][h[1] != 0], want[1][h[1] != 0])
    assert torch.isfinite(c.y[[0, 2, 4]].float()).all()


@pytest.mark.parametrize("cols", [40, 700, 5000])
def test_squares_past_32_bits(P, cols):
    """r is 0: y is 0 wherever h is finite."""
    x = np.random.default_rng(cols).standard_normal((3, cols))
    x[1] *= 1e25
    c = Call(P, 3, cols, "f32", "f32", "int8", add=False, x=x)
    c.forward()
    assert c.rstd[1] == 0 and (c.y[1] == 0).all()
    assert torch.isfinite(c.y).all() and (c.y[[0, 2]] != 0).any()


@pytest.mark.parametrize("cols", [4097, 5001, 5120])
@pytest.mark.parametrize("pad,start", [(0, 0), (8, 0), (3, 1)])
@pytest.mark.parametrize("dtype,over,p", [("bf16", "bf16", 0.0), ("f16", "f16", 0.2), ("bf16", "f32", 0.0),
                                          ("bf16", "f32", 0.2), ("f32", "f32", 0.0)])
def test_widths_with_two_kinds_of_team(P, cols, pad, start, dtype, over, p):
    """Which one depends on the alignment, the stream, dropout and the pass."""
    c = Call(P, 333, cols, dtype, over, "int8", p, pad, start)
    c.forward()
    c.check_forward()
    for from_8 in (False, True):
        c.backward(from_8)
        c.check_backward(from_8)
