"""poseidon_qk_forward and poseidon_qk_backward with infinities and NaNs in weights,
rows and gradients: they reach what the formulas say, and nothing else.  Finite values
keep the tolerances of test_gpu_qk.py."""
import numpy as np
import pytest

from test_gpu_qk import Case, near

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2609_06086_gb300 as P
    P.lib()
    return P


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dim,rot,half", [(128, 128, True), (64, 20, True), (80, 48, False),
                                          (30, 10, False)])
def test_padding_under_weights_that_are_not_finite(P, dim, rot, half, dtype, bad):
    """A padding token's outputs and gradients are zeros under any weights, in place too."""
    pos = np.array([3, -1, 0, -7, 49, 7, 7])
    c = Case(P, 7, 5, 2, dim, rot, dtype, "int8", half, positions=pos, seed=1)
    c.dw_weights[:, 3] = bad
    y = c.forward()
    for from_x in (False, True):
        dx, _ = c.backward(from_x)
        for k in range(2):
            for a in (y[k], dx[k]):
                assert (a[pos < 0] == 0).all() and not np.isfinite(a[pos >= 0]).all()
    dx, _ = c.backward(dx=c.d_g)
    assert all((a[pos < 0] == 0).all() for a in dx)
