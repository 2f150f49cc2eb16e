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


# rotations of a part of the head, the elements from rot on beside one another in a
# lane (adjacent pairs), in lanes of their own (rot / 2 = 32) or anywhere
PARTS = [(80, 48, False), (128, 64, False), (31, 10, False), (128, 64, True), (72, 36, True),
         (128, 100, True), (29, 10, True)]


def agree(got, want, room):
    """The same infinities and NaNs; finite values as near as they have to be."""
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine], equal_nan=True)
    assert (np.abs(got - want)[fine] <= room[fine]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dim,rot,half", PARTS)
@pytest.mark.parametrize("at", [0, 1, -1])
def test_infinities_beyond_the_rotation(P, dim, rot, half, dtype, at):
    """An infinite element, gradient or weight from rot on reaches its own column and
    the head's norm, and no neighbour's rotation."""
    e = rot + at if at >= 0 else dim - 1
    with np.errstate(invalid="ignore", over="ignore"):
        c = Case(P, 5, 3, 2, dim, rot, dtype, half=half)
        c.dx_in[0][2, 1, e], c.x[0][2, 1, e] = float("inf"), np.inf
        for got, (want, room) in zip(c.forward(), c.want_forward()):
            agree(got, want, room)
        c = Case(P, 5, 3, 2, dim, rot, dtype, half=half)
        c.dw_weights[0, e], c.w[0, e] = float("-inf"), -np.inf
        for got, (want, room) in zip(c.forward(), c.want_forward()):
            agree(got, want, room)
        c = Case(P, 5, 3, 2, dim, rot, dtype, half=half)
        c.forward()
        c.d_g[0][2, 1, e], c.g[0][2, 1, e] = float("inf"), np.inf
        for from_x in (False, True):
            dx, dw = c.backward(from_x)
            want_dx, want_dw = c.want_backward(from_x)
            for k in range(2):
                agree(dw[k], *want_dw[k])
            agree(dx[1], *want_dx[1])
            rest = [(t, h) for t in range(5) for h in range(3) if (t, h) != (2, 1)]
            for t, h in rest:
                agree(dx[0][t, h], want_dx[0][0][t, h], want_dx[0][1][t, h])
