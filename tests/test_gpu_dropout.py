"""poseidon_dropout against its definition in 64 bits."""
import numpy as np
import pytest

import dropout_util as D
import layer_util as U

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2609_06086_gb300 as P
    return P


def stream():
    return torch.cuda.current_stream().cuda_stream


def matrix(rng, rows, cols, dtype, ld, start=0):
    """A [rows][cols] view with rows `ld` elements apart, `start` elements into a buffer
    of NaNs."""
    buf = torch.full((start + max(rows - 1, 0) * ld + cols,), float("nan"), dtype=U.DTYPES[dtype],
                     device="cuda")
    x = buf.as_strided((rows, cols), (ld, 1), start)
    x.copy_(torch.from_numpy(rng.standard_normal((rows, cols)) * 3))
    return x


def f64(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("rows,cols,pad,start", [(1, 1, 0, 0), (1, 7, 0, 0), (5, 8, 0, 0),
                                                 (3, 9, 0, 0), (40, 264, 0, 0), (17, 130, 6, 0),
                                                 (9, 61, 3, 1), (6, 700, 1, 5), (33, 48, 0, 3)])
@pytest.mark.parametrize("dtype,dtype_y", [("bf16", "bf16"), ("f16", "f16"), ("f32", "f32"),
                                           ("bf16", "f32"), ("f32", "bf16"), ("f16", "bf16")])
@pytest.mark.parametrize("p,add", [(0.1, True), (0.5, False), (0.0, True), (0.0, False),
                                   (1.0, True)])
def test_definition(P, rows, cols, pad, start, dtype, dtype_y, p, add):
    """y is one rounding in 32 bits and one to its type away from the definition; what lies
    beside its rows is not touched."""
    rng = np.random.default_rng([rows, cols, pad])
    x = matrix(rng, rows, cols, dtype, cols + pad, start)
    res = matrix(rng, rows, cols, dtype_y, cols + pad, start) if add else None
    y = matrix(rng, rows, cols + pad, dtype_y, cols + pad, start)
    before = y.clone()
    seed, offset, at = 0x123456789abcdef0 + rows, 2 ** 40 + cols, 2 ** 63 - 2 ** 40 + 17
    d_at = torch.tensor([at], dtype=torch.int64, device="cuda")
    P.poseidon_dropout(P.pos_dropout(p, seed, offset, d_at.data_ptr()), rows, cols, x.data_ptr(),
                       U.CODES[dtype], x.stride(0), res.data_ptr() if add else 0, cols + pad,
                       y.data_ptr(), U.CODES[dtype_y], y.stride(0), stream())
    kept, factor = D.mask(range(rows), cols, seed, offset + at, p)
    want = np.where(kept, f64(x) * factor, 0) + (f64(res) if add else 0)
    u, tiny = U.ROUND[dtype_y], U.TINY[dtype_y]
    off = np.abs(f64(y[:, :cols]) - want)
    assert (off <= (u + U.ROUND["f32"]) * 1.001 * np.abs(want) + tiny).all()
    if not add:
        assert ((f64(y[:, :cols]) != 0) <= kept).all()
    assert torch.equal(y[:, cols:], before[:, cols:])


def test_what_is_dropped_has_no_effect(P):
    """Infinities and NaNs in dropped places, in x alone and with a residual; the
    gradient's call drops the same places."""
    rows, cols, p = 37, 203, 0.3
    kept, _ = D.mask(range(rows), cols, 7, 8, p)
    drop = P.pos_dropout(p, 7, 8, 0)
    x = torch.ones(rows, cols, device="cuda")
    x[torch.from_numpy(~kept).cuda()] = float("nan")
    x.view(-1)[::3] = torch.where(x.view(-1)[::3].isnan(), float("inf"), x.view(-1)[::3])
    y, dx = torch.empty_like(x), torch.empty_like(x)
    for res in (None, torch.ones_like(x)):
        P.poseidon_dropout(drop, rows, cols, x.data_ptr(), 2, cols,
                           0 if res is None else res.data_ptr(), cols, y.data_ptr(), 2, cols,
                           stream())
        assert torch.isfinite(y).all()
    P.poseidon_dropout(drop, rows, cols, torch.ones_like(x).data_ptr(), 2, cols, 0, 0,
                       dx.data_ptr(), 2, cols, stream())
    assert np.array_equal(dx.cpu().numpy() != 0, kept)
    assert np.array_equal(y.cpu().numpy() != 1, kept)


def test_in_place(P):
    """y as x, and y as the residual."""
    rng = np.random.default_rng(3)
    drop = P.pos_dropout(0.2, 1, 2, 0)
    for start in (0, 3):
        x, res = matrix(rng, 21, 77, "bf16", 80, start), matrix(rng, 21, 77, "bf16", 80, start)
        y = torch.empty(21, 77, dtype=torch.bfloat16, device="cuda")
        call = lambda x, res, y: P.poseidon_dropout(  # noqa: E731
            drop, 21, 77, x.data_ptr(), 0, x.stride(0), res.data_ptr(), res.stride(0),
            y.data_ptr(), 0, y.stride(0), stream())
        call(x, res, y)
        for which in (0, 1):
            pair = [x.clone(memory_format=torch.preserve_format) for x in (x, res)]
            pair = [matrix(rng, 21, 77, "bf16", 80, start).copy_(t) for t in (x, res)]
            call(*pair, pair[which])
            assert torch.equal(pair[which], y)


def test_empty(P):
    drop = P.pos_dropout(0.2, 1, 2, 0)
    P.poseidon_dropout(drop, 0, 8, 0, 0, 8, 0, 0, 0, 0, 8, stream())
    P.poseidon_dropout(drop, 8, 0, 0, 0, 8, 0, 0, 0, 0, 8, stream())


def test_offsets_past_32_bits(P):
    """2^21 + 5 rows of 8192: elements, bytes and groups of 8 past 2^31; x is one row."""
    rows, cols, p = 2 ** 21 + 5, 8192, 0.5
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB")
    x = torch.ones(cols, dtype=torch.bfloat16, device="cuda")
    y = torch.full((rows, cols), 9, dtype=torch.bfloat16, device="cuda")
    P.poseidon_dropout(P.pos_dropout(p, 11, 12, 0), rows, cols, x.data_ptr(), 0, 0, 0, 0,
                       y.data_ptr(), 0, cols, stream())
    some = [0, 1, 2 ** 20 - 1, 2 ** 20, 2 ** 21 - 3, 2 ** 21 - 2, 2 ** 21 - 1, 2 ** 21, rows - 1]
    kept, _ = D.mask(some, cols, 11, 12, p)
    assert np.array_equal(f64(y[some]), 2.0 * kept)
    # every element was written: the row sums are those of 0 and 2
    assert bool((y.view(-1, 64)[::7].float().amax(1) <= 2).all())


def test_a_captured_step_draws_new_masks(P):
    """d_offset is read at each replay."""
    rows, cols, p = 16, 256, 0.5
    x = torch.ones(rows, cols, device="cuda")
    y = torch.empty_like(x)
    at = torch.zeros(1, dtype=torch.int64, device="cuda")
    drop = P.pos_dropout(p, 3, 100, at.data_ptr())
    call = lambda: P.poseidon_dropout(drop, rows, cols, x.data_ptr(), 2, cols, 0, 0,  # noqa: E731
                                      y.data_ptr(), 2, cols, stream())
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
        at.add_(1)
    for step in range(3):
        graph.replay()
        kept, _ = D.mask(range(rows), cols, 3, 100 + step, p)
        assert np.array_equal(y.cpu().numpy() != 0, kept)
