"""poseidon_norm_forward and poseidon_norm_backward against their formulas in 64 bits,
and the gradients against differences of the forward formula."""
import numpy as np
import pytest

import dropout_util as D
import layer_util as U

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

EPS, F32 = 1e-6, U.ROUND["f32"]
# roundings of 32 bits in a sum of a row's squares or products: 32 elements a thread one
# after another, ten steps over the block, the factors' own
SUM = 32 + 10 + 6


@pytest.fixture(scope="module")
def P():
    import paper_2609_06086_gb300 as P
    return P


def stream():
    return torch.cuda.current_stream().cuda_stream


def matrix(values, dtype, ld, start=0):
    """A view of the values with rows `ld` elements apart, `start` elements into a buffer of
    NaNs."""
    rows, cols = values.shape
    buf = torch.full((start + max(rows - 1, 0) * ld + cols,), float("nan"), dtype=U.DTYPES[dtype],
                     device="cuda")
    x = buf.as_strided((rows, cols), (ld, 1), start)
    x.copy_(torch.as_tensor(values))
    return x


def f64(t):
    return t.double().cpu().numpy()


def kept_of(ckpt, rows, cols, fmt):
    """(codes, scales) of a checkpoint buffer."""
    groups, pitch, spitch, _ = U.layout(rows, cols)
    raw = ckpt.cpu().numpy()
    return (raw[:rows * pitch].reshape(rows, pitch),
            raw[rows * pitch:].reshape(rows, spitch)[:, :groups])


class Call:
    """One forward pass and its outputs, and the backward pass."""

    def __init__(self, P, rows, cols, dtype, over, fmt, p=0.0, pad=0, start=0, add=True, weight=True,
                 seed=0, x=None):
        rng = np.random.default_rng([rows, cols, seed])
        self.P, self.rows, self.cols, self.dtype, self.over, self.fmt = P, rows, cols, dtype, over, fmt
        self.p, ld = p, cols + pad
        new = lambda t, scale: matrix(rng.standard_normal((rows, cols)) * scale, t, ld,  # noqa: E731
                                      start)
        self.x = new(dtype, 1.0)  # (drawn in any case, so that the others are the same)
        if x is not None:
            self.x.copy_(torch.from_numpy(x))
        self.res = new(over, 2.0) if add else None
        self.w = torch.from_numpy(1 + 0.2 * rng.standard_normal(cols)).float().cuda() if weight \
            else None
        self.h, self.y = new(over, 1.0), new(dtype, 1.0)
        size = U.layout(rows, cols)[3]
        self.ckpt_h, self.ckpt_y = (torch.zeros(max(size, 16), dtype=torch.uint8, device="cuda")
                                    for _ in range(2))
        self.rstd = torch.empty(rows, device="cuda")
        self.dy, self.dh_in = new(dtype, 1.0), new(over, 1.0)
        self.dh, self.dx = new(over, 1.0), new(dtype, 1.0)
        self.dw_in = torch.from_numpy(rng.standard_normal(cols)).float().cuda()
        self.dw = torch.empty(cols, device="cuda")
        self.seed, self.offset = 12345 + 2 ** 33 * seed, 2 ** 35 + rows
        self.n = P.pos_norm(rows, cols, U.CODES[dtype], U.CODES[over], U.FORMATS[fmt], EPS,
                            self.w.data_ptr() if weight else 0,
                            P.pos_dropout(p, self.seed, self.offset, 0))

    def forward(self, **over):
        a = dict(res=self.res, h=self.h, y=self.y)
        a.update(over)
        at = lambda t: (0, 0) if t is None else (t.data_ptr(), t.stride(0))  # noqa: E731
        self.P.poseidon_norm_forward(self.n, *at(self.x), *at(a["res"]), *at(a["h"]), *at(a["y"]),
                                     self.ckpt_h.data_ptr(), self.ckpt_y.data_ptr(),
                                     self.rstd.data_ptr(), stream())

    def backward(self, from_8, dh_in=True, dh=None, dx=None, dw=True, dw_in=True):
        at = lambda t: (t.data_ptr(), t.stride(0))  # noqa: E731
        dh, dx = self.dh if dh is None else dh, self.dx if dx is None else dx
        self.P.poseidon_norm_backward(
            self.n, *((0, 0) if from_8 else at(self.h)), self.ckpt_h.data_ptr() if from_8 else 0,
            self.rstd.data_ptr(), *at(self.dy), *(at(self.dh_in) if dh_in else (0, 0)), *at(dh),
            *at(dx), self.dw_in.data_ptr() if dw and dw_in else 0, self.dw.data_ptr() if dw else 0,
            stream())

    def mask(self):
        if self.p == 0:
            return np.ones((self.rows, self.cols), bool), 1.0
        return D.mask(range(self.rows), self.cols, self.seed, self.offset, self.p)

    def check_forward(self):
        kept, factor = self.mask()
        want = np.where(kept, f64(self.x) * factor, 0) + (f64(self.res) if self.res is not None else 0)
        h = f64(self.h)
        assert (np.abs(h - want) <= (U.ROUND[self.over] + F32) * 1.001 * np.abs(want) +
                U.TINY[self.over]).all()
        r = 1 / np.sqrt((h * h).mean(1) + EPS)
        assert (np.abs(f64(self.rstd) - r) <= SUM * F32 * r).all()
        w = f64(self.w) if self.w is not None else 1.0
        want = h * r[:, None] * w
        assert (np.abs(f64(self.y) - want) <=
                (U.ROUND[self.dtype] + (SUM + 2) * F32) * 1.001 * np.abs(want) +
                U.TINY[self.dtype]).all()
        # the checkpoints are those of the tensors written, bit for bit
        for ckpt, t in ((self.ckpt_h, h), (self.ckpt_y, f64(self.y))):
            codes, scales = kept_of(ckpt, self.rows, self.cols, self.fmt)
            want_codes, want_scales = U.encode(t, self.fmt)
            assert np.array_equal(scales, want_scales)
            if self.fmt == "e4m3":  # a negative value that rounds to nothing may keep its sign
                codes, want_codes = (np.where(c == 128, 0, c) for c in (codes, want_codes))
            assert np.array_equal(codes, want_codes)

    def formulas(self, from_8, dh_in=True):
        """(dh, dx, dw) and the sums of the magnitudes that they are made of."""
        h = f64(self.h)
        if from_8:
            h = U.decode(*kept_of(self.ckpt_h, self.rows, self.cols, self.fmt), self.cols, self.fmt)
        r, g = f64(self.rstd)[:, None], f64(self.dy)
        w = f64(self.w) if self.w is not None else np.ones(self.cols)
        n, a = h * r, g * w
        kept, factor = self.mask()
        first = f64(self.dh_in) if dh_in else 0.0
        dh = first + r * (a - n * (a * n).mean(1, keepdims=True))
        parts = np.abs(first) + r * (np.abs(a) + np.abs(n) * np.abs(a * n).mean(1, keepdims=True))
        dw, dw_parts = (g * n).sum(0), np.abs(g * n).sum(0)
        return (dh, parts), (np.where(kept, dh * factor, 0), np.where(kept, parts * factor, 0)), \
            (dw, dw_parts)

    def check_backward(self, from_8, dh_in=True, dw=True):
        (dh, parts), (dx, dx_parts), (want, dw_parts) = self.formulas(from_8, dh_in)
        for got, v, m, t in ((self.dh, dh, parts, self.over), (self.dx, dx, dx_parts, self.dtype)):
            assert (np.abs(f64(got) - v) <= U.ROUND[t] * 1.001 * np.abs(v) + (SUM + 4) * F32 * m +
                    U.TINY[t]).all()
        if dw:
            first = f64(self.dw_in)
            assert (np.abs(f64(self.dw) - first - want) <=
                    (self.rows + 8) * F32 * (dw_parts + np.abs(first))).all()


SIZES = [(1, 1, 0, 0), (3, 8, 0, 0), (9, 31, 0, 0), (20, 100, 5, 1), (11, 256, 0, 0),
         (10, 264, 0, 0), (7, 1024, 8, 0), (5, 1025, 0, 0), (40, 1100, 3, 2), (3, 8192, 0, 0),
         (3, 8197, 0, 0), (2, 16384, 0, 0), (2, 16390, 0, 0), (2, 32768, 0, 0), (700, 48, 0, 0),
         (3, 4097, 0, 0), (5, 5001, 7, 0), (4, 5001, 0, 0), (3, 5120, 0, 0), (3, 2100, 4, 3),
         (333, 1290, 0, 0)]


@pytest.mark.parametrize("rows,cols,pad,start", SIZES)
@pytest.mark.parametrize("dtype,over,fmt,p", [("bf16", "bf16", "int8", 0.1),
                                              ("f16", "f16", "e4m3", 0.0),
                                              ("f32", "f32", "int8", 0.0),
                                              ("bf16", "f32", "e4m3", 0.5),
                                              ("f16", "f32", "int8", 0.25)])
def test_both_passes(P, rows, cols, pad, start, dtype, over, fmt, p):
    c = Call(P, rows, cols, dtype, over, fmt, p, pad, start)
    c.forward()
    c.check_forward()
    for from_8 in (False, True):
        c.backward(from_8)
        c.check_backward(from_8)


@pytest.mark.parametrize("p", [0.0, 0.3])
def test_what_may_be_left_out(P, p):
    """No residual, weight, gradient from other ways or sums; no dropout of a plain norm."""
    c = Call(P, 13, 200, "bf16", "bf16", "int8", p, add=False, weight=False)
    c.forward()
    c.check_forward()
    c.backward(False, dh_in=False, dw=False)
    c.check_backward(False, dh_in=False, dw=False)
    # sums alone
    dh, dx = c.dh.clone(), c.dx.clone()
    P.poseidon_norm_backward(c.n, c.h.data_ptr(), c.h.stride(0), 0, c.rstd.data_ptr(),
                             c.dy.data_ptr(), c.dy.stride(0), d_dw=c.dw.data_ptr(), stream=stream())
    want, parts = c.formulas(False, False)[2]
    assert (np.abs(f64(c.dw) - want) <= (c.rows + 8) * F32 * parts).all()
    assert torch.equal(c.dh, dh) and torch.equal(c.dx, dx)
    # y alone, the same as among all outputs
    y = torch.empty(13, 200, dtype=torch.bfloat16, device="cuda")
    P.poseidon_norm_forward(c.n, c.x.data_ptr(), c.x.stride(0), d_y=y.data_ptr(), ldy=200,
                            stream=stream())
    assert torch.equal(y, c.y)


def test_no_rows(P):
    c = Call(P, 0, 64, "bf16", "bf16", "int8")
    c.forward()
    c.backward(False)
    assert torch.equal(c.dw, c.dw_in)
    c.backward(False, dw_in=False)
    assert not c.dw.any()


def test_in_place(P):
    """h as the residual, y as x; dh as dh_in, dx as dy, dw as dw_in."""
    for start in (0, 1):
        args = (19, 520, "bf16", "f32", "int8", 0.2, 8, start)
        a, b = Call(P, *args), Call(P, *args)
        a.forward()
        a.backward(False)
        b.forward(h=b.res, y=b.x)
        assert torch.equal(b.res, a.h) and torch.equal(b.x, a.y)
        b.h.copy_(a.h)
        P.poseidon_norm_backward(b.n, b.h.data_ptr(), b.h.stride(0), 0, b.rstd.data_ptr(),
                                 b.dy.data_ptr(), b.dy.stride(0), b.dh_in.data_ptr(),
                                 b.dh_in.stride(0), b.dh_in.data_ptr(), b.dh_in.stride(0),
                                 b.dy.data_ptr(), b.dy.stride(0), b.dw_in.data_ptr(),
                                 b.dw_in.data_ptr(), stream())
        assert torch.equal(b.dh_in, a.dh) and torch.equal(b.dy, a.dx)
        assert torch.equal(b.dw_in, a.dw)


def test_nan_stays_in_its_row(P):
    """A NaN or an infinity makes its own row's outputs NaN (its group's codes in the
    checkpoints, and those behind the last column stay zeros); the others are as without."""
    rows, cols = 12, 100
    clean = Call(P, rows, cols, "bf16", "bf16", "e4m3")
    clean.forward()
    clean.backward(True)
    values = f64(clean.x)
    values[4, 50], values[9, 3] = np.nan, np.inf
    c = Call(P, rows, cols, "bf16", "bf16", "e4m3", x=values)
    c.forward()
    c.backward(True)
    bad = np.zeros(rows, bool)
    bad[[4, 9]] = True
    for got, want in ((c.y, clean.y), (c.dh, clean.dh), (c.dx, clean.dx)):
        assert torch.equal(got[~bad], want[~bad])
    assert c.y[4].isnan().all() and c.dh[bad].isnan().all()
    codes, scales = kept_of(c.ckpt_h, rows, cols, "e4m3")
    assert (scales[4] == 255).tolist() == [False, True, False, False]
    assert (scales[9] == 255).tolist() == [True, False, False, False]
    codes, scales = kept_of(c.ckpt_y, rows, cols, "e4m3")
    assert (scales[4] == 255).all() and (codes[:, cols:] == 0).all()


@pytest.mark.parametrize("rows,cols", [(20, 100), (40, 1100), (9, 4096), (5, 5001), (3, 8192),
                                       (2, 20001)])
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_y_is_rounded_once(P, rows, cols, dtype):
    """Of whole numbers, whose squares' sums are exact in 32 bits, y is the formula's value
    rounded to f32 (or to the neighbour next to a border, by 2^-20 of a step) and then to its
    type: r and the products come with their roundings, so 2^-45 of a value is all else."""
    values = np.random.default_rng(cols).integers(-8, 9, (rows, cols)).astype(float)
    c = Call(P, rows, cols, dtype, dtype, "int8", add=False, x=values)
    c.forward()
    want = values / np.sqrt((values * values).mean(1, keepdims=True) + np.float32(EPS)) * f64(c.w)
    if dtype == "f32":
        assert (np.abs(f64(c.y) - want) <= F32 * (1 + 2.0 ** -20) * np.abs(want)).all()
    else:
        assert torch.equal(c.y, torch.from_numpy(want).float().to(U.DTYPES[dtype]).cuda())


def test_weights_that_are_not_finite(P):
    """They reach their own columns as the formula has it: infinities stay infinities."""
    for dtype in ("bf16", "f32"):
        clean, c = (Call(P, 6, 300, dtype, dtype, "int8") for _ in range(2))
        c.w[7], c.w[150] = np.inf, np.nan
        clean.forward()
        c.forward()
        sign = f64(clean.h)[:, 7]
        assert (f64(c.y)[:, 7] == np.where(sign > 0, np.inf, -np.inf)).all()
        assert c.y[:, 150].isnan().all()
        rest = np.ones(300, bool)
        rest[[7, 150]] = False
        # beside them in a thread's columns, y has two more roundings of 32 bits
        a, b = f64(c.y)[:, rest], f64(clean.y)[:, rest]
        assert (np.abs(a - b) <= (2 * U.ROUND[dtype] + 4 * F32) * np.abs(b)).all()


def test_gradients_against_differences(P):
    """dx, dh and dw in f32 against central differences of the formula in 64 bits, whose own
    error is of the order of step^2."""
    rows, cols, p = 5, 37, 0.3
    c = Call(P, rows, cols, "f32", "f32", "int8", p)
    c.forward()
    c.backward(False, dw_in=False)
    kept, factor = c.mask()
    x, res, w, dy, dh_in = (f64(t) for t in (c.x, c.res, c.w, c.dy, c.dh_in))

    def loss(x, res, w):
        h = res + np.where(kept, x * factor, 0)
        y = h / np.sqrt((h * h).mean(1, keepdims=True) + EPS) * w
        return (y * dy).sum() + (h * dh_in).sum()

    rng, step = np.random.default_rng(5), 1e-4
    for _ in range(40):
        i, j = rng.integers(rows), rng.integers(cols)
        for k, got in ((0, c.dx[i, j]), (1, c.dh[i, j]), (2, c.dw[j])):
            a = [x.copy(), res.copy(), w.copy()]
            b = [x.copy(), res.copy(), w.copy()]
            at = j if k == 2 else (i, j)
            a[k][at] += step
            b[k][at] -= step
            want = (loss(*a) - loss(*b)) / (2 * step)
            # third derivatives of order 10 here; SUM roundings of parts of order 10
            assert abs(float(got) - want) <= 10 * step ** 2 + SUM * F32 * (10 + abs(want))


def test_same_bits_again_and_on_another_stream(P):
    """Two passes at once, on two streams, and captured: the same results."""
    c = Call(P, 600, 4096, "bf16", "f32", "int8", 0.1)
    c.forward()
    c.backward(True)
    torch.cuda.synchronize()
    want = [t.clone() for t in (c.h, c.y, c.ckpt_y, c.rstd, c.dh, c.dx, c.dw)]
    others = [Call(P, 600, 4096, "bf16", "f32", "int8", 0.1) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in others]
    torch.cuda.synchronize()
    for _ in range(3):
        for o, s in zip(others, streams):
            with torch.cuda.stream(s):
                o.forward()
                o.backward(True)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward()
        c.backward(True)
    for t in (c.h, c.y, c.dh, c.dx, c.dw):
        t.zero_()
    graph.replay()
    graph.replay()
    for o in (*others, c):
        for t, v in zip((o.h, o.y, o.ckpt_y, o.rstd, o.dh, o.dx, o.dw), want):
            assert torch.equal(t, v)


def test_norm_then_weight_gradient(P):
    """The checkpoint of y goes into the weight gradient of the next linear operation: the
    same bits as from a checkpoint packed of y."""
    rows, cols, n = 300, 512, 192
    c = Call(P, rows, cols, "bf16", "bf16", "int8", 0.1)
    c.forward()
    packed = torch.zeros_like(c.ckpt_y)
    P.poseidon_ckpt_pack(c.y.data_ptr(), 0, rows, cols, c.y.stride(0), 0, packed.data_ptr(),
                         stream())
    dy = torch.randn(rows, n, device="cuda").bfloat16()
    out = [torch.empty(n, cols, device="cuda") for _ in range(2)]
    for ckpt, dw in zip((c.ckpt_y, packed), out):
        P.poseidon_ckpt_wgrad(ckpt.data_ptr(), 0, dy.data_ptr(), 0, n, rows, n, cols, 0,
                              dw.data_ptr(), cols, stream())
    assert torch.equal(*out)
