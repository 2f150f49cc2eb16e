"""poseidon_qk_forward and poseidon_qk_backward against their formulas in 64
bits, and the backward pass against differences of the formula.

Tolerances, from the formulas in 32 bits (u = 2^-24): a head's sum of dim
squares is off by at most dim u, so r by (dim / 2 + 2) u; every product and sum
of a few terms adds a few u of the magnitudes that it is made of; the result is
rounded once to its type."""
import numpy as np
import pytest

import layer_util as U

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture(scope="module")
def P():
    import paper_2609_06086_gb300 as P
    P.lib()
    return P


class Case:
    """Inputs on the CPU in f64 (exact in their type) and on the GPU."""

    def __init__(self, P, T, hq, hk, dim, rot, dtype="f32", fmt="int8", half=True, fused=False,
                 positions=None, n_pos=50, seed=0, weights=True, shift=0, pad=0):
        import torch
        self.P, self.T, self.heads, self.dim, self.rot = P, T, (hq, hk), dim, rot
        self.dtype, self.fmt, self.half, self.n_pos = dtype, fmt, half, n_pos
        rng = np.random.default_rng(seed)
        t = U.DTYPES[dtype]
        stride = (hq + 2 * hk) * (dim + pad)
        flat = torch.full((T * stride + shift + 8,), float("nan"), dtype=t, device="cuda")
        self.dx_in = []
        for k, h in enumerate(self.heads):
            start = shift + (hq * (dim + pad) if k else 0)
            if fused:
                v = flat[start:].as_strided((T, h, dim), (stride, dim + pad, 1))
            else:
                v = torch.empty(T, h, dim, dtype=t, device="cuda")
            x = rng.standard_normal((T, h, dim)) * np.exp(rng.uniform(-2, 2, (1, 1, dim)))
            v.copy_(torch.from_numpy(x))
            self.dx_in.append(v)
        self.x = [v.double().cpu().numpy() for v in self.dx_in]
        self.w = 1 + 0.3 * rng.standard_normal((2, dim)) if weights else np.ones((2, dim))
        self.w = self.w.astype(np.float32).astype(np.float64)
        self.dw_weights = torch.from_numpy(self.w).float().cuda()
        ang = rng.uniform(-3, 3, (n_pos, rot // 2))
        self.cos = np.cos(ang).astype(np.float32).astype(np.float64)
        self.sin = np.sin(ang).astype(np.float32).astype(np.float64)
        self.d_cos, self.d_sin = (torch.from_numpy(a).float().cuda() for a in (self.cos, self.sin))
        self.pos = np.arange(T) if positions is None else np.asarray(positions)
        self.d_pos = None if positions is None else \
            torch.from_numpy(self.pos.astype(np.int32)).cuda()
        ptr = lambda a: a.data_ptr() if a is not None else 0  # noqa: E731
        w0 = self.dw_weights.data_ptr() if weights else 0
        self.qk = P.pos_qk(T, hq, hk, dim, rot, 0 if half else 1, U.CODES[dtype], U.FORMATS[fmt],
                           EPS, w0, w0 + 4 * dim if weights else 0, ptr(self.d_cos),
                           ptr(self.d_sin), n_pos, ptr(self.d_pos))
        g = [torch.from_numpy(rng.standard_normal((T, h, dim))).to(t) for h in self.heads]
        self.g = [a.double().numpy() for a in g]
        self.d_g = [a.cuda() for a in g]

    def pair(self, tensors):
        return self.P.qk_heads(*(v for t in tensors for v in (t.data_ptr(), t.stride(0),
                                                              t.stride(1))))

    def new(self, fill=5.0):
        import torch
        return [torch.full((self.T, h, self.dim), fill, dtype=U.DTYPES[self.dtype], device="cuda")
                for h in self.heads]

    def forward(self, keep=True, y=None, stream=None):
        import torch
        s = stream or torch.cuda.current_stream()
        self.y = y or self.new()
        self.r = [torch.empty(self.T, h, device="cuda") for h in self.heads]
        self.c = [torch.full((U.layout(self.T * h, self.dim)[3] + 16,), 0xAB, dtype=torch.uint8,
                             device="cuda") for h in self.heads]
        some = lambda a: tuple(t.data_ptr() for t in a) if keep else (0, 0)  # noqa: E731
        self.P.poseidon_qk_forward(self.qk, self.pair(self.dx_in), self.pair(self.y),
                                   rstd=some(self.r), ckpt=some(self.c), stream=s.cuda_stream)
        torch.cuda.synchronize()
        return [t.double().cpu().numpy() for t in self.y]

    def backward(self, from_x=False, dw_in=None, dx=None, dy=None, dw=True):
        import torch
        self.dx = dx or self.new()
        self.dw = torch.full((2, self.dim), 7.0, device="cuda")
        self.P.poseidon_qk_backward(
            self.qk, self.pair(dy or self.d_g), self.pair(self.dx),
            tuple(t.data_ptr() for t in self.r),
            ckpt=(0, 0) if from_x else tuple(t.data_ptr() for t in self.c),
            x=self.pair(self.dx_in) if from_x else None,
            dw_in=0 if dw_in is None else dw_in.data_ptr(),
            dw=self.dw.data_ptr() if dw else 0, stream=torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        return [t.double().cpu().numpy() for t in self.dx], self.dw.double().cpu().numpy()

    # the formulas
    def turn(self):
        at = np.clip(self.pos, 0, self.n_pos - 1)
        return self.cos[at][:, None], self.sin[at][:, None]

    def live(self):
        return (self.pos >= 0)[:, None, None]

    def norm(self, k):
        return 1 / np.sqrt((self.x[k] ** 2).mean(-1, keepdims=True) + EPS)

    def want_forward(self):
        """(values, allowed errors)."""
        cos, sin = self.turn()
        out = []
        for k in range(2):
            u = self.x[k] * self.norm(k) * self.w[k]
            y = np.where(self.live(), U.turned(u, cos, sin, self.rot, self.half), 0)
            room = (self.dim / 2 + 8) * 2.0 ** -24 * U.spread(u, cos, sin, self.rot, self.half)
            out.append((y, room + U.ROUND[self.dtype] * np.abs(y) * 1.01 + U.TINY[self.dtype]))
        return out

    def want_backward(self, from_x=False):
        cos, sin = self.turn()
        dxs, dws = [], []
        for k in range(2):
            x = self.x[k] if from_x else U.kept(
                self.x[k].reshape(-1, self.dim), self.fmt).reshape(self.x[k].shape)
            r = self.norm(k)
            n = x * r
            g = np.where(self.live(), U.turned(self.g[k], cos, sin, self.rot, self.half, True), 0)
            ga = np.where(self.live(), U.spread(self.g[k], cos, sin, self.rot, self.half), 0)
            h, ha = g * self.w[k], ga * np.abs(self.w[k])
            dx = r * (h - n * (h * n).mean(-1, keepdims=True))
            room = (2 * self.dim + 24) * 2.0 ** -24 * r * (
                ha + np.abs(n) * (ha * np.abs(n)).mean(-1, keepdims=True))
            dxs.append((dx, room + U.ROUND[self.dtype] * np.abs(dx) * 1.01 + U.TINY[self.dtype]))
            rows = self.T * self.heads[k]
            dws.append(((g * n).sum((0, 1)),
                        (rows + self.dim / 2 + 24) * 2.0 ** -24 * (ga * np.abs(n)).sum((0, 1))))
        return dxs, dws


def near(got, want):
    for g, (w, room) in zip(got, want):
        assert g.shape == w.shape
        bad = ~(np.abs(g - w) <= room)
        assert not bad.any(), (np.argwhere(bad)[:3], np.max(np.abs(g - w) / room))


SHAPES = [(1, 1, 1, 1, 0), (1, 1, 0, 2, 2), (2, 3, 1, 8, 4), (5, 4, 2, 31, 10), (3, 2, 2, 64, 64),
          (7, 5, 1, 72, 48), (9, 20, 4, 80, 80), (4, 3, 3, 96, 30), (11, 8, 2, 128, 128),
          (33, 0, 2, 128, 64), (2, 9, 1, 200, 16), (6, 2, 1, 256, 256), (40, 40, 8, 128, 128),
          (700, 3, 1, 64, 32)]


@pytest.mark.parametrize("T,hq,hk,dim,rot", SHAPES)
@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("dtype,fmt", [("f32", "int8"), ("bf16", "e4m3"), ("f16", "int8")])
def test_against_64_bits(P, T, hq, hk, dim, rot, half, dtype, fmt):
    c = Case(P, T, hq, hk, dim, rot, dtype, fmt, half, n_pos=max(T, 1), seed=dim + T)
    near(c.forward(), c.want_forward())
    for k, h in enumerate(c.heads):
        if not h:
            continue
        groups, pitch, spitch, size = U.layout(T * h, dim)
        b = c.c[k].cpu().numpy()
        assert (b[size:] == 0xAB).all()
        codes, scales = U.encode(c.x[k].reshape(-1, dim), fmt)
        assert np.array_equal(b[:T * h * pitch].reshape(-1, pitch), codes)
        assert np.array_equal(b[T * h * pitch:size].reshape(-1, spitch)[:, :groups], scales)
        r = c.r[k].double().cpu().numpy()[..., None]
        assert (np.abs(r / c.norm(k) - 1) <= (dim / 2 + 4) * 2.0 ** -24).all()
    for from_x in (False, True):
        dx, dw = c.backward(from_x)
        want_dx, want_dw = c.want_backward(from_x)
        near(dx, want_dx)
        near(dw, want_dw)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dim,rot", [(64, 36), (72, 72), (80, 34), (88, 84), (128, 100), (256, 124),
                                     (192, 190)])
def test_partners_that_are_not_whole_vectors_apart(P, dtype, dim, rot):
    """rot / 2 = 18, 36, 17, 42, 50, 62 and 95: partners by pairs or one by one, heads of
    whole vectors that fill their lanes or leave some idle."""
    c = Case(P, 21, 9, 2, dim, rot, dtype, "e4m3", seed=rot)
    near(c.forward(), c.want_forward())
    for from_x in (False, True):
        dx, dw = c.backward(from_x)
        want_dx, want_dw = c.want_backward(from_x)
        near(dx, want_dx)
        near(dw, want_dw)


@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("dim,rot", [(24, 24), (128, 64), (36, 20)])
def test_gradients_against_differences(P, half, dim, rot):
    """The formula's differences in 64 bits, x exact in 8 bits so that the
    checkpoint is x itself.  Central differences of step 1e-4 are off by about
    1e-8 of a third derivative of order one; the gradients of order one are in
    32 bits with sums of up to 256 terms: 1e-4 holds both."""
    import torch
    c = Case(P, 2, 2, 1, dim, rot, "f32", "int8", half, seed=dim)
    rng = np.random.default_rng(8)
    for k in range(2):
        c.x[k] = rng.integers(-100, 101, c.x[k].shape) / 64.0
        c.dx_in[k].copy_(torch.from_numpy(c.x[k]))
    c.forward()
    dx, dw = c.backward()
    cos, sin = c.turn()

    def loss(k, x, w):
        r = 1 / np.sqrt((x ** 2).mean(-1, keepdims=True) + EPS)
        return (U.turned(x * r * w, cos, sin, rot, half) * c.g[k]).sum()

    d = 1e-4
    for k in range(2):
        for _ in range(25):
            i = tuple(rng.integers(0, s) for s in c.x[k].shape)
            up, down = c.x[k].copy(), c.x[k].copy()
            up[i] += d
            down[i] -= d
            slope = (loss(k, up, c.w[k]) - loss(k, down, c.w[k])) / (2 * d)
            assert abs(slope - dx[k][i]) <= 1e-4 * (1 + abs(slope))
            up, down = c.w[k].copy(), c.w[k].copy()
            up[i[2]] += d
            down[i[2]] -= d
            slope = (loss(k, c.x[k], up) - loss(k, c.x[k], down)) / (2 * d)
            assert abs(slope - dw[k][i[2]]) <= 1e-4 * (1 + abs(slope))


@pytest.mark.parametrize("half", [True, False])
@pytest.mark.parametrize("dtype,dim,rot", [("bf16", 128, 128), ("f16", 80, 24), ("f32", 30, 10)])
def test_padding_and_positions_outside(P, half, dtype, dim, rot):
    """Padding tokens give zeros and add nothing, whatever they hold; a
    position past the tables gives NaN for its token."""
    pos = np.array([3, -1, 0, -2 ** 31, 49, 7, 7])
    c = Case(P, 7, 3, 2, dim, rot, dtype, "int8", half, positions=pos, seed=1)
    for k in range(2):
        c.dx_in[k][1] = float("nan")
        c.d_g[k][1] = float("inf")
        c.x[k][1], c.g[k][1] = 1.0, 1.0
    near(c.forward(), c.want_forward())
    for from_x in (False, True):
        dx, dw = c.backward(from_x)
        want_dx, want_dw = c.want_backward(from_x)
        near(dx, want_dx)
        near(dw, want_dw)
    c = Case(P, 7, 3, 2, dim, rot, dtype, "int8", half, positions=[3, 50, 0, -1, 49, 2 ** 31 - 1, 7])
    y = c.forward()
    dx, dw = c.backward()
    for k in range(2):
        for a in (y[k], dx[k]):
            assert np.isnan(a[[1, 5]]).all() and np.isfinite(a[[0, 2, 3, 4, 6]]).all()
    assert np.isnan(dw).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,shift,pad", [(128, 0, 0), (128, 1, 0), (64, 0, 4), (40, 8, 8),
                                           (128, 3, 5)])
def test_inside_a_fused_projection(P, dtype, dim, shift, pad):
    """Strided heads at any start, outputs in place."""
    c = Case(P, 6, 4, 2, dim, dim, dtype, fused=True, shift=shift, pad=pad, seed=2)
    near(c.forward(), c.want_forward())
    near(c.forward(keep=False, y=c.dx_in), c.want_forward())  # x becomes y
    c = Case(P, 6, 4, 2, dim, dim, dtype, fused=True, shift=shift, pad=pad, seed=2)
    c.forward()
    want_dx, want_dw = c.want_backward()
    dx, dw = c.backward(dx=c.d_g)  # dy becomes dx
    near(dx, want_dx)
    near(dw, want_dw)


def test_repeated_gradient(P):
    """dy of strides 0, one head for every token and head."""
    c = Case(P, 5, 3, 2, 64, 32, "bf16", seed=3)
    c.forward()
    one = [g[:1, :1].expand(5, h, 64) for g, h in zip(c.d_g, c.heads)]
    c.g = [np.broadcast_to(g[:1, :1], g.shape) for g in c.g]
    dx, dw = c.backward(dy=one)
    want_dx, want_dw = c.want_backward()
    near(dx, want_dx)
    near(dw, want_dw)


def test_added_to_earlier_gradients(P):
    import torch
    c = Case(P, 50, 4, 2, 96, 96, "f32", seed=4)
    c.forward()
    _, dw = c.backward()
    add = torch.randn(2, 96, device="cuda")
    _, got = c.backward(dw_in=add)
    assert np.array_equal(got, (add + torch.from_numpy(dw).float().cuda()).double().cpu().numpy())
    c.backward(dw=False)
    assert (c.dw == 7).all()


def test_nothing_to_do(P):
    import torch
    c = Case(P, 0, 2, 1, 16, 16)
    assert all(y.size == 0 for y in c.forward())
    add = torch.randn(2, 16, device="cuda")
    _, dw = c.backward(dw_in=add)
    assert np.array_equal(dw, add.double().cpu().numpy())
    _, dw = c.backward()
    assert (dw == 0).all()
    c = Case(P, 3, 0, 0, 16, 16)
    c.forward()
    _, dw = c.backward()
    assert (dw == 0).all()


def test_without_weights_and_rotation(P):
    c = Case(P, 4, 2, 1, 48, 0, "f32", weights=False, n_pos=4)
    near(c.forward(), c.want_forward())


def test_rows_beyond_32_bit_offsets(P):
    import torch
    c = Case(P, 2, 2, 1, 64, 64, "bf16", seed=6)
    big = torch.empty((1 << 32) + 4096, dtype=torch.bfloat16, device="cuda")
    far = [big.as_strided((2, 2, 64), (1 << 32, 256, 1)),
           big[1024:].as_strided((2, 1, 64), (1 << 32, 64, 1))]
    for k in range(2):
        far[k].copy_(c.dx_in[k])
    near_x, c.dx_in = c.dx_in, far
    near(c.forward(), c.want_forward())
    c.dx_in = near_x
    near(c.forward(y=far), c.want_forward())


def test_same_bits_every_time(P):
    """Weights' gradients of many tokens, the same on every call and stream."""
    import torch
    c = Case(P, 3000, 8, 2, 128, 128, "bf16", n_pos=3000, seed=7)
    c.forward(stream=torch.cuda.Stream())
    first = c.backward()
    for _ in range(4):
        again = c.backward()
        assert np.array_equal(first[1], again[1])
        assert all(np.array_equal(a, b) for a, b in zip(first[0], again[0]))
