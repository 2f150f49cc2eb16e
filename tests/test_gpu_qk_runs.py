"""poseidon_qk_forward and poseidon_qk_backward where a warp takes many steps:
heads one after another within a task, a ring of rows in shared memory that is used
again and passes from token to token, sums over a thread's steps.  Compared with the
formulas in 64 bits, with the tolerances of test_gpu_qk.py."""
import numpy as np
import pytest

import layer_util as U
from test_gpu_qk import Case, near

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2609_06086_gb300 as P
    P.lib()
    return P


def moved(tensors, shift):
    """The tensors at a start `shift` elements past an aligned one, rows one element wider."""
    import torch
    out = []
    for t in tensors:
        T, h, d = t.shape
        flat = torch.full((T * h * (d + 1) + shift,), float("nan"), dtype=t.dtype, device="cuda")
        v = flat[shift:].as_strided((T, h, d), (h * (d + 1), d + 1, 1))
        v.copy_(t)
        out.append(v)
    return out


# 41 + 7 heads (the last step of a token is not whole).  On 152 SMs a warp takes 2 to 8
# steps of a task forward and 3 to 15 of one to four tokens backward, most runs starting
# within a token.
SHAPES = [(900, 128, 128, True, 0), (900, 128, 128, False, 0), (900, 128, 64, True, 0),
          (900, 80, 48, False, 0), (900, 72, 36, True, 0), (900, 200, 16, False, 0),
          (700, 256, 256, True, 0), (2000, 64, 64, True, 0), (2000, 40, 20, True, 0),
          (900, 128, 128, True, 1), (900, 70, 30, True, 3)]


@pytest.mark.parametrize("T,dim,rot,half,shift", SHAPES)
@pytest.mark.parametrize("dtype,fmt", [("bf16", "int8"), ("f16", "e4m3"), ("f32", "int8")])
def test_many_steps(P, T, dim, rot, half, shift, dtype, fmt):
    """Outputs, codes, scale bytes, 1 / rms, gradients from the checkpoints and from x,
    in place too, with padding tokens that hold NaNs and infinities."""
    rng = np.random.default_rng(T + dim)
    pos = rng.integers(0, 50, T)
    pos[rng.random(T) < 0.08] = -1
    live = pos >= 0

    def make():
        c = Case(P, T, 41, 7, dim, rot, dtype, fmt, half, positions=pos, seed=dim)
        for k in range(2):
            c.dx_in[k][~live] = float("nan")
            c.d_g[k][~live] = float("inf")
            c.x[k][~live] = 1.0
            c.g[k][~live] = 1.0
        if shift:
            c.dx_in, c.d_g = moved(c.dx_in, shift), moved(c.d_g, shift)
        return c

    c = make()
    near(c.forward(), c.want_forward())
    for k, h in enumerate(c.heads):
        groups, pitch, spitch, size = U.layout(T * h, dim)
        b = c.c[k].cpu().numpy()
        assert (b[size:] == 0xAB).all()
        codes, scales = U.encode(c.x[k][live].reshape(-1, dim), fmt)
        got = b[:T * h * pitch].reshape(T, h, pitch)[live].reshape(-1, pitch)
        assert np.array_equal(got, codes) if fmt == "int8" else \
            np.array_equal(U.E4M3[got], U.E4M3[codes])
        got = b[T * h * pitch:size].reshape(T, h, spitch)[live][:, :, :groups]
        assert np.array_equal(got.reshape(-1, groups), scales)
        r = c.r[k].double().cpu().numpy()[..., None]
        assert (np.abs(r / c.norm(k) - 1) <= (dim / 2 + 4) * 2.0 ** -24)[live].all()
    for from_x in (False, True):
        want_dx, want_dw = c.want_backward(from_x)
        dx, dw = c.backward(from_x)
        near(dx, want_dx)
        near(dw, want_dw)
    want = c.want_forward()
    near(c.forward(keep=False, y=c.dx_in), want)  # x becomes y
    c = make()
    c.forward()
    want_dx, want_dw = c.want_backward()
    dx, dw = c.backward(dx=c.d_g)  # dy becomes dx
    near(dx, want_dx)
    near(dw, want_dw)


def test_same_bits_on_two_streams(P):
    """Forward passes on two streams, each behind the stream that made its inputs, and
    backward passes that overlap on them with outputs and partial sums of their own."""
    import torch
    c = Case(P, 3000, 8, 2, 128, 128, "bf16", n_pos=3000, seed=7)
    first = c.forward()
    kept = [t.clone() for t in (*c.c, *c.r)]
    first_dx, first_dw = c.backward()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for i in range(6):
        y, dx = c.new(), c.new()
        ck, r = [torch.full_like(t, 0xAB) for t in c.c], [torch.empty_like(t) for t in c.r]
        outs.append((y, dx, ck, r, torch.full((2, 128), 7.0, device="cuda")))
    torch.cuda.synchronize()
    for i, (y, dx, ck, r, dw) in enumerate(outs):
        s = streams[i % 2].cuda_stream
        rp, cp = tuple(t.data_ptr() for t in r), tuple(t.data_ptr() for t in ck)
        P.poseidon_qk_forward(c.qk, c.pair(c.dx_in), c.pair(y), rstd=rp, ckpt=cp, stream=s)
        P.poseidon_qk_backward(c.qk, c.pair(c.d_g), c.pair(dx), rp, ckpt=cp, dw=dw.data_ptr(),
                               stream=s)
    torch.cuda.synchronize()
    for y, dx, ck, r, dw in outs:
        for a, b in zip(first, y):
            assert np.array_equal(a, b.double().cpu().numpy())
        for a, b in zip(kept, (*ck, *r)):
            assert torch.equal(a, b)
        for a, b in zip(first_dx, dx):
            assert np.array_equal(a, b.double().cpu().numpy())
        assert np.array_equal(first_dw, dw.double().cpu().numpy())
