"""poseidon_ckpt_wgrad against the sum of exact products in 64 bits.

Tolerance: products are exact, and a sum of T of them in 32 bits is off by at
most (T / 16 + 16) 2^-23 times the sum of their magnitudes (16 products of a
tensor core's step are aligned to the largest and cut, then added to the sum,
which is cut or rounded), plus one rounding of 2^-24 for every later addition."""
import numpy as np
import pytest

import layer_util as U

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2609_06086_gb300 as P
    P.lib()
    return P


def stream():
    import torch
    return torch.cuda.current_stream().cuda_stream


def make(rows, n, cols, dtype, fmt, seed):
    """(codes, scale bytes, x in f64 as dy's type has it, dy on the CPU)."""
    import torch
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * np.exp(rng.uniform(-3, 3, (1, cols)))
    codes, scales = U.encode(x, fmt)
    dy = torch.from_numpy(rng.standard_normal((rows, n)) * 0.1).to(U.DTYPES[dtype])
    return codes, scales, U.as_type(U.decode(codes, scales, cols, fmt), dtype), dy


def call(P, ckpt, fmt, dy, dtype, rows, n, cols, ld_dy, add, out, ld):
    import torch
    P.poseidon_ckpt_wgrad(ckpt.data_ptr(), U.FORMATS[fmt], dy.data_ptr(), U.CODES[dtype], ld_dy,
                          rows, n, cols, 0 if add is None else add.data_ptr(), out.data_ptr(), ld,
                          stream())
    torch.cuda.synchronize()


def near(got, x, dy, add=None):
    y = dy.double().numpy()
    want = y.T @ x + (0 if add is None else add)
    room = (len(x) / 16 + 16) * 2.0 ** -23 * (np.abs(y).T @ np.abs(x)) + 2.0 ** -22 * np.abs(want)
    assert (np.abs(got - want) <= room).all(), np.max(np.abs(got - want) / room)


SIZES = [(1, 1, 1), (1, 300, 40), (5, 8, 32), (16, 64, 64), (63, 100, 33), (64, 256, 256),
         (65, 257, 129), (130, 31, 300), (513, 520, 264), (1100, 24, 1000)]


@pytest.mark.parametrize("rows,n,cols", SIZES)
@pytest.mark.parametrize("dtype,fmt", [("bf16", "int8"), ("bf16", "e4m3"), ("f16", "int8"),
                                       ("f16", "e4m3")])
def test_against_64_bits(P, rows, n, cols, dtype, fmt):
    import torch
    codes, scales, x, dy = make(rows, n, cols, dtype, fmt, rows + n)
    out = torch.full((n + 1, cols + 3), 9.0, device="cuda")
    call(P, U.buffer(codes, scales), fmt, dy.cuda(), dtype, rows, n, cols, n, None, out, cols + 3)
    near(out[:n, :cols].double().cpu().numpy(), x, dy)
    assert (out[n:] == 9).all() and (out[:, cols:] == 9).all()  # nothing else is written


@pytest.mark.parametrize("rows,n,cols", [(200, 70, 90), (4200, 300, 520), (9000, 40, 64)])
def test_added_to_earlier_gradients(P, rows, n, cols):
    """dw_in in a buffer of its own, and dw_in = dw_out."""
    import torch
    codes, scales, x, dy = make(rows, n, cols, "bf16", "int8", 7)
    ckpt, d = U.buffer(codes, scales), dy.cuda()
    add = torch.randn(n, cols, device="cuda")
    before = add.clone()
    out = torch.empty_like(add)
    call(P, ckpt, "int8", d, "bf16", rows, n, cols, n, add, out, cols)
    near(out.double().cpu().numpy(), x, dy, before.double().cpu().numpy())
    assert torch.equal(add, before)
    call(P, ckpt, "int8", d, "bf16", rows, n, cols, n, add, add, cols)
    assert torch.equal(add, out)  # the same sums in the same order


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shift,pad", [(1, 0), (0, 3), (8, 8), (3, 5)])
def test_strides_and_alignment_of_dy(P, dtype, shift, pad):
    """Rows of a wider buffer, at a start that need not be 16-byte aligned;
    NaNs lie between the rows."""
    import torch
    rows, n, cols = 100, 72, 96
    codes, scales, x, dy = make(rows, n, cols, dtype, "e4m3", 11)
    flat = torch.full((rows * (n + pad) + shift + 8,), float("nan"), dtype=dy.dtype, device="cuda")
    view = flat[shift:].as_strided((rows, n), (n + pad, 1))
    view.copy_(dy)
    out = torch.empty(n, cols, device="cuda")
    call(P, U.buffer(codes, scales), "e4m3", view, dtype, rows, n, cols, n + pad, None, out, cols)
    near(out.double().cpu().numpy(), x, dy)


def test_broadcast_dy(P):
    """A gradient repeated over the rows (stride 0), as the sum's is."""
    import torch
    codes, scales, x, dy = make(70, 40, 50, "bf16", "int8", 12)
    row = dy[:1].contiguous()
    out = torch.empty(40, 50, device="cuda")
    call(P, U.buffer(codes, scales), "int8", row.cuda(), "bf16", 70, 40, 50, 0, None, out, 50)
    near(out.double().cpu().numpy(), x, row.expand(70, 40))


def test_dy_rows_beyond_32_bit_offsets(P):
    import torch
    rows, n, cols, ld = 3, 16, 40, 1 << 31
    codes, scales, x, dy = make(rows, n, cols, "bf16", "int8", 13)
    big = torch.empty(2 * ld + n, dtype=torch.bfloat16, device="cuda")
    view = big.as_strided((rows, n), (ld, 1))
    view.copy_(dy)
    out = torch.empty(n, cols, device="cuda")
    call(P, U.buffer(codes, scales), "int8", view, "bf16", rows, n, cols, ld, None, out, cols)
    near(out.double().cpu().numpy(), x, dy)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_extreme_scales(P, dtype, fmt):
    """Every exponent that the sums still hold; f16 rounds and saturates as
    poseidon_ckpt_unpack does.  One row: the products are the result, exact in
    f32 (an f16 product of two 11-bit numbers has 22 bits)."""
    import torch
    n, cols = 8, 32 * 230
    exps = np.arange(-110, 120)
    rng = np.random.default_rng(2)
    codes = rng.integers(0, 127, (1, cols)).astype(np.uint8)
    scales = (exps + 127).astype(np.uint8)[None]
    x = U.as_type(U.decode(codes, scales, cols, fmt), dtype)
    dy = torch.tensor([[1, -1, 0.5, 2, 0, -0.25, 1.5, -1.75]], dtype=U.DTYPES[dtype])
    out = torch.empty(n, cols, device="cuda")
    call(P, U.buffer(codes, scales), fmt, dy.cuda(), dtype, 1, n, cols, n, None, out, cols)
    want = dy.double().numpy().T @ x
    got = out.double().cpu().numpy()
    # a product past 2^128 overflows to infinity, as f32 does
    fits = np.abs(want) < 2.0 ** 127
    assert np.array_equal(got[fits], want[fits])


def test_nan_groups_stay_in_their_columns(P):
    """A group that stands for NaNs makes its 32 columns of dW NaN and no
    others; an infinite gradient makes its row of dW infinite or NaN only."""
    import torch
    rows, n, cols = 90, 40, 200
    codes, scales, x, dy = make(rows, n, cols, "bf16", "int8", 14)
    scales[17, 2] = 255
    codes[17, 64:96] = 0
    out = torch.empty(n, cols, device="cuda")
    call(P, U.buffer(codes, scales), "int8", dy.cuda(), "bf16", rows, n, cols, n, None, out, cols)
    got = out.double().cpu().numpy()
    assert np.isnan(got[:, 64:96]).all()
    rest = np.r_[0:64, 96:200]
    near(got[:, rest], x[:, rest], dy)
    codes, scales, x, dy = make(rows, n, cols, "bf16", "int8", 14)
    dy[3, 5] = float("inf")
    call(P, U.buffer(codes, scales), "int8", dy.cuda(), "bf16", rows, n, cols, n, None, out, cols)
    got = out.double().cpu().numpy()
    assert not np.isfinite(got[5]).any()
    keep = [i for i in range(n) if i != 5]
    near(got[keep], x, dy[:, keep])


@pytest.mark.parametrize("add", [False, True])
def test_no_rows(P, add):
    """No rows: dw_in, or zeros."""
    import torch
    a = torch.randn(5, 7, device="cuda")
    out = torch.full((5, 7), 3.0, device="cuda")
    P.poseidon_ckpt_wgrad(0, 0, 0, 0, 0, 0, 5, 7, a.data_ptr() if add else 0, out.data_ptr(), 7,
                          stream())
    torch.cuda.synchronize()
    assert torch.equal(out, a if add else torch.zeros_like(a))
    P.poseidon_ckpt_wgrad(0, 0, 0, 0, 0, 9, 0, 7, 0, out.data_ptr(), 7, stream())
    P.poseidon_ckpt_wgrad(0, 0, 0, 0, 0, 9, 5, 0, 0, out.data_ptr(), 7, stream())


def test_long_sums_keep_their_precision(P):
    """16384 rows whose products share their sign: cutting every step of one
    32-bit sum would lose 16384 / 16 / 2 * 2^-24 = 3e-5 of the result; sums of
    at most 1024 rows added by rounding lose less than a tenth of that."""
    import torch
    rows, n, cols = 16384, 128, 128
    rng = np.random.default_rng(3)
    codes, scales = U.encode(np.abs(rng.standard_normal((rows, cols))) + 0.1, "int8")
    x = U.decode(codes, scales, cols, "int8")
    dy = torch.from_numpy(np.abs(rng.standard_normal((rows, n))) + 0.1).to(torch.bfloat16)
    out = torch.empty(n, cols, device="cuda")
    call(P, U.buffer(codes, scales), "int8", dy.cuda(), "bf16", rows, n, cols, n, None, out, cols)
    want = dy.double().numpy().T @ x
    assert np.max(np.abs(out.double().cpu().numpy() / want - 1)) <= 3e-6


@pytest.mark.parametrize("rows,n,cols", [(300, 200, 300), (5000, 300, 600), (2048, 2048, 1024)])
def test_same_bits_every_time(P, rows, n, cols):
    """Also while calls on two streams overlap."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(5)
    codes = torch.randint(0, 127, (rows, U.layout(rows, cols)[1]), generator=gen, device="cuda")
    spitch = U.layout(rows, cols)[2]
    ckpt = torch.cat([codes.to(torch.uint8).flatten(),
                      torch.randint(120, 130, (rows * spitch,), generator=gen,
                                    device="cuda").to(torch.uint8)])
    dy = torch.randn(rows, n, generator=gen, device="cuda").to(torch.bfloat16)
    first = torch.empty(n, cols, device="cuda")
    call(P, ckpt, "int8", dy, "bf16", rows, n, cols, n, None, first, cols)
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.full((n, cols), 5.0, device="cuda") for _ in range(6)]
    torch.cuda.synchronize()
    for i, o in enumerate(outs):
        P.poseidon_ckpt_wgrad(ckpt.data_ptr(), 0, dy.data_ptr(), 0, n, rows, n, cols, 0,
                              o.data_ptr(), cols, streams[i % 2].cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(first, o) for o in outs)


@pytest.mark.parametrize("rows,n,cols,fmt", [(4096, 6144, 4096, "int8"), (8192, 2048, 2048, "e4m3"),
                                             (1500, 5000, 3000, "int8")])
def test_many_tiles_added_to_earlier_gradients(P, rows, n, cols, fmt):
    """Several tiles per pair of SMs with dw_in to read in between, which lets
    the loads run as far ahead as their buffers allow; several calls, since what
    overtakes what differs from one to the next.  The sums in 64 bits are the
    GPU's, of the values that poseidon_ckpt_unpack gives."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x = torch.randn(rows, cols, device="cuda", generator=gen)
    ckpt = torch.empty(U.layout(rows, cols)[3], dtype=torch.uint8, device="cuda")
    P.poseidon_ckpt_pack(x.data_ptr(), 2, rows, cols, cols, U.FORMATS[fmt], ckpt.data_ptr(), stream())
    P.poseidon_ckpt_unpack(ckpt.data_ptr(), U.FORMATS[fmt], rows, cols, x.data_ptr(), 2, cols,
                           stream())
    dy = torch.randn(rows, n, device="cuda", generator=gen).to(torch.bfloat16)
    add = torch.randn(n, cols, device="cuda", generator=gen)
    want = add.double() + dy.double().t() @ x.double()
    size = dy.double().abs().t() @ x.double().abs()
    room = (rows / 16 + 16) * 2.0 ** -23 * size + 2.0 ** -22 * want.abs()
    for _ in range(8):
        out = torch.full((n, cols), 5.0, device="cuda")
        call(P, ckpt, fmt, dy, "bf16", rows, n, cols, n, add, out, cols)
        assert bool(((out.double() - want).abs() <= room).all())
