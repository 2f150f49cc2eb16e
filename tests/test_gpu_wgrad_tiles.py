"""poseidon_ckpt_wgrad on the tiles and cuts that large sizes take: last tiles narrower
than the others, cut and whole, and sums of many rows in one tile.  The sums in 64 bits
are the GPU's, of the values that poseidon_ckpt_unpack gives (compared bit for bit in
test_gpu_ckpt.py); tolerances as in test_gpu_wgrad.py."""
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


def kept(P, x, fmt, dtype):
    """(checkpoint of f32 x, what it stands for in the type)."""
    import torch
    rows, cols = x.shape
    ckpt = torch.empty(U.layout(rows, cols)[3], dtype=torch.uint8, device="cuda")
    y = torch.empty(rows, cols, dtype=U.DTYPES[dtype], device="cuda")
    P.poseidon_ckpt_pack(x.data_ptr(), 2, rows, cols, cols, U.FORMATS[fmt], ckpt.data_ptr(), stream())
    P.poseidon_ckpt_unpack(ckpt.data_ptr(), U.FORMATS[fmt], rows, cols, y.data_ptr(),
                           U.CODES[dtype], cols, stream())
    return ckpt, y


def wgrad(P, ckpt, fmt, dy, dtype, cols, add=None):
    import torch
    rows, n = dy.shape
    out = torch.full((n + 1, cols + 3), 9.0, device="cuda")
    if add is not None:
        out[:n, :cols] = add
    P.poseidon_ckpt_wgrad(ckpt.data_ptr(), U.FORMATS[fmt], dy.data_ptr(), U.CODES[dtype],
                          dy.stride(0), rows, n, cols, 0 if add is None else out.data_ptr(),
                          out.data_ptr(), cols + 3, stream())
    torch.cuda.synchronize()
    assert bool((out[n:] == 9).all()) and bool((out[:, cols:] == 9).all())
    return out[:n, :cols]


# Tiles of 256 columns of dy and last ones for 3 (64 wide), 100 (128 wide) or 128
# columns; on 76 pairs of SMs the first two sizes take all rows in one unit, the next
# cut every tile into three parts, the last the narrow tiles and a few others only.
@pytest.mark.parametrize("rows,n,cols", [(4093, 1283, 5120), (4093, 1380, 5120), (4093, 1283, 1024),
                                         (4093, 1408, 1024), (4093, 1380, 4096)])
@pytest.mark.parametrize("dtype,fmt", [("bf16", "int8"), ("bf16", "e4m3"), ("f16", "int8"),
                                       ("f16", "e4m3")])
@pytest.mark.parametrize("added", [False, True])
def test_narrow_last_tiles(P, rows, n, cols, dtype, fmt, added):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(n)
    ckpt, x = kept(P, torch.randn(rows, cols, device="cuda", generator=gen), fmt, dtype)
    # rows of whole 16-byte words, so that the tensor copies read dy itself
    wide = torch.randn(rows, -(-n // 8) * 8, device="cuda", generator=gen).to(U.DTYPES[dtype])
    dy = wide[:, :n]
    add = torch.randn(n, cols, device="cuda", generator=gen) if added else None
    got = wgrad(P, ckpt, fmt, dy, dtype, cols, add).double()
    want = dy.double().t() @ x.double()
    size = dy.double().abs().t() @ x.double().abs()
    if added:
        want += add.double()
    room = (rows / 16 + 16) * 2.0 ** -23 * size + 2.0 ** -22 * want.abs()
    assert bool(((got - want).abs() <= room).all())


# tiles of 128 columns (cut) and of 256 (cut) in f16, which the smaller sizes of
# test_gpu_wgrad.py give tiles of 64 only
@pytest.mark.parametrize("rows,n,cols", [(4200, 300, 520), (2048, 2048, 1024), (2000, 700, 520),
                                         (1500, 5000, 3000)])
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_wide_tiles_in_f16(P, rows, n, cols, fmt):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(cols)
    ckpt, x = kept(P, torch.randn(rows, cols, device="cuda", generator=gen), fmt, "f16")
    dy = torch.randn(rows, n, device="cuda", generator=gen).half()
    got = wgrad(P, ckpt, fmt, dy, "f16", cols).double()
    want = dy.double().t() @ x.double()
    room = (rows / 16 + 16) * 2.0 ** -23 * (dy.double().abs().t() @ x.double().abs()) + \
        2.0 ** -22 * want.abs()
    assert bool(((got - want).abs() <= room).all())


def test_precision_of_tiles_that_are_not_cut(P):
    """16384 rows in one unit (64 tiles on 76 pairs), all products positive.  An
    accumulator of 768 rows adds 48 times, and each addition cuts off less than 2^-23 of
    the sum so far: less than 24.5 * 2^-23 = 2.9e-6 of its result on average over its
    growth; adding such sums rounds to both sides.  One accumulator of all rows drifts
    by what 2.6e-6 over 4096 rows gives for 16384, 1e-5."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.rand(16384, 2048, device="cuda", generator=gen) + 0.5
    ckpt, y = kept(P, x, "int8", "bf16")
    dy = (torch.rand(16384, 2048, device="cuda", generator=gen) + 0.5).bfloat16()
    got = wgrad(P, ckpt, "int8", dy, "bf16", 2048).double()
    off = got / (dy.double().t() @ y.double()) - 1
    assert abs(float(off.mean())) <= 24.5 * 2.0 ** -23
