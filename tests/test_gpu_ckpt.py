"""poseidon_ckpt_pack and poseidon_ckpt_unpack against the definition in 64
bits.  Both are exact: codes, scale bytes and values are compared bit for bit."""
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


def pack(P, x, fmt, dtype):
    """(codes, scale bytes) of a device matrix x (its rows may be strided)."""
    import torch
    rows, cols = x.shape
    groups, pitch, spitch, size = U.layout(rows, cols)
    assert P.poseidon_ckpt_bytes(rows, cols) == size
    buf = torch.full((size + 64,), 0xAB, dtype=torch.uint8, device="cuda")
    P.poseidon_ckpt_pack(x.data_ptr(), U.CODES[dtype], rows, cols, x.stride(0), U.FORMATS[fmt],
                         buf.data_ptr(), stream())
    torch.cuda.synchronize()
    b = buf.cpu().numpy()
    assert (b[size:] == 0xAB).all()  # nothing past the checkpoint is written
    return b[:rows * pitch].reshape(rows, pitch), \
        b[rows * pitch:size].reshape(rows, spitch)[:, :groups]


def unpack(P, codes, scales, cols, fmt, dtype, pad):
    import torch
    rows = len(codes)
    buf = U.buffer(codes, scales)
    y = torch.full((rows, cols + pad), 77.0, dtype=U.DTYPES[dtype], device="cuda")
    P.poseidon_ckpt_unpack(buf.data_ptr(), U.FORMATS[fmt], rows, cols, y.data_ptr(),
                           U.CODES[dtype], cols + pad, stream())
    torch.cuda.synchronize()
    assert (y[:, cols:] == 77).all()
    return y[:, :cols].double().cpu().numpy()


def values(rows, cols, dtype, seed):
    """Values of every magnitude that the type has, halves of codes, zeros."""
    import torch
    rng = np.random.default_rng(seed)
    wide = {"bf16": 80, "f16": 8, "f32": 80}[dtype]
    x = rng.standard_normal((rows, cols)) * np.exp(rng.uniform(-wide, wide, (rows, 1)))
    x[rng.random((rows, cols)) < 0.1] = 0
    ties = rng.integers(-255, 256, (rows, cols)) / 2.0
    x = np.where(rng.random((rows, 1)) < 0.3, ties, x)
    if rows > 2:
        x[rows // 2] = 0
    return torch.from_numpy(x).to(U.DTYPES[dtype])


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 31, 1), (3, 32, 0), (2, 33, 3), (5, 64, 8),
                                           (7, 100, 4), (33, 129, 0), (64, 1000, 8), (130, 517, 5)])
def test_round_trip(P, rows, cols, pad, dtype, fmt):
    import torch
    x = values(rows, cols, dtype, rows * 1000 + cols)
    wide = torch.full((rows, cols + pad), float("nan"), dtype=x.dtype)
    wide[:, :cols] = x
    codes, scales = pack(P, wide.cuda()[:, :cols], fmt, dtype)
    want_codes, want_scales = U.encode(x.double().numpy(), fmt)
    assert np.array_equal(scales, want_scales)
    if fmt == "e4m3":  # zeros of either sign are one value
        same = U.E4M3[codes] == U.E4M3[want_codes]
        assert same.all()
    else:
        assert np.array_equal(codes, want_codes)
    for out in ("bf16", "f16", "f32"):
        got = unpack(P, codes, scales, cols, fmt, out, pad)
        want = U.as_type(U.decode(codes, scales, cols, fmt), out)
        assert np.array_equal(got, want)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_extreme_groups(P, dtype, fmt):
    """Infinities and NaNs make their own group NaN and no other; the type's
    largest and lowest values saturate or stay; the smallest ones vanish."""
    import torch
    t = U.DTYPES[dtype]
    top, tiny = torch.finfo(t).max, torch.finfo(t).tiny
    x = torch.ones(9, 96, dtype=t)
    x[0, 40] = float("inf")
    x[1, 40] = float("-inf")
    x[2, 40] = float("nan")
    x[3, :] = top
    x[4, :] = -top
    x[5, 0] = -top
    x[6, :] = tiny
    x[7, :] = tiny / 8
    x[8, 64:] = 0
    codes, scales = pack(P, x.cuda(), fmt, dtype)
    want_codes, want_scales = U.encode(x.double().numpy(), fmt)
    assert np.array_equal(scales, want_scales) and (scales[:3, 1] == 255).all()
    assert np.array_equal(codes, want_codes)
    got = unpack(P, codes, scales, 96, fmt, dtype, 0)
    assert np.array_equal(got, U.as_type(U.decode(codes, scales, 96, fmt), dtype), equal_nan=True)
    assert np.isnan(got[:3, 32:64]).all() and np.isfinite(got[:3, :32]).all()
    assert np.isfinite(got[3:]).all()


@pytest.mark.parametrize("rows,cols", [(0, 5), (5, 0), (0, 0)])
def test_nothing_to_do(P, rows, cols):
    P.poseidon_ckpt_pack(0, 0, rows, cols, cols, 0, 0, stream())
    P.poseidon_ckpt_unpack(0, 0, rows, cols, 0, 0, cols, stream())


def test_repeated_row(P):
    """A stride of 0 reads one row again and again."""
    import torch
    x = values(1, 70, "bf16", 3).cuda()
    codes, scales = pack(P, x.expand(6, 70), "int8", "bf16")
    want = U.encode(x.double().cpu().numpy(), "int8")
    assert np.array_equal(codes, np.repeat(want[0], 6, 0))
    assert np.array_equal(scales, np.repeat(want[1], 6, 0))


def test_rows_beyond_32_bit_offsets(P):
    """Rows 2^31 elements apart: element and byte offsets pass 32 bits."""
    import torch
    ld, cols = 1 << 31, 40
    big = torch.empty(2 * ld + cols, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((3, cols), (ld, 1))
    v = values(3, cols, "bf16", 4)
    x.copy_(v)
    codes, scales = pack(P, x, "int8", "bf16")
    want = U.encode(v.double().numpy(), "int8")
    assert np.array_equal(codes, want[0]) and np.array_equal(scales, want[1])
    x.zero_()
    buf = U.buffer(*want)
    P.poseidon_ckpt_unpack(buf.data_ptr(), 0, 3, cols, x.data_ptr(), 0, ld, stream())
    torch.cuda.synchronize()
    assert np.array_equal(x.double().cpu().numpy(), U.decode(*want, cols, "int8"))


def test_on_another_stream(P):
    """The calls are ordered on the stream they are given."""
    import torch
    s = torch.cuda.Stream()
    x = values(512, 1024, "bf16", 5)
    with torch.cuda.stream(s):
        d = torch.zeros(512, 1024, dtype=torch.bfloat16, device="cuda")
        buf = torch.zeros(U.layout(512, 1024)[3], dtype=torch.uint8, device="cuda")
        y = torch.zeros(512, 1024, device="cuda")
        torch.cuda._sleep(20_000_000)
        d.copy_(x.pin_memory(), non_blocking=True)
        P.poseidon_ckpt_pack(d.data_ptr(), 0, 512, 1024, 1024, 1, buf.data_ptr(), s.cuda_stream)
        P.poseidon_ckpt_unpack(buf.data_ptr(), 1, 512, 1024, y.data_ptr(), 2, 1024, s.cuda_stream)
    s.synchronize()
    assert np.array_equal(y.double().cpu().numpy(), U.kept(x.double().numpy(), "e4m3"))
