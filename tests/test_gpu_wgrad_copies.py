"""poseidon_ckpt_wgrad in blocks: where dy has to be copied first, 256 MB at a time, of
columns, and of rows where there are many; and of the largest row counts.  Values are whole numbers and sums stay
below 2^24, so that gradients are exact in any order of the sums."""
import pytest

import layer_util as U

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2609_06086_gb300 as P
    P.lib()
    return P


def make(rows, n, cols, seed):
    """(checkpoint, dy [rows][n] of odd stride): codes of scale 1, dy in {-1, 0, 1}."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    groups, pitch, spitch, size = U.layout(rows, cols)
    ckpt = torch.full((size,), 127, dtype=torch.uint8, device="cuda")
    codes = ckpt[:rows * pitch].view(rows, pitch)
    codes.zero_()
    codes[:, :cols] = torch.randint(-127, 128, (rows, cols), dtype=torch.int8, device="cuda",
                                    generator=gen).view(torch.uint8)
    ld = n | 1
    dy = torch.randint(-1, 2, (rows, ld), dtype=torch.int8, device="cuda", generator=gen).bfloat16()
    return ckpt, dy[:, :n]


def same(got, ckpt, dy, cols, add=None):
    rows, n = dy.shape
    pitch = U.layout(rows, cols)[1]
    x = ckpt[:rows * pitch].view(rows, pitch)[:, :cols].contiguous().view(dtype=U.torch.int8).double()
    for j in range(0, n, 1024):
        want = dy[:, j:j + 1024].double().t() @ x
        if add is not None:
            want += add[j:j + 1024].double()
        assert bool((got[j:j + 1024].double() == want).all()), j


def call(P, ckpt, dy, cols, add, out):
    import torch
    rows, n = dy.shape
    P.poseidon_ckpt_wgrad(ckpt.data_ptr(), 0, dy.data_ptr(), 0, dy.stride(0), rows, n, cols,
                          0 if add is None else add.data_ptr(), out.data_ptr(), out.stride(0),
                          torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()


def test_the_pool_keeps_no_large_copy(P):
    """dy of 4.3 GB: the library holds 256 MB for a copy and 64 MB for partial sums at most."""
    import torch
    ckpt, dy = make(65536, 32769, 64, 1)
    out = torch.empty(32769, 64, device="cuda")
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    free = torch.cuda.mem_get_info()[0]
    call(P, ckpt, dy, 64, None, out)
    assert free - torch.cuda.mem_get_info()[0] <= 352 << 20
    same(out, ckpt, dy, 64)


@pytest.mark.parametrize("rows,n,cols", [(16384, 20001, 300),  # three blocks of columns
                                         (8_500_001, 9, 40),   # two of rows
                                         (600_001, 301, 33)])  # two of either
def test_blocks(P, rows, n, cols):
    """Alone, added to other gradients, and added in place."""
    import torch
    ckpt, dy = make(rows, n, cols, 2)
    out = torch.full((n + 1, cols + 2), 9.0, device="cuda")
    call(P, ckpt, dy, cols, None, out)
    same(out[:n, :cols], ckpt, dy, cols)
    add = torch.randint(-1000, 1000, (n + 1, cols + 2), device="cuda").float()
    before = add.clone()
    call(P, ckpt, dy, cols, add, out)
    same(out[:n, :cols], ckpt, dy, cols, add[:n, :cols])
    assert torch.equal(add, before)
    call(P, ckpt, dy, cols, add, add)
    same(add[:n, :cols], ckpt, dy, cols, before[:n, :cols])
    for a, b in ((out, torch.full_like(out, 9.0)), (add, before)):  # nothing else is written
        assert torch.equal(a[n:], b[n:]) and torch.equal(a[:, cols:], b[:, cols:])


def test_most_rows(P):
    """The largest row count: all zeros but for rows on either side of the places where
    sums begin and end.  111 GB: skipped where they are not free."""
    import torch
    rows, n, cols = 2 ** 31 - 65, 8, 32
    pitch, size = U.layout(rows, cols)[1], U.layout(rows, cols)[3]
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 130 << 30:
        pytest.skip("needs 130 GB of device memory")
    ckpt = torch.zeros(size, dtype=torch.uint8, device="cuda")
    dy = torch.zeros(rows, n, dtype=torch.bfloat16, device="cuda")
    want = torch.zeros(n, cols, dtype=torch.float64)
    gen = torch.Generator().manual_seed(5)
    marked = [0, 1, 767, 768, 2 ** 30 - 1, 2 ** 30, 2 ** 30 + 768, 2 ** 31 - 833, 2 ** 31 - 769,
              2 ** 31 - 768, rows - 64, rows - 1]
    for r in marked:
        code = torch.randint(-127, 128, (cols,), dtype=torch.int8, generator=gen)
        g = torch.randint(-8, 9, (n,), generator=gen).bfloat16()
        ckpt[r * pitch:(r + 1) * pitch] = code.view(torch.uint8).cuda()
        ckpt[rows * pitch + 4 * r] = 127
        dy[r] = g.cuda()
        want += torch.outer(g.double(), code.double())
    out = torch.full((n, cols), 5.0, device="cuda")
    call(P, ckpt, dy, cols, None, out)
    del ckpt, dy
    torch.cuda.empty_cache()
    assert torch.equal(out.double().cpu(), want)
