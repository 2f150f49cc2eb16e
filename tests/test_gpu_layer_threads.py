"""Norm, dropout and attention called from several host threads at once, and the norm in place
at widths of every kind of team of threads."""
import threading

import pytest

from test_gpu_attn import Call as Attn
from test_gpu_norm import Call as Norm

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2609_06086_gb300 as P
    return P


def test_host_threads(P):
    """Four threads, a stream each, sizes of their own: the results of one after another."""
    def make(i):
        return (Attn(P, [100 * i + 3, 700], 8, 2, (64, 80, 128, 72)[i], ("bf16", "f16")[i % 2],
                     ("fused", "odd")[i // 2]),
                Norm(P, 300, 1000 + 999 * i, "bf16", "f32", "int8", 0.1))

    def passes(calls, times):
        for _ in range(times):
            calls[0].forward()
            calls[0].backward()
            calls[1].forward()
            calls[1].backward(True)

    def results(calls):
        a, n = calls
        return [a.o, a.lse, *a.dx, n.h, n.y, n.dh, n.dx, n.dw]

    want, got, errors = [make(i) for i in range(4)], [make(i) for i in range(4)], []
    for calls in want:
        passes(calls, 1)
    torch.cuda.synchronize()

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                passes(got[i], 20)
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    for a, b in zip(want, got):
        for x, y in zip(results(a), results(b)):
            assert torch.equal(x, y)


@pytest.mark.parametrize("rows,cols", [(40, 200), (9, 4096), (5, 5001), (5, 5120), (3, 8192), (2, 16390),
                                       (3, 32768)])
@pytest.mark.parametrize("start", [0, 1])
@pytest.mark.parametrize("over", ["bf16", "f32"])
def test_norm_in_place(P, rows, cols, start, over):
    """h as the residual, y as x; dh as dh_in, dx as dy, dw as dw_in."""
    args = (rows, cols, "bf16", over, "int8", 0.2, 8, start)
    a, b = Norm(P, *args), Norm(P, *args)
    a.forward()
    a.backward(False)
    b.forward(h=b.res, y=b.x)
    assert torch.equal(b.res, a.h) and torch.equal(b.x, a.y)
    b.h.copy_(a.h)
    s = torch.cuda.current_stream().cuda_stream
    P.poseidon_norm_backward(b.n, b.h.data_ptr(), b.h.stride(0), 0, b.rstd.data_ptr(),
                             b.dy.data_ptr(), b.dy.stride(0), b.dh_in.data_ptr(), b.dh_in.stride(0),
                             b.dh_in.data_ptr(), b.dh_in.stride(0), b.dy.data_ptr(), b.dy.stride(0),
                             b.dw_in.data_ptr(), b.dw_in.data_ptr(), s)
    assert torch.equal(b.dh_in, a.dh) and torch.equal(b.dy, a.dx) and torch.equal(b.dw_in, a.dw)
