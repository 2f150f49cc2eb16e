"""What attention's calls take from the library's pools, and what stays taken."""
import pytest

from test_gpu_attn import Call

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2609_06086_gb300 as P
    return P


def test_large_scratch_is_given_back(P):
    """Tensors off the alignment, which are copied: 0.5 GB forward and 0.9 GB back, of which at
    most 320 MB may be kept (and 32 MB that the driver rounds up); the results are those of
    aligned tensors."""
    args = ([1000] * 64, 32, 2, 100, "bf16")
    c, want = Call(P, *args, "odd"), Call(P, *args, "apart")
    for x, y in zip((*c.x, c.g), (*want.x, want.g)):
        x.copy_(y)
    want.forward()
    want.backward()
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    for _ in range(3):
        c.forward()
        c.backward()
    torch.cuda.synchronize()
    torch.cuda.synchronize()
    assert before - torch.cuda.mem_get_info()[0] <= (320 + 32) << 20
    for x, y in zip((c.o, c.lse, *c.dx), (want.o, want.lse, *want.dx)):
        assert torch.equal(x, y)


def test_large_scratch_in_a_captured_call(P):
    """The same captured and replayed, beside a call of its own."""
    args = ([1000] * 64, 32, 2, 100, "bf16", "odd")
    c, want = Call(P, *args), Call(P, *args)
    want.forward()
    want.backward()
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward()
        c.backward()
    for t in (c.o, c.lse, *c.dx):
        t.fill_(77)
    graph.replay()
    want.forward()
    graph.replay()
    torch.cuda.synchronize()
    for x, y in zip((c.o, c.lse, *c.dx), (want.o, want.lse, *want.dx)):
        assert torch.equal(x, y)
