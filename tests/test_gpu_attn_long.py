"""Attention of long rows: what thousands of small probabilities add up to."""
import math

import pytest

import layer_util as U
from test_gpu_attn import F32, Call

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2609_06086_gb300 as P
    return P


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("bits", [8.3, 17.4, 24.6, 25.4, 27.0])
@pytest.mark.parametrize("n", [3000, 30000])
def test_one_large_score_and_many_small_ones(P, dtype, bits, n):
    """One key, near the end, has 2^bits times the weight of every other and a value of 0, the
    others' values are 1: a row behind it is the share of the others.  Their probabilities are
    rounded to dtype (all the same way) as they are relative to the row's reference, in f16
    with 2^7 of it, so that half of the smallest step is 2^-32 of the large one."""
    t = n - 50
    c = Call(P, [n], 2, 1, 64, dtype, starts=False, scale=1.0)
    q, k, v = c.x
    q.zero_(), k.zero_(), v.fill_(1.0)
    q[:, :, 3] = 1
    k[t, :, 3] = bits * math.log(2)
    v[t] = 0
    c.forward()
    u = U.ROUND[dtype]
    weight = math.exp(-float(k[t, 0, 3]))
    others = torch.arange(n, device="cuda", dtype=torch.float64)  # seen beside t, for rows from t on
    total = torch.where(others < t, others + 1, 1 + others * weight)
    share = torch.where(others < t, 1.0, others * weight / total)
    lse = torch.log(total) + torch.where(others < t, 0.0, float(k[t, 0, 3]))
    step = 2.0 ** -32 if dtype == "f16" else 0.0
    # P and o rounded; a sum of n that the tensor cores cut (2^-23 an addition of 16)
    tol = (2 * u + (n / 16 + 70) * 2 * F32) * 1.01 * share + step * others + U.TINY[dtype]
    assert ((c.o.double() - share[:, None, None]).abs() <= tol[:, None, None]).all()
    assert ((c.lse.double() - lse).abs() <= (n + 70) * 2 * F32 + 4 * F32 * lse.abs()).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("longer", [129, 256, 700])
def test_gradients_of_first_queries_do_not_depend_on_the_length(P, dtype, longer):
    """A query sees no later token: the first 128 queries' outputs and gradients have the same
    bits in a sequence of 128 tokens as in a longer one that begins with them."""
    short, c = Call(P, [128], 4, 2, 64, dtype), Call(P, [longer], 4, 2, 64, dtype)
    for a, b in zip((*short.x, short.g), (*c.x, c.g)):
        a.copy_(b[:128])
    for x in (short, c):
        x.forward()
        x.backward()
    assert torch.equal(short.o, c.o[:128]) and torch.equal(short.lse, c.lse[:, :128])
    assert torch.equal(short.dx[0], c.dx[0][:128])


def test_short_rows_of_a_longer_sequence(P):
    """dq of the first queries of a longer sequence is as near to the formula as its own
    rounding allows: 2^-9 of a value at most, less than half of that on average, and what
    cancels."""
    for n in (2, 128, 129, 500):
        c = Call(P, [n], 8, 4, 64, "bf16", seed=5)
        c.forward()
        c.backward()
        want = c.formulas()[0][0][:100]
        assert float((c.dx[0][:100].double() - want).norm() / want.norm()) < 1.5 * 2.0 ** -9


@pytest.mark.parametrize("dtype,q,k,scale", [("f16", 3e4, 2.0 ** 16, 0.125), ("f16", 6e4, 2.0 ** 16, 1.0),
                                             ("bf16", 1e5, 2.0 ** 17, 0.125),
                                             ("bf16", 1e15, 2.0 ** 50, 0.125),
                                             ("bf16", 1e18, 2.0 ** 60, 0.7)])
def test_scores_far_past_the_steps_of_32_bits(P, dtype, q, k, scale):
    """One element of queries and keys, 300 different keys: a row is the value of the largest
    key that it sees, the others' weights being less than e^-1000."""
    n = 300
    c = Call(P, [n], 2, 1, 64, dtype, "apart", scale=scale)
    for x in c.x[:2]:
        x.zero_()
    gen = torch.Generator().manual_seed(7)
    steps = torch.randperm(3 * 128, generator=gen)[:n].cuda()
    sign = torch.where(torch.randperm(n, generator=gen).cuda() % 2 == 0, 1.0, -1.0)
    values = 2.0 ** (-(steps // 128).double()) * (1 + (steps % 128).double() / 128) / 2 * k * sign
    c.x[0][:, :, 5] = q
    c.x[1][:, 0, 5] = values.to(c.dt)
    key = c.x[1][:, 0, 5].double()
    assert len(key.unique()) == n
    c.forward()
    top, at = key.cummax(0)
    want = c.x[2][at, 0]
    # The one weight is 2^d, |d| up to half a step of its score, rounded to 16 bits for the product
    # (half of eps) and not in the sum (64 + 2 roundings in 32 bits); their ratio's product with the
    # value is rounded once more (half of eps).
    eps = torch.finfo(c.dt).eps
    want = want[:, None].double()
    bound = (eps + eps * eps / 4 + 100 * 2.0 ** -24) * want.abs()
    assert ((c.o.double() - want).abs() <= bound).all()
    lse = top * float(c.x[0][0, 0, 5]) * scale
    assert ((c.lse.double() - lse).abs() <= 8 * F32 * lse.abs()).all()
