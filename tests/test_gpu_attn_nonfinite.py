"""Attention of inputs that are not finite, or too large for 16 bits on the way: rows that do
not see them are as the formulas have them, whatever the tensor cores made of them first."""
import pytest

from test_gpu_attn import Call

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def P():
    import paper_2609_06086_gb300 as P
    return P


def test_rows_beside_a_nan(P):
    """Values of one token in a tile are NaN: the rows before it in that tile, which the product
    of the tile multiplies by 0, are as they are, the same every time."""
    n, t = 250, 230
    at = torch.arange(n, device="cuda")
    c = Call(P, [n], 64, 8, 128, "bf16", starts=False)
    c.x[2][t] = float("nan")
    want = None
    for _ in range(20):
        c.o.fill_(77)
        c.forward()
        if want is None:
            want = c.o.clone()
        assert torch.isfinite(c.o[:t].double()).all() and c.o[t:].isnan().all()
        assert torch.equal(c.o[:t], want[:t])
    c.without_what_is_not_finite()
    c.check_forward(at < t)


def passes(c):
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    return [t.clone() for t in (c.o, c.lse, *c.dx)]


def seconds(c):
    """The fastest of three calls of both passes, on the device."""
    best = 1e9
    for _ in range(3):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        torch.cuda.synchronize()
        a.record()
        c.forward()
        c.backward()
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b) / 1e3)
    return best


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("what", ["dO late", "dO all", "v first", "v late", "k late", "q late", "all"])
def test_the_time_of_what_is_not_finite(P, dtype, what):
    """A tile of the diagonal that holds something is looked over column by column, some ten
    microseconds each, beside the products: no call takes twice its time."""
    n = 4096
    c = Call(P, [n], 32, 8, 128, dtype, starts=False)
    passes(c)
    clean = seconds(c)
    for name, t in (("q", c.x[0]), ("k", c.x[1]), ("v", c.x[2]), ("dO", c.g)):
        if what == "all" or what == name + " all":
            t.fill_(float("nan"))
        elif what == name + " late":
            t[n - 10, 0] = float("inf")
        elif what == name + " first":
            t[0] = float("nan")
    assert seconds(c) < 2 * clean


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 100])
@pytest.mark.parametrize("lengths", [[40], [128], [300], [129, 5, 700], [1500], [30] * 20 + [257]], ids=str)
def test_rows_that_do_not_see_it(P, dtype, dim, lengths):
    """Infinities and NaNs in the queries, keys, values and gradients of some tokens of every
    sequence: rows and keys that do not see them are as the formulas have them with 0 in their
    place.  Many units a block, and keys' tiles that several blocks share."""
    hq, hk = 8, 2
    for which in range(4):  # of queries, keys, values, gradients
        c = Call(P, lengths, hq, hk, dim, dtype, behind=2, seed=which)
        t = (*c.x, c.g)[which]
        gen = torch.Generator().manual_seed(which)
        at = torch.arange(c.T, device="cuda")
        # per sequence: one token, one of the heads that hold it
        first = torch.full((c.T, t.shape[1]), c.T, device="cuda")  # of the row's sequence and head
        for a, b in zip(c.at, c.at[1:]):
            if b - a < 2:
                continue
            i = a + int(torch.randint(1, b - a, (1,), generator=gen))
            h = int(torch.randint(t.shape[1], (1,), generator=gen))
            t[i, h, int(torch.randint(dim, (1,), generator=gen))] = (float("nan"), float("inf"))[i % 2]
            first[a:b, h] = i
        got = passes(c)
        for x in got:  # nothing left as it was
            assert not (x[c.live] == 77).any() if x.shape[0] == c.T else not (x[:, c.live] == 77).any()
        c.check_untouched()
        c.without_what_is_not_finite()
        out, tol = c.formulas()
        group = hq // hk
        q_first = first if which in (0, 3) else first.repeat_interleave(group, 1)
        k_first = first if which in (1, 2) else None
        before = at[:, None] < q_first  # rows of queries that do not see it
        if which in (0, 3):
            same = at[:, None] != first
            rows = same
            # keys behind it, or of heads without it
            hit = torch.where(first < c.T, first, -1).view(c.T, hk, group).amax(2)
            keys = at[:, None] > hit
        else:
            rows = before
            hit = k_first < c.T
            keys = ~hit  # a key's gradients are sums over rows that see the token
        live = c.live[:, None]
        if which == 3:
            rows_o = live.expand(c.T, hq)
        else:
            rows_o = rows & live
        assert torch.isfinite(got[0][rows_o].double()).all()
        for g, want, tl, pick in zip(got[2:], out, tol, (rows, keys, keys)):
            pick = pick & live
            assert ((g.double() - want).abs() <= tl)[pick].all(), which
        c.check_forward((rows_o | ~live).all(1))


def test_values_next_to_the_largest(P):
    """Sums of exponentials times values near bf16's largest pass it, their quotients do not."""
    c = Call(P, [200], 2, 1, 64, "bf16")
    c.x[2] *= 2e37
    c.forward()
    c.check_forward()
    assert float(c.o.abs().max()) > 1e37


@pytest.mark.parametrize("lengths,hq,hk", [([200], 2, 1), ([1000], 8, 1), ([90] * 40, 4, 4)])
def test_large_values_in_f16(P, lengths, hq, hk):
    """dS beyond f16's range under a factor that dO alone would give, in some sequences and
    heads only: results as the formulas have them."""
    c = Call(P, lengths, hq, hk, 64, "f16")
    c.x[2][:c.at[1] // 2, 0] *= 300
    c.forward()
    c.check_forward()
    c.backward()
    out, tol = c.formulas()
    for got, want, t in zip(c.dx, out, tol):
        fits = want.abs() < 60000
        assert ((got.double() - want).abs() <= t)[fits].all() and fits.float().mean() > 0.9


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("t", [1, 60, 127, 128, 255, 256, 299])
def test_a_key_of_no_weight(P, dtype, t):
    """An infinite element of a key whose scores are all minus infinity: it has no weight, and
    outputs and gradients are those of the others, but for the column of dq, where the formula
    multiplies the infinity by 0.  (Token t may be the first that a tile's rows see.)"""
    n = 300
    at = torch.arange(n, device="cuda")
    c, want = Call(P, [n], 4, 2, 64, dtype, "apart"), Call(P, [n], 4, 2, 64, dtype, "apart")
    for x in (c, want):
        x.x[0][:, :, 5] = -x.x[0][:, :, 5].abs() - 0.1
    c.x[1][t, :, 5] = float("inf")
    # as a key that is finite but far away: its weight is 0 in 32 bits
    want.x[1][t, :, 5] = 60000.0 if dtype == "f16" else 1e6
    for x in (c, want):
        x.forward()
        x.backward()
    assert torch.equal(c.o, want.o) and torch.equal(c.lse, want.lse)
    assert not torch.isfinite(c.dx[0][t:, :, 5].double()).any()
    rest = torch.ones(64, dtype=torch.bool, device="cuda")
    rest[5] = False
    # (the other columns' products are the same; sums with 0 in t's place)
    assert torch.equal(c.dx[0][:, :, rest], want.dx[0][:, :, rest])
    assert torch.equal(c.dx[0][:t], want.dx[0][:t])
    # (its own key's gradients may be NaN: behind the sequence its scores are 0 times infinity)
    for x, y in zip(c.dx[1:], want.dx[1:]):
        assert torch.equal(x[at != t], y[at != t])
