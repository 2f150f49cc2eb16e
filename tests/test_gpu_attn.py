"""poseidon_attn_forward and poseidon_attn_backward against their formulas in 64 bits, and
the gradients against differences of the forward formula."""
import math

import pytest

import layer_util as U

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32 = U.ROUND["f32"]
CUT = 2 * F32  # the tensor cores cut what they add to a sum
# 2^x below 2^-126 may be 0, as may 16-bit values below it: off by as much, so a product
# with the gradient d by 2^-126 (1 + |d|)
FLUSH = 2.0 ** -126


@pytest.fixture(scope="module")
def P():
    import paper_2609_06086_gb300 as P
    return P


def stream():
    return torch.cuda.current_stream().cuda_stream


def heads_of(t):
    return (t.data_ptr(), t.stride(0), t.stride(1))


class Call:
    """Inputs, outputs and both passes of one call.  lengths: of the sequences; before,
    behind: tokens that belong to none, whose inputs are NaN; None: one sequence without
    starts.  layout: "fused" (one tensor holds queries, keys and values), "apart", or "odd"
    (an odd start and odd strides, which are copied)."""

    def __init__(self, P, lengths, hq, hk, dim, dtype, layout="fused", before=0, behind=0, seed=0,
                 starts=True, spread=1.0, grad=1.0, scale=None):
        g = torch.Generator(device="cuda").manual_seed(1000 * seed + 7 * dim + hq)
        self.P, self.hq, self.hk, self.dim, self.dtype = P, hq, hk, dim, dtype
        self.T = T = before + sum(lengths) + behind
        self.dt = U.DTYPES[dtype]
        at = [before]
        for n in lengths:
            at.append(at[-1] + n)
        self.at = at
        self.live = torch.zeros(T, dtype=torch.bool, device="cuda")
        self.live[at[0]:at[-1]] = True
        self.starts = torch.tensor(at, dtype=torch.int32, device="cuda") if starts else None
        self.scale = scale or 1 / math.sqrt(dim)

        def values(n, size):
            x = torch.randn(T, n, dim, device="cuda", generator=g) * size
            x[~self.live] = float("nan")
            return x.to(self.dt)

        def placed(x, pad):
            """x in a buffer at an odd element with odd strides"""
            n = x.shape[1]
            buf = torch.full((3 + T * (n * (dim + pad) + 1),), float("nan"), dtype=self.dt,
                             device="cuda")
            y = buf.as_strided(x.shape, (n * (dim + pad) + 1, dim + pad, 1), 3)
            return y.copy_(x)

        q, k, v = values(hq, 1.5 * spread), values(hk, 1.2 * spread), values(hk, 1.0)
        if layout == "fused":
            x = torch.cat((q, k, v), 1)
            q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
        elif layout == "odd":
            q, k, v = placed(q, 1), placed(k, 3), placed(v, 0)
        self.x = [q, k, v]
        self.g = values(hq, grad)
        if layout == "odd":
            self.g = placed(self.g, 1)
        new = lambda n: torch.full((T, n, dim), 77.0, dtype=self.dt, device="cuda")  # noqa: E731
        self.o, self.dx = new(hq), [new(hq), new(hk), new(hk)]
        if layout == "odd":
            self.o, self.dx = placed(self.o, 2), [placed(t, 1) for t in self.dx]
        self.lse = torch.full((hq, T), 77.0, device="cuda")
        self.a = P.pos_attn(T, hq, hk, dim, U.CODES[dtype], self.scale,
                            len(lengths) if starts else 0,
                            self.starts.data_ptr() if starts else 0)

    def triple(self, ts):
        return self.P.attn_heads(*(v for t in ts for v in heads_of(t)))

    def forward(self, lse=True):
        self.P.poseidon_attn_forward(self.a, self.triple(self.x), self.P.pos_heads(*heads_of(self.o)),
                                     lse=self.lse.data_ptr() if lse else 0, stream=stream())

    def backward(self):
        self.P.poseidon_attn_backward(self.a, self.triple(self.x),
                                      self.P.pos_heads(*heads_of(self.o)), self.lse.data_ptr(),
                                      self.P.pos_heads(*heads_of(self.g)), self.triple(self.dx),
                                      stream=stream())

    def sequences(self):
        """(tokens, query head, key head, Q, K, V, scores, what a score's 32 bits may be off)"""
        q, k, v = (t.double() for t in self.x)
        for a, b in zip(self.at, self.at[1:]):
            if a == b:
                continue
            future = torch.ones(b - a, b - a, dtype=torch.bool, device="cuda").triu(1)
            for h in range(self.hq):
                j = h // (self.hq // self.hk)
                Q, K, V = q[a:b, h], k[a:b, j], v[a:b, j]
                s = (self.scale * Q @ K.t()).masked_fill(future, -math.inf)
                # dim products added up and cut, scale times log2 e rounded, the difference
                # from a reference rounded, 2^x to two units
                off = (self.dim + 2) * CUT * self.scale * (Q.abs() @ K.abs().t()).masked_fill(future, 0)
                off = off + 4 * F32 * s.abs().masked_fill(future, 0) + 8 * F32
                yield a, b, h, j, Q, K, V, s, off

    def check_forward(self, rows=None):
        """rows: of the call's tokens, a mask of those compared."""
        u, tiny = U.ROUND[self.dtype], U.TINY[self.dtype]
        for a, b, h, _, _, _, V, s, off in self.sequences():
            n = b - a
            pick = slice(None) if rows is None else rows[a:b]
            want = torch.logsumexp(s, 1)
            p = torch.exp(s - want[:, None])
            # scores' errors act on a probability and on the sum; sums of n are cut
            r = 2 * off.amax(1) + (n + 8) * CUT
            lse = self.lse[h, a:b].double()
            assert ((lse - want).abs() <= r + 4 * F32 * want.abs())[pick].all()
            o = p @ V
            tol = (u + r)[:, None] * 1.01 * (p @ V.abs()) + u * 1.01 * o.abs() + tiny
            tol = tol + FLUSH * V.abs().cumsum(0)  # (relative to a sum of at least 1)
            if self.dtype == "f16":  # small probabilities: half the smallest step
                tol = tol + tiny * (V.abs().cumsum(0))
            assert ((self.o[a:b, h].double() - o).abs() <= tol)[pick].all()

    def without_what_is_not_finite(self):
        """For comparisons of rows that do not see it: 0 in the place of every infinity and
        NaN, so that the formulas' products with 0 are 0."""
        for t in (*self.x, self.g, self.o, self.lse):
            t.copy_(torch.where(torch.isfinite(t), t, 0))

    def formulas(self):
        """(dq, dk, dv) of the given o and lse, and how far they may be off."""
        u, tiny = U.ROUND[self.dtype], U.TINY[self.dtype]
        zeros = lambda n: torch.zeros(self.T, n, self.dim, dtype=torch.float64,  # noqa: E731
                                      device="cuda")
        out = [zeros(self.hq), zeros(self.hk), zeros(self.hk)]
        tol = [zeros(self.hq), zeros(self.hk), zeros(self.hk)]
        f16 = self.dtype == "f16"
        g = self.g.double()
        # f16: half the smallest step of P times 2^12 and of dS under its factor, by which the
        # largest dO of the sequence and key head is 2^8 at least
        step_p = tiny / 4096 if f16 else 0.0
        for a, b, h, j, Q, K, V, s, off in self.sequences():
            n, G, O = b - a, g[a:b, h], self.o[a:b, h].double()
            group = self.hq // self.hk
            large = float(g[a:b, j * group:(j + 1) * group].abs().max())
            step_ds = tiny * large / 256 if f16 else 0.0
            lse = self.lse[h, a:b, None].double()
            seen = s > -math.inf
            p = torch.exp(s - lse)
            off = off + 4 * F32 * (s.masked_fill(~seen, 0).abs() + lse.abs())
            dp = G @ V.t()
            # D, the sum over a row of p dp, as a guess, do o, and the sum e of p (dp - guess):
            # the same but for guess * (1 - sum p), and p is of an lse of 32 bits here, so that
            # its sum is 1 only up to lse's rounding
            guess = (G * O).sum(1, keepdim=True)
            D = guess + (p * (dp - guess)).sum(1, keepdim=True)
            dp_off = (self.dim + 2) * CUT * (G.abs() @ V.abs().t())
            terms = (p * (dp - guess)).abs()
            D_off = (p * dp_off + 1.01 * off * terms + (n + 64) * F32 * terms).sum(1, keepdim=True) + \
                2 * F32 * D.abs()
            ds, first = p * (dp - D), p * (dp - guess)
            ds[0] = first[0] = 0  # sees itself only
            e = D - guess
            e[0] = 0
            rest = p * 1.01 * (dp_off + D_off) + (step_ds + FLUSH * (1 + (dp - D).abs())) * seen
            # one rounding; of one tile, what a second value of 16 bits leaves
            inner = u if n > 128 else u * u
            ds_off = (inner + 1.01 * off + 4 * F32) * ds.abs() + rest
            p_off = (inner + 1.01 * off) * p + (step_p + FLUSH) * seen
            # dq = (p (dp - guess)) k - e p k
            q_off = (inner + 1.01 * off + 4 * F32) * first.abs() + rest + e.abs() * p_off + \
                (n + 2) * CUT * (first.abs() + e.abs() * p)
            out[0][a:b, h] = self.scale * ds @ K
            tol[0][a:b, h] = self.scale * q_off @ K.abs()
            n = n * (self.hq // self.hk)
            out[1][a:b, j] += self.scale * ds.t() @ Q
            tol[1][a:b, j] += self.scale * (ds_off + (n + 2) * CUT * ds.abs()).t() @ Q.abs()
            out[2][a:b, j] += p.t() @ G
            tol[2][a:b, j] += (p_off + (n + 2) * CUT * p).t() @ G.abs()
        return out, [1.01 * (t + (u + 2 * F32) * v.abs()) + tiny for t, v in zip(tol, out)]

    def check_backward(self, rows=(None, None, None)):
        out, tol = self.formulas()
        for got, want, t, pick in zip(self.dx, out, tol, rows):
            pick = self.live if pick is None else self.live & pick
            assert ((got.double() - want).abs() <= t)[pick].all()

    def check_untouched(self):
        for t in (self.o, *self.dx):
            assert (t[~self.live] == 77).all()
        assert (self.lse[:, ~self.live] == 77).all()

    def check(self):
        self.forward()
        self.check_forward()
        self.backward()
        self.check_backward()
        self.check_untouched()


LENGTHS = [[1], [2], [63], [127], [128], [129], [255], [256], [257], [385], [1, 1, 1],
           [0, 5, 0, 130, 1], [300, 64, 513], [700], []]


@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
@pytest.mark.parametrize("hq,hk,dim,dtype", [(4, 2, 128, "bf16"), (2, 2, 64, "f16"),
                                             (5, 1, 80, "bf16")])
def test_lengths(P, lengths, hq, hk, dim, dtype):
    Call(P, lengths, hq, hk, dim, dtype, before=3, behind=5).check()


@pytest.mark.parametrize("dim", [1, 7, 8, 16, 40, 50, 56, 64, 72, 96, 100, 120, 128])
@pytest.mark.parametrize("dtype,layout", [("bf16", "fused"), ("f16", "apart"), ("bf16", "odd"),
                                          ("f16", "odd")])
def test_dims_and_layouts(P, dim, dtype, layout):
    Call(P, [140, 33, 200], 6, 2, dim, dtype, layout, before=1, behind=2).check()


@pytest.mark.parametrize("hq,hk", [(1, 1), (3, 3), (8, 1), (9, 3), (64, 8)])
def test_heads(P, hq, hk):
    Call(P, [150], hq, hk, 64, "bf16").check()


@pytest.mark.parametrize("tokens", [1, 128, 256, 300, 1030])
def test_one_sequence_without_starts(P, tokens):
    Call(P, [tokens], 4, 1, 128, "bf16", starts=False).check()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("spread,grad", [(0.01, 1e-3), (3.0, 1.0), (1.0, 30.0), (8.0, 1e-4)])
def test_distributions(P, dtype, spread, grad):
    """Flat and sharp probabilities, whose largest score moves by far more than 2^8 from
    tile to tile, and small and large gradients."""
    Call(P, [600], 2, 1, 128, dtype, spread=spread, grad=grad).check()


def test_gradients_of_sequences_far_apart_in_size(P):
    """Of the second sequence, and of the first's second key head, dO is 1e-7 of the first
    one's in f16: their own dS keep their bits.  Alone or beside the others, the same
    results."""
    c = Call(P, [200, 150, 40], 4, 2, 64, "f16", grad=3000.0, starts=True)
    c.g[200:350] *= 1e-7
    c.g[:200, 2:] *= 1e-7
    c.check()
    alone = Call(P, [200, 150, 40], 4, 2, 64, "f16")
    for a, b in zip((*alone.x, alone.g), (*c.x, c.g)):
        a.copy_(b)
    alone.g[:200] = 0
    alone.g[350:] = 0
    alone.forward()
    alone.backward()
    for a, b in zip(alone.dx, c.dx):
        assert torch.equal(a[200:350], b[200:350])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("what", ["nan", "inf"])
def test_other_sequences_are_not_read(P, dtype, what):
    """Sequences of values that are not finite on both sides of one, within its tiles: its
    rows are as the formulas have them, and the others' are written and not finite."""
    c = Call(P, [150, 200, 90], 4, 2, 64, dtype)
    around = torch.ones(440, dtype=torch.bool, device="cuda")
    around[150:350] = False
    for t in (*c.x, c.g):
        t[around] = float(what)
    c.forward()
    c.backward()
    for t in (c.o, *c.dx):
        assert not torch.isfinite(t[around].double()).any()
    c.without_what_is_not_finite()
    c.check_forward(~around)
    c.check_backward((~around,) * 3)


def test_heads_outermost(P):
    """Tensors [heads][tokens][dim], inputs and results."""
    c = Call(P, [130, 60], 4, 2, 80, "bf16", "apart", behind=2)
    outer = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    c.x, c.g, c.o, c.dx = [outer(t) for t in c.x], outer(c.g), outer(c.o), [outer(t) for t in c.dx]
    c.check()


def test_more_sequences_than_tokens(P):
    """Most of them empty."""
    for dtype in ("bf16", "f16"):
        lengths = [0] * 700
        for i in (3, 4, 299, 699):
            lengths[i] = 70 + i % 7
        Call(P, lengths, 2, 1, 64, dtype, behind=1).check()


def test_a_scale_of_its_own(P):
    Call(P, [200], 2, 2, 64, "bf16", scale=0.37).check()


def test_a_stride_of_zero(P):
    """Keys and values that all heads share, and queries that all tokens share."""
    c = Call(P, [200], 4, 4, 64, "bf16", "apart")
    c.x = [c.x[0][:1].expand(200, 4, 64), c.x[1][:, :1].expand(200, 4, 64),
           c.x[2][:, :1].expand(200, 4, 64)]
    c.check()


def test_many_sequences(P):
    """More sequences than a warp or a block holds at once, most of them short."""
    lengths = [(i * 37) % 23 if i % 50 else 400 for i in range(1500)]
    Call(P, lengths, 2, 1, 64, "bf16", behind=9).check()


def test_starts_in_disorder(P):
    """A start below one before it counts as that one, one outside as the nearest inside."""
    c = Call(P, [60, 0, 100, 40], 2, 1, 64, "bf16")
    c.starts.copy_(torch.tensor([-7, 60, 20, 160, 10 ** 6], dtype=torch.int32))
    c.check()


def test_no_sequences_write_nothing(P):
    c = Call(P, [], 2, 1, 64, "bf16", behind=300)
    c.forward()
    c.backward()
    c.check_untouched()


def test_without_lse(P):
    c = Call(P, [300], 4, 2, 128, "bf16")
    c.forward(lse=False)
    o = c.o.clone()
    assert (c.lse == 77).all()
    c.forward()
    assert torch.equal(c.o, o)


@pytest.mark.parametrize("what", ["nan", "inf"])
@pytest.mark.parametrize("which", [0, 1, 2])
def test_later_tokens_do_not_reach_earlier_ones(P, which, what):
    """A NaN or an infinity in the queries, keys or values of a token: forward, its own
    row (queries) or it and what is behind it are lost, the rows before are as the formula
    has them; backward likewise, so far as the formula keeps them apart."""
    n, t = 300, 140
    c = Call(P, [n], 2, 1, 64, "bf16")
    c.x[which][t, :, 5] = float(what)
    c.forward()
    c.backward()
    assert not torch.isfinite(c.o[t].double()).all()
    if which and what == "nan":
        assert c.o[t:].isnan().any(2).all()
    at = torch.arange(n, device="cuda")
    c.without_what_is_not_finite()
    c.check_forward(at != t if which == 0 else at < t)
    # a key's gradients are sums over the queries behind it, which see the token in t
    rest = at > t if which == 0 else at < 0
    c.check_backward((at != t if which == 0 else at < t, rest, rest))


def test_a_gradient_that_is_not_finite(P):
    """dO of a token reaches its dq, and dk and dv of the tokens that it sees."""
    n, t = 300, 140
    c = Call(P, [n], 2, 1, 64, "bf16")
    c.g[t, :, 3] = float("inf")
    c.forward()
    c.backward()
    at = torch.arange(n, device="cuda")
    assert not torch.isfinite(c.dx[2][:t + 1].double()).all(2).any()
    c.without_what_is_not_finite()
    c.check_backward((at != t, at > t, at > t))


def test_gradients_too_large_for_f16(P):
    """dS beyond f16's range under its factor: the rows are done again in 32 bits."""
    c = Call(P, [200], 2, 1, 64, "f16", grad=1.0)
    c.x[2] *= 400  # values
    c.forward()
    c.check_forward()
    c.backward()
    out, tol = c.formulas()
    for got, want, t in zip(c.dx, out, tol):
        fits = want.abs() < 60000
        assert ((got.double() - want).abs() <= t)[fits].all() and fits.float().mean() > 0.9


def test_gradients_against_differences(P):
    """Along random directions: what the gradients promise of sum(o * g) against central
    differences of the formula in 64 bits.  Their own error is of the third derivative's
    order, 1e-6 of the terms here; the gradients' tolerances are those above."""
    for dtype in ("bf16", "f16"):
        c = Call(P, [90, 45], 4, 2, 64, dtype)
        c.forward()
        c.backward()
        _, tol = c.formulas()
        base, g = [t.double() for t in c.x], c.g.double()

        def loss(x):
            total = 0.0
            for a, b in zip(c.at, c.at[1:]):
                future = torch.ones(b - a, b - a, dtype=torch.bool, device="cuda").triu(1)
                q, k, v = (t[a:b].transpose(0, 1) for t in x)
                k, v = k.repeat_interleave(2, 0), v.repeat_interleave(2, 0)
                s = (c.scale * q @ k.mT).masked_fill(future, -math.inf)
                total += float((torch.softmax(s, -1) @ v * g[a:b].transpose(0, 1)).sum())
            return total

        gen = torch.Generator(device="cuda").manual_seed(3)
        for i in range(3):
            d = torch.randn(base[i].shape, device="cuda", generator=gen, dtype=torch.float64)
            h = 1e-4
            up, down = list(base), list(base)
            up[i], down[i] = base[i] + h * d, base[i] - h * d
            want = (loss(up) - loss(down)) / (2 * h)
            got = float((c.dx[i].double() * d).sum())
            assert abs(got - want) <= float((tol[i] * d.abs()).sum()) + \
                1e-6 * float((c.dx[i].double() * d).abs().sum())


def test_the_roundings_of_o_have_no_effect(P):
    """Short rows, where do o differs from the sum of p dp by o's rounding, and that is
    more than anything else: dq and dk are as near as their own roundings allow, two of
    16 bits each (2^-9 of a value, less than half of it on average) and what cancels."""
    for lengths in ([2], [3, 2, 2], [5], [2] * 40):
        c = Call(P, lengths, 8, 4, 64, "bf16", seed=5)
        c.forward()
        c.backward()
        out, _ = c.formulas()
        for got, want in zip(c.dx, out):
            assert float((got.double() - want).norm() / want.norm()) < 1.5 * 2.0 ** -9


def test_same_bits_again_on_streams_and_captured(P):
    make = lambda: Call(P, [700, 1, 290], 8, 2, 128, "bf16", behind=3)  # noqa: E731
    c = make()
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    want = [t.clone() for t in (c.o, c.lse, *c.dx)]
    others = [make(), make()]
    streams = [torch.cuda.Stream() for _ in others]
    torch.cuda.synchronize()
    for _ in range(3):
        for o, s in zip(others, streams):
            with torch.cuda.stream(s):
                o.forward()
                o.backward()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward()
        c.backward()
    for t in (c.o, c.lse, *c.dx):
        t.fill_(77)
    graph.replay()
    graph.replay()
    for o in (*others, c):
        for t, v in zip((o.o, o.lse, *o.dx), want):
            assert torch.equal(t, v)


def test_captured_with_other_lengths(P):
    """The lengths are read when the kernels run: a captured call serves others of the same
    total and number."""
    c = Call(P, [200, 100, 84], 4, 2, 64, "f16")
    c.forward()
    c.backward()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward()
        c.backward()
    c.at = [0, 10, 11, 384]
    c.starts.copy_(torch.tensor(c.at, dtype=torch.int32))
    graph.replay()
    c.check_forward()
    c.check_backward()


def test_offsets_past_32_bits(P):
    """Elements and bytes past 2^31 and 2^32 in every tensor."""
    lengths, hq, hk, dim = [40] * 700 + [129], 640, 640, 128
    T = sum(lengths)
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("needs 100 GB")
    assert T * hq * dim > 2 ** 31
    c = Call(P, lengths, hq, hk, dim, "bf16", "apart")
    c.forward()
    c.backward()
    # the same tokens and heads alone
    for h in (0, 300, hq - 1):
        for n in (0, 350, 700):
            a, b = c.at[n], c.at[n + 1]
            d = Call(P, [b - a], 1, 1, dim, "bf16", "apart")
            d.x = [t[a:b, h:h + 1].contiguous() for t in c.x]
            d.g = c.g[a:b, h:h + 1].contiguous()
            d.forward()
            d.backward()
            for got, want in zip((c.o, *c.dx), (d.o, *d.dx)):
                assert torch.equal(got[a:b, h:h + 1], want)
            assert torch.equal(c.lse[h:h + 1, a:b], d.lse)


def test_norm_rotation_and_attention(P):
    """As a layer uses them: queries, keys and values in one projection's output, the norm and
    rotation in place, attention, and both backward passes; against 64-bit autograd."""
    T, hq, hk, dim, eps = 260, 4, 2, 64, 1e-6
    gen = torch.Generator(device="cuda").manual_seed(11)
    x = torch.randn(T, hq + 2 * hk, dim, device="cuda", generator=gen).bfloat16()
    w = 1 + 0.1 * torch.randn(2, dim, device="cuda", generator=gen)
    ang = torch.arange(T, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (
        -torch.arange(dim // 2, device="cuda", dtype=torch.float64) / (dim // 2))
    cos, sin = ang.cos().float(), ang.sin().float()
    starts = torch.tensor([0, 100, T], dtype=torch.int32, device="cuda")
    g = torch.randn(T, hq, dim, device="cuda", generator=gen).bfloat16()
    qk = P.pos_qk(T, hq, hk, dim, dim, 0, 0, 0, eps, w[0].data_ptr(), w[1].data_ptr(),
                  cos.data_ptr(), sin.data_ptr(), T, 0)
    a = P.pos_attn(T, hq, hk, dim, 0, dim ** -0.5, 2, starts.data_ptr())

    def parts(t):
        return t[:, :hq], t[:, hq:hq + hk], t[:, hq + hk:]

    def pair(t):
        q, k, _ = parts(t)
        return P.qk_heads(*heads_of(q), *heads_of(k))

    y, dy, dx = x.clone(), torch.empty_like(x), torch.empty_like(x)
    rstd = [torch.empty(T, n, device="cuda") for n in (hq, hk)]
    o, lse = torch.empty_like(g), torch.empty(hq, T, device="cuda")
    at = tuple(r.data_ptr() for r in rstd)
    P.poseidon_qk_forward(qk, pair(x), pair(y), rstd=at, stream=stream())
    triple = P.attn_heads(*(v for t in parts(y) for v in heads_of(t)))
    one = P.pos_heads(*heads_of(o))
    P.poseidon_attn_forward(a, triple, one, lse=lse.data_ptr(), stream=stream())
    P.poseidon_attn_backward(a, triple, one, lse.data_ptr(), P.pos_heads(*heads_of(g)),
                             P.attn_heads(*(v for t in parts(dy) for v in heads_of(t))),
                             stream=stream())
    P.poseidon_qk_backward(qk, pair(dy), pair(dx), at, x=pair(x), stream=stream())

    X = x.double().requires_grad_()
    q, k, v = parts(X)
    turned = []
    for i, t in enumerate((q, k)):
        t = t / torch.sqrt(t.square().mean(-1, keepdim=True) + eps) * w[i].double()
        c, s = ang.cos()[:, None], ang.sin()[:, None]
        b, e = t[..., :dim // 2], t[..., dim // 2:]
        turned.append(torch.cat((b * c - e * s, e * c + b * s), -1))
    q, k, v = (t.transpose(0, 1) for t in (*turned, v))
    k, v = k.repeat_interleave(hq // hk, 0), v.repeat_interleave(hq // hk, 0)
    tok = torch.arange(T, device="cuda")
    seen = (tok[:, None] >= tok) & ((tok[:, None] < 100) == (tok < 100))
    s = (q @ k.mT * dim ** -0.5).masked_fill(~seen, -math.inf)
    O = (torch.softmax(s, -1) @ v).transpose(0, 1)
    (O * g.double()).sum().backward()
    got = torch.cat((parts(dx)[0], parts(dx)[1], parts(dy)[2]), 1).double()
    # six roundings to bf16 on the way, of 2^-9 of a value each on average at worst, the
    # gradients' sums twice their size or less
    far = lambda p, q: float((p - q).norm() / q.norm())  # noqa: E731
    assert far(o.double(), O.detach()) < 4 * 2.0 ** -9
    assert far(got, X.grad) < 12 * 2.0 ** -9
