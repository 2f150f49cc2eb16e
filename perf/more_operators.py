"""The measured calls of what a layer computes between its linear operations:
the residual's addition with its norm, dropout, and attention.

Kinds of a case
  norm    h = residual + x, RMS norm of h, the result also as an 8-bit checkpoint
  step    the same in a training step, with dropout of x where p > 0: the forward
          pass keeps h (or h in 8 bits), the backward pass reads it: outputs,
          gradients of h, x and the norm's weights
  drop    y = residual + dropout(x), and the gradient of x, which is the dropout
          of y's under the same mask; the mask is never stored
  prompt  causal attention with grouped heads over packed sequences, outputs only
  attn    the same in a training step: outputs, logarithms of the softmax sums,
          gradients of queries, keys and values

h is the sum in 32 bits (one rounding), rounded to its type; the norm and the
checkpoint of h are those of h as it is written, the checkpoint of y that of y as
it is written.  A checkpoint of [rows][cols] values: one byte per value, groups of
32 columns with one scale byte e + 127; a value is code * 2^e, the code an int8
in [-127, 127] ("int8") or a float8 e4m3 ("e4m3"); e is the smallest that keeps
the group's largest magnitude within 127 or 448 (at least -110).

The dropout's mask: element (r, c) is kept where its 16 random bits are at least
t = round(p * 65536), and then scaled by 65536 / (65536 - t).  The bits are the
(c mod 8)-th half word (low half first) of the four words that Philox-4x32 of ten
rounds gives for the counter (c / 8, r, offset low, offset high) under the key
(seed low, seed high).

Attention: token i of a sequence sees its tokens 0..i; tokens behind the last
sequence are left as they were (their inputs are NaN here).

Sizes follow the repository's own workloads: widths of 4096, 5120 and 8192,
sequences of 4096, micro-batch 1 and a few, 32 or 64 query and 8 key heads of 128.
"""
import math
import random
from types import SimpleNamespace

import numpy as np
import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
CODE = {"bf16": 0, "f16": 1, "f32": 2}
FORMAT = {"int8": 0, "e4m3": 1}
TOP = {"int8": 127.0, "e4m3": 448.0}
E_HI = {"int8": 121, "e4m3": 119}
E_LO = -110
EPS = 1e-6


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _norm(name, kind, rows, cols, dtype="bf16", stream="", fmt="int8", p=0.0, pad=0, kept="h8"):
    """stream: the residual stream's type (the same as dtype's unless given)."""
    return dict(name=name, kind=kind, rows=rows, cols=cols, dtype=dtype, stream=stream or dtype,
                fmt=fmt, p=p, pad=pad, kept=kept)


def _drop(name, rows, cols, dtype="bf16", stream="", p=0.1, pad=0):
    return dict(name=name, kind="drop", rows=rows, cols=cols, dtype=dtype, stream=stream or dtype,
                p=p, pad=pad)


def _attn(name, kind, tokens, hq, hk, dim, dtype="bf16", parts=0, cut=0, behind=0, fused=True):
    """parts: sequences that the tokens are cut into, at places drawn from `cut`
    (0: one sequence of all tokens); behind: tokens behind the last of them."""
    return dict(name=name, kind=kind, tokens=tokens, hq=hq, hk=hk, dim=dim, dtype=dtype,
                parts=parts, cut=cut, behind=behind, fused=fused)


def listed():
    return [
        # a short micro-batch of a narrow layer: latency of the call
        _norm("norm_small", "norm", 128, 1024),
        # f16, odd sizes, slices of wider buffers, dropout, h kept as it is
        _norm("norm_odd", "step", 3001, 5001, dtype="f16", fmt="e4m3", p=0.1, pad=7, kept="h"),
        # a 7B-like layer's norm with dropout, micro-batch 1, sequence 4096
        _norm("norm_7b", "step", 4096, 4096, p=0.1),
        # a 70B-like layer, four sequences, residual stream in f32
        _norm("norm_70b", "step", 16384, 8192, stream="f32", fmt="e4m3"),
        # latency of two calls
        _drop("drop_small", 128, 1024),
        # odd sizes, slices of wider buffers
        _drop("drop_odd", 5003, 5001, dtype="f16", pad=7),
        # four sequences of a 70B-like layer
        _drop("drop_70b", 16384, 8192, p=0.25),
        # a short prompt of a 7B-like model: latency of the call
        _attn("prompt_short", "prompt", 100, 32, 8, 128),
        # a long prompt, one device's share of the heads
        _attn("prompt_long", "prompt", 32768, 4, 1, 128),
        # packed sequences of odd lengths, heads of 80, in f16, padding behind them
        _attn("attn_odd", "attn", 3001, 20, 4, 80, dtype="f16", parts=7, cut=1, behind=45),
        # a training step of a 7B-like layer, sequence 4096, micro-batch 1
        _attn("attn_7b", "attn", 4096, 32, 8, 128),
        # a training step of a 70B-like layer, 8192 tokens of packed sequences
        _attn("attn_70b", "attn", 8192, 64, 8, 128, parts=5, cut=2),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("norm", "step", "step", "drop", "prompt", "attn", "attn", "attn"))
    dtype = rng.choice(("bf16", "bf16", "f16", "f32"))
    stream = rng.choice((dtype, "f32"))
    pad = rng.choice((0, 0, 8, 3))
    if kind in ("norm", "step", "drop"):
        rows, cols = _log_int(rng, 1, 16384), _log_int(rng, 1, 8192)
        if kind == "drop":
            return _drop("", rows, cols, dtype, stream, rng.choice((0.05, 0.1, 0.5)), pad)
        return _norm("", kind, rows, cols, dtype, stream, rng.choice(("int8", "e4m3")),
                     0.0 if kind == "norm" else rng.choice((0.0, 0.1, 0.3)), pad,
                     rng.choice(("h8", "h")))
    dim = rng.choice((64, 64, 72, 80, 96, 128, 128, 128))
    hk = rng.choice((1, 2, 4, 8))
    hq = hk * rng.choice((1, 2, 4, 5, 8))
    tokens = _log_int(rng, 1, 8192)
    parts = rng.choice((0, 1, 3, 8, 20))
    behind = rng.randint(0, tokens // 8) if parts else 0
    return _attn("", kind, tokens, hq, hk, dim, rng.choice(("bf16", "bf16", "f16")), parts,
                 rng.randint(1, 10 ** 6), behind, rng.random() < 0.7)


def _starts(case):
    """Where the sequences start, and behind them where the last one ends; some
    may be empty, others a single token."""
    live = case["tokens"] - case["behind"]
    if not case["parts"]:
        return [0, live]
    rng = random.Random(case["cut"])
    return [0] + sorted(rng.randint(0, live) for _ in range(case["parts"] - 1)) + [live]


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _activation(gen, rows, cols):
    """f32 values as activations have them: per-column widths, a few columns
    far larger than the others."""
    x = torch.randn(rows, cols, device="cuda", generator=gen)
    width = torch.exp(0.5 * torch.randn(cols, device="cuda", generator=gen))
    loud = torch.rand(cols, device="cuda", generator=gen) < 0.005
    x *= torch.where(loud, width * 20, width)
    return x


def _strided(x, dtype, pad):
    """x as rows of a buffer that is `pad` columns wider."""
    buf = torch.empty(x.shape[0], x.shape[1] + pad, dtype=dtype, device="cuda")
    buf[:, :x.shape[1]] = x
    buf[:, x.shape[1]:] = float("nan")
    return buf[:, :x.shape[1]]


def _ckpt_bytes(rows, cols):
    groups = -(-cols // 32)
    return rows * (32 * groups + 4 * -(-groups // 4))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s = SimpleNamespace(case=dict(case))
    c, dt = case, DTYPE[case["dtype"]]
    if c["kind"] in ("prompt", "attn"):
        T, hq, hk, dim = c["tokens"], c["hq"], c["hk"], c["dim"]
        starts = _starts(c)
        s.starts = torch.tensor(starts, dtype=torch.int32, device="cuda") if c["parts"] else None

        def heads(n, scale):
            x = torch.randn(T, n, dim, device="cuda", generator=gen)
            x *= scale * torch.exp(0.4 * torch.randn(n, 1, device="cuda", generator=gen))
            x[starts[-1]:] = float("nan")
            return x.to(dt)

        q, k, v = heads(hq, 1.2), heads(hk, 1.2), heads(hk, 1.0)
        if c["fused"]:  # inside one projection's output
            x = torch.cat((q, k, v), 1)
            q, k, v = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
        s.q, s.k, s.v = q, k, v
        s.scale = 1 / math.sqrt(dim)
        s.o = torch.zeros(T, hq, dim, dtype=dt, device="cuda")
        if c["kind"] == "attn":
            s.do = heads(hq, 0.02)
            s.lse = torch.zeros(hq, T, device="cuda")
            x = torch.zeros(T, hq + 2 * hk, dim, dtype=dt, device="cuda")
            s.dq, s.dk, s.dv = x[:, :hq], x[:, hq:hq + hk], x[:, hq + hk:]
        return s
    rows, cols, pad, stream = c["rows"], c["cols"], c["pad"], DTYPE[c["stream"]]
    s.x = _strided(_activation(gen, rows, cols), dt, pad)
    s.res = _strided(2 * _activation(gen, rows, cols), stream, pad)
    s.h = _strided(s.res, stream, pad)
    host = random.Random(int(seed))
    s.seed, s.offset = host.getrandbits(64), host.getrandbits(40)
    # the step's number, which a captured program reads on the device
    s.at = torch.tensor([host.getrandbits(62)], dtype=torch.int64, device="cuda")
    if c["kind"] == "drop":
        s.dy = _strided(torch.randn(rows, cols, device="cuda", generator=gen) * 0.02, stream, pad)
        s.dx = _strided(s.x, dt, pad)
        return s
    s.w = 1 + 0.1 * torch.randn(cols, device="cuda", generator=gen)
    s.y = torch.empty(rows, cols, dtype=dt, device="cuda")
    s.kept = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    s.ckpt_y = torch.empty(_ckpt_bytes(rows, cols), dtype=torch.uint8, device="cuda")
    if c["kind"] == "step":
        s.ckpt_h = torch.empty(_ckpt_bytes(rows, cols), dtype=torch.uint8, device="cuda")
        s.rstd = torch.empty(rows, device="cuda")
        s.dy = _strided(torch.randn(rows, cols, device="cuda", generator=gen) * 0.02, dt, pad)
        s.dh_in = _strided(torch.randn(rows, cols, device="cuda", generator=gen) * 0.02, stream, pad)
        s.dh = torch.empty(rows, cols, dtype=stream, device="cuda")
        s.dx = torch.empty(rows, cols, dtype=dt, device="cuda")
        s.dw = torch.empty(cols, device="cuda")
    return s


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------
def _run_own(s):
    import paper_2609_06086_gb300 as P
    c = s.case
    stream = torch.cuda.current_stream().cuda_stream
    if c["kind"] in ("prompt", "attn"):
        a = P.pos_attn(c["tokens"], c["hq"], c["hk"], c["dim"], CODE[c["dtype"]], s.scale,
                       len(s.starts) - 1 if c["parts"] else 0,
                       s.starts.data_ptr() if c["parts"] else 0)

        def heads(*ts):
            return P.attn_heads(*(v for t in ts for v in (t.data_ptr(), t.stride(0), t.stride(1))))

        x = heads(s.q, s.k, s.v)
        o = P.pos_heads(s.o.data_ptr(), s.o.stride(0), s.o.stride(1))
        if c["kind"] == "prompt":
            P.poseidon_attn_forward(a, x, o, stream=stream)
            return s.o
        P.poseidon_attn_forward(a, x, o, lse=s.lse.data_ptr(), stream=stream)
        do = P.pos_heads(s.do.data_ptr(), s.do.stride(0), s.do.stride(1))
        P.poseidon_attn_backward(a, x, o, s.lse.data_ptr(), do, heads(s.dq, s.dk, s.dv),
                                 stream=stream)
        return s.o, s.lse, s.dq, s.dk, s.dv
    rows, cols = c["rows"], c["cols"]
    dtype, over = CODE[c["dtype"]], CODE[c["stream"]]
    drop = P.pos_dropout(c["p"], s.seed, s.offset, s.at.data_ptr())
    if c["kind"] == "drop":
        P.poseidon_dropout(drop, rows, cols, s.x.data_ptr(), dtype, s.x.stride(0),
                           s.res.data_ptr(), s.res.stride(0), s.h.data_ptr(), over,
                           s.h.stride(0), stream)
        P.poseidon_dropout(drop, rows, cols, s.dy.data_ptr(), over, s.dy.stride(0), 0, 0,
                           s.dx.data_ptr(), dtype, s.dx.stride(0), stream)
        return s.h, s.dx
    fmt = FORMAT[c["fmt"]]
    n = P.pos_norm(rows, cols, dtype, over, fmt, EPS, s.w.data_ptr(), drop)
    step, from_8 = c["kind"] == "step", c["kept"] == "h8"
    P.poseidon_norm_forward(n, s.x.data_ptr(), s.x.stride(0), s.res.data_ptr(), s.res.stride(0),
                            s.h.data_ptr(), s.h.stride(0), s.y.data_ptr(), s.y.stride(0),
                            s.ckpt_h.data_ptr() if step and from_8 else 0, s.ckpt_y.data_ptr(),
                            s.rstd.data_ptr() if step else 0, stream)
    P.poseidon_ckpt_unpack(s.ckpt_y.data_ptr(), fmt, rows, cols, s.kept.data_ptr(), 0,
                           s.kept.stride(0), stream)
    if not step:
        return s.h, s.y, s.kept
    P.poseidon_norm_backward(n, 0 if from_8 else s.h.data_ptr(), s.h.stride(0),
                             s.ckpt_h.data_ptr() if from_8 else 0, s.rstd.data_ptr(),
                             s.dy.data_ptr(), s.dy.stride(0), s.dh_in.data_ptr(),
                             s.dh_in.stride(0), s.dh.data_ptr(), s.dh.stride(0), s.dx.data_ptr(),
                             s.dx.stride(0), 0, s.dw.data_ptr(), stream)
    return s.h, s.y, s.kept, s.dh, s.dx, s.dw


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _power(e):
    """2^e in f32, e a tensor of whole numbers in [-126, 127]."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _in_8_bits(x, fmt):
    """What a checkpoint of f32 values [rows][cols] stands for."""
    rows, cols = x.shape
    groups = -(-cols // 32)
    x = torch.nn.functional.pad(x, (0, 32 * groups - cols)).view(rows, groups, 32)
    top = TOP[fmt]
    big = x.abs().amax(2)
    m, e = torch.frexp(big)  # big = m 2^e, 0.5 <= m < 1
    width = 7 if fmt == "int8" else 9  # top = m 2^width
    e = e - width + (m > top / 2 ** width)
    e = torch.where(big > 0, e, E_LO).clamp(E_LO, E_HI[fmt])
    v = (x * _power(-e)[:, :, None]).clamp(-top, top)
    code = v.round() if fmt == "int8" else v.to(torch.float8_e4m3fn).float()
    return (code * _power(e)[:, :, None]).flatten(1)[:, :cols]


def _philox_round(x, k):
    """One round on four int64 tensors that hold 32 bits each.  Products of 32 by
    32 bits by halves, so that none passes 2^63."""
    low = 0xffffffff
    hi0 = (0xD2511F53 * (x[0] >> 16) + (0xD2511F53 * (x[0] & 0xffff) >> 16)) >> 16
    hi1 = (0xCD9E8D57 * (x[2] >> 16) + (0xCD9E8D57 * (x[2] & 0xffff) >> 16)) >> 16
    return [hi1 ^ x[1] ^ k[0], 0xCD9E8D57 * x[2] & low, hi0 ^ x[3] ^ k[1], 0xD2511F53 * x[0] & low]


def _mask(s):
    """(kept [rows][cols], factor of what is kept)."""
    c = s.case
    t = round(c["p"] * 65536)
    low = 0xffffffff
    groups = -(-c["cols"] // 8)
    at = s.at + s.offset  # wraps as 64 bits do
    zero = torch.zeros(c["rows"], groups, dtype=torch.int64, device="cuda")
    x = [zero + torch.arange(groups, device="cuda"),
         zero + torch.arange(c["rows"], device="cuda")[:, None], zero + (at & low),
         zero + (at >> 32 & low)]
    k = [s.seed & low, s.seed >> 32]
    for _ in range(10):
        x = _philox_round(x, k)
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    u = torch.stack([h for w in x for h in (w & 0xffff, w >> 16)], -1).flatten(1)[:, :c["cols"]]
    return u >= t, float(np.float32(65536 / (65536 - t)))


def _run_plain_attn(s):
    c, dt = s.case, s.q.dtype
    T, hq, hk, dim = c["tokens"], c["hq"], c["hk"], c["dim"]
    group = hq // hk
    at = torch.arange(T, device="cuda", dtype=torch.int32)
    if s.starts is None:
        seq, live = torch.zeros_like(at), at >= 0
    else:
        seq = torch.searchsorted(s.starts[1:].contiguous(), at, right=True)
        live = at < s.starts[-1]

    def rows(x, heads):  # [key head][its heads x tokens][dim] in f32
        x = torch.where(live[:, None, None], x, 0).float()
        return x.view(T, hk, heads, dim).permute(1, 2, 0, 3).reshape(hk, heads * T, dim)

    def back(x, heads):
        return x.view(hk, heads, T, dim).permute(2, 0, 1, 3).reshape(T, hk * heads, dim).to(dt)

    q, k, v = rows(s.q, group), rows(s.k, 1), rows(s.v, 1)
    seen = (at[:, None] >= at) & (seq[:, None] == seq)
    p = (q * s.scale @ k.mT).view(hk, group, T, T)
    p = torch.where(seen, p, float("-inf"))
    big = p.amax(-1, keepdim=True)
    p = (p - big).exp_()
    total = p.sum(-1, keepdim=True)
    p = (p / total).view(hk, group * T, T)
    o = torch.where(live[:, None, None], back(p @ v, group), 0)
    if c["kind"] == "prompt":
        return o
    lse = torch.where(live, (big + total.log()).view(hq, T), 0.0)
    do = rows(s.do, group)
    ds = do @ v.mT
    # D = do o, which is the same sum before its order is changed
    ds = p * (ds - (p * ds).sum(-1, keepdim=True)) * s.scale
    return o, lse, back(ds @ k, group), back(ds.mT @ q, 1), back(p.mT @ do, 1)


def _run_plain(s):
    c = s.case
    if c["kind"] in ("prompt", "attn"):
        return _run_plain_attn(s)
    dt, stream = DTYPE[c["dtype"]], DTYPE[c["stream"]]
    x = s.x.double()
    if c["p"] > 0:
        kept, factor = _mask(s)
        x = torch.where(kept, x * factor, 0.0)
    # in 64 bits: one rounding to f32, next to the borders of the 8 bits
    h = (s.res.double() + x).float().to(stream)
    if c["kind"] == "drop":
        return h, torch.where(kept, s.dy.float() * factor, 0.0).to(dt)
    n = h.float()
    r = torch.rsqrt(n.square().mean(1, keepdim=True) + EPS)
    y = (n * r * s.w).to(dt)
    y8 = _in_8_bits(y.float(), c["fmt"]).to(torch.bfloat16)
    if c["kind"] == "norm":
        return h, y, y8
    n = (_in_8_bits(n, c["fmt"]) if c["kept"] == "h8" else n) * r
    g = s.dy.float()
    a = g * s.w
    dh = s.dh_in.float() + r * (a - n * (a * n).mean(1, keepdim=True))
    dx = torch.where(kept, dh * factor, 0.0) if c["p"] > 0 else dh
    return h, y, y8, dh.to(stream), dx.to(dt), (g * n).sum(0)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    c = case
    size = 4 if c["dtype"] == "f32" else 2
    if c["kind"] in ("prompt", "attn"):
        starts = _starts(c)
        pairs = sum(n * (n + 1) // 2 for n in (b - a for a, b in zip(starts, starts[1:])))
        per = c["dim"] * size * starts[-1]
        forward = {"bytes": per * (2 * c["hq"] + 2 * c["hk"]), "flops": 4 * pairs * c["dim"] * c["hq"]}
        if c["kind"] == "prompt":
            return forward
        # backward: q, k, v, o, do and the sums' logarithms in, three gradients out
        return {"bytes": forward["bytes"] + per * (4 * c["hq"] + 4 * c["hk"]) +
                8 * c["hq"] * starts[-1], "flops": 14 * pairs * c["dim"] * c["hq"]}
    n, over = c["rows"] * c["cols"], 4 if c["stream"] == "f32" else 2
    if c["kind"] == "drop":
        return {"bytes": n * (2 * size + 3 * over), "flops": 4 * n}
    kept = c["rows"] * (c["cols"] + -(-c["cols"] // 32))
    forward = n * (2 * size + 2 * over) + 2 * kept + 2 * n  # and the 8 bits as values
    if c["kind"] == "norm":
        return {"bytes": forward, "flops": 6 * n}
    h = 2 * kept if c["kept"] == "h8" else n * over
    return {"bytes": forward + h + n * (2 * size + 2 * over), "flops": 18 * n}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _two_to(e):
    """2^e in f64 from its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_8_bits(x, fmt):
    """What 8 bits keep of f64 values [rows][cols]."""
    rows, cols = x.shape
    pad = -cols % 32
    x = torch.cat((x, x.new_zeros(rows, pad)), 1).view(rows, -1, 32)
    top = TOP[fmt]
    big = x.abs().max(2).values
    e = torch.log2(big.clamp(min=2.0 ** -140) / top).round()
    e = e + (big > top * _two_to(e)).double()
    e = e - (big <= top * _two_to(e - 1)).double()
    scale = _two_to(e.clamp(E_LO, E_HI[fmt]))[:, :, None]
    v = x / scale
    if fmt == "int8":
        step = 1.0
    else:  # three bits after the leading one, exponents down to -6
        leading = ((v.view(torch.int64) >> 52) & 2047) - 1023
        step = _two_to(leading.clamp(min=-6) - 3)
    return ((v / step).round() * step).clamp(-top, top).mul(scale).view(rows, -1)[:, :cols]


def _exact_mask(case, seed, offset):
    """The generator in unsigned 64-bit words on the host, a block of rows at a time."""
    rows, cols = case["rows"], case["cols"]
    t = round(case["p"] * 65536)
    groups, low = -(-cols // 8), np.uint64(0xffffffff)
    m = (np.uint64(0xD2511F53), np.uint64(0xCD9E8D57))
    kept = np.empty((rows, cols), bool)
    for r0 in range(0, rows, 256):
        n = min(256, rows - r0)
        a = np.broadcast_to(np.arange(groups, dtype=np.uint64), (n, groups))
        b = np.broadcast_to(np.arange(r0, r0 + n, dtype=np.uint64)[:, None], (n, groups))
        c = np.full((n, groups), offset & 0xffffffff, np.uint64)
        d = np.full((n, groups), offset >> 32, np.uint64)
        for i in range(10):
            k0 = np.uint64((seed + i * 0x9E3779B9) & 0xffffffff)
            k1 = np.uint64(((seed >> 32) + i * 0xBB67AE85) & 0xffffffff)
            u, v = m[0] * a, m[1] * c
            a, b, c, d = (v >> np.uint64(32)) ^ b ^ k0, v & low, (u >> np.uint64(32)) ^ d ^ k1, u & low
        words = np.stack((a, b, c, d), -1).astype("<u4").view("<u2").reshape(n, -1)
        kept[r0:r0 + n] = words[:, :cols] >= t
    return torch.from_numpy(kept).cuda(), 65536 / (65536 - t)


def _exact_attn(case, s):
    hq, hk, scale = case["hq"], case["hk"], s.scale
    q, k, v = s.q.double(), s.k.double(), s.v.double()
    train = case["kind"] == "attn"
    o = torch.zeros_like(q)
    outs = [o]
    if train:
        do = s.do.double()
        lse = torch.zeros(hq, case["tokens"], dtype=torch.float64, device="cuda")
        dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
        outs = [o, lse, dq, dk, dv]
    starts = _starts(case)
    for a, b in zip(starts, starts[1:]):
        future = torch.ones(b - a, b - a, dtype=torch.bool, device="cuda").triu(1)
        for h in range(hq):
            if b == a:
                continue
            g = h // (hq // hk)
            Q, K, V = q[a:b, h], k[a:b, g], v[a:b, g]
            score = (Q @ K.t()).mul_(scale).masked_fill_(future, -math.inf)
            if not train:
                o[a:b, h] = torch.softmax(score, 1) @ V
                continue
            lse[h, a:b] = torch.logsumexp(score, 1)
            P = score.sub_(lse[h, a:b, None]).exp_()
            o[a:b, h] = P @ V
            G = do[a:b, h]
            dv[a:b, g] += P.t() @ G
            P.mul_(G @ V.t() - (G * o[a:b, h]).sum(1, keepdim=True))
            dq[a:b, h] = scale * (P @ K)
            dk[a:b, g] += scale * (P.t() @ Q)
    return tuple(outs) if train else o


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] in ("prompt", "attn"):
        return _exact_attn(c, s)
    factor = 1.0
    x = s.x.double()
    if c["p"] > 0:
        at = (s.offset + int(s.at.item())) & (2 ** 64 - 1)
        kept, factor = _exact_mask(c, s.seed, at)
        x = (x * float(np.float32(factor))).masked_fill_(~kept, 0.0)
    h32 = (x + s.res.double()).float()  # the definition's one rounding to f32,
    h = h32.to(DTYPE[c["stream"]]).double()  # and h as it is written
    if c["kind"] == "drop":
        return h32.double(), (s.dy.double() * factor).masked_fill_(~kept, 0.0)
    rms = torch.sqrt((h * h).sum(1, keepdim=True) / c["cols"] + EPS)
    y = h / rms * s.w.double()
    y8 = _exact_8_bits(y.to(DTYPE[c["dtype"]]).double(), c["fmt"])
    if c["kind"] == "norm":
        return h32.double(), y, y8
    n = (_exact_8_bits(h, c["fmt"]) if c["kept"] == "h8" else h) / rms
    g = s.dy.double()
    dw = (g * n).sum(0)
    g = g * s.w.double()
    dh = s.dh_in.double() + (g - n * (g * n).sum(1, keepdim=True) / c["cols"]) / rms
    dx = (dh * factor).masked_fill_(~kept, 0.0) if c["p"] > 0 else dh
    return h32.double(), y, y8, dh, dx, dw
