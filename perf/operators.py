"""The measured operator calls: what a pipeline stage keeps of a micro-batch in
8 bits between its forward and its backward pass, and what it computes from it.

Kinds of a case
  keep    an activation is packed into an 8-bit checkpoint and restored from it
  wgrad   the weight gradient of a linear layer, read from the checkpoint of
          its input: dw_out = dw_in + dY^T X (dw_in may be absent)
  serve   per-head RMS norm of queries and keys with the position rotation in
          the same pass, as generation calls it (nothing kept)
  train   the same for a training step: the forward pass keeps q and k in 8
          bits, the backward pass reads them: outputs, gradients of q, k and
          both norm weights

A checkpoint of [rows][cols] values: one byte per value, rows of
pitch = 32 * ceil(cols / 32) bytes, then one scale byte e + 127 per group of 32
columns, rows of spitch = 4 * ceil(groups / 4) bytes.  A value is code * 2^e,
the code an int8 in [-127, 127] ("int8") or a float8 e4m3 ("e4m3"); e is the
smallest that keeps the group's largest magnitude within 127 or 448, at least
-110 and at most 121 or 119, and the code saturates.  A group that holds an
infinity or a NaN has scale byte 255 and stands for NaN.

Sizes follow the repository's own workloads: widths of 4096, 5120 and 8192,
sequences of 4096, micro-batch 1 and a few.
"""
import math
from types import SimpleNamespace

import torch

own = False

DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
CODE = {"bf16": 0, "f16": 1, "f32": 2}
FORMAT = {"int8": 0, "e4m3": 1}
PAIRING = {"half": 0, "adjacent": 1}
TOP = {"int8": 127.0, "e4m3": 448.0}
E_HI = {"int8": 121, "e4m3": 119}
E_LO = -110
EPS = 1e-6


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _keep(name, rows, cols, dtype="bf16", fmt="int8", pad=0):
    return dict(name=name, kind="keep", rows=rows, cols=cols, dtype=dtype, fmt=fmt, pad=pad)


def _wgrad(name, rows, n, cols, dtype="bf16", fmt="int8", add=False, pad=0):
    return dict(name=name, kind="wgrad", rows=rows, n=n, cols=cols, dtype=dtype, fmt=fmt, add=add,
                pad=pad)


def _qk(name, kind, tokens, hq, hk, dim, rot, dtype="bf16", fmt="int8", pairing="half",
        padding=0.0, fused=True, n_pos=4096):
    return dict(name=name, kind=kind, tokens=tokens, hq=hq, hk=hk, dim=dim, rot=rot, dtype=dtype,
                fmt=fmt, pairing=pairing, padding=padding, fused=fused, n_pos=n_pos)


def listed():
    return [
        # a short micro-batch's slice of a narrow layer: latency of two calls
        _keep("keep_small", 128, 1024),
        # the input of a 7B-like layer's linears, micro-batch 1, sequence 4096
        _keep("keep_7b", 4096, 4096, fmt="e4m3"),
        # an fp16 activation of odd sizes, a slice of a wider buffer
        _keep("keep_odd", 5003, 5001, dtype="f16", pad=7),
        # four micro-batches of a 70B-like layer, residual stream in f32
        _keep("keep_70b", 16384, 8192, dtype="f32"),
        # a small projection of a short micro-batch, few output tiles
        _wgrad("wgrad_small", 512, 1024, 1024),
        # fp16, odd token count and odd widths, gradients in a padded buffer
        _wgrad("wgrad_odd", 4093, 1283, 5120, dtype="f16", fmt="e4m3", pad=5),
        # the fused q, k, v projection of a 7B-like layer (8 key heads),
        # added to the gradients of earlier micro-batches
        _wgrad("wgrad_7b", 4096, 6144, 4096, add=True),
        # the same projection of a 70B-like layer, two sequences
        _wgrad("wgrad_70b", 8192, 10240, 8192, fmt="e4m3"),
        # one token of a 7B-like model: latency of the call
        _qk("serve_one", "serve", 1, 32, 8, 128, 128, n_pos=32768),
        # a batch of generating sequences of a 70B-like model at scattered
        # positions, q and k inside one fused projection's output
        _qk("serve_batch", "serve", 509, 64, 8, 128, 128, n_pos=32768),
        # a training step of odd head width, partly rotated in adjacent pairs,
        # with padding tokens
        _qk("train_odd", "train", 3001, 20, 4, 80, 48, dtype="f16", fmt="e4m3",
            pairing="adjacent", padding=0.1),
        # a training step of a 70B-like layer, sequence 4096, micro-batch 2
        _qk("train_70b", "train", 8192, 64, 8, 128, 128, padding=0.02),
    ]


def _log_int(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return v + 1 if v == 3072 else v


def draw(rng):
    kind = rng.choice(("keep", "wgrad", "wgrad", "serve", "train", "train"))
    fmt = rng.choice(("int8", "e4m3"))
    if kind == "keep":
        return _keep("", _log_int(rng, 1, 16384), _log_int(rng, 33, 8192),
                     rng.choice(("bf16", "bf16", "f16", "f32")), fmt, rng.choice((0, 0, 8, 3)))
    if kind == "wgrad":
        size = lambda lo, hi: (_log_int(rng, lo, hi) if rng.random() < 0.4 else  # noqa: E731
                               64 * _log_int(rng, max(1, lo // 64), hi // 64))
        rows, n, cols = size(1, 8192), size(64, 10240), size(64, 8192)
        rows, n, cols = (v + (v == 3072) for v in (rows, n, cols))
        return _wgrad("", rows, n, cols, rng.choice(("bf16", "bf16", "f16")), fmt,
                      rng.random() < 0.5, rng.choice((0, 0, 8, 3)))
    dim = rng.choice((64, 80, 96, 128, 128, 128, 192, 256, 72))
    hk = rng.choice((1, 2, 4, 8))
    hq = hk * rng.choice((1, 2, 4, 8))
    while hq * dim * (1 if kind == "serve" else 2) > 16384 or \
            3072 in (hq * dim, (hq + hk) * dim, (hq + 2 * hk) * dim):
        hq = hq // 2 or hq + 1
        hk = min(hk, hq)
    rot = dim if rng.random() < 0.6 else 2 * rng.randint(1, dim // 2)
    tokens = _log_int(rng, 1, 2048) if kind == "serve" else _log_int(rng, 17, 8192)
    return _qk("", kind, tokens, hq, hk, dim, rot, rng.choice(("bf16", "bf16", "f16", "f32")), fmt,
               rng.choice(("half", "adjacent")), rng.choice((0.0, 0.0, 0.1)), rng.random() < 0.5,
               rng.choice((4096, 32768)))


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


def _layout(rows, cols):
    groups = -(-cols // 32)
    pitch, spitch = 32 * groups, 4 * -(-groups // 4)
    return groups, pitch, spitch, rows * (pitch + spitch)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    s = SimpleNamespace(case=dict(case))
    dt = DTYPE[case["dtype"]]
    if case["kind"] == "keep":
        rows, cols = case["rows"], case["cols"]
        s.x = _strided(_activation(gen, rows, cols), dt, case["pad"])
        s.y = torch.empty(rows, cols, dtype=dt, device="cuda")
        s.ckpt = torch.empty(_layout(rows, cols)[3], dtype=torch.uint8, device="cuda")
    elif case["kind"] == "wgrad":
        rows, n, cols = case["rows"], case["n"], case["cols"]
        groups, pitch, spitch, size = _layout(rows, cols)
        code, e = _codes(_activation(gen, rows, cols).to(dt).float(), case["fmt"])
        s.ckpt = torch.zeros(size, dtype=torch.uint8, device="cuda")
        kind = torch.int8 if case["fmt"] == "int8" else torch.float8_e4m3fn
        s.ckpt[:rows * pitch].view(rows, pitch).copy_(
            code.reshape(rows, pitch).to(kind).view(torch.uint8))
        s.ckpt[rows * pitch:].view(rows, spitch)[:, :groups] = (e + 127).to(torch.uint8)
        del code, e
        s.dy = _strided(torch.randn(rows, n, device="cuda", generator=gen) * 0.02, dt, case["pad"])
        s.dw_in = torch.randn(n, cols, device="cuda", generator=gen) if case["add"] else None
        s.dw = torch.empty(n, cols, device="cuda")
    else:
        T, hq, hk, dim = case["tokens"], case["hq"], case["hk"], case["dim"]
        half = case["rot"] // 2
        # one fused projection's output holds q, k and as many value heads as
        # key heads; otherwise q and k are tensors of their own
        x = _activation(gen, T, (hq + 2 * hk) * dim).to(dt).view(T, hq + 2 * hk, dim)
        if case["fused"]:
            s.q, s.k = x[:, :hq], x[:, hq:hq + hk]
        else:
            s.q, s.k = x[:, :hq].contiguous(), x[:, hq:hq + hk].contiguous()
        s.w = 1 + 0.1 * torch.randn(2, dim, device="cuda", generator=gen)
        ang = torch.arange(case["n_pos"], device="cuda", dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / max(half, 1))
        s.cos, s.sin = ang.cos().float(), ang.sin().float()
        if case["kind"] == "serve":
            s.pos = torch.randint(0, case["n_pos"], (T,), device="cuda", generator=gen)
        else:  # sequences of at most 4096, packed one after another
            s.pos = torch.arange(T, device="cuda") % min(4096, case["n_pos"])
        drop = torch.rand(T, device="cuda", generator=gen) < case["padding"]
        s.pos = torch.where(drop, -1, s.pos).to(torch.int32)
        s.yq, s.yk = torch.empty(T, hq, dim, dtype=dt, device="cuda"), \
            torch.empty(T, hk, dim, dtype=dt, device="cuda")
        if case["kind"] == "train":
            s.gq = torch.randn(T, hq, dim, device="cuda", generator=gen).to(dt)
            s.gk = torch.randn(T, hk, dim, device="cuda", generator=gen).to(dt)
            s.rq, s.rk = torch.empty(T, hq, device="cuda"), torch.empty(T, hk, device="cuda")
            s.cq = torch.empty(_layout(T * hq, dim)[3], dtype=torch.uint8, device="cuda")
            s.ck = torch.empty(_layout(T * hk, dim)[3], dtype=torch.uint8, device="cuda")
            s.dq, s.dk = torch.empty_like(s.gq), torch.empty_like(s.gk)
            s.dw = torch.empty(2, dim, device="cuda")
    return s


# ---------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------
def _run_own(s):
    import paper_2609_06086_gb300 as P
    c = s.case
    stream = torch.cuda.current_stream().cuda_stream
    dtype, fmt = CODE[c["dtype"]], FORMAT[c["fmt"]]
    if c["kind"] == "keep":
        P.poseidon_ckpt_pack(s.x.data_ptr(), dtype, c["rows"], c["cols"], s.x.stride(0), fmt,
                             s.ckpt.data_ptr(), stream)
        P.poseidon_ckpt_unpack(s.ckpt.data_ptr(), fmt, c["rows"], c["cols"], s.y.data_ptr(), dtype,
                               s.y.stride(0), stream)
        return s.y
    if c["kind"] == "wgrad":
        P.poseidon_ckpt_wgrad(s.ckpt.data_ptr(), fmt, s.dy.data_ptr(), dtype, s.dy.stride(0),
                              c["rows"], c["n"], c["cols"],
                              0 if s.dw_in is None else s.dw_in.data_ptr(), s.dw.data_ptr(),
                              s.dw.stride(0), stream)
        return s.dw

    def heads(q, k):
        return P.qk_heads(q.data_ptr(), q.stride(0), q.stride(1), k.data_ptr(), k.stride(0),
                          k.stride(1))

    qk = P.pos_qk(c["tokens"], c["hq"], c["hk"], c["dim"], c["rot"], PAIRING[c["pairing"]], dtype,
                  fmt, EPS, s.w[0].data_ptr(), s.w[1].data_ptr(), s.cos.data_ptr(),
                  s.sin.data_ptr(), c["n_pos"], s.pos.data_ptr())
    x, y = heads(s.q, s.k), heads(s.yq, s.yk)
    if c["kind"] == "serve":
        P.poseidon_qk_forward(qk, x, y, stream=stream)
        return s.yq, s.yk
    rstd, ckpt = (s.rq.data_ptr(), s.rk.data_ptr()), (s.cq.data_ptr(), s.ck.data_ptr())
    P.poseidon_qk_forward(qk, x, y, rstd=rstd, ckpt=ckpt, stream=stream)
    P.poseidon_qk_backward(qk, heads(s.gq, s.gk), heads(s.dq, s.dk), rstd=rstd, ckpt=ckpt,
                           dw=s.dw.data_ptr(), stream=stream)
    return s.yq, s.yk, s.dq, s.dk, s.dw


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------
def _power(e):
    """2^e in f32, e a tensor of whole numbers in [-126, 127]."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _codes(x, fmt):
    """(codes as f32 [rows][groups][32], exponents [rows][groups]) of f32 values
    [rows][cols]; columns past the last are zeros."""
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
    return code, e


def _values(code, e, cols, dtype):
    """What the codes stand for, as f32 [rows][cols]; an f16 value saturates."""
    v = (code * _power(e)[:, :, None]).flatten(1)[:, :cols]
    return v.clamp(-65504, 65504).half().float() if dtype == "f16" else v


def _rotated(u, cos, sin, rot, pairing):
    """Rot u over the last dimension; cos, sin [tokens][1][rot / 2]."""
    if rot == 0:
        return u
    if pairing == "half":
        a, b = u[..., :rot // 2], u[..., rot // 2:rot]
        out = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = u[..., 0:rot:2], u[..., 1:rot:2]
        out = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    return torch.cat((out, u[..., rot:]), -1)


def _run_plain(s):
    c = s.case
    dt = DTYPE[c["dtype"]]
    if c["kind"] == "keep":
        code, e = _codes(s.x.float(), c["fmt"])
        return _values(code, e, c["cols"], c["dtype"]).to(dt)
    if c["kind"] == "wgrad":
        rows, cols = c["rows"], c["cols"]
        groups, pitch, spitch, _ = _layout(rows, cols)
        kind = torch.int8 if c["fmt"] == "int8" else torch.float8_e4m3fn
        code = s.ckpt[:rows * pitch].view(kind).float().view(rows, groups, 32)
        e = s.ckpt[rows * pitch:].view(rows, spitch)[:, :groups].int() - 127
        dw = s.dy.float().t() @ _values(code, e, cols, c["dtype"])
        return dw if s.dw_in is None else dw + s.dw_in
    live = (s.pos >= 0)[:, None, None]
    at = s.pos.clamp(min=0).long()
    cos, sin = s.cos[at][:, None], s.sin[at][:, None]
    outs, grads, dws = [], [], []
    for i, x in enumerate((s.q, s.k)):
        x = x.float()
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
        y = _rotated(x * r * s.w[i], cos, sin, c["rot"], c["pairing"])
        outs.append(torch.where(live, y, 0.0).to(dt))
        if c["kind"] == "train":
            code, e = _codes(x.reshape(-1, c["dim"]), c["fmt"])
            n = _values(code, e, c["dim"], "f32").view(x.shape) * r
            g = (s.gq, s.gk)[i].float()
            g = torch.where(live, _rotated(g, cos, -sin, c["rot"], c["pairing"]), 0.0)
            h = g * s.w[i]
            grads.append((r * (h - n * (h * n).mean(-1, keepdim=True))).to(dt))
            dws.append((g * n).sum((0, 1)))
    if c["kind"] == "serve":
        return tuple(outs)
    return (*outs, *grads, torch.stack(dws))


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "keep":
        rows, cols = case["rows"], case["cols"]
        kept = rows * (cols + -(-cols // 32))
        return {"bytes": 2 * rows * cols * size + 2 * kept, "flops": 4 * rows * cols}
    if case["kind"] == "wgrad":
        rows, n, cols = case["rows"], case["n"], case["cols"]
        kept = rows * (cols + -(-cols // 32))
        return {"bytes": kept + rows * n * size + n * cols * 4 * (2 if case["add"] else 1),
                "flops": 2 * rows * n * cols}
    T, heads, dim = case["tokens"], case["hq"] + case["hk"], case["dim"]
    table = 4 * case["rot"] * min(T, case["n_pos"] if case["kind"] == "serve" else 4096)
    if case["kind"] == "serve":
        return {"bytes": 2 * T * heads * dim * size + table + 4 * T, "flops": 9 * T * heads * dim}
    kept = T * heads * (dim + -(-dim // 32) + 4)
    return {"bytes": 4 * T * heads * dim * size + 2 * kept + 2 * (table + 4 * T),
            "flops": 27 * T * heads * dim}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def _two_to(e):
    """2^e in f64 from its bits (a power function may be off by a unit in the
    last place, and then a value halfway between two codes goes either way)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_kept(x, fmt):
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


def exact(case, seed):
    s = prepare(case, seed)
    fmt, half_type = case["fmt"], case["dtype"] == "f16"
    if case["kind"] == "keep":
        y = _exact_kept(s.x.double(), fmt)
        return y.clamp(-65504, 65504) if half_type else y
    if case["kind"] == "wgrad":
        rows, cols = case["rows"], case["cols"]
        groups, pitch, spitch, _ = _layout(rows, cols)
        raw = s.ckpt[:rows * pitch].view(rows, pitch)[:, :cols].long()
        if fmt == "int8":
            x = (raw - 256 * (raw > 127)).double()
        else:
            low, field = (raw & 7).double(), (raw >> 3) & 15
            x = torch.where(field == 0, low * 2.0 ** -9, (8 + low) * _two_to(field - 10))
            x = torch.where(raw > 127, -x, x)
        e = s.ckpt[rows * pitch:].view(rows, spitch)[:, :groups].double() - 127
        x = x * _two_to(e).repeat_interleave(32, 1)[:, :cols]
        if half_type:
            x = x.clamp(-65504, 65504).half().double()
        dw = s.dy.double().t().contiguous() @ x
        return dw if s.dw_in is None else s.dw_in.double() + dw
    pos = s.pos.long()
    dim, rot = case["dim"], case["rot"]
    # the rotation as complex factors of the pairs
    turn = torch.complex(s.cos.double(), s.sin.double())[pos.clamp(min=0)][:, None]
    first = torch.arange(rot // 2, device="cuda") * (1 if case["pairing"] == "half" else 2)
    second = first + (rot // 2 if case["pairing"] == "half" else 1)

    def turned(u, by):
        z = torch.complex(u[..., first], u[..., second]) * by
        u = u.clone()
        u[..., first], u[..., second] = z.real, z.imag
        return u

    ys, dxs, dws = [], [], []
    for x, w, g in ((s.q, s.w[0], getattr(s, "gq", None)), (s.k, s.w[1], getattr(s, "gk", None))):
        x, w = x.double(), w.double()
        norm = torch.sqrt((x * x).sum(-1, keepdim=True) / dim + EPS)
        y = turned(x / norm * w, turn)
        y[pos < 0] = 0
        ys.append(y)
        if g is None:
            continue
        n = _exact_kept(x.reshape(-1, dim), fmt).view(x.shape) / norm
        g = turned(g.double(), turn.conj())
        g[pos < 0] = 0
        dws.append((g * n).sum((0, 1)))
        g = g * w
        dxs.append((g - n * (g * n).sum(-1, keepdim=True) / dim) / norm)
    if case["kind"] == "serve":
        return tuple(ys)
    return (*ys, *dxs, torch.stack(dws))
