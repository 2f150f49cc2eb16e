"""The layer operators together, as a transformer layer's attention half uses them in a
training step: the residual's addition with dropout and the norm (kept in 8 bits for the
weight gradient), one projection, norm and rotation of queries and keys, attention, the
output projection from an 8-bit checkpoint, dropout and the residual; forward and
backward, against 64-bit automatic differentiation of the same formulas."""
import math

import numpy as np
import pytest

import dropout_util as D

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

T, HQ, HK, DIM, EPS, P_DROP = 200, 4, 2, 64, 1e-6, 0.2
HIDDEN, STARTS = HQ * DIM, (0, 70, 200)


@pytest.fixture(scope="module")
def P():
    import paper_2609_06086_gb300 as P
    return P


def ptr(t):
    return t.data_ptr(), t.stride(0)


def test_attention_half_of_a_layer(P):
    gen = torch.Generator(device="cuda").manual_seed(4)
    new = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    bf = torch.bfloat16
    x, res = new(T, HIDDEN).to(bf), new(T, HIDDEN)
    w_norm = 1 + 0.1 * new(HIDDEN)
    n_out = (HQ + 2 * HK) * DIM
    w_qkv = (new(n_out, HIDDEN) / math.sqrt(HIDDEN)).to(bf)
    w_o = (new(HIDDEN, HIDDEN) / math.sqrt(HIDDEN)).to(bf)
    w_head = 1 + 0.1 * new(2, DIM)
    ang = torch.arange(T, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (
        -torch.arange(DIM // 2, device="cuda", dtype=torch.float64) / (DIM // 2))
    cos, sin = ang.cos().float(), ang.sin().float()
    starts = torch.tensor(STARTS, dtype=torch.int32, device="cuda")
    g_out = new(T, HIDDEN)
    s = torch.cuda.current_stream().cuda_stream

    # forward
    n = P.pos_norm(T, HIDDEN, 0, 2, 0, EPS, w_norm.data_ptr(), P.pos_dropout(P_DROP, 21, 1, 0))
    h, y = torch.empty(T, HIDDEN, device="cuda"), torch.empty(T, HIDDEN, dtype=bf, device="cuda")
    ckpt = lambda: torch.empty(P.poseidon_ckpt_bytes(T, HIDDEN), dtype=torch.uint8,  # noqa: E731
                               device="cuda")
    ckpt_h, ckpt_y, ckpt_o = ckpt(), ckpt(), ckpt()
    rstd = torch.empty(T, device="cuda")
    P.poseidon_norm_forward(n, *ptr(x), *ptr(res), *ptr(h), *ptr(y), ckpt_h.data_ptr(),
                            ckpt_y.data_ptr(), rstd.data_ptr(), s)
    qkv = (y @ w_qkv.t()).view(T, HQ + 2 * HK, DIM)
    at = lambda t: (t.data_ptr(), t.stride(0), t.stride(1))  # noqa: E731
    parts = lambda t: (t[:, :HQ], t[:, HQ:HQ + HK], t[:, HQ + HK:])  # noqa: E731
    pair = lambda t: P.qk_heads(*at(parts(t)[0]), *at(parts(t)[1]))  # noqa: E731
    triple = lambda t: P.attn_heads(*(v for u in parts(t) for v in at(u)))  # noqa: E731
    qk = P.pos_qk(T, HQ, HK, DIM, DIM, 0, 0, 0, EPS, w_head[0].data_ptr(), w_head[1].data_ptr(),
                  cos.data_ptr(), sin.data_ptr(), T, 0)
    r_qk = [torch.empty(T, k, device="cuda") for k in (HQ, HK)]
    c_qk = [torch.empty(P.poseidon_ckpt_bytes(T * k, DIM), dtype=torch.uint8, device="cuda")
            for k in (HQ, HK)]
    rp, cp = tuple(t.data_ptr() for t in r_qk), tuple(t.data_ptr() for t in c_qk)
    P.poseidon_qk_forward(qk, pair(qkv), pair(qkv), rstd=rp, ckpt=cp, stream=s)  # in place
    a = P.pos_attn(T, HQ, HK, DIM, 0, DIM ** -0.5, len(STARTS) - 1, starts.data_ptr())
    o = torch.empty(T, HQ, DIM, dtype=bf, device="cuda")
    lse = torch.empty(HQ, T, device="cuda")
    P.poseidon_attn_forward(a, triple(qkv), P.pos_heads(*at(o)), lse=lse.data_ptr(), stream=s)
    o2 = o.view(T, HIDDEN)
    P.poseidon_ckpt_pack(o2.data_ptr(), 0, T, HIDDEN, HIDDEN, 0, ckpt_o.data_ptr(), s)
    proj = o2 @ w_o.t()
    drop2 = P.pos_dropout(P_DROP, 21, 2, 0)
    out = torch.empty_like(h)
    P.poseidon_dropout(drop2, T, HIDDEN, *[proj.data_ptr(), 0, HIDDEN], h.data_ptr(), HIDDEN,
                       out.data_ptr(), 2, HIDDEN, s)

    # backward
    d_proj = torch.empty_like(proj)
    P.poseidon_dropout(drop2, T, HIDDEN, g_out.data_ptr(), 2, HIDDEN, 0, 0, d_proj.data_ptr(), 0,
                       HIDDEN, s)
    dw_o, dw_qkv = torch.empty(HIDDEN, HIDDEN, device="cuda"), torch.empty(n_out, HIDDEN, device="cuda")
    P.poseidon_ckpt_wgrad(ckpt_o.data_ptr(), 0, *[d_proj.data_ptr(), 0, HIDDEN], T, HIDDEN, HIDDEN, 0,
                          dw_o.data_ptr(), HIDDEN, s)
    d_o = (d_proj @ w_o).view(T, HQ, DIM)
    d_qkv = torch.empty_like(qkv)
    P.poseidon_attn_backward(a, triple(qkv), P.pos_heads(*at(o)), lse.data_ptr(),
                             P.pos_heads(*at(d_o)), triple(d_qkv), stream=s)
    dw_head = torch.empty(2, DIM, device="cuda")
    P.poseidon_qk_backward(qk, pair(d_qkv), pair(d_qkv), rp, ckpt=cp, dw=dw_head.data_ptr(), stream=s)
    dy2 = d_qkv.view(T, n_out)
    P.poseidon_ckpt_wgrad(ckpt_y.data_ptr(), 0, *[dy2.data_ptr(), 0, n_out], T, n_out, HIDDEN, 0,
                          dw_qkv.data_ptr(), HIDDEN, s)
    d_y = dy2 @ w_qkv
    dh, dx, dw_norm = torch.empty_like(h), torch.empty_like(x), torch.empty(HIDDEN, device="cuda")
    P.poseidon_norm_backward(n, 0, 0, ckpt_h.data_ptr(), rstd.data_ptr(), *ptr(d_y), *ptr(g_out),
                             *ptr(dh), *ptr(dx), 0, dw_norm.data_ptr(), s)

    # the same in 64 bits
    X, R, W, Wq, Wo, Wh = (t.double().requires_grad_() for t in (x, res, w_norm, w_qkv, w_o, w_head))
    masks = []
    for k in (1, 2):
        kept, factor = D.mask(range(T), HIDDEN, 21, k, P_DROP)
        masks.append(torch.from_numpy(kept * factor).cuda())
    H = R + X * masks[0]
    Y = H / torch.sqrt(H.square().mean(1, keepdim=True) + EPS) * W
    q, k, v = parts((Y @ Wq.t()).view(T, -1, DIM))
    turned = []
    for i, t in enumerate((q, k)):
        t = t / torch.sqrt(t.square().mean(-1, keepdim=True) + EPS) * Wh[i]
        c, e = ang.cos()[:, None], ang.sin()[:, None]
        b, d = t[..., :DIM // 2], t[..., DIM // 2:]
        turned.append(torch.cat((b * c - d * e, d * c + b * e), -1))
    q, k, v = (t.transpose(0, 1) for t in (*turned, v))
    k, v = k.repeat_interleave(HQ // HK, 0), v.repeat_interleave(HQ // HK, 0)
    tok = torch.arange(T, device="cuda")
    seen = (tok[:, None] >= tok) & ((tok[:, None] < STARTS[1]) == (tok < STARTS[1]))
    score = (q @ k.mT * DIM ** -0.5).masked_fill(~seen, -math.inf)
    O = (torch.softmax(score, -1) @ v).transpose(0, 1).reshape(T, HIDDEN)
    OUT = H + (O @ Wo.t()) * masks[1]
    (OUT * g_out.double()).sum().backward()

    far = lambda got, want: float((got.double() - want).norm() / want.norm())  # noqa: E731
    # forward: bf16 roundings of y, qkv, q and k, o and proj one after another, 2^-9 of a
    # value each at worst on average, added as if they were alike; the residual is larger
    assert far(out, OUT.detach()) < 6 * 2.0 ** -9
    # backward: the same number again, and what 8 bits keep: at most 2^-8 of a group's
    # largest magnitude, which is about three times the mean, evenly spread
    # (3 / (2^8 sqrt 3) = 0.007), of h, y, o and the heads
    for got, want in ((dh, R.grad), (dx, X.grad), (dw_norm, W.grad), (dw_qkv, Wq.grad),
                      (dw_o, Wo.grad), (dw_head, Wh.grad)):
        assert far(got, want) < 12 * 2.0 ** -9 + 2 * 0.007
    dropped = torch.from_numpy(~D.mask(range(T), HIDDEN, 21, 1, P_DROP)[0]).cuda()
    assert not dx[dropped].any() and np.isclose(dropped.float().mean().item(), P_DROP, atol=0.02)
