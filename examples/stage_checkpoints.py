"""A plan, and a stage of it that keeps its activations in 8 bits.

1. Searches the pipeline plan of a 7B-like model on one device of 80 GB and three
   slower ones of 24 GB twice: with the tables as profiled (activations in bf16),
   and with the memory per micro-batch that is left when the inputs of a layer's
   four linear operations are kept as 8-bit checkpoints.  The queries and keys that
   attention's backward pass reads stay as they are; those before their norm, which
   the profile has no norm for, are kept in 8 bits besides.  The second search may
   use plans that did not fit before.
2. Runs the q/k/v projections of the first stage of that plan in its 1F1B order
   on the GPU: W_s slots of checkpoints, one per micro-batch in flight; the
   forward pass fills a slot, the backward pass reads it, and the weights'
   gradients add up over the micro-batches.

    python examples/stage_checkpoints.py [--layers 2] [--seq 4096]
"""
import argparse
import math
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import numpy as np  # noqa: E402
import torch  # noqa: E402

import gen  # noqa: E402
import paper_2609_06086_gb300 as P  # noqa: E402
from paper_2609_06086_gb300.binding import POS_BF16, POS_CKPT_INT8, POS_ROT_HALF  # noqa: E402

EPS = 1e-6


def kept_bytes(seq, widths, heads, dim):
    """(bf16, 8 bits): bytes of one micro-batch's activations of the given widths
    (inputs of linear operations) and of q and k with their norms' factors."""
    plain = 2 * seq * (sum(widths) + sum(heads) * dim)
    packed = sum(P.poseidon_ckpt_bytes(seq, w) for w in widths)
    packed += sum(P.poseidon_ckpt_bytes(seq * h, dim) + 4 * seq * h for h in heads)
    return plain, packed


def workload(checkpoints):
    """Layers of width 4096, 32 query and 8 key heads, sequences of 4096."""
    w = gen.config2()
    w.placement, w.type_counts = gen.workloads.PLACE_EXACT, [1, 3]
    w.cap = np.array([80, 24], np.int64) * 10 ** 9
    if checkpoints:
        # instead of bf16: inputs of the q/k/v and output projections, of the MLP's two
        plain, packed = kept_bytes(4096, (4096, 4096, 4096, 4 * 4096), (), 128)
        # besides: q and k before their norm
        w.mem_a = w.mem_a - (plain - packed) + kept_bytes(4096, (), (32, 8), 128)[1]
    return w


def search(w):
    problem, keep = P.make_problem(w, prune=2)
    return P.poseidon_search(problem)[0]


class Slot:
    """What a layer keeps of one micro-batch."""

    def __init__(self, seq, hidden, heads, dim):
        self.x = torch.empty(P.poseidon_ckpt_bytes(seq, hidden), dtype=torch.uint8, device="cuda")
        self.qk = [torch.empty(P.poseidon_ckpt_bytes(seq * h, dim), dtype=torch.uint8,
                               device="cuda") for h in heads]
        self.rstd = [torch.empty(seq, h, device="cuda") for h in heads]

    def bytes(self):
        return sum(t.numel() * t.element_size() for t in (self.x, *self.qk, *self.rstd))


class Projection:
    """qkv = x W^T, then norm and rotation of q and k."""

    def __init__(self, seq, hidden, heads_q, heads_k, dim, gen_):
        self.shape = seq, hidden, heads_q, heads_k, dim
        n = (heads_q + 2 * heads_k) * dim
        self.w = (torch.randn(n, hidden, device="cuda", generator=gen_) / math.sqrt(hidden)).bfloat16()
        self.norm = 1 + 0.1 * torch.randn(2, dim, device="cuda", generator=gen_)
        self.dw = torch.zeros(n, hidden, device="cuda")
        self.dnorm = torch.zeros(2, dim, device="cuda")
        ang = torch.arange(seq, device="cuda", dtype=torch.float64)[:, None] * 10000.0 ** (
            -torch.arange(dim // 2, device="cuda", dtype=torch.float64) / (dim // 2))
        self.cos, self.sin = ang.cos().float(), ang.sin().float()
        self.qk = P.pos_qk(seq, heads_q, heads_k, dim, dim, POS_ROT_HALF, POS_BF16, POS_CKPT_INT8,
                           EPS, self.norm[0].data_ptr(), self.norm[1].data_ptr(),
                           self.cos.data_ptr(), self.sin.data_ptr(), seq, 0)

    def heads(self, qkv):
        """The queries and keys inside a fused [seq][heads][dim] tensor."""
        hq = self.shape[2]
        q, k = qkv[:, :hq], qkv[:, hq:]
        return P.qk_heads(q.data_ptr(), q.stride(0), q.stride(1), k.data_ptr(), k.stride(0),
                          k.stride(1))

    def forward(self, x, slot):
        seq, hidden, hq, hk, dim = self.shape
        s = torch.cuda.current_stream().cuda_stream
        P.poseidon_ckpt_pack(x.data_ptr(), POS_BF16, seq, hidden, x.stride(0), POS_CKPT_INT8,
                             slot.x.data_ptr(), s)
        qkv = (x @ self.w.t()).view(seq, hq + 2 * hk, dim)
        t = self.heads(qkv)
        P.poseidon_qk_forward(self.qk, t, t, rstd=tuple(r.data_ptr() for r in slot.rstd),
                              ckpt=tuple(c.data_ptr() for c in slot.qk), stream=s)  # in place
        return qkv

    def backward(self, dqkv, slot):
        """dqkv [seq][heads][dim], the gradients of forward()'s result, becomes
        that of x W^T; returns x's."""
        seq, hidden, hq, hk, dim = self.shape
        s = torch.cuda.current_stream().cuda_stream
        t = self.heads(dqkv)
        P.poseidon_qk_backward(self.qk, t, t, tuple(r.data_ptr() for r in slot.rstd),
                               ckpt=tuple(c.data_ptr() for c in slot.qk),
                               dw_in=self.dnorm.data_ptr(), dw=self.dnorm.data_ptr(), stream=s)
        dy = dqkv.view(seq, -1)
        P.poseidon_ckpt_wgrad(slot.x.data_ptr(), POS_CKPT_INT8, dy.data_ptr(), POS_BF16,
                              dy.stride(0), seq, dy.shape[1], hidden, self.dw.data_ptr(),
                              self.dw.data_ptr(), hidden, s)
        return dy @ self.w


def one_f_one_b(stage, stages, micro_batches):
    """The operations of a stage (0-based) in 1F1B order: ('F' or 'B', micro-batch)."""
    w = min(stages - stage, micro_batches)
    order = [("F", m) for m in range(w)]
    for m in range(micro_batches - w):
        order += [("B", m), ("F", w + m)]
    return w, order + [("B", m) for m in range(micro_batches - w, micro_batches)]


def run_stage(plan, stage, layers, seq, hidden, heads_q, heads_k, dim, seed=0):
    """Both passes of every micro-batch; returns (layers, slots, inputs, output
    gradients), the layers with the gradients summed over the micro-batches."""
    gen_ = torch.Generator(device="cuda").manual_seed(seed)
    stack = [Projection(seq, hidden, heads_q, heads_k, dim, gen_) for _ in range(layers)]
    w, order = one_f_one_b(stage, len(plan["layers"]), plan["M"])
    slots = [[Slot(seq, hidden, (heads_q, heads_k), dim) for _ in stack] for _ in range(w)]
    shape = (plan["M"], layers, seq)
    xs = torch.randn(*shape, hidden, device="cuda", generator=gen_).bfloat16()
    gs = torch.randn(*shape, heads_q + 2 * heads_k, dim, device="cuda", generator=gen_).bfloat16()
    for op, m in order:
        for i, layer in enumerate(stack):
            slot = slots[m % w][i]
            if op == "F":
                layer.forward(xs[m, i], slot)
            else:
                layer.backward(gs[m, i].clone(), slot)
    torch.cuda.synchronize()
    return stack, slots, xs, gs


def plain_gradients(layer, xs, gs):
    """(dW, dnorm) of one layer by automatic differentiation in f32, with
    nothing kept in 8 bits."""
    seq, hidden, hq, hk, dim = layer.shape
    w = layer.w.float().requires_grad_()
    norm = layer.norm.clone().requires_grad_()
    cos, sin = layer.cos[:, None], layer.sin[:, None]
    for x, g in zip(xs, gs):
        y = (x.float() @ w.t()).view(seq, -1, dim)
        parts = []
        for k, t in enumerate((y[:, :hq], y[:, hq:hq + hk])):
            u = t * torch.rsqrt(t.square().mean(-1, keepdim=True) + EPS) * norm[k]
            a, b = u[..., :dim // 2], u[..., dim // 2:]
            parts.append(torch.cat((a * cos - b * sin, b * cos + a * sin), -1))
        out = torch.cat((*parts, y[:, hq + hk:]), 1)
        (out * g.float()).sum().backward()
    return w.grad, norm.grad


def main(argv=None):
    a = argparse.ArgumentParser()
    a.add_argument("--layers", type=int, default=2, help="layers of the stage that are run")
    a.add_argument("--seq", type=int, default=4096)
    a.add_argument("--hidden", type=int, default=4096)
    a.add_argument("--heads", type=int, nargs=2, default=(32, 8), help="query and key heads")
    a.add_argument("--micro-batches", type=int, default=0, help="run fewer than the plan's")
    o = a.parse_args(argv)
    hq, hk = o.heads
    dim = o.hidden // hq
    plan, leaner = search(workload(False)), search(workload(True))
    for name, p in (("bf16", plan), ("8 bits", leaner)):
        print(f"kept in {name:6s}: iteration {p['T']} us, M = {p['M']}, layers {p['layers']}, "
              f"device types {p['types']}")
    run = dict(leaner, M=min(leaner["M"], o.micro_batches or leaner["M"]))
    stack, slots, xs, gs = run_stage(run, 0, o.layers, o.seq, o.hidden, hq, hk, dim)
    plain, packed = kept_bytes(o.seq, (o.hidden,), (hq, hk), dim)
    print(f"stage 0: {len(slots)} slots of {packed / 2**20:.1f} MiB a layer (bf16: "
          f"{plain / 2**20:.1f})")
    off = []
    for i, layer in enumerate(stack):
        dw, dnorm = plain_gradients(layer, xs[:, i], gs[:, i])
        off.append([float((got - want).norm() / want.norm())
                    for got, want in ((layer.dw, dw), (layer.dnorm, dnorm))])
        print(f"layer {i}: gradients off by {off[-1][0]:.4f} (weights) and {off[-1][1]:.4f} (norms) "
              f"of their norm against f32 with nothing in 8 bits")
    return plan, leaner, off


if __name__ == "__main__":
    main()
