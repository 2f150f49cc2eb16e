"""Attention whose waits run out.  Limits of no time or of a few microseconds, in processes
of their own: every result that is lost by that is NaN and every other one is right, whatever
was in memory; nothing faults, and a call after it is none the worse.  (With no time a first
try that fails ends the wait; copies and products in flight end by themselves.)"""
import os
import subprocess
import sys

import pytest

pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))

# lengths, hq, hk, dim, dtype: several units a block, packed and single, parts of key blocks
CALLS = [([300] * 40, 8, 2, 64, "bf16"), ([90] * 50 + [700], 8, 2, 128, "f16"),
         ([1024], 8, 1, 128, "bf16"), ([100, 2000], 8, 1, 64, "f16")]

PROGRAM = """
import os, sys
sys.path.insert(0, %r)
import torch
import paper_2609_06086_gb300 as P
from test_gpu_attn import Call

calls = [Call(P, lengths, *rest, behind=3) for lengths, *rest in %r]
out = []
for c in calls:
    for _ in range(3):
        for t in (c.o, c.lse, *c.dx):
            t.fill_(77)
        c.forward()
        torch.cuda.synchronize()
        forward = [t.clone() for t in (c.o, c.lse)]
        if len(sys.argv) > 2:  # the right forward pass's results, to see the backward pass alone
            for t, w in zip((c.o, c.lse), torch.load(sys.argv[2])[len(out) // 3]):
                t.copy_(w)
        c.backward()
        torch.cuda.synchronize()
        c.check_untouched()
        out.append([t[c.live].cpu() if t.shape[0] == c.T else t[:, c.live].cpu()
                    for t in (*forward, *c.dx)])
torch.save(out, sys.argv[1])
if "POSEIDON_ATTN_WAIT_NS" not in os.environ:
    torch.save([(c.o, c.lse) for c in calls], sys.argv[1] + ".forward")
"""


def results(tmp_path, name, limit=None, forward=None):
    env = {k: v for k, v in os.environ.items() if k != "POSEIDON_ATTN_WAIT_NS"}
    env["PYTHONPATH"] = os.path.dirname(HERE)
    if limit is not None:
        env["POSEIDON_ATTN_WAIT_NS"] = str(limit)
    import torch
    subprocess.run([sys.executable, "-c", PROGRAM % (HERE, CALLS), str(tmp_path / name)] +
                   ([forward] if forward else []), check=True, env=env, timeout=300)
    return torch.load(tmp_path / name)


def test_what_is_lost_is_nan(tmp_path):
    import torch
    right = results(tmp_path, "right")
    for run in right:
        assert all(torch.isfinite(t.double()).all() for t in run)
    forward = str(tmp_path / "right.forward")
    for limit in (0, 300, 1000, 3000, 10 ** 9):
        for first in (None, forward):
            lost = 0
            for i, run in enumerate(results(tmp_path, "lost", limit, first)):
                for k, (got, want) in enumerate(zip(run, right[i])):
                    nan = got.isnan()
                    assert torch.equal(got.masked_fill(nan, 0), want.masked_fill(nan, 0)), (limit, i, k)
                    lost += int(nan.sum())
            # (a try of no time may sleep long enough for some units all the same)
            assert lost > 0 if limit == 0 else limit < 10 ** 9 or lost == 0


def test_a_limit_that_is_no_number(tmp_path):
    """It counts as none given, not as no time."""
    import torch
    right = results(tmp_path, "right")
    for got, want in zip(results(tmp_path, "got", "2s"), right, strict=True):
        assert all(torch.equal(a, b) for a, b in zip(got, want, strict=True))
