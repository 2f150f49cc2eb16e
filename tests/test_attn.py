"""Attention without a GPU: refused arguments and the structs' layouts."""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P16, ODD = 1 << 20, (1 << 20) + 1  # addresses that are never read: a refusal comes first


@pytest.fixture(scope="module")
def P():
    from paper_2609_06086_gb300 import build
    build.build()
    import paper_2609_06086_gb300 as P
    P.lib()
    return P


def refused(P, status, text):
    assert status == P.binding.POS_EINVAL
    assert text in P.lib().poseidon_last_error().decode()


def attn(P, **over):
    f = dict(tokens=4, heads_q=4, heads_k=2, dim=8, dtype=0, scale=0.5, sequences=0, starts=None)
    f.update(over)
    return P.pos_attn(*f.values())


def triple(P, which=0, **over):
    """queries, keys, values of heads one after another; `over` in one of them"""
    f = [dict(data=P16, token=32, head=8), dict(data=P16, token=16, head=8),
         dict(data=P16, token=16, head=8)]
    f[which].update(over)
    return P.attn_heads(*(v for t in f for v in t.values()))


def calls(P):
    L, one = P.lib(), P.pos_heads(P16, 32, 8)

    def forward(a, x=triple(P), o=one, lse=None):
        return L.poseidon_attn_forward(C.byref(a) if a else None, x, o, lse, None)

    def backward(a, x=triple(P), o=one, lse=P16, d_o=one, dx=triple(P)):
        return L.poseidon_attn_backward(C.byref(a) if a else None, x, o, lse, d_o, dx, None)

    return forward, backward


BAD = ((dict(tokens=-1), "token count"), (dict(tokens=1 << 31), "token count"),
       (dict(heads_q=-1), "multiple"), (dict(heads_k=-1), "multiple"), (dict(heads_q=3), "multiple"),
       (dict(heads_k=0), "multiple"), (dict(heads_q=65537, heads_k=1), "multiple"),
       (dict(dim=0), "dim"), (dict(dim=129), "dim"), (dict(dtype=2), "bf16 or f16"),
       (dict(dtype=-1), "bf16 or f16"), (dict(scale=0.0), "scale"), (dict(scale=-1.0), "scale"),
       (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"),
       (dict(sequences=-1), "sequence count"), (dict(sequences=1 << 25), "sequence count"),
       (dict(starts=P16 + 2), "misaligned starts"))


@pytest.mark.parametrize("over,text", BAD)
def test_refused_descriptions(P, over, text):
    for call in calls(P):
        refused(P, call(attn(P, **over)), text)


def test_refused_tensors(P):
    forward, backward = calls(P)
    a = attn(P)
    for call in (forward, backward):
        refused(P, call(None), "NULL")
        refused(P, call(a, x=None), "NULL")
        refused(P, call(a, o=None), "NULL")
        refused(P, call(a, o=P.pos_heads(0, 32, 8)), "NULL o")
        refused(P, call(a, o=P.pos_heads(ODD, 32, 8)), "misaligned o")
        for which, name in enumerate(("queries", "keys", "values")):
            refused(P, call(a, x=triple(P, which, data=0)), "NULL the " + name)
            refused(P, call(a, x=triple(P, which, data=ODD)), "misaligned the " + name)
            refused(P, call(a, x=triple(P, which, token=-1)), "stride of the " + name)
            refused(P, call(a, x=triple(P, which, head=1 << 38)), "stride of the " + name)
    refused(P, forward(a, o=P.pos_heads(P16, 32, 4)), "overlapping rows of o")
    refused(P, forward(a, o=P.pos_heads(P16, 0, 8)), "overlapping rows of o")
    refused(P, forward(a, lse=P16 + 2), "misaligned lse")
    refused(P, backward(a, lse=None), "NULL lse")
    refused(P, backward(a, lse=P16 + 1), "misaligned lse")
    refused(P, backward(a, d_o=P.pos_heads(0, 32, 8)), "NULL o's gradient")
    refused(P, backward(a, d_o=None), "NULL")
    refused(P, backward(a, dx=None), "NULL")
    for which, name in enumerate(("queries", "keys", "values")):
        refused(P, backward(a, dx=triple(P, which, head=4)),
                "overlapping rows of the gradients of the " + name)
        refused(P, backward(a, dx=triple(P, which, data=ODD)),
                "misaligned the gradients of the " + name)
    with pytest.raises(P.PoseidonError):
        P.poseidon_attn_forward(attn(P, dim=0), triple(P), P.pos_heads(P16, 32, 8))
    with pytest.raises(ValueError):
        P.poseidon_attn_forward(a, [P.pos_heads(P16, 32, 8)], P.pos_heads(P16, 32, 8))


def test_triples_of_pos_heads(P):
    """Three pos_heads, as a sequence or an array, mean what attn_heads() does."""
    from paper_2609_06086_gb300 import binding
    t = [P.pos_heads(1, 2, 3), P.pos_heads(4, 5, 6), P.pos_heads(7, 8, 9)]
    want = bytes(P.attn_heads(1, 2, 3, 4, 5, 6, 7, 8, 9))
    for x in (t, tuple(t), (P.pos_heads * 3)(*t)):
        assert bytes(binding._triple(x)) == want


def test_struct_layout(P, tmp_path):
    lines = ['#include <stdio.h>', '#include <stddef.h>',
             f'#include "{os.path.join(ROOT, "include", "poseidon.h")}"', "int main(void) {",
             'printf("size %zu\\n", sizeof(pos_attn));']
    for f, _ in P.pos_attn._fields_:
        lines.append(f'printf("{f} %zu\\n", offsetof(pos_attn, {f}));')
    lines += ["return 0;", "}"]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines))
    subprocess.run(["gcc", "-std=c99", "-o", str(tmp_path / "layout"), str(src)], check=True)
    got = dict(line.split() for line in subprocess.run(
        [str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout.splitlines())
    assert int(got["size"]) == C.sizeof(P.pos_attn)
    for f, _ in P.pos_attn._fields_:
        assert int(got[f]) == getattr(P.pos_attn, f).offset, f
