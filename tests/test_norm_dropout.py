"""Norm and dropout without a GPU: refused arguments, the structs' layouts, and the
generator that the GPU tests compare with."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

import dropout_util as D

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


def test_generator_known_answers():
    """The published answers of Philox-4x32-10."""
    ones = 0xffffffff
    for counter, key, want in (
            ((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
            ((ones,) * 4, (ones,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
            ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0),
             (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))):
        assert D.philox(counter, key) == want


def test_mask_keeps_what_it_should():
    """64,000 elements at p = 0.25: the share that is kept is within five standard
    deviations, sqrt(0.25 * 0.75 / 64000) = 0.0017 each."""
    kept, factor = D.mask(range(8), 8000, 5, 6, 0.25)
    assert abs(kept.mean() - 0.75) < 5 * 0.0017 and factor == np.float32(4 / 3)


def test_dropout_refused(P):
    def call(p=0.1, rows=2, cols=8, x=P16, dtype=0, ldx=8, res=None, ldr=8, y=P16, dtype_y=0,
             ldy=8, d_offset=None, drop=True):
        d = P.pos_dropout(p, 1, 2, d_offset)
        return P.lib().poseidon_dropout(C.byref(d) if drop else None, rows, cols, x, dtype, ldx,
                                        res, ldr, y, dtype_y, ldy, None)

    refused(P, call(drop=False), "NULL")
    refused(P, call(x=None), "NULL")
    refused(P, call(y=None), "NULL")
    for p in (-0.1, 1.1, float("nan")):
        refused(P, call(p=p), "p must be")
    for over in (dict(rows=-1), dict(cols=-1), dict(rows=1 << 31), dict(cols=1 << 31)):
        refused(P, call(**over), "rows or cols")
    refused(P, call(dtype=3), "dtype")
    refused(P, call(dtype_y=-1), "dtype")
    for over in (dict(ldx=-1), dict(ldr=-1), dict(ldy=7), dict(ldx=1 << 31)):
        refused(P, call(**over), "stride")
    for over in (dict(x=ODD), dict(y=ODD), dict(res=ODD), dict(x=P16 + 2, dtype=2)):
        refused(P, call(**over), "aligned to its elements")
    refused(P, call(d_offset=P16 + 4), "d_offset")
    with pytest.raises(P.PoseidonError):
        P.poseidon_dropout(P.pos_dropout(2.0, 0, 0, 0), 1, 1, P16, 0, 1, 0, 0, P16, 0, 1)


def test_norm_refused(P):
    L = P.lib()

    def norm(**over):
        f = dict(rows=2, cols=8, dtype=0, dtype_h=0, format=0, eps=1e-6, w=P16)
        drop = P.pos_dropout(over.pop("p", 0.0), 0, 0, over.pop("d_offset", 0))
        f.update(over)
        return C.byref(P.pos_norm(*f.values(), drop))

    def forward(n, x=P16, ldx=8, res=P16, ldr=8, h=P16, ldh=8, y=P16, ldy=8, ch=None, cy=None,
                rstd=None):
        return L.poseidon_norm_forward(n, x, ldx, res, ldr, h, ldh, y, ldy, ch, cy, rstd, None)

    def backward(n, h=P16, ldh=8, ch=None, rstd=P16, dy=P16, lddy=8, add=P16, ldadd=8, dh=P16,
                 lddh=8, dx=P16, lddx=8, dw_in=None, dw=None):
        return L.poseidon_norm_backward(n, h, ldh, ch, rstd, dy, lddy, add, ldadd, dh, lddh, dx,
                                        lddx, dw_in, dw, None)

    for call in (forward, backward):
        refused(P, call(None), "NULL")
        for over, text in ((dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"),
                           (dict(cols=0), "cols"), (dict(cols=32769), "cols"),
                           (dict(dtype=4), "dtype"), (dict(dtype_h=1), "dtype_h"),
                           (dict(dtype=2, dtype_h=0), "dtype_h"), (dict(format=2), "format"),
                           (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"),
                           (dict(w=P16 + 2), "misaligned w"), (dict(p=1.5), "p must be"),
                           (dict(d_offset=P16 + 4), "d_offset")):
            refused(P, call(norm(**over)), text)
    refused(P, forward(norm(), x=None), "NULL x")
    for name in ("x", "res", "h", "y"):
        refused(P, forward(norm(), **{name: ODD}), "misaligned")
    for name in ("ldx", "ldr", "ldh", "ldy"):
        refused(P, forward(norm(), **{name: -1}), "row stride")
    for name in ("ldh", "ldy"):
        refused(P, forward(norm(), **{name: 7}), "row stride")
    for name in ("ch", "cy"):
        refused(P, forward(norm(), **{name: P16 + 8}), "16-byte")
    refused(P, forward(norm(), rstd=P16 + 2), "rstd")
    for name in ("h", "dy", "add", "dh", "dx"):
        refused(P, backward(norm(), **{name: ODD}), "misaligned")
    for name in ("lddh", "lddx"):
        refused(P, backward(norm(), **{name: 7}), "row stride")
    refused(P, backward(norm(), h=None), "neither h nor its checkpoint")
    refused(P, backward(norm(), ch=P16 + 8), "16-byte")
    refused(P, backward(norm(), rstd=None), "NULL rstd or dy")
    refused(P, backward(norm(), dy=None), "NULL rstd or dy")
    refused(P, backward(norm(), rstd=P16 + 2), "misaligned rstd")
    refused(P, backward(norm(), dw=P16 + 2), "misaligned dw")
    refused(P, backward(norm(), dw_in=P16), "dw_in without dw")


def test_struct_layouts(P, tmp_path):
    structs = {"pos_dropout": P.pos_dropout, "pos_norm": P.pos_norm}
    lines = ['#include <stdio.h>', '#include <stddef.h>',
             f'#include "{os.path.join(ROOT, "include", "poseidon.h")}"', "int main(void) {"]
    for name, cls in structs.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        for f, _ in cls._fields_:
            lines.append(f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));')
    lines += ["return 0;", "}"]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines))
    subprocess.run(["gcc", "-std=c99", "-o", str(tmp_path / "layout"), str(src)], check=True)
    got = dict(line.split() for line in subprocess.run(
        [str(tmp_path / "layout")], capture_output=True, text=True, check=True).stdout.splitlines())
    for name, cls in structs.items():
        assert int(got[name]) == C.sizeof(cls)
        for f, _ in cls._fields_:
            assert int(got[f"{name}.{f}"]) == getattr(cls, f).offset, (name, f)
