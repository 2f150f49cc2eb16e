"""The layer operators without a GPU: refused arguments, checkpoint sizes, the
structs' layouts, and the definitions that the GPU tests compare with."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

import layer_util as U

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


@pytest.mark.parametrize("rows,cols", [(0, 0), (1, 1), (3, 32), (7, 33), (5, 128), (5, 129),
                                       (4096, 5120), (1 << 31, 8192)])
def test_checkpoint_bytes(P, rows, cols):
    groups = (cols + 31) // 32
    assert P.poseidon_ckpt_bytes(rows, cols) == rows * (32 * groups + 4 * ((groups + 3) // 4))


def test_checkpoint_sizes_refused(P):
    L, out = P.lib(), C.c_int64()
    for rows, cols in ((-1, 4), (4, -1), (1, 1 << 31), (1 << 62, 1)):
        refused(P, L.poseidon_ckpt_bytes(rows, cols, C.byref(out)), "rows or cols")
    refused(P, L.poseidon_ckpt_bytes(1, 1, None), "NULL")


def test_pack_and_unpack_refused(P):
    L = P.lib()
    pack = lambda x=P16, dtype=0, rows=2, cols=8, ld=8, fmt=0, c=P16: \
        L.poseidon_ckpt_pack(x, dtype, rows, cols, ld, fmt, c, None)  # noqa: E731
    refused(P, pack(x=None), "NULL")
    refused(P, pack(c=None), "NULL")
    refused(P, pack(c=P16 + 8), "16-byte")
    refused(P, pack(x=ODD), "aligned to its elements")
    refused(P, pack(dtype=3), "dtype")
    refused(P, pack(fmt=-1), "format")
    refused(P, pack(rows=-1), "rows")
    refused(P, pack(ld=-1), "stride")
    unpack = lambda ld: L.poseidon_ckpt_unpack(P16, 0, 2, 8, P16, 0, ld, None)  # noqa: E731
    refused(P, unpack(7), "stride")  # rows that are written would overlap
    with pytest.raises(P.PoseidonError):
        P.poseidon_ckpt_pack(0, 0, 1, 1, 1, 0, P16)


def test_wgrad_refused(P):
    L = P.lib()

    def wgrad(ckpt=P16, fmt=0, dy=P16, dtype=0, ld_dy=8, rows=2, n=8, cols=8, add=None, out=P16,
              ld=8):
        return L.poseidon_ckpt_wgrad(ckpt, fmt, dy, dtype, ld_dy, rows, n, cols, add, out, ld, None)

    refused(P, wgrad(ckpt=None), "NULL")
    refused(P, wgrad(dy=None), "NULL")
    refused(P, wgrad(out=None), "NULL")
    refused(P, wgrad(ckpt=P16 + 8), "16-byte")
    refused(P, wgrad(dy=ODD), "aligned to its elements")
    refused(P, wgrad(out=P16 + 2), "aligned to its elements")
    refused(P, wgrad(add=P16 + 2), "aligned to its elements")
    refused(P, wgrad(dtype=2), "bf16 or f16")
    refused(P, wgrad(fmt=2), "format")
    refused(P, wgrad(ld=7), "stride")
    refused(P, wgrad(ld_dy=-1), "stride")
    for size in ("rows", "n", "cols"):
        refused(P, wgrad(**{size: -1}), "bad rows")
        refused(P, wgrad(**{size: 1 << 31}), "bad rows")


def test_qk_refused(P):
    L = P.lib()

    def qk(**over):
        f = dict(tokens=2, heads_q=2, heads_k=1, dim=8, rot=8, pairing=0, dtype=0, format=0,
                 eps=1e-6, w_q=None, w_k=None, cos=P16, sin=P16, n_pos=4, positions=None)
        f.update(over)
        return P.pos_qk(*f.values())

    t = P.qk_heads(P16, 24, 8, P16, 24, 8)

    def forward(q, x=t, y=t, ckpt=None):
        return L.poseidon_qk_forward(C.byref(q) if q else None, x, y, None, None, ckpt, None, None)

    def backward(q, x=t, ckpt=None, r=P16, dy=t, dx=t, add=None, dw=None):
        return L.poseidon_qk_backward(C.byref(q), x, ckpt, ckpt, r, r, dy, dx, add, dw, None)

    refused(P, forward(None), "NULL")
    for call in (forward, backward):
        for over, text in ((dict(tokens=-1), "count"), (dict(heads_q=-1), "count"),
                           (dict(dim=0), "dim"), (dict(dim=257), "dim"), (dict(rot=3), "rot"),
                           (dict(rot=10), "rot"), (dict(pairing=2), "pairing"),
                           (dict(dtype=5), "dtype"), (dict(format=2), "format"),
                           (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"),
                           (dict(n_pos=-1), "n_pos"), (dict(cos=None), "tables")):
            refused(P, call(qk(**over)), text)
    refused(P, forward(qk(), x=None), "NULL x")
    refused(P, forward(qk(), x=P.qk_heads(P16, 24, 8, 0, 24, 8)), "NULL x")
    refused(P, forward(qk(), x=P.qk_heads(ODD, 24, 8, P16, 24, 8)), "misaligned x")
    refused(P, forward(qk(), x=P.qk_heads(P16, -8, 8, P16, 24, 8)), "stride of x")
    refused(P, forward(qk(), y=P.qk_heads(P16, 24, 4, P16, 24, 8)), "overlapping rows of y")
    refused(P, forward(qk(), y=P.qk_heads(P16, 0, 8, P16, 24, 8)), "overlapping rows of y")
    refused(P, forward(qk(), ckpt=P16 + 8), "16-byte")
    refused(P, backward(qk(), x=None), "neither x nor its checkpoint")
    refused(P, backward(qk(), r=None), "NULL rstd")
    refused(P, backward(qk(), add=P16), "dw_in without dw")
    refused(P, backward(qk(), dx=P.qk_heads(P16, 24, 0, P16, 24, 8)), "overlapping rows of dx")


def test_qk_misaligned_refused(P):
    """Weights, tables, positions, rstd and dw off their elements."""
    t = P.qk_heads(P16, 24, 8, P16, 24, 8)
    for name in ("w_q", "w_k", "cos", "sin", "positions"):
        f = dict(tokens=2, heads_q=2, heads_k=1, dim=8, rot=8, pairing=0, dtype=0, format=0,
                 eps=1e-6, w_q=P16, w_k=P16, cos=P16, sin=P16, n_pos=4, positions=P16)
        f[name] += 2
        refused(P, P.lib().poseidon_qk_forward(C.byref(P.pos_qk(*f.values())), t, t, None, None,
                                               None, None, None), "misaligned weights, tables")
        f[name] -= 2
    q = C.byref(P.pos_qk(*f.values()))

    def forward(rq=P16, rk=P16):
        return P.lib().poseidon_qk_forward(q, t, t, rq, rk, None, None, None)

    def backward(rq=P16, rk=P16, add=P16, dw=P16):
        return P.lib().poseidon_qk_backward(q, t, None, None, rq, rk, t, t, add, dw, None)

    for call in (forward, backward):
        refused(P, call(rq=P16 + 2), "misaligned rstd")
        refused(P, call(rk=ODD), "misaligned rstd")
    refused(P, backward(add=P16 + 2), "misaligned dw")
    refused(P, backward(dw=P16 + 2), "misaligned dw")


@pytest.mark.parametrize("make", [lambda P, q, k: (P.pos_heads * 2)(q, k), lambda P, q, k: (q, k),
                                  lambda P, q, k: [q, k]])
def test_pairs_of_pos_heads(P, make):
    """Both q/k calls take two pos_heads as they take qk_heads(): every field arrives,
    which the refusal of one field after another shows."""
    q = P.pos_qk(2, 2, 1, 8, 8, 0, 0, 0, 1e-6, None, None, P16, P16, 4, None)
    good = make(P, P.pos_heads(P16, 24, 8), P.pos_heads(P16, 24, 8))
    for over, text in ((dict(), "16-byte"), (dict(q=(ODD, 24, 8)), "misaligned"),
                       (dict(q=(P16, -1, 8)), "stride"), (dict(q=(P16, 24, 4)), "overlapping"),
                       (dict(k=(ODD, 24, 8)), "misaligned"), (dict(k=(P16, 0, 8)), "overlapping"),
                       (dict(k=(P16, 24, -1)), "stride")):
        f = dict(q=(P16, 24, 8), k=(P16, 24, 8))
        f.update(over)
        t = make(P, *(P.pos_heads(*v) for v in f.values()))
        for x, y in ((good, t), (t, t)):
            with pytest.raises(P.PoseidonError, match=text):
                P.poseidon_qk_forward(q, x, y, ckpt=(P16 + 8, 0))
            with pytest.raises(P.PoseidonError, match=text):
                P.poseidon_qk_backward(q, x, t, (P16, P16), x=x, ckpt=(P16 + 8, 0))
    with pytest.raises(ValueError):
        P.poseidon_qk_forward(q, [P.pos_heads(P16, 24, 8)], good)


@pytest.mark.parametrize("seed", range(3))
def test_written_rows_that_overlap_are_refused(P, seed):
    """Against all pairs of rows, for small shapes and strides; the checkpoint that is
    refused next shows that a tensor whose rows are apart got past."""
    rng = np.random.default_rng(seed)
    met = set()
    for _ in range(400):
        tokens, heads, dim = (int(v) for v in rng.integers(1, 6, 3))
        ts, hs = (int(v) for v in rng.integers(0, 24, 2))
        starts = sorted(i * ts + j * hs for i in range(tokens) for j in range(heads))
        apart = all(b - a >= dim for a, b in zip(starts, starts[1:]))
        met.add(apart)
        q = P.pos_qk(tokens, heads, 0, dim, 0, 0, 0, 0, 1e-6, None, None, None, None, 0, None)
        t = P.qk_heads(P16, ts, hs, 0, 0, 0)
        refused(P, P.lib().poseidon_qk_forward(C.byref(q), t, t, None, None, P16 + 8, None, None),
                "16-byte" if apart else "overlapping rows of y")
    assert met == {True, False}


def test_struct_layouts(P, tmp_path):
    structs = {"pos_qk": P.pos_qk, "pos_heads": P.pos_heads}
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


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_the_definition_by_its_properties(fmt):
    """The tests' own encoder: codes stand for values within half a step of a
    group's largest code, the largest magnitude fits, the next smaller scale
    would not hold it, and kept values are kept again unchanged."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((40, 70)) * np.exp(rng.uniform(-60, 60, (40, 1)))
    x[3] = 0
    codes, scales = U.encode(x, fmt)
    v = U.decode(codes, scales, 70, fmt)
    top = 127.0 if fmt == "int8" else 448.0
    e = np.repeat(scales.astype(int) - 127, 32, 1)[:, :70]
    step = 2.0 ** e if fmt == "int8" else 2.0 ** e * 32
    assert (np.abs(v - x) <= step / 2).all()
    for g in range(3):
        a, s = np.abs(x[:, 32 * g:32 * g + 32]).max(1), scales[:, g].astype(int) - 127
        assert (a <= top * 2.0 ** s).all()
        assert ((a > top * 2.0 ** (s - 1)) | (s == -110)).all()
    assert np.array_equal(U.kept(v, fmt), v)
    assert (codes[:, 70:] == 0).all()
