"""examples/stage_checkpoints.py: its schedule on the CPU, and the whole of it,
plan and stage, on the GPU with a small layer."""
import importlib.util
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    from paper_2609_06086_gb300 import build
    build.build()
    spec = importlib.util.spec_from_file_location(
        "stage_checkpoints", os.path.join(ROOT, "examples", "stage_checkpoints.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("stages,micro_batches", [(1, 1), (4, 8), (4, 2), (3, 3)])
def test_slots_of_the_schedule(example, stages, micro_batches):
    """Every micro-batch goes forward once, then backward once, and its slot,
    m modulo W_s, is free when it starts."""
    for stage in range(stages):
        w, order = example.one_f_one_b(stage, stages, micro_batches)
        assert w == min(stages - stage, micro_batches)
        held, done = {}, []
        for op, m in order:
            if op == "F":
                assert m % w not in held
                held[m % w] = m
            else:
                assert held.pop(m % w) == m
                done.append(m)
        assert done == list(range(micro_batches)) and not held


def test_checkpoints_take_about_half(example):
    plain, packed = example.kept_bytes(4096, (4096, 5120), (32, 8), 128)
    assert packed < 0.54 * plain


def test_memory_of_the_planned_layer(example):
    """What 8 bits save of 34 s h (2 s h the inputs of three linear operations, 8 s h the
    fourth's) and what the norm of q and k adds; q and k as attention reads them (2 s
    each of their widths) stay.  The plans' times are the oracle's."""
    import oracle
    s, h, width = 4096, 4096, (32 + 8) * 128
    plain, packed = example.workload(False), example.workload(True)
    saved = 14 * s * h - 7 * s * h * 33 // 32          # a byte and a scale of 32 instead of two
    norm = s * width * 33 // 32 + 4 * s * (32 + 8)     # their codes, scales and 1 / rms
    assert (plain.mem_a - packed.mem_a == saved - norm).all()
    times = [oracle.search(w, prune=False)[0]["T"] for w in (plain, packed)]
    assert times == [11078885, 10480313]


@pytest.mark.gpu
def test_plan_and_stage(example):
    """Smaller activations let the search find a faster plan, and the gradients
    differ from f32's by what rounding does: what is kept by at most 2^-7 of a
    group's largest magnitude, which is three to four times the values' root mean
    square here, evenly spread over that range at worst: 2^-7 * 4 / sqrt(3), 0.018;
    bf16's y, x and dy add 2^-9 each."""
    plan, leaner, off = example.main(["--layers", "1", "--seq", "512", "--hidden", "512",
                                      "--heads", "4", "2", "--micro-batches", "6"])
    assert leaner["T"] * plan["M"] < plan["T"] * leaner["M"]
    assert all(d < 0.018 + 3 * 2.0 ** -9 for pair in off for d in pair)
