"""Poseidon's search hot path on one GB300: batched DAG-makespan evaluation,
memory feasibility, the stage-level prune and the exact search, in CUDA
kernels behind the C ABI of include/poseidon.h (libposeidon.so); and the
operators of a layer that keeps its activations in 8 bits between a
micro-batch's forward and backward pass.

The Python side is the ctypes binding in ``binding``; it loads the in-tree
library and never computes anything itself.
"""
from .binding import (  # noqa: F401
    EXPORTS, Handle, PoseidonError, Tables, lib, make_problem, pos_heads, pos_qk,
    poseidon_argmin, poseidon_ckpt_bytes, poseidon_ckpt_pack, poseidon_ckpt_unpack,
    poseidon_ckpt_wgrad, poseidon_eval_batch, poseidon_eval_batch_ex, poseidon_eval_batch_host,
    poseidon_qk_backward, poseidon_qk_forward, poseidon_search, qk_heads,
)
