"""Shared-prefix attention of small and large queries.

Queries times a power of two with the softmax scale divided by it are the same
attention, and every step of it is the same but for exponents: the results
have to be equal bit for bit.
"""
import pytest
import torch

from paper_2609_04263_amd import configs, synth

from test_gpu_append import CASES
from test_gpu_shared import call, close, filled, reference

pytestmark = pytest.mark.gpu

NAMES = ["tiny_b1", "tiny_b16", "kivi", "kivi_meta16", "gqa12b", "hadamard", "perch_k4v2_window64", "had_affine_window",
         "perch8_meta16", "affine8", "kvarn_sink", "sink32_window", "sink64"]
MORE = {
    "kivi_d256": (dict(configs.WORKLOADS["llama8b_kivi"].fmt), 256),
    "had_perch_window": (configs.make_format(4, 2, k_axis=1, k_group=32, v_group=32, residual=32, flush=32,
                                             rotate=128), 128),
}


@pytest.mark.parametrize("first,C", [([0, 3], 1), ([0, 33], 1), ([0, 2], 20)])
@pytest.mark.parametrize("name", NAMES + list(MORE))
def test_queries_of_any_size(name, first, C):
    fmt, D = {**CASES, **MORE}[name]
    H, B = 2, first[-1]
    prefix = filled(fmt, 1, H, D, 333, 80, "prefix")
    suffix = filled(fmt, B, H, D, 70, 81, "suffix")
    Q = synth.queries(82, B * C, 2 * H, D).reshape(B, C, 2 * H, D)
    sm = D ** -0.5
    want = reference(prefix, suffix, first, Q, sm)
    for k in range(3):
        base = call(prefix, suffix, first, Q, sm, chunk=C > 1, kernels=k)
        close(base, want, what=f"kernels={k}")
        for power in (-60, -24, -10, -4, 9, 40):
            scaled = synth.to_bf16_bits(synth.bf16_bits_to_f32(Q) * 2.0 ** power)
            got = call(prefix, suffix, first, scaled, sm * 2.0 ** -power, chunk=C > 1, kernels=k)
            assert torch.equal(got, base), f"kernels={k} power={power}: {(got - base).abs().max()}"


@pytest.mark.parametrize("name", ["tiny_b16", "kivi", "gqa12b", "hadamard"])
def test_queries_of_zero_weigh_every_token_alike(name):
    fmt, D = CASES[name]
    prefix, suffix = filled(fmt, 1, 2, D, 200, 83, "prefix"), filled(fmt, 3, 2, D, 50, 84, "suffix")
    Q = synth.queries(85, 3, 4, D).reshape(3, 1, 4, D)
    for zeros in (slice(0, 3), slice(1, 2)):  # all rows, and rows beside others
        Q[zeros] = 0
        want = reference(prefix, suffix, [0, 3], Q, D ** -0.5)
        for k in range(3):
            close(call(prefix, suffix, [0, 3], Q, D ** -0.5, kernels=k), want, what=f"kernels={k}")
