"""Calls over a shared prefix stay within the workspace that they ask for.

The size comes from a bound for any lengths, groups and fewer queries; what a
call writes is (D + 2) floats per partial of its plan.  Plans of many calls are
compared with the bound on the host, and a few calls with the memory behind
their workspace.
"""
import ctypes as C
import random

import pytest

from paper_2609_04263_amd import configs

from test_gather_plan import cache
from test_host_abi import FAKE, kvq  # noqa: F401  (kvq: the fixture)

FORMATS = [(configs.make_format(k_group=32), D) for D in (64, 128, 256)]
FORMATS += [(configs.make_format(8, 8, k_group=64), 64), (configs.make_format(k_group=64, sink=64), 128),
            (configs.make_format(4, 2, k_mode=1, v_mode=1, k_group=128, v_group=32, rotate=128), 128),
            (configs.WORKLOADS["llama8b_kivi"].fmt, 128), (configs.WORKLOADS["llama8b_kivi"].fmt, 256)]


def log_int(rng, lo, hi):
    return min(hi, int(lo * (hi / lo) ** rng.random() + 0.5))


@pytest.mark.parametrize("seed", range(len(FORMATS)))
def test_plans_fit_their_workspace(kvq, seed):
    f, D = FORMATS[seed]
    plan = kvq.lib().kvq_internal_shared_partials
    plan.argtypes, plan.restype = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int], C.c_size_t
    rng = random.Random(seed)
    for _ in range(150):
        H, G, P = log_int(rng, 1, 8), rng.randint(1, 16), log_int(rng, 1, 256)
        B, n_p = log_int(rng, 1, 300), rng.choice([0, log_int(rng, 1, 40000)])
        p = cache(kvq, f, P, H, D, max(n_p, 1), n=n_p)
        s = cache(kvq, f, B, H, D, 3000, addr=FAKE + (1 << 44))
        cuts = sorted(rng.randint(0, B) for _ in range(P - 1))
        first = (C.c_int32 * (P + 1))(0, *cuts, B)
        most = log_int(rng, 1, 400)  # the workspace is one of calls of up to so many queries
        bytes_ = s.shared_workspace_bytes(p, H * G, most)
        for c in {1, most, rng.randint(1, most)}:
            s.restore(rng.choice([c, 3000, rng.randint(c, 3000)]))
            for kernels in range(3):
                assert plan(p.handle, s.handle, first, c, H * G, kernels) * (D + 2) * 4 <= bytes_, \
                    (H, G, P, B, n_p, s.n, c, most, list(first), kernels)


@pytest.mark.gpu
@pytest.mark.parametrize("first", [[0, 1], [0, 2, 3], [0, 40], [0, 7, 64]])
@pytest.mark.parametrize("name", ["tiny_b16", "kivi", "gqa12b", "hadamard"])
def test_nothing_is_written_behind_the_workspace(name, first):
    import torch
    from test_gpu_append import CASES
    from test_gpu_shared import call, filled
    from paper_2609_04263_amd import synth
    fmt, D = CASES[name]
    B, H_q = first[-1], 8
    prefix = filled(fmt, len(first) - 1, 2, D, 3000, 90, "prefix")
    suffix = filled(fmt, B, 2, D, 100, 91, "suffix")
    for c in (1, 6):
        Q = synth.queries(92, B * c, H_q, D).reshape(B, c, H_q, D)
        need = suffix.gpu.shared_workspace_bytes(prefix.gpu, H_q, c)
        memory = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        for kernels in range(3):
            call(prefix, suffix, first, Q, D ** -0.5, ws=memory[:need], chunk=c > 1, kernels=kernels)
            assert (memory[need:] == 0xA5).all()
