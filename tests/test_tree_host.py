"""Host side of the attention of drafted trees, without a GPU: refusals,
workspaces against plans, and the bits of a tree."""
import ctypes as C
import random

import numpy as np
import pytest
import torch

from paper_2609_04263_amd import configs

from test_gather_plan import cache, status
from test_host_abi import FAKE, FakeStorage, kvq  # noqa: F401  (kvq: the fixture)
from test_shared_host import pair
from test_shared_workspace import FORMATS, log_int


def call(kvq, p, s, H_q=8, C_len=2, first=None, Q=FAKE, O=FAKE, ws=FAKE, nbytes=1 << 30, sm=0.125, tree=FAKE, **kw):
    arr = None if first is None else (C.c_int32 * len(first))(*first)
    return kvq.lib().kvq_tree_attn_shared(p and p.handle, s and s.handle, arr, Q, C_len, H_q, sm, tree, O, ws, nbytes, 0)


def test_refusals(kvq):
    p, s = pair(kvq)
    for kw in (dict(H_q=3), dict(H_q=34), dict(H_q=0), dict(C_len=0), dict(C_len=-1), dict(C_len=11), dict(Q=0), dict(O=0),
               dict(ws=0), dict(tree=0), dict(tree=FAKE + 2), dict(Q=FAKE + 8), dict(sm=float("nan")),
               dict(first=[0, 2, 3]), dict(first=[1, 2, 4]), dict(first=[0, 5, 4]), dict(C_len=1 << 27)):
        assert call(kvq, p, s, **kw) == kvq.ERR_ARG, kw
    assert call(kvq, None, s) == kvq.ERR_ARG and call(kvq, p, None) == kvq.ERR_ARG
    need = s.shared_workspace_bytes(p, 8, 2)
    assert call(kvq, p, s, nbytes=need - 1) == kvq.ERR_WORKSPACE
    assert call(kvq, p, pair(kvq, f2=configs.make_format(4, 4, k_group=32))[1]) == kvq.ERR_FORMAT
    assert (p.n, s.n) == (50, 10)


def test_bits_indexed_in_32_bits(kvq):
    f = configs.make_format()
    p, s = cache(kvq, f, 1, 1, 64, 1, n=0), cache(kvq, f, 1, 1, 64, 1 << 20, n=1 << 20, addr=FAKE + (1 << 40))
    assert call(kvq, p, s, H_q=1, C_len=1 << 18, nbytes=1 << 60) == kvq.ERR_ARG   # 2^18 rows of 2^13 words


def test_shapes(kvq):
    p, s = pair(kvq)
    q, w = FakeStorage(0), FakeStorage(1 << 30)
    for bad in (torch.zeros(4, 2, 2, dtype=torch.int32), torch.zeros(4, 2, 1, dtype=torch.int64),
                torch.zeros(4, 4, 1, dtype=torch.int32)[:, ::2]):
        with pytest.raises(ValueError):
            s.tree_attn_shared(p, q, 2, 8, 0.125, bad, q, w, stream=0)


def test_tree_words(kvq):
    rng = np.random.default_rng(0)
    B, n = 3, 70
    parents = np.stack([[rng.integers(-1, i) for i in range(n)] for _ in range(B)])
    parents[1, 50:] = -2  # no drafts
    got = kvq.tree_words(parents).numpy().view(np.uint32)
    assert got.shape == (B, n, 3)
    for b in range(B):
        for i in range(n):
            want, j = set(), i
            while j >= 0 and parents[b, i] > -2:
                want.add(j)
                j = int(parents[b, j])
            assert {j for j in range(96) if got[b, i, j // 32] >> (j % 32) & 1} == want
    for bad in ([[0]], [[-1, 1]], [[-1, 2, 0]]):
        with pytest.raises(ValueError):
            kvq.tree_words(bad)
    assert kvq.tree_words(torch.tensor([[-1, 0, 0]])).tolist() == [[[1], [3], [5]]]


@pytest.mark.parametrize("seed", range(len(FORMATS)))
def test_plans_fit_their_workspace(kvq, seed):
    f, D = FORMATS[seed]
    plan = kvq.lib().kvq_internal_tree_partials
    plan.argtypes, plan.restype = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int], C.c_size_t
    rng = random.Random(100 + seed)
    for _ in range(150):
        H, G, P = log_int(rng, 1, 8), rng.randint(1, 16), log_int(rng, 1, 256)
        B, n_p = log_int(rng, 1, 300), rng.choice([0, log_int(rng, 1, 40000)])
        p = cache(kvq, f, P, H, D, max(n_p, 1), n=n_p)
        s = cache(kvq, f, B, H, D, 3000, addr=FAKE + (1 << 44))
        cuts = sorted(rng.randint(0, B) for _ in range(P - 1))
        first = (C.c_int32 * (P + 1))(0, *cuts, B)
        most = log_int(rng, 1, 400)
        bytes_ = s.shared_workspace_bytes(p, H * G, most)
        for c in {1, most, rng.randint(1, most)}:
            s.restore(rng.choice([c, 3000, rng.randint(c, 3000)]))
            for kernels in range(3):
                parts = plan(p.handle, s.handle, first, c, H * G, kernels)
                assert parts * (D + 2) * 4 <= bytes_, (H, G, P, B, n_p, s.n, c, most, list(first), kernels)
                assert parts >= B * c * H * G
