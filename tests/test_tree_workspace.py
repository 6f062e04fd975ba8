"""The workspace of calls behind a shared prefix: those without a tree take what they
write and no more, and one that is enough for drafted trees has a partial more for
every row, or, where a row has many, as many."""
import ctypes
import random

import numpy as np
import pytest
import torch

from paper_2609_04263_amd import configs, synth

from test_gather_plan import cache
from test_host_abi import FAKE, kvq  # noqa: F401  (kvq: the fixture)
from test_shared_workspace import log_int


WORKLOADS = {"tiny_b16": (configs.WORKLOADS["tiny_b16"].fmt, 64), "kivi": (configs.WORKLOADS["llama8b_kivi"].fmt, 128),
             "gqa12b": (configs.WORKLOADS["gqa12b_b8"].fmt, 256)}


def partials(B, H, D, C, G):
    """Partials of calls without trees: of either cache one per row, or what a round of workgroups of the image kernel
    (256 of 256 rows, 128 at D = 256) or the direct one (512 of 32, 16) is cut into."""
    def segment(units, u):
        return max(units * u, 256 * min(u, 128 if D == 256 else 256), 512 * min(u, 16 if D == 256 else 32))
    return segment(H, B * C * G) + segment(B * H, C * G)


def nbytes(parts, D):
    return -(-parts * D * 4 // 256) * 256 + parts * 8


def test_sizes(kvq):
    rng = random.Random(1)
    f, more = configs.make_format(k_group=32), 0
    for _ in range(400):
        D, H, G = rng.choice((64, 128, 256)), log_int(rng, 1, 16), rng.randint(1, 16)
        B, C = log_int(rng, 1, 300), log_int(rng, 1, 2000)
        p = cache(kvq, f, 1, H, D, 100, n=50)
        s = cache(kvq, f, B, H, D, 100, n=10, addr=FAKE + (1 << 44))
        parts, rows = partials(B, H, D, C, G), B * C * H * G
        few = parts < 64 * rows
        assert s.shared_workspace_bytes(p, H * G, C) == nbytes(parts + few * rows, D)
        more += few
    assert 40 < more < 360


@pytest.mark.gpu
@pytest.mark.parametrize("name,B,C,G", [("tiny_b16", 8, 512, 8), ("gqa12b", 8, 512, 4)])
def test_calls_of_many_rows(name, B, C, G):
    # each with the least workspace that it takes, and nothing behind it written
    from paper_2609_04263_amd import kvq
    from test_gpu_append import CASES
    from test_gpu_shared import close
    fmt, D = CASES[name]
    H, H_q, n_p, n_s = 2, 2 * G, 100, C + 45
    parts, rows = partials(B, H, D, C, G), B * C * H_q
    assert parts < 64 * rows
    gen = torch.Generator(device="cuda").manual_seed(3)
    p, s = kvq.Cache(fmt, 1, H, D, n_p), kvq.Cache(fmt, B, H, D, n_s)
    for c, n in ((p, n_p), (s, n_s)):
        c.append(*(torch.randn((c.B, n, H, D), generator=gen, device="cuda").bfloat16() for _ in "kv"))
    Q = torch.randn((B, C, H_q, D), generator=gen, device="cuda").bfloat16()
    chain = np.tril(np.ones((C, C), bool))
    words = (chain.reshape(C, -1, 32).astype(np.uint64) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32)
    tree = torch.from_numpy(words.view(np.int32)).cuda().expand(B, -1, -1).contiguous()
    need = {"causal": nbytes(parts, D), "tree": nbytes(parts + rows, D)}
    assert s.shared_workspace_bytes(p, H_q, C) == need["tree"]
    out = {}
    for kind in need:
        memory = torch.full((need[kind] + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        O = out[kind] = torch.empty(Q.shape, dtype=torch.float32, device="cuda")

        def call(n, **kw):
            ws = memory[:n]
            if kind == "tree":
                s.tree_attn_shared(p, Q, C, H_q, D ** -0.5, tree, O, ws, **kw)
            else:
                s.prefill_attn_shared(p, Q, C, H_q, D ** -0.5, O, ws, **kw)
        with pytest.raises(kvq.KvqError) as e:
            call(need[kind] - 1)
        assert e.value.status == kvq.ERR_WORKSPACE
        call(need[kind])
        torch.cuda.synchronize()
        assert (memory[need[kind]:] == 0xA5).all()
    close(out["tree"], out["causal"].double().cpu().numpy(), 2.0)
    one = torch.empty((B, H_q, D), dtype=torch.float32, device="cuda")
    ws = torch.empty(nbytes(partials(B, H, D, 1, G), D), dtype=torch.uint8, device="cuda")
    s.decode_attn_shared(p, Q[:, -1].contiguous(), H_q, D ** -0.5, one, ws)
    torch.cuda.synchronize()
    close(one[:, None], out["causal"][:, -1:].double().cpu().numpy(), 2.0)


# (B, H, G, C and lengths that cut either cache into 64 ranges: the drafts' partial takes the place of some)
FULL = [("tiny_b16", 1, 8, 16, 2, 8192, 8194), ("kivi", 1, 8, 8, 2, 8192, 8194), ("gqa12b", 2, 4, 8, 2, 8192, 8194)]


@pytest.mark.parametrize("name,B,H,G,C,n_p,n_s", FULL)
def test_plans_give_up_a_range(kvq, name, B, H, G, C, n_p, n_s):
    fmt, D = WORKLOADS[name]
    plan = kvq.lib().kvq_internal_tree_partials
    plan.argtypes, plan.restype = [ctypes.c_void_p] * 3 + [ctypes.c_int] * 3, ctypes.c_size_t
    p = cache(kvq, fmt, B, H, D, n_p, n=n_p)
    s = cache(kvq, fmt, B, H, D, n_s, n=n_s, addr=FAKE + (1 << 44))
    first, rows = (ctypes.c_int32 * (B + 1))(*range(B + 1)), B * C * H * G
    assert partials(B, H, D, C, G) == 128 * rows
    assert plan(p.handle, s.handle, first, C, H * G, 0) < 129 * rows
    s.restore(n_s - 200)
    assert plan(p.handle, s.handle, first, C, H * G, 0) <= 128 * rows


@pytest.mark.gpu
@pytest.mark.parametrize("name,B,H,G,C,n_p,n_s", FULL)
def test_trees_that_give_up_a_range(name, B, H, G, C, n_p, n_s):
    import test_gpu_tree as trees
    trees.run(name, list(range(B + 1)), n_p, n_s, C, G=G, H=H, seed=40)
