"""Attention of drafted trees against 64-bit attention over the oracle's
reconstruction of both caches.  Bounds as in test_gpu_shared.py: the same
products, summed in the same steps."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2609_04263_amd import synth

from gpu_util import dev_bf16
from test_gpu_append import CASES
from test_gpu_shared import GUARD, close, filled, hadamard

pytestmark = pytest.mark.gpu


def words_of(sees):
    B, C, _ = sees.shape
    bits = np.zeros((B, C, -(-C // 32) * 32), np.uint64)
    bits[:, :, :C] = sees
    return (bits.reshape(B, C, -1, 32) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32).view(np.int32)


def random_tree(B, C, seed, padded=True):
    rng = synth.stream(seed, "tree")
    sees = np.zeros((B, C, C), bool)
    for b in range(B):
        for i in range(C):
            parent = int(rng.integers(-1, i)) if i else -1
            if parent >= 0:
                sees[b, i] = sees[b, parent]
            sees[b, i, i] = True
        if padded and b % 2:
            sees[b, C - C // 3:] = False
    return sees


def reference(prefix, suffix, first, Q, sm, sees):
    """fp64 [B, C, H_q, D]; rows that see nothing are zeros."""
    fmt, D = prefix.ref.fmt, prefix.ref.D
    B, C, H_q, _ = Q.shape
    H = prefix.ref.H
    q = synth.bf16_bits_to_f32(Q).astype(np.float64)
    if fmt["rotate"]:
        q = q @ hadamard(D)
    q = q.reshape(B, C, H, H_q // H, D)
    kp, vp = prefix.dequant()
    ks, vs = suffix.dequant()
    n = kp.shape[2] + ks.shape[2]
    out = np.zeros((B, C, H, H_q // H, D))
    for g in range(len(first) - 1):
        for b in range(first[g], first[g + 1]):
            k, v = np.concatenate([kp[g], ks[b]], 1), np.concatenate([vp[g], vs[b]], 1)
            for c in range(C):
                keep = np.concatenate([np.ones(n - C, bool), sees[b, c]])
                if not keep.any():
                    continue
                s = sm * np.einsum("hgd,htd->hgt", q[b, c], k[:, keep])
                p = np.exp(s - s.max(-1, keepdims=True))
                out[b, c] = np.einsum("hgt,htd->hgd", p / p.sum(-1, keepdims=True), v[:, keep])
    out = out.reshape(B, C, H_q, D)
    return out @ hadamard(D) if fmt["rotate"] else out


def call_kernel(prefix, suffix, first, Q, H_q, C, sm, tree, O, ws, kernels):
    from paper_2609_04263_amd import kvq
    f = kvq._lib.kvq_internal_tree_attn
    V, I = ctypes.c_void_p, ctypes.c_int
    f.argtypes = [V, V, V, V, I, I, ctypes.c_float, V, V, V, ctypes.c_size_t, V, I]
    arr = None if first is None else (ctypes.c_int32 * len(first))(*first)
    assert f(prefix.handle, suffix.handle, arr, Q.data_ptr(), C, H_q, sm, tree.data_ptr(), O.data_ptr(), ws.data_ptr(),
             ws.numel(), torch.cuda.current_stream().cuda_stream, kernels) == 0


def call(prefix, suffix, first, Q, sm, tree, kernels=0, **kw):
    """The output of a call, with the floats around it and the memory behind its workspace checked."""
    B, C, H_q, D = Q.shape
    s, p = suffix.gpu, prefix.gpu
    flat = torch.full((Q.size + 2 * GUARD,), 7.5, dtype=torch.float32, device="cuda")
    O = flat[GUARD:-GUARD]
    need = s.shared_workspace_bytes(p, H_q, C)
    memory = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")
    ws, dq = memory[:need], dev_bf16(Q)
    if kernels:
        call_kernel(p, s, first, dq, H_q, C, sm, tree, O, ws, kernels)
    else:
        s.tree_attn_shared(p, dq, C, H_q, sm, tree, O, ws, first=first, **kw)
    torch.cuda.synchronize()
    assert (flat[:GUARD] == 7.5).all() and (flat[-GUARD:] == 7.5).all() and (memory[need:] == 255).all()
    return O.view(B, C, H_q, D)


def run(name, first, n_p, n_s, C, G=4, H=2, seed=0, sm=None, sees=None):
    fmt, D = CASES[name]
    P, B = len(first) - 1, first[-1]
    prefix = filled(fmt, P, H, D, n_p, seed + 1, "prefix")
    suffix = filled(fmt, B, H, D, n_s, seed + 2, "suffix")
    H_q = H * G
    Q = synth.queries(seed + 3, B * C, H_q, D).reshape(B, C, H_q, D)
    sees = random_tree(B, C, seed) if sees is None else sees
    tree = torch.from_numpy(words_of(sees)).cuda()
    sm0 = D ** -0.5
    sm = sm0 if sm is None else sm
    want = reference(prefix, suffix, first, Q, sm, sees)
    empty = ~sees.any(-1) & (n_p + n_s == C)
    for k in (0, 1, 2):
        got = call(prefix, suffix, first, Q, sm, tree, k)
        assert not got[torch.from_numpy(empty).cuda()].any()
        close(got, want, max(1.0, abs(sm) / sm0), f"{name} first={first} n={n_p}+{n_s} G={G} C={C} kernels={k}")
    return prefix, suffix, Q, tree, got


@pytest.mark.parametrize("name", list(CASES))
@pytest.mark.parametrize("C,n_s", [(1, 1), (5, 5), (8, 165), (37, 70), (100, 131)])
def test_formats(name, C, n_s):
    run(name, [0, 1, 3], 290, n_s, C, seed=C + n_s)


@pytest.mark.parametrize("C", [1, 2, 31, 32, 33, 63, 64, 65, 96, 129, 300])
@pytest.mark.parametrize("name", ["tiny_b16", "kivi", "gqa12b"])
def test_numbers_of_drafts(name, C):
    # words and blocks of the tree, at any offset in the cache's blocks
    for n_s in (C, C + 1, C + 31, C + 47):
        run(name, [0, 2], 40, n_s, C, G=2, H=1, seed=C)


@pytest.mark.parametrize("name", ["tiny_b16", "kivi", "hadamard", "gqa12b", "kvarn_sink", "sink32_window"])
@pytest.mark.parametrize("C,n_s", [(7, 7), (7, 300), (40, 40)])
def test_one_cache(name, C, n_s):
    run(name, [0, 3], 0, n_s, C, seed=8)


@pytest.mark.parametrize("name", ["tiny_b16", "kivi", "hadamard"])
def test_rows_that_see_nothing(name):
    C = 45
    sees = random_tree(3, C, 5)
    sees[0] = False
    sees[1, ::2] = False
    run(name, [0, 3], 0, C, C, seed=9, sees=sees)
    run(name, [0, 3], 50, C, C, seed=9, sees=sees)


@pytest.mark.parametrize("name", ["tiny_b16", "kivi", "gqa12b"])
def test_any_pattern(name):
    # not only trees: all, none of the earlier ones, later ones, the ends of the words
    C = 67
    rng = synth.stream(6, "pattern")
    sees = rng.random((4, C, C)) < 0.5
    sees[1] = True
    sees[2] = np.triu(np.ones((C, C), bool))
    sees[3] = False
    sees[3, :, [0, 31, 32, 63, 64, 66]] = True
    run(name, [0, 1, 4], 100, 80, C, seed=10, sees=sees)


@pytest.mark.parametrize("name", ["kvarn_sink", "sink32_window", "sink64"])
@pytest.mark.parametrize("n_s", [1, 31, 32, 33, 63, 64, 127, 128, 129, 160, 200])
def test_drafts_in_the_sink(name, n_s):
    run(name, [0, 2], 150, n_s, min(n_s, 40), seed=11)
    run(name, [0, 2], 0, n_s, min(n_s, 33), seed=12)


@pytest.mark.parametrize("n_s", [100, 128, 129, 159, 160, 161, 191, 192, 700])
def test_drafts_in_and_before_the_window(n_s):
    run("kivi", [0, 2], 200, n_s, 90, seed=13)
    run("kivi", [0, 2], 200, n_s, 10, seed=14)


@pytest.mark.parametrize("G", [1, 2, 3, 7, 16])
@pytest.mark.parametrize("name", ["tiny_b16", "kivi", "hadamard", "gqa12b"])
def test_head_groups(name, G):
    run(name, [0, 1, 4], 321, 65, 9, G=G, seed=20 + G)


@pytest.mark.parametrize("first", [[0, 0, 5], [0, 5, 5], [0, 0, 0, 2, 2, 3, 3], [0, 1], [0, 33]])
def test_groups_with_and_without_sequences(first):
    run("tiny_b16", first, 200, 40, 6, H=1, seed=30)


@pytest.mark.parametrize("name", ["tiny_b16", "gqa12b", "hadamard"])
def test_enough_work_for_the_image_kernel(name):
    run(name, [0, 12], 1700, 40, 40, G=16, H=1, seed=31)
    run(name, [0, 2], 0, 2300, 64, G=16, H=1, seed=32)


def test_peaked_flat_and_negative_scales():
    for sm in (4.0, 1e-4, -0.1, 0.0):
        run("tiny_b16", [0, 3], 400, 50, 20, sm=sm, seed=33)


@pytest.mark.parametrize("name", ["tiny_b16", "kivi", "gqa12b", "hadamard"])
def test_a_chain_is_the_causal_chunk(name):
    fmt, D = CASES[name]
    C, n_s = 40, 70
    sees = np.tril(np.ones((3, C, C), bool))
    prefix, suffix, Q, tree, got = run(name, [0, 1, 3], 290, n_s, C, seed=34, sees=sees)
    O = torch.empty(Q.shape, dtype=torch.float32, device="cuda")
    s, p = suffix.gpu, prefix.gpu
    s.prefill_attn_shared(p, dev_bf16(Q), C, Q.shape[2], D ** -0.5, O, s.shared_workspace(p, Q.shape[2], C), first=[0, 1, 3])
    torch.cuda.synchronize()
    close(got, O.double().cpu().numpy(), 2.0)


def test_the_same_bits_every_time_captured_and_on_another_stream():
    fmt, D = CASES["kivi"]
    C, first = 20, [0, 2, 5]
    prefix, suffix, Q, tree, _ = run("kivi", first, 700, 60, C, seed=35)
    s, p, H_q = suffix.gpu, prefix.gpu, Q.shape[2]
    other = torch.from_numpy(words_of(random_tree(5, C, 77))).cuda()
    sm, dq, ws = D ** -0.5, dev_bf16(Q), s.shared_workspace(p, H_q, C)
    want = [call(prefix, suffix, first, Q, sm, t) for t in (tree, other)]
    O, bits = torch.empty(Q.shape, dtype=torch.float32, device="cuda"), tree.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    s.tree_attn_shared(p, dq, C, H_q, sm, bits, O, ws, first=first, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(O, want[0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.tree_attn_shared(p, dq, C, H_q, sm, bits, O, ws, first=first)
    for t, w in ((other, want[1]), (tree, want[0]), (other, want[1])):  # (the bits are read when the graph runs)
        bits.copy_(t)
        O.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, w)
        assert torch.equal(call(prefix, suffix, first, Q, sm, t), w)


def test_default_groups():
    fmt, D = CASES["tiny_b16"]
    prefix, suffix, Q, tree, _ = run("tiny_b16", [0, 2, 4, 6], 100, 10, 7, seed=36)
    assert torch.equal(call(prefix, suffix, None, Q, D ** -0.5, tree), call(prefix, suffix, [0, 2, 4, 6], Q, D ** -0.5, tree))
