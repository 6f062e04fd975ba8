"""Attention over a shared prefix and own suffixes against 64-bit attention
over the oracle's reconstruction of both caches.

Bound.  The matrix products are exact (binary16 operands, hi + lo where a value
has more bits: 22 of them) and sums are binary32.  A score sums D / 32 products
of 32 channels and up to D / 32 scaled groups, at most 16 steps at D = 256, each
off by 2^-24 of a partial sum of at most |q| |k| sm, which with four outlier
channels of 20 is about sm sqrt(D) sqrt(1 + 4 * 400 / D) <= 5 natural units, and
the codes' centre up to eight times that.  Taken as random that is 4 * 2^-25 * 40 =
5e-6, and an output, an average of values weighted by e^score, is off by as much
relatively; its own sums add as much again.  2^-14 = 6e-5 of the norm leaves a
factor of six; without the lo half of an operand the error would be 2^-12.  A
larger softmax scale scales it.
"""
import ctypes

import numpy as np
import pytest
import torch

import oracle
from paper_2609_04263_amd import configs, synth

from gpu_util import dev_bf16, image
from test_gpu_append import CASES

pytestmark = pytest.mark.gpu


def hadamard(D):
    h = np.ones((1, 1))
    while h.shape[0] < D:
        h = np.block([[h, h], [h, -h]])
    return h / np.sqrt(D)


class Pair:
    """A cache on the GPU, over storage full of NaN, and in the oracle."""

    def __init__(self, fmt, B, H, D, T):
        from paper_2609_04263_amd import kvq
        n = kvq.cache_bytes(fmt, B, H, D, T)
        self.gpu = kvq.Cache(fmt, B, H, D, T, storage=torch.full((n,), 255, dtype=torch.uint8, device="cuda"))
        self.ref = oracle.Cache(fmt, B, H, D, T)

    def append(self, K, V):
        if K.shape[1]:
            self.gpu.append(dev_bf16(K), dev_bf16(V))
            self.ref.append(K, V)
        return self

    def dequant(self):
        return self.ref.dequant()


def filled(fmt, B, H, D, n, seed, name, spare=8):
    outlier = ("student_t", 3.0) if fmt["rotate"] else ("scale", 4, 20.0)
    return Pair(fmt, B, H, D, n + spare).append(*synth.kv_tokens(seed, B, n, H, D, outlier=outlier, name=name))


def reference(prefix, suffix, first, Q, sm):
    """fp64 [B, C, H_q, D]."""
    fmt, D = prefix.ref.fmt, prefix.ref.D
    B, C, H_q, _ = Q.shape
    H = prefix.ref.H
    q = synth.bf16_bits_to_f32(Q).astype(np.float64)
    if fmt["rotate"]:
        q = q @ hadamard(D)
    q = q.reshape(B, C, H, H_q // H, D)
    kp, vp = prefix.dequant()
    ks, vs = suffix.dequant()
    n_p, n_s = kp.shape[2], ks.shape[2]
    out = np.zeros((B, C, H, H_q // H, D))
    for g in range(len(first) - 1):
        for b in range(first[g], first[g + 1]):
            k, v = np.concatenate([kp[g], ks[b]], 1), np.concatenate([vp[g], vs[b]], 1)
            for c in range(C):
                t = n_p + (n_s - C + c + 1 if n_s else 0)
                s = sm * np.einsum("hgd,htd->hgt", q[b, c], k[:, :t])
                p = np.exp(s - s.max(-1, keepdims=True))
                out[b, c] = np.einsum("hgt,htd->hgd", p / p.sum(-1, keepdims=True), v[:, :t])
    out = out.reshape(B, C, H_q, D)
    return out @ hadamard(D) if fmt["rotate"] else out


GUARD = 64


def call_kernel(prefix, suffix, first, Q, H_q, C, sm, O, ws, chunk, kernels):
    """The same call by one of the two kernels alone (1: direct, 2: image)."""
    from paper_2609_04263_amd import kvq
    f = kvq._lib.kvq_internal_shared_attn
    V, I = ctypes.c_void_p, ctypes.c_int
    f.argtypes = [V, V, V, V, I, I, ctypes.c_float, V, V, ctypes.c_size_t, I, V, I]
    arr = None if first is None else (ctypes.c_int32 * len(first))(*first)
    assert f(prefix.handle, suffix.handle, arr, Q.data_ptr(), C, H_q, sm, O.data_ptr(), ws.data_ptr(), ws.numel(),
             int(chunk), torch.cuda.current_stream().cuda_stream, kernels) == 0


def call(prefix, suffix, first, Q, sm, chunk=None, ws=None, kernels=0, **kw):
    """The output of a shared call, with the floats around it checked."""
    B, C, H_q, D = Q.shape
    s, p = suffix.gpu, prefix.gpu
    flat = torch.full((Q.size + 2 * GUARD,), 7.5, dtype=torch.float32, device="cuda")
    O = flat[GUARD:-GUARD]
    if ws is None:
        ws = s.shared_workspace(p, H_q, C)
        ws.fill_(255)
    dq = dev_bf16(Q)
    if chunk is None:
        chunk = C > 1
    if kernels:
        call_kernel(p, s, first, dq, H_q, C, sm, O, ws, chunk, kernels)
    elif chunk:
        s.prefill_attn_shared(p, dq, C, H_q, sm, O, ws, first=first, **kw)
    else:
        s.decode_attn_shared(p, dq, H_q, sm, O, ws, first=first, **kw)
    torch.cuda.synchronize()
    assert (flat[:GUARD] == 7.5).all() and (flat[-GUARD:] == 7.5).all()
    return O.view(B, C, H_q, D)


def close(got, want, factor=1.0, what=""):
    got, tol = got.double().cpu().numpy(), 2.0 ** -14 * factor
    assert np.isfinite(got).all(), what
    err = np.linalg.norm(got - want, axis=-1)  # per row
    norm = np.linalg.norm(want, axis=-1)
    rms = np.sqrt((norm ** 2).mean())
    assert np.sqrt((err ** 2).mean()) <= tol * rms, (what, np.sqrt((err ** 2).mean()) / rms)
    # a single row: its own norm may be small beside its values', whose average it is
    assert (err <= 8 * tol * np.maximum(norm, rms)).all(), (what, (err / np.maximum(norm, rms)).max())


def run(name, first, n_p, n_s, G=4, H=2, C=1, seed=0, sm=None, chunk=None):
    fmt, D = CASES[name]
    P, B = len(first) - 1, first[-1]
    prefix = filled(fmt, P, H, D, n_p, seed + 1, "prefix")
    suffix = filled(fmt, B, H, D, n_s, seed + 2, "suffix")
    H_q = H * G
    Q = synth.queries(seed + 3, B * C, H_q, D).reshape(B, C, H_q, D)
    sm0 = D ** -0.5
    sm = sm0 if sm is None else sm
    got = call(prefix, suffix, first, Q, sm, chunk)
    want = reference(prefix, suffix, first, Q, sm)
    for k, o in ((0, got), (1, call(prefix, suffix, first, Q, sm, chunk, kernels=1)),
                 (2, call(prefix, suffix, first, Q, sm, chunk, kernels=2))):
        close(o, want, max(1.0, sm / sm0), f"{name} first={first} n={n_p}+{n_s} G={G} C={C} kernels={k}")
    return prefix, suffix, Q, got


@pytest.mark.parametrize("name", list(CASES))
@pytest.mark.parametrize("n_p,n_s", [(1, 1), (33, 31), (257, 70), (1500, 200)])
def test_decode(name, n_p, n_s):
    run(name, [0, 3, 5], n_p, n_s, seed=n_p)


@pytest.mark.parametrize("name", list(CASES))
def test_decode_of_many_samples(name):
    # groups of 36 and 124 rows
    run(name, [0, 9, 40], 1500, 70, seed=3)


@pytest.mark.parametrize("G,count", [(2, 16), (3, 11), (2, 32), (5, 13), (16, 8), (15, 9), (16, 16), (15, 18)])
@pytest.mark.parametrize("name", ["tiny_b16", "gqa12b", "hadamard"])
def test_rows_around_whole_tiles(name, G, count):
    # one to sixteen tiles and a row more, of one wave, several and all of a workgroup
    run(name, [0, count, 2 * count], 700, 40, G=G, H=1, seed=4)


@pytest.mark.parametrize("C,n_s", [(40, 40), (3, 70)])
def test_enough_work_for_the_image_kernel(C, n_s):
    # 480 tiles of 54 blocks; the suffix has units of 640 rows, and of 48
    first = [0, 4 * (120 // C)]
    run("gqa12b", first, 1700, n_s, G=16, H=1, C=C, seed=5)


@pytest.mark.parametrize("name", list(CASES))
@pytest.mark.parametrize("C,n_s", [(5, 5), (5, 165), (37, 70), (130, 131)])
def test_chunk(name, C, n_s):
    run(name, [0, 1, 3], 290, n_s, C=C, seed=C + n_s)


@pytest.mark.parametrize("name", ["tiny_b16", "kivi", "hadamard", "gqa12b", "kvarn_sink", "sink32_window"])
@pytest.mark.parametrize("n_p,n_s", [(0, 1), (0, 300), (300, 0), (1, 0)])
def test_one_side_empty(name, n_p, n_s):
    run(name, [0, 2, 3], n_p, n_s, seed=9)


@pytest.mark.parametrize("name", ["tiny_b16", "kivi", "gqa12b"])
def test_empty_prefix_is_decode_attention(name):
    fmt, D = CASES[name]
    prefix, suffix, Q, got = run(name, [0, 3], 0, 411, seed=10)
    O = torch.empty((3, 8, D), dtype=torch.float32, device="cuda")
    suffix.gpu.decode_attn(dev_bf16(Q[:, 0]), 8, D ** -0.5, O, suffix.gpu.decode_workspace(8))
    torch.cuda.synchronize()
    close(got[:, 0], O.double().cpu().numpy(), 2.0)


@pytest.mark.parametrize("G", [1, 2, 3, 7, 16])
@pytest.mark.parametrize("name", ["tiny_b16", "kivi", "hadamard", "gqa12b"])
def test_head_groups_and_group_sizes(name, G):
    # rows of a group from one to several tiles, odd and even
    run(name, [0, 1, 12], 321, 65, G=G, seed=20 + G)


@pytest.mark.parametrize("first", [[0, 0, 5], [0, 5, 5], [0, 0, 0, 2, 2, 3, 3], [0, 1], [0, 33], [0, 70]])
def test_groups_with_and_without_sequences(first):
    run("tiny_b16", first, 200, 40, H=1, seed=30)


def test_equal_groups_by_default():
    prefix, suffix, Q, got = run("tiny_b16", [0, 2, 4, 6], 100, 10, seed=31)
    assert torch.equal(call(prefix, suffix, None, Q, 64 ** -0.5), got)


def test_the_most_prefixes():
    # as many as a call takes, groups of zero to two sequences
    first = [0]
    for g in range(256):
        first.append(first[-1] + g % 3)
    run("tiny_b16", first, 40, 5, H=1, G=2, seed=32)


@pytest.mark.parametrize("name", ["tiny_b1", "kivi", "gqa12b", "hadamard"])
def test_many_splits(name):
    # one group of few rows and a long prefix: as many splits as there are CUs for
    run(name, [0, 2], 9001, 33, H=1, seed=33)


@pytest.mark.parametrize("name", ["tiny_b16", "gqa12b", "hadamard"])
def test_one_split_per_tile(name):
    # more tiles than a round of workgroups: nothing is split, waves walk several blocks
    run(name, [0, 40, 80, 120, 160], 700, 300, H=2, G=16, seed=34)


@pytest.mark.parametrize("n_s", [1, 31, 32, 33, 127, 128, 129, 160, 200])
@pytest.mark.parametrize("name", ["kvarn_sink", "sink32_window", "sink64"])
def test_sinks_of_both_caches(name, n_s):
    run(name, [0, 2], 150, n_s, C=min(n_s, 40), chunk=True, seed=35)
    run(name, [0, 2], n_s, 150, C=3, seed=36)


@pytest.mark.parametrize("n_s", [100, 128, 129, 159, 160, 161, 191, 192, 700])
def test_kivi_window_boundaries(n_s):
    run("kivi", [0, 2], n_s, 200, seed=37)
    run("kivi", [0, 2], 200, n_s, C=100, seed=38)


@pytest.mark.parametrize("name", ["tiny_b16", "kivi", "hadamard"])
def test_peaked_flat_and_negative_scales(name):
    for sm in (4.0, 1e-4, -0.1, 0.0):
        run(name, [0, 3], 400, 50, sm=sm, seed=39)


def ramp(D, n, span, lo, total):
    """r_t u of tokens lo .. lo + n - 1 of `total`: logits climb by span from the first to the last."""
    u = np.where(np.arange(D) % 2 == 0, 1.0, -1.0)
    t = (lo + np.arange(n)) / (total - 1)
    return (abs(span) / np.sqrt(D) * (t if span > 0 else 1 - t))[:, None] * u


@pytest.mark.parametrize("span", [40.0, -40.0])
@pytest.mark.parametrize("name", ["tiny_b16", "kivi", "gqa12b"])
def test_the_largest_scores_on_one_side(name, span):
    """The suffix (or the prefix) holds all of the weight: partials far apart, many rescales."""
    fmt, D = CASES[name]
    n_p, n_s, H, B = 1111, 257, 2, 4
    caches = []
    for n, U, lo, nm in ((n_p, 1, 0, "p"), (n_s, B, n_p, "s")):
        K, V = synth.kv_tokens(41, U, n, H, D, name=nm)
        K = synth.to_bf16_bits(synth.bf16_bits_to_f32(K) + ramp(D, n, span, lo, n_p + n_s)[None, :, None, :])
        caches.append(Pair(fmt, U, H, D, n).append(K, V))
    u = np.where(np.arange(D) % 2 == 0, 1.0, -1.0).astype(np.float32)
    Q = synth.queries(42, B, 2 * H, D).reshape(B, 1, 2 * H, D)
    Q = synth.to_bf16_bits(synth.bf16_bits_to_f32(Q) * np.float32(0.25) + u)
    # (partial sums of these scores reach 8 (40 + 5) units: nine times the bound's)
    want = reference(*caches, [0, B], Q, D ** -0.5)
    for k in range(3):
        close(call(*caches, [0, B], Q, D ** -0.5, kernels=k), want, 9.0, f"kernels={k}")


@pytest.mark.parametrize("first", [[0, 3], [0, 33]])
@pytest.mark.parametrize("name", [n for n in CASES if n in ("tiny_b1", "tiny_b16", "kivi", "gqa12b", "hadamard", "sink64")
                                  or CASES[n][0]["k_bits"] == 8])
def test_values_of_all_magnitudes(name, first):
    """Runs of tokens whose values are tiny, large, all equal and zero: blocks whose scales are far apart."""
    fmt, D = CASES[name]
    caches = []
    for n, U, nm in ((777, 1, "p"), (301, first[-1], "s")):
        K, V = synth.kv_tokens(45, U, n, 2, D, name=nm)
        f = synth.bf16_bits_to_f32(V) * np.repeat(np.float32([1, 1e-6, 300, 0, 1e-3, 1e-20]), 37)[
            np.arange(n) % 222][None, :, None, None]
        f[:, 100:140] = 3.0
        caches.append(Pair(fmt, U, 2, D, n).append(K, synth.to_bf16_bits(f.astype(np.float32))))
    Q = synth.queries(46, first[-1], 8, D).reshape(first[-1], 1, 8, D)
    want = reference(*caches, first, Q, D ** -0.5)
    for k in range(3):
        close(call(*caches, first, Q, D ** -0.5, kernels=k), want, what=f"kernels={k}")


@pytest.mark.parametrize("first", [[0, 3], [0, 33]])
@pytest.mark.parametrize("name", ["tiny_b16", "gqa12b", "hadamard"])
def test_values_beside_enormous_ones(name, first):
    """Powers of two of blocks further apart than one binary32 number reaches (fp32 metadata, no fp16 tokens)."""
    fmt, D = CASES[name]
    caches = []
    for n, U, nm in ((300, 1, "p"), (200, first[-1], "s")):
        K, V = synth.kv_tokens(49, U, n, 2, D, name=nm)
        f = synth.bf16_bits_to_f32(V) * np.where(np.arange(n) // 64 % 2 == 0, np.float32(1e32), np.float32(0))[
            None, :, None, None]
        caches.append(Pair(fmt, U, 2, D, n).append(K, synth.to_bf16_bits(f.astype(np.float32))))
    Q = synth.queries(50, first[-1], 8, D).reshape(first[-1], 1, 8, D)
    want = reference(*caches, first, Q, D ** -0.5)
    for k in range(3):
        close(call(*caches, first, Q, D ** -0.5, kernels=k), want, what=f"kernels={k}")


@pytest.mark.parametrize("first", [[0, 3], [0, 33]])
@pytest.mark.parametrize("name", ["tiny_b16", "kivi", "hadamard"])
def test_values_of_zero(name, first):
    fmt, D = CASES[name]
    caches = []
    for n, U in ((300, 1), (200, first[-1])):
        K, V = synth.kv_tokens(47, U, n, 2, D)
        caches.append(Pair(fmt, U, 2, D, n).append(K, np.zeros_like(V)))
    Q = synth.queries(48, first[-1], 8, D).reshape(first[-1], 1, 8, D)
    # An affine token of zeros has the least scale, 1e-8, and is 1e-8 (c - mid) + 1e-8 mid with c = 0 and mid
    # <= 7.5.  Both terms are taken with a weight rounded to 22 bits and summed in binary32 (some 2^-24 of a
    # partial sum per step): they cancel to 2^-20 of one of them.
    for k in range(3):
        assert (call(*caches, first, Q, D ** -0.5, kernels=k).abs() <= 2.0 ** -20 * 7.5e-8).all(), k


def test_same_bits_every_time_and_after_a_larger_call():
    prefix, suffix, Q, got = run("hadamard", [0, 5, 9], 777, 99, seed=43)
    ws = suffix.gpu.shared_workspace(prefix.gpu, 8, 30)  # larger than needed, dirty
    ws.fill_(255)
    for _ in range(3):
        assert torch.equal(call(prefix, suffix, [0, 5, 9], Q, 128 ** -0.5, ws=ws), got)
    side = torch.cuda.Stream()
    assert torch.equal(call(prefix, suffix, [0, 5, 9], Q, 128 ** -0.5, stream=side), got)


@pytest.mark.parametrize("C", [1, 16, 17, 32])
def test_a_workspace_of_more_queries(C):
    # fewer rows are cut into more ranges
    prefix, suffix, Q, got = run("tiny_b16", [0, 1], 9000, 50, G=1, H=1, C=C, chunk=True, seed=51)
    ws = suffix.gpu.shared_workspace(prefix.gpu, 1, 33)
    ws.fill_(255)
    assert torch.equal(call(prefix, suffix, [0, 1], Q, 64 ** -0.5, chunk=True, ws=ws), got)


@pytest.mark.parametrize("name,C", [("kivi", 1), ("tiny_b16", 20), ("hadamard", 1)])
def test_captured_calls_replay(name, C):
    fmt, D = CASES[name]
    prefix, suffix, Q, got = run(name, [0, 2, 5], 500, 77, C=C, seed=44)
    dq, H_q = dev_bf16(Q), Q.shape[2]
    outs = [torch.zeros_like(got) for _ in range(2)]
    wss = [suffix.gpu.shared_workspace(prefix.gpu, H_q, C) for _ in range(2)]
    graphs = []
    for O, ws in zip(outs, wss):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            suffix.gpu.prefill_attn_shared(prefix.gpu, dq, C, H_q, D ** -0.5, O, ws, first=[0, 2, 5])
        graphs.append(g)
    for i in range(4):
        for O, g in zip(outs, graphs):
            O.zero_()
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(O, got) for O in outs), i
        assert torch.equal(call(prefix, suffix, [0, 2, 5], Q, D ** -0.5), got)


@pytest.mark.parametrize("kernels", [1, 2])
@pytest.mark.parametrize("name", ["kivi", "gqa12b"])
def test_each_kernel_replays_beside_another_graph(name, kernels):
    """Two captured calls of one kernel, each with a workspace of its own, replayed at once on two streams."""
    fmt, D = CASES[name]
    prefix, suffix, Q, _ = run(name, [0, 20], 700, 77, C=3, seed=52)
    want = call(prefix, suffix, [0, 20], Q, D ** -0.5, kernels=kernels)
    dq, H_q, C = dev_bf16(Q), Q.shape[2], 3
    outs, graphs = [], []
    for _ in range(2):
        O, ws = torch.zeros_like(want), suffix.gpu.shared_workspace(prefix.gpu, H_q, C)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call_kernel(prefix.gpu, suffix.gpu, [0, 20], dq, H_q, C, D ** -0.5, O, ws, True, kernels)
        outs.append(O)
        graphs.append((g, ws, torch.cuda.Stream()))
    for i in range(4):
        for O in outs:
            O.zero_()
        torch.cuda.synchronize()
        for g, _, stream in graphs:
            with torch.cuda.stream(stream):
                g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(O, want) for O in outs), i


@pytest.mark.parametrize("name", ["tiny_b1", "kivi", "gqa12b", "hadamard", "sink32_window"])
def test_serving_a_prompt_with_samples(name):
    """The calls together, as a sampling loop makes them: two prompts, three samples each behind them, the
    samples' own prompt in one chunk, decode steps, a beam reorder in place, steps, the survivors in a smaller
    batch, steps.  Every output is checked against attention over what each sequence has seen."""
    fmt, D = CASES[name]
    H, G, n_p, C, T = 2, 2, 200, 45, 90
    H_q, sm = H * G, D ** -0.5
    from paper_2609_04263_amd import kvq
    prefix = filled(fmt, 2, H, D, n_p, 50, "prompt", spare=0)
    suffix, first, step = Pair(fmt, 6, H, D, T), [0, 3, 6], [100]

    def new(count):
        step[0] += 1
        B = suffix.gpu.B
        suffix.append(*synth.kv_tokens(step[0], B, count, H, D))
        Q = synth.queries(step[0], B * count, H_q, D).reshape(B, count, H_q, D)
        close(call(prefix, suffix, first, Q, sm), reference(prefix, suffix, first, Q, sm), what=f"step {step[0]}")

    def as_gathered(ref, rows, T_max):
        """The oracle's cache of the chosen sequences: their images put together."""
        out = oracle.Cache(fmt, len(rows), H, D, T_max)
        for i in range(10):
            if ref.lengths[i]:
                a = ref.section(i).reshape(ref.B, H, -1)
                b = out.image[out.offsets[i]:out.offsets[i] + out.lengths[i]].reshape(len(rows), H, -1)
                b[:] = a[rows]
        out.n = ref.n
        return out
    new(C)
    for _ in range(3):
        new(1)
    rows = [1, 1, 0, 4, 3, 4]  # beams of a prompt take over each other's caches
    suffix.gpu.gather(suffix.gpu, rows)
    suffix.ref = as_gathered(suffix.ref, rows, T)
    for _ in range(2):
        new(1)
    rows, first = [0, 2, 5], [0, 2, 3]  # three go on, in a smaller cache
    small = Pair(fmt, 3, H, D, T)
    small.gpu.gather(suffix.gpu, rows)
    small.ref = as_gathered(suffix.ref, rows, T)
    suffix = small
    for _ in range(20):
        new(1)
    assert suffix.gpu.n == C + 25
    assert kvq.SCRATCH_BYTES  # (the binding is the one under test)
