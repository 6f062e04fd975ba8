"""Gathering sequences of packed caches on the GPU, byte for byte.

The expected image is made on the host from the images before the call and
the layout that kvq_cache_section reports: for every section, the live bytes
of (b, h) are those of (rows[b], h), and every other byte of the destination
is what it was (the destinations start as noise).
"""
import random

import numpy as np
import pytest
import torch

from paper_2609_04263_amd import configs, synth

from gpu_util import dev_bf16, image

pytestmark = pytest.mark.gpu

KIVI = configs.WORKLOADS["llama8b_kivi"].fmt
FORMATS = {
    "affine4": (configs.make_format(4, 4, k_group=32, v_group=64), 64),
    "kivi": (KIVI, 128),
    "kivi_meta16": (dict(KIVI, meta_fp16=1), 64),
    "had": (configs.WORKLOADS["llama8b_had"].fmt, 128),
    "bits8_d256": (configs.make_format(8, 8, k_group=64, v_group=128), 256),
    "sink": (configs.make_format(4, 2, k_mode=1, v_mode=1, k_group=64, v_group=32, rotate=128, sink=64), 128),
    "sink_window": (dict(KIVI, sink=32), 128),
}


def noise_cache(fmt, B, H, D, T, seed):
    from paper_2609_04263_amd import kvq
    n = kvq.cache_bytes(fmt, B, H, D, T)
    g = torch.Generator().manual_seed(seed)
    return kvq.Cache(fmt, B, H, D, T, storage=torch.randint(0, 256, (n,), dtype=torch.uint8, generator=g).cuda())


def filled(fmt, B, H, D, T, n, seed):
    c = noise_cache(fmt, B, H, D, T, seed)
    if n:
        K, V = synth.kv_tokens(seed, B, n, H, D)
        c.append(dev_bf16(K), dev_bf16(V))
    return c


def live_ranges(c, n):
    """(section, first byte, end) within a (sequence, head) slab of the first n tokens' bytes."""
    f, D = c.fmt, c.D
    tail = max(0, n - f.sink)
    nq = tail if not f.flush else max(0, tail - f.residual) // f.flush * f.flush
    T_alloc = (max(c.T_max - f.sink, 0) + 31) // 32 * 32
    out = []
    for s in range(6):
        if T_alloc and nq:
            per_block = c.section(s)[1] // (c.B * c.H) // (T_alloc // 32)
            out.append((s, 0, per_block * ((nq + 31) // 32)))
    ring = f.residual + f.flush
    for t in range(nq, tail if ring else nq):
        out += [(s, t % ring * 2 * D, (t % ring + 1) * 2 * D) for s in (6, 7)]
    out += [(s, 0, min(n, f.sink) * 2 * D) for s in (8, 9)]
    return out


def expected(src, src_img, dst, dst_img, rows, n):
    out = dst_img.copy()
    for s, lo, hi in live_ranges(src, n):
        (so, sl), (do, dl) = src.section(s), dst.section(s)
        if hi <= lo or sl == 0:
            continue
        a = src_img[so:so + sl].reshape(src.B, src.H, -1)
        b = out[do:do + dl].reshape(dst.B, dst.H, -1)
        for d, r in enumerate(rows):
            if r >= 0:
                b[d, :, lo:hi] = a[r, :, lo:hi]
    return out


def check(src, dst, rows, n=None, **kw):
    a, b = image(src), image(dst)
    m = src.n if n is None else n
    want = expected(src, a, dst, b, rows, m)
    dst.gather(src, rows, n, **kw)
    got = image(dst)
    assert dst.n == m
    assert np.array_equal(got, want), f"{(got != want).sum()} bytes differ"
    if dst is not src:
        assert np.array_equal(image(src), a), "the source changed"


@pytest.mark.parametrize("name", list(FORMATS))
@pytest.mark.parametrize("n", [1, 31, 33, 160, 161, 500])
def test_between_caches(name, n):
    fmt, D = FORMATS[name]
    src = filled(fmt, 3, 2, D, n + 5, n, seed=n)
    dst = noise_cache(fmt, 5, 2, D, n + 100, seed=n + 1)  # other B and capacity
    check(src, dst, [2, -1, 0, 0, 2])


@pytest.mark.parametrize("name", list(FORMATS))
@pytest.mark.parametrize("kind", ["swap", "cycle9", "beam", "shift", "mixed"])
def test_in_place(name, kind):
    fmt, D = FORMATS[name]
    B = 11
    rows = {"swap": [1, 0] + list(range(2, B)),
            "cycle9": [(b + 1) % 9 if b < 9 else b for b in range(B)],
            "beam": [0, 1, 2, 0, 4, 2, 2, 7, 4, 0, -1],
            "shift": [1, 2, 4, 5, 9, 10, -1, -1, -1, -1, -1],  # the survivors move to the front
            "mixed": [3, 3, 0, 1, 4, 10, 5, 6, -1, 7, 9]}[kind]
    n = 333
    c = filled(fmt, B, 2, D, n + 40, n, seed=5)
    check(c, c, rows)


def test_many_sequences_in_place_and_between():
    # several launches of 256 operations, and cycles longer than a launch
    fmt, D = configs.make_format(2, 2, k_group=64, v_group=64), 64
    B, n = 700, 40
    rng = random.Random(7)
    c = filled(fmt, B, 1, D, n, n, seed=6)
    check(c, c, [(b + 1) % B for b in range(B)])
    check(c, c, rng.sample(range(B), B))
    check(c, c, [rng.randrange(-1, B) for _ in range(B)])
    d = noise_cache(fmt, 900, 1, D, n, seed=8)
    check(c, d, [rng.randrange(-1, B) for _ in range(900)])


def test_shorter_copies():
    for name in ("affine4", "had", "sink"):
        fmt, D = FORMATS[name]
        src = filled(fmt, 2, 3, D, 300, 300, seed=9)
        for n in (0, 1, 40, 64, 65, 299):
            check(src, noise_cache(fmt, 3, 3, D, max(n, 1), seed=10), [1, 0, 1], n=n)
        check(src, src, [1, 0], n=77)  # in place, and shorter from then on


@pytest.mark.parametrize("name", list(FORMATS))
def test_a_copy_goes_on_like_its_source(name):
    """A forked sequence appended to equals a cache that had the tokens from the start."""
    fmt, D = FORMATS[name]
    H, n, m = 2, 150, 77
    K, V = synth.kv_tokens(20, 1, n, H, D)
    K2, V2 = synth.kv_tokens(21, 3, m, H, D)
    from paper_2609_04263_amd import kvq
    one = kvq.Cache(fmt, 1, H, D, n)
    one.append(dev_bf16(K), dev_bf16(V))
    fork = kvq.Cache(fmt, 3, H, D, n + m)
    fork.gather(one, [0, 0, 0])
    whole = kvq.Cache(fmt, 3, H, D, n + m)
    whole.append(dev_bf16(np.repeat(K, 3, 0)), dev_bf16(np.repeat(V, 3, 0)))
    assert fork.length() == whole.length()
    for c in (fork, whole):
        c.append(dev_bf16(K2), dev_bf16(V2))
    H_q = 2 * H
    Q = dev_bf16(synth.queries(22, 3, H_q, D))
    outs = []
    for c in (fork, whole):
        O = torch.empty((3, H_q, D), dtype=torch.float32, device="cuda")
        c.decode_attn(Q, H_q, D ** -0.5, O, c.decode_workspace(H_q))
        outs.append(O)
    torch.cuda.synchronize()
    assert torch.equal(*outs)
    a, b = image(fork), image(whole)
    for s, lo, hi in live_ranges(fork, n + m):  # (the window slots of tokens coded since are dead)
        off, ln = fork.section(s)
        va, vb = (x[off:off + ln].reshape(3, H, -1)[:, :, lo:hi] for x in (a, b))
        assert np.array_equal(va, vb), s


def test_capture_and_another_stream():
    fmt, D = FORMATS["kivi"]
    n = 333
    src = filled(fmt, 4, 2, D, n, n, seed=11)
    dst = noise_cache(fmt, 4, 2, D, n, seed=12)
    rows = [3, 1, 1, 0]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    check(src, dst, rows, stream=side)
    # a captured in-place rotation: every replay turns the batch once more
    start = image(src)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        src.gather(src, [1, 2, 3, 0])
    want = start
    for _ in range(5):
        want = expected(src, want, src, want.copy(), [1, 2, 3, 0], n)
        graph.replay()
        assert np.array_equal(image(src), want)
        check(src, dst, rows)  # eager work between the replays
