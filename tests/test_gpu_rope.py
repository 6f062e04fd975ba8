"""Positions and per-head norms (kvq_rope_qk), and appends of keys that take
them on the way (kvq_append_rope).

Bounds.  The result is one bf16 rounding (half a step, 2^-8 of the value) of a
binary32 evaluation whose roundings are 2^-24 each: of r, x r, (x r) w, the two
products, their sum, c and s, at most 7 of them on each term |a c| + |b s|.  So
|out - exact| <= 2^-8 |exact| + 2^-21 (|a c| + |b s|).  Against the documented
steps evaluated with extended angles the bits are the same unless a cosine, sine
or r falls within 2^-53 of a binary32 border (1 in 10^8) and the bf16 rounding
within that step of its own (1 in 10^4): no difference is allowed for.
"""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_04263_amd import configs, synth

from gpu_util import dev_bf16, host_bits, image
from rope_ref import steps, wide
from test_gpu_append import CASES

pytestmark = pytest.mark.gpu

GUARD = 256


def guarded(shape):
    """A bf16 tensor with numbers around it that nobody may touch."""
    n = int(np.prod(shape))
    flat = torch.full((n + 2 * GUARD,), 7.5, dtype=torch.bfloat16, device="cuda")
    return flat, flat[GUARD:GUARD + n].view(shape)


def untouched(flat):
    return bool((flat[:GUARD] == 7.5).all() and (flat[-GUARD:] == 7.5).all())


def weights(seed, name, D):
    return synth.to_bf16_bits(1 + 0.3 * synth.stream(seed, name).standard_normal(D).astype(np.float32))


def positions(kind, B, n, seed):
    if kind == "consecutive":
        return None, 1000, 1000 + np.arange(n)[None].repeat(B, 0)
    g = synth.stream(seed, "pos")
    if kind == "far":
        p = g.integers(0, 2 ** 31 - 1, (B, n))
    elif kind == "zero":
        p = np.zeros((B, n), np.int64)
    else:
        p = g.integers(-3000, 200000, (B, n))
    return torch.from_numpy(p.astype(np.int32)).cuda(), 5, p


def check(B, n, H_q, H, D, rot, interleaved=False, norm=0, kind="mixed", scale=None, eps=1e-6, seed=7, in_place=False):
    from paper_2609_04263_amd import kvq
    rope = kvq.Rope(rot, 500000.0 if rot > 64 else 10000.0, interleaved=interleaved, scale=scale, eps=eps)
    turns = np.array(rope.c.turns[:rot // 2])
    pos, pos0, at = positions(kind, B, n, seed)
    w = [weights(seed, k, D) if norm & (i + 1) else None for i, k in enumerate("qk")]
    ins = [synth.normal_bf16(seed, (k, "rows"), (B, n, h, D)) if h else None for k, h in zip("qk", (H_q, H))]
    dev = [None if x is None else dev_bf16(x) for x in ins]
    flats, outs = zip(*[(None, None) if x is None else guarded(x.shape) for x in ins])
    if in_place:
        for o, d in zip(outs, dev):
            if o is not None:
                o.copy_(d)
        dev, given = list(outs), (None, None)
    else:
        given = outs
    rope.qk(*dev, *given, *[None if x is None else dev_bf16(x) for x in w], pos=pos, pos0=pos0)
    for x, weight, o, flat in zip(ins, w, outs, flats):
        if x is None:
            continue
        got = host_bits(o)
        assert untouched(flat)
        m = 1.0 if scale is None else scale
        ref, size = wide(x, weight, eps, turns, rot, interleaved, at, m)
        err = np.abs(synth.bf16_bits_to_f32(got).astype(np.float64) - ref)
        assert (err <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -21 * size).all(), (err - 2.0 ** -8 * np.abs(ref)).max()
        want = steps(x, weight, eps, turns, rot, interleaved, at, m)
        # (zeros of either sign are one value)
        assert ((got == want) | ((got | want) & 0x7FFF == 0)).all(), np.argwhere(got != want)[:3]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D,H_q,H", [(64, 32, 4), (128, 32, 8), (256, 16, 8), (128, 5, 1), (64, 1, 1), (256, 7, 3)])
def test_layers(D, H_q, H, interleaved):
    check(2, 3, H_q, H, D, D, interleaved, norm=3)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_part_of_the_head(D, interleaved):
    for rot in {0, 16, 48, D // 2, D - 16, D}:
        check(1, 5, 6, 2, D, rot, interleaved, norm=rot // 16 % 4)


@pytest.mark.parametrize("kind", ["consecutive", "far", "zero", "mixed"])
def test_positions(kind):
    check(3, 17, 8, 2, 128, 128, kind=kind)
    check(2, 9, 4, 4, 64, 32, True, kind=kind)


@pytest.mark.parametrize("norm", [0, 1, 2, 3])
def test_norms_of_either(norm):
    check(2, 7, 5, 3, 128, 96, norm=norm, eps=1e-2)


def test_queries_or_keys_alone_and_in_place():
    for D in (64, 128, 256):
        check(2, 11, 9, 0, D, D, norm=3)
        check(2, 11, 0, 3, D, D, norm=3)
        check(2, 11, 9, 3, D, D, norm=3, in_place=True)
        check(2, 11, 9, 3, D, 32, True, norm=1, in_place=True)


@pytest.mark.parametrize("B,n,H_q,H", [(1, 1, 32, 8), (1, 300, 32, 8), (2, 777, 32, 8), (5, 401, 16, 8), (1, 2048, 71, 1)])
def test_many_tokens(B, n, H_q, H):
    # (every split of a token's heads over waves)
    check(B, n, H_q, H, 128, 128, norm=3, kind="consecutive")


def test_scaled_cosines():
    check(2, 9, 4, 2, 64, 64, scale=1.1386294)


def test_zero_rows_and_large_values():
    from paper_2609_04263_amd import kvq
    x = torch.zeros((1, 4, 2, 64), dtype=torch.bfloat16, device="cuda")
    x[0, 1], x[0, 2] = 2.0 ** 100, 2.0 ** -100
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    out = torch.empty_like(x)
    kvq.Rope(64).qk(x, None, out, q_norm=w, pos0=0)
    o = out.float().cpu()
    assert (o[0, 0] == 0).all() and (o[0, 3] == 0).all()
    # rows of equal numbers: 1, and 2^-100 / sqrt(eps); position 1 and 2 leave a pair's length
    a, b = o[0, 1, 0, :32], o[0, 1, 0, 32:]
    assert ((a * a + b * b - 2).abs() <= 4 * 2.0 ** -8).all()
    assert (o[0, 2].abs() <= 2.0 ** -89).all() and (o[0, 2] != 0).any()


def test_another_stream_and_a_captured_call():
    from paper_2609_04263_amd import kvq
    rope = kvq.Rope(128)
    B, n, D = 2, 5, 128
    Q = dev_bf16(synth.normal_bf16(3, "q", (B, n, 8, D)))
    K = dev_bf16(synth.normal_bf16(3, "k", (B, n, 2, D)))
    pos = torch.arange(B * n, dtype=torch.int32, device="cuda").view(B, n)
    want = torch.empty_like(Q), torch.empty_like(K)
    rope.qk(Q, K, *want, pos=pos)
    got = torch.zeros_like(Q), torch.zeros_like(K)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    rope.qk(Q, K, *got, pos=pos, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rope.qk(Q, K, *got, pos=pos)
    for shift in (3, 50, 7):  # (positions are read when the graph runs, frequencies were when it was made)
        pos += shift
        rope.c.turns[0] = 0.25
        g.replay()
        rope.c.turns[0] = kvq.Rope(128).c.turns[0]
        rope.qk(Q, K, *want, pos=pos)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


# ------------------------------------------------------------------ appends

def append_case(name, B, H, cuts, seed, rot=None, interleaved=False, norm=0, kind="consecutive", H_q=0, drafts=0):
    """Tokens cuts[0] .. cuts[-1] in pieces: the storage's bytes against the oracle's append of keys turned on the host,
    and against kvq_append of kvq_rope_qk's."""
    from paper_2609_04263_amd import kvq
    fmt, D = CASES[name]
    n = cuts[-1]
    rot = D if rot is None else rot
    rope = kvq.Rope(rot, interleaved=interleaved)
    outlier = ("student_t", 3.0) if fmt["rotate"] else ("scale", 4, 20.0)
    K, V = synth.kv_tokens(seed, B, n, H, D, outlier=outlier)
    wq, wk = (weights(seed, k, D) if norm else None for k in "qk")
    pos, pos0, at = positions(kind, B, n, seed)
    two, one = (kvq.Cache(fmt, B, H, D, n + 5) for _ in range(2))
    ref = oracle.Cache(fmt, B, H, D, n + 5)
    ref.append(steps(K, wk, 1e-6, np.array(rope.c.turns[:rot // 2]), rot, interleaved, at), V)
    Kd, Vd = dev_bf16(K), dev_bf16(V)
    norms = dict(k_norm=None if wk is None else dev_bf16(wk))
    for a, b in zip(cuts[:-1], cuts[1:]):
        k, v = Kd[:, a:b].contiguous(), Vd[:, a:b].contiguous()
        p = None if pos is None else pos[:, a:b].contiguous()
        kw = dict(pos=p, pos0=pos0 + a, **norms)
        ko = torch.empty_like(k)
        rope.qk(None, k, None, ko, **kw)
        two.append(ko, v)
        if H_q:
            q = dev_bf16(synth.normal_bf16(seed, ("q", a), (B, b - a, H_q, D)))
            want, (flat, got) = torch.empty_like(q), guarded(q.shape)
            qw = None if wq is None else dev_bf16(wq)
            rope.qk(q, None, want, None, q_norm=qw, pos=p, pos0=pos0 + a)
            one.append_rope(rope, k, v, Q=q, Qo=got, q_norm=qw, **kw)
            assert torch.equal(want, got) and untouched(flat)
        elif drafts:  # the rows somewhere among more
            g = synth.stream(seed, "rows", a)
            rows = torch.from_numpy(np.stack([g.permutation(b - a + drafts)[:b - a] for _ in range(B)]).astype(np.int32))
            wide_k, wide_v = (torch.full((B, b - a + drafts, H, D), 99.0, dtype=torch.bfloat16, device="cuda") for _ in "kv")
            for i in range(B):
                wide_k[i, rows[i].long().cuda()], wide_v[i, rows[i].long().cuda()] = k[i], v[i]
            one.append_rope(rope, wide_k, wide_v, rows=rows.cuda(), **kw)
        else:
            one.append_rope(rope, k, v, **kw)
    assert one.length() == two.length() == (n, ref.n_coded)
    assert np.array_equal(image(one), image(two)), f"{name}: not the bytes of the two calls"
    assert np.array_equal(image(one), ref.image), f"{name}: not the oracle's bytes"


@pytest.mark.parametrize("name", list(CASES))
def test_append_ragged_chunks(name):
    append_case(name, 2, 3, [0, 1, 2, 31, 64, 100, 131, 200, 233], seed=41)


@pytest.mark.parametrize("name", list(CASES))
def test_append_with_norms_part_of_the_head(name):
    D = CASES[name][1]
    append_case(name, 2, 2, [0, 70, 71, 150], seed=42, rot=D // 2 + 16, norm=1, kind="mixed", H_q=4)


@pytest.mark.parametrize("name", ["tiny_b16", "kivi", "gqa12b", "hadamard", "kvarn_sink", "had_affine_window"])
def test_append_interleaved(name):
    append_case(name, 1, 2, [0, 33, 34, 170], seed=43, interleaved=True, norm=1, kind="far")
    append_case(name, 1, 2, [0, 33, 34, 170], seed=43, rot=48, interleaved=True)


@pytest.mark.parametrize("name", ["tiny_b16", "kivi", "hadamard", "kvarn_sink", "sink32_window"])
def test_append_token_by_token(name):
    append_case(name, 1, 2, list(range(171)), seed=44, H_q=2)


@pytest.mark.parametrize("name", ["tiny_b16", "kivi", "gqa12b", "hadamard", "kvarn_sink", "sink32_window", "affine8"])
def test_append_of_chosen_rows(name):
    append_case(name, 3, 2, [0, 1, 6, 140, 141, 165], seed=45, drafts=13, kind="mixed")


def test_append_without_rotation_is_append():
    from paper_2609_04263_amd import kvq
    fmt, D = CASES["gqa12b"]
    K, V = synth.kv_tokens(46, 2, 90, 2, D)
    a, b = (kvq.Cache(fmt, 2, 2, D, 100) for _ in range(2))
    a.append(dev_bf16(K), dev_bf16(V))
    b.append_rope(kvq.Rope(0), dev_bf16(K), dev_bf16(V), pos0=17)
    assert np.array_equal(image(a), image(b))


def test_rows_outside_are_the_nearest_and_may_repeat():
    from paper_2609_04263_amd import kvq
    fmt, D = CASES["tiny_b16"]
    K, V = synth.kv_tokens(47, 1, 6, 2, D)
    a, b = (kvq.Cache(fmt, 1, 2, D, 100) for _ in range(2))
    rows = [[-5, 2, 2, 6, 2 ** 31 - 1, -2 ** 31, 0]]
    pick = [0, 2, 2, 5, 5, 0, 0]
    rope = kvq.Rope(64)
    a.append_rope(rope, dev_bf16(K), dev_bf16(V), rows=torch.tensor(rows, dtype=torch.int32, device="cuda"), pos0=3)
    b.append_rope(rope, dev_bf16(K[:, pick]), dev_bf16(V[:, pick]), pos0=3)
    assert a.n == 7 and np.array_equal(image(a), image(b))


def test_append_first_rows_of_more():
    from paper_2609_04263_amd import kvq
    fmt, D = CASES["kivi"]
    K, V = synth.kv_tokens(48, 3, 40, 2, D)
    a, b = (kvq.Cache(fmt, 3, 2, D, 100) for _ in range(2))
    rope = kvq.Rope(D)
    a.append_rope(rope, dev_bf16(K), dev_bf16(V), n_new=29)
    b.append_rope(rope, dev_bf16(K[:, :29]), dev_bf16(V[:, :29]))
    assert a.n == 29 and np.array_equal(image(a), image(b))


def test_a_refused_append_changes_nothing():
    from paper_2609_04263_amd import kvq
    fmt, D = CASES["tiny_b1"]
    K, V = synth.kv_tokens(49, 1, 40, 1, D)
    c = kvq.Cache(fmt, 1, 1, D, 40)
    q = dev_bf16(K[:, :11])
    out = torch.zeros_like(q)
    c.append_rope(kvq.Rope(D), dev_bf16(K[:, :30]), dev_bf16(V[:, :30]))
    before = image(c).copy()
    with pytest.raises(kvq.KvqError) as e:
        c.append_rope(kvq.Rope(D), dev_bf16(K[:, :11]), dev_bf16(V[:, :11]), Q=q, Qo=out)
    assert e.value.status == kvq.ERR_CAPACITY
    assert c.n == 30 and np.array_equal(image(c), before) and not out.any()


@pytest.mark.parametrize("name,B,H,n", [("kivi", 8, 9, 1000), ("gqa12b", 8, 9, 1000), ("tiny_b16", 8, 17, 2030),
                                        ("hadamard", 8, 17, 1000), ("had_affine_window", 8, 9, 1001),
                                        ("sym4_window", 8, 17, 2100), ("affine8", 8, 17, 2030), ("kivi", 1, 1, 1000)])
@pytest.mark.parametrize("norm", [0, 1])
def test_append_several_heads_of_a_workgroup(name, B, H, n, norm):
    # calls so large that a workgroup codes several heads, the last ones fewer: the bytes of the two calls
    from paper_2609_04263_amd import kvq
    fmt, D = CASES[name]
    g = torch.Generator(device="cuda")
    g.manual_seed(50)
    K, V, Q = (torch.randn((B, n, h, D), generator=g, device="cuda").to(torch.bfloat16) for h in (H, H, 2 * H))
    w = dev_bf16(weights(50, "k", D)) if norm else None
    rope = kvq.Rope(D if norm else D // 2, 500000.0)
    one, two = (kvq.Cache(fmt, B, H, D, n + 40) for _ in range(2))
    for lo, hi in ((0, 37), (37, n)):
        k, v, q = (x[:, lo:hi].contiguous() for x in (K, V, Q))
        kw = dict(k_norm=w, q_norm=w, pos0=lo)
        a, b = torch.empty_like(q), torch.empty_like(q)
        kk = torch.empty_like(k)
        rope.qk(q, k, a, kk, **kw)
        two.append(kk, v)
        one.append_rope(rope, k, v, Q=q, Qo=b, **kw)
        assert torch.equal(a, b)
    assert torch.equal(one.storage, two.storage)


def test_append_of_one_token_without_its_axis():
    from paper_2609_04263_amd import kvq
    fmt, D = CASES["tiny_b16"]
    K, V = synth.kv_tokens(51, 3, 1, 2, D)
    a, b = (kvq.Cache(fmt, 3, 2, D, 100) for _ in range(2))
    a.append_rope(kvq.Rope(D), dev_bf16(K), dev_bf16(V), pos0=9)
    b.append_rope(kvq.Rope(D), dev_bf16(K[:, 0]), dev_bf16(V[:, 0]), pos0=9)
    assert a.n == b.n == 1 and np.array_equal(image(a), image(b))


def test_more_workgroups_than_a_row_of_the_grid():
    # 2^22 + 5 tokens of one head: 2^20 + 2 workgroups of four waves
    from paper_2609_04263_amd import kvq
    n = (1 << 22) + 5
    x = torch.ones((1, n, 1, 64), dtype=torch.bfloat16, device="cuda")
    rope = kvq.Rope(64)
    rope.qk(x, None, pos0=1)
    at = [0, 1 << 21, (1 << 22) - 1, 1 << 22, n - 1]
    y = torch.ones((1, len(at), 1, 64), dtype=torch.bfloat16, device="cuda")
    rope.qk(y, None, pos=torch.tensor([[i + 1 for i in at]], dtype=torch.int32, device="cuda"))
    assert torch.equal(x[0, at], y[0])
    # every row has the length of its two halves' pairs
    z = x.float().square()
    assert ((z[..., :32] + z[..., 32:] - 2).abs() <= 4 * 2.0 ** -8).all()


def test_one_token_of_more_workgroups_than_a_row_of_the_grid():
    # 2^14 keys and 2^20 rows of queries, a workgroup each
    from paper_2609_04263_amd import kvq
    fmt, B, H_q, D = configs.make_format(k_group=32, v_group=32), 1 << 14, 64, 64
    gen = torch.Generator(device="cuda").manual_seed(5)
    q, k, v = (torch.randn((B, 1, h, D), device="cuda", generator=gen).bfloat16() for h in (H_q, 1, 1))
    rope, w = kvq.Rope(D), torch.rand(D, device="cuda", generator=gen).bfloat16()
    one, two = (kvq.Cache(fmt, B, 1, D, 32) for _ in range(2))
    guard = torch.full((q.numel() + 4096,), 7.0, dtype=torch.bfloat16, device="cuda")
    qo, want, kk = guard[:q.numel()].view_as(q), torch.empty_like(q), torch.empty_like(k)
    one.append_rope(rope, k, v, Q=q, Qo=qo, q_norm=w, k_norm=w, pos0=77)
    rope.qk(q, k, want, kk, q_norm=w, k_norm=w, pos0=77)
    two.append(kk, v)
    assert torch.equal(qo, want) and torch.equal(one.storage, two.storage)
    assert (guard[q.numel():] == 7.0).all()


@pytest.mark.parametrize("n", (1, 3))
def test_more_heads_than_a_row_of_the_grid_without_queries(n):
    from paper_2609_04263_amd import kvq
    fmt, B, D = configs.make_format(k_group=32, v_group=32), (1 << 20) + 5, 64
    gen = torch.Generator(device="cuda").manual_seed(6)
    k, v = (torch.randn((B, n, 1, D), device="cuda", generator=gen).bfloat16() for _ in range(2))
    rope, kk = kvq.Rope(D), torch.empty_like(k)
    one, two = (kvq.Cache(fmt, B, 1, D, 32) for _ in range(2))
    one.append_rope(rope, k, v, pos0=77)
    rope.qk(None, k, None, kk, pos0=77)
    two.append(kk, v)
    assert torch.equal(one.storage, two.storage)
