"""The norm of a key is the same number in kvq_rope_qk and in kvq_append_rope.

A row's sum of squares is rounded at every step, so it depends on the order of its
additions, which both calls have to share.  Another order moves the last bit of the sum
in one of 10^4 rows and the stored key in one of 10^13: the rows here are made so that
it would move the key.  Their sums lie at every number around the one at which 1 / sqrt
passes a border of binary32 (all of them, so that one is at the border of the
evaluation itself, which is off by some units of its last place), two orders leave
neighbours of them, and channel 0, a one, times its weight lies at a border of bf16.
"""
import numpy as np
import pytest
import torch

from paper_2609_04263_amd import configs, synth

from gpu_util import dev_bf16

SPAN = 20  # numbers on either side of the border: the evaluation is off by 2^-51, at most 8 of them


def squares(x):
    """[.., D] -> the pieces' sums of squares [.., D / 8], each in binary64 steps (a square of bf16 is exact)."""
    v = x.astype(np.float64).reshape(x.shape[:-1] + (-1, 8)) ** 2
    s = np.zeros(v.shape[:-1])
    for e in range(8):
        s = s + v[..., e]
    return s


def by_pieces(p):
    """Neighbours first, then pairs of them, .."""
    while p.shape[-1] > 1:
        p = p[..., 0::2] + p[..., 1::2]
    return p[..., 0]


def by_pairs(p, rot):
    """A rotated pair's two pieces first."""
    hp = rot // 16
    a = p[..., :hp] + p[..., hp:2 * hp]
    return by_pieces(np.concatenate([a, p[..., 2 * hp::2] + p[..., 2 * hp + 1::2]], -1))


def bf16(x):
    return synth.bf16_bits_to_f32(synth.to_bf16_bits(np.asarray(x, np.float32)))


def border(k):
    """A weight and neighbouring binary32 factors whose products with it round to different bf16 numbers."""
    w = np.float32(1 + (2 * k + 1) / 128)
    r = np.float32((1 + 1 / 256) / w)
    r = np.nextafter(r, np.float32(0))
    while bf16(r * w) == bf16(np.nextafter(r, np.float32(2)) * w):
        r = np.nextafter(r, np.float32(2))
    return w, r, np.nextafter(r, np.float32(2))


def rows(D, rot, k=3):
    """Rows [2 SPAN + 1, D] as described above, and channel 0's weight."""
    w, low, high = border(k)
    mid = (np.float64(low) + np.float64(high)) / 2
    at = np.float64(D) / (mid * mid)
    ulp = np.spacing(at)
    rng = np.random.default_rng(D + rot)
    found = {}
    for _ in range(4000):
        # squares of bf16 numbers that add up to some number near `at`, and small ones that meet or do not
        rest, x = at + ulp * rng.integers(-SPAN - 3, SPAN + 1) - 1.0, []
        tiny = float(bf16([np.sqrt(0.3 * ulp)])[0])
        rest -= 8 * tiny * tiny
        while rest > 0.5 * ulp and len(x) < D // 2:
            t = synth.to_bf16_bits(np.array([np.sqrt(rest)], np.float32))
            t = float(synth.bf16_bits_to_f32(t)[0])
            if t * t > rest:
                t = float(synth.bf16_bits_to_f32(synth.to_bf16_bits(np.array([t], np.float32)) - 1)[0])
            x.append(t)
            rest -= t * t
        x = np.array(x + [tiny] * 8 + [0.0] * (D - 9 - len(x)))
        trials = np.concatenate([np.ones((64, 1)), rng.permuted(np.tile(x, (64, 1)), axis=1)], 1)
        p = squares(trials)
        one, other = by_pieces(p), by_pairs(p, rot)
        for i in np.flatnonzero(np.abs(one - other) == ulp):
            j = int(round((min(one[i], other[i]) - at) / ulp))
            if abs(j) <= SPAN:
                found.setdefault(j, trials[i])
        if len(found) == 2 * SPAN + 1:
            return np.stack([found[j] for j in sorted(found)]).astype(np.float32), w
    raise AssertionError(f"D = {D}: rows for {len(found)} of {2 * SPAN + 1} sums")


# (rotated channels: all, a power of two of them and not)
CASES = [(64, 64), (64, 32), (64, 48), (128, 128), (128, 32), (128, 64), (128, 96), (256, 256), (256, 32), (256, 64), (256, 128),
         (256, 208)]


@pytest.mark.parametrize("D,rot", CASES)
def test_the_rows_have_two_sums(D, rot):
    x, w = rows(D, rot)
    p = squares(x)
    one, other = by_pieces(p), by_pairs(p, rot)
    at = np.sort(np.minimum(one, other))
    assert (np.abs(one - other) == np.spacing(at)).all() and (np.diff(at) == np.spacing(at[:-1])).all()
    assert np.array_equal(bf16(x), x) and (x[:, 0] == 1).all()
    r = np.float32(1 / np.sqrt(at / D))
    products = set(bf16(r * w).tolist())
    assert len(products) == 2, products


@pytest.mark.gpu
@pytest.mark.parametrize("D,rot", CASES)
def test_the_same_norm_in_both_calls(D, rot):
    # a window's rows, which hold the keys as they are; and one token at a time
    from paper_2609_04263_amd import kvq
    x, w = rows(D, rot)
    n = x.shape[0]
    weight = np.ones(D, np.float32)
    weight[0] = w
    norm = dev_bf16(synth.to_bf16_bits(weight))
    fmt = configs.make_format(2, 2, k_axis=1, k_group=32, v_group=32, residual=128, flush=32)
    K = dev_bf16(synth.to_bf16_bits(x)).view(1, n, 1, D)
    rope = kvq.Rope(rot, eps=0.0)
    pos = torch.zeros((1, n), dtype=torch.int32, device="cuda")
    turned = torch.empty_like(K)
    rope.qk(None, K, None, turned, k_norm=norm, pos=pos)
    assert len(turned[0, :, 0, 0].unique()) == 2
    want, once, single = (kvq.Cache(fmt, 1, 1, D, 128) for _ in range(3))
    want.append(turned, K)
    once.append_rope(rope, K, K, k_norm=norm, pos=pos)
    for i in range(n):
        single.append_rope(rope, K[:, i:i + 1], K[:, i:i + 1], k_norm=norm, pos=pos[:, :1])
    assert torch.equal(once.storage, want.storage) and torch.equal(single.storage, want.storage)
    # as queries, beside keys, and beside an append
    for q, k in ((K, None), (K, K)):
        a, b = torch.empty_like(K), torch.empty_like(K)
        rope.qk(q, k, a, None if k is None else b, q_norm=norm, k_norm=norm, pos=pos)
        assert torch.equal(a, turned) and (k is None or torch.equal(b, turned))
    a = torch.empty_like(K)
    want.append_rope(rope, K, K, Q=K, Qo=a, q_norm=norm, k_norm=norm, pos=pos)
    assert torch.equal(a, turned)
