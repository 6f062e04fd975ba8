"""Eq. (3)'s edge cases through kvq_append_rope: its coders take other steps than
kvq_append's, and the bytes have to be the same for every finite input.

The groups of test_gpu_edge_groups.py (constant, zero, signed zeros, ranges around
the scale's floor) and those of test_gpu_append_range.py.  Keys are
appended without rotation (they are coded as they are) in one call and in ragged
ones: single tokens, a few, whole blocks of several heads.  Against the oracle's
bytes and kvq_append's.
"""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_04263_amd import configs, synth

from gpu_util import dev_bf16, image
from test_gpu_append_range import CUTS, LARGE, large_tokens
from test_gpu_edge_groups import FORMATS, edge_tokens

pytestmark = pytest.mark.gpu


def compare(name, fmt, D, K, V, cuts):
    from paper_2609_04263_amd import kvq
    B, n, H, _ = K.shape
    ref = oracle.Cache(fmt, B, H, D, n + 12)
    ref.append(K, V)
    one, two = (kvq.Cache(fmt, B, H, D, n + 12) for _ in range(2))
    two.append(dev_bf16(K), dev_bf16(V))
    rope = kvq.Rope(0)
    for a, b in zip(cuts[:-1], cuts[1:]):
        one.append_rope(rope, dev_bf16(K[:, a:b]), dev_bf16(V[:, a:b]), pos0=a)
    x, y = image(one), image(two)
    for i in range(10):
        part = slice(ref.offsets[i], ref.offsets[i] + ref.lengths[i])
        for what, other in (("the oracle's", ref.image), ("kvq_append's", y)):
            diff = np.flatnonzero(x[part] != other[part])
            assert not diff.size, f"{name}: section {i} is not {what} at {diff.size} bytes, first at {diff[0]}"


@pytest.mark.parametrize("cuts", list(CUTS))
@pytest.mark.parametrize("name", list(FORMATS))
def test_edge_groups(name, cuts):
    fmt, D = FORMATS[name]
    B, H, n = 2, 2, 420
    K = edge_tokens(1000 + D, B, n, H, D, fmt["k_mode"], fmt["k_bits"], fmt["meta_fp16"], True)
    V = edge_tokens(2000 + D, B, n, H, D, fmt["v_mode"], fmt["v_bits"], fmt["meta_fp16"], False)
    compare(name, fmt, D, K, V, CUTS[cuts])


@pytest.mark.parametrize("cuts", list(CUTS))
@pytest.mark.parametrize("name", list(LARGE))
def test_the_top_of_the_range(name, cuts):
    fmt, D = LARGE[name]
    K, V = (large_tokens(s + D, 2, 420, 3, D) for s in (3000, 4000))
    compare(name, fmt, D, K, V, CUTS[cuts])


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("meta16", [0, 1])
@pytest.mark.parametrize("mode", [0, 1])
def test_channels_up_to_the_window_s_range(mode, meta16, D):
    # per-channel keys of constants and ranges up to +-65504, fp16's largest
    fmt = configs.make_format(4, 4, k_mode=mode, v_mode=mode, k_axis=1, k_group=32, v_group=32, residual=32, flush=32,
                              meta_fp16=meta16)
    g = np.random.default_rng(5000 + D)
    B, n, H = 2, 420, 2
    kinds = np.array([(65504.0, 65504.0), (-65504.0, 65504.0), (-65504.0, -65504.0), (0.0, 6e-8), (-1.0, 1.0)])

    def tokens():
        lo, hi = kinds[g.integers(0, len(kinds), (B, 1, H, D))].transpose(4, 0, 1, 2, 3)
        x = lo + (hi - lo) * (g.integers(0, 5, (B, n, H, D)) / 4)
        return synth.to_bf16_bits(np.clip(x, -65280.0, 65280.0).astype(np.float32))
    for cuts in CUTS.values():
        compare(f"mode {mode}", fmt, D, tokens(), tokens(), cuts)


def test_scales_of_a_turned_row():
    # positions and a transform: numbers up to 2^110, far from overflow in any sum
    from paper_2609_04263_amd import kvq
    for name in ("hadamard_sym", "affine2_g64_d128"):
        fmt, D = FORMATS[name]
        g = np.random.default_rng(6)
        K, V = (dev_bf16(synth.to_bf16_bits((2.0 ** g.integers(90, 110, (2, 300, 3, 1)) *
                                             g.standard_normal((2, 300, 3, D))).astype(np.float32))) for _ in "kv")
        rope = kvq.Rope(D)
        one, two = (kvq.Cache(fmt, 2, 3, D, 300) for _ in range(2))
        for a, b in ((0, 1), (1, 40), (40, 300)):
            k, v = K[:, a:b].contiguous(), V[:, a:b].contiguous()
            kk = torch.empty_like(k)
            rope.qk(None, k, None, kk, pos0=a)
            two.append(kk, v)
            one.append_rope(rope, k, v, pos0=a)
        assert torch.equal(one.storage, two.storage), name
