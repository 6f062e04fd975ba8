"""Codes at the top of binary32: ranges that overflow it (the scale is infinite and
every code 0), scales above 2^126 (their reciprocals are subnormal), constants
beside which fp16's largest offset is nothing.  Every number that the coder sees is
finite, so the bytes are the oracle's, whichever kernel writes them: kvq_append of
single tokens, of parts of blocks and of whole ones, and the projection's fused append.
"""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_04263_amd import configs, synth

from gpu_util import dev_bf16, image
from test_gpu_edge_groups import FORMATS

pytestmark = pytest.mark.gpu

TOP = float(synth.bf16_bits_to_f32(np.array([0x7F7F], np.uint16))[0])  # the largest bf16, 3.39e38
CUTS = {"at once": [0, 420], "ragged": [0, 1, 33, 200, 201, 206, 240, 420], "tokens": list(range(41)) + [420]}

# (lo, hi) of groups; a window would round all of these to infinity
RANGES = [(-TOP, TOP), (0.0, TOP), (-TOP, 0.0), (-TOP / 2, TOP / 2), (TOP / 2, TOP), (-1.0, TOP), (-1.7e38, 1.7e38),
          (-1.5e38, 1.2e38), (0.0, 2.6e38), (0.0, 8.6e37), (TOP, TOP), (-TOP, -TOP), (2.0 ** 110, 2.0 ** 110),
          (-2.0 ** 104, -2.0 ** 104), (2.0 ** 103, 2.0 ** 103), (1e20, 1.01e20), (65504.0, 1e6), (-1e6, -65504.0),
          (-3e5, 3e5), (1e10, 1e10), (-1.0, 1.0)]


def large_tokens(seed, B, n, H, D):
    """Tokens whose numbers lie in one of RANGES, its ends among them, half of them on quarters of it."""
    g = np.random.default_rng(seed)
    lo, hi = np.array(RANGES)[g.integers(0, len(RANGES), (B, n, H))].transpose(3, 0, 1, 2)[..., None]
    u = g.random((B, n, H, D))
    u = np.where(g.random((B, n, H, 1)) < 0.5, np.rint(u * 4) / 4, u)
    x = lo * (1 - u) + hi * u
    x[..., 0::32], x[..., 1::32] = lo, hi
    bits = synth.to_bf16_bits(np.clip(x, -TOP, TOP).astype(np.float32))
    assert np.isfinite(synth.bf16_bits_to_f32(bits)).all()
    return bits


LARGE = {k: FORMATS[k] for k in ("affine4_g32", "affine2_g64_d128", "sym4_g64", "sym_k4v2_g128", "affine4_meta16",
                                 "sym4_meta16_d256", "affine8", "sym8_meta16")}
LARGE |= {"sym2_d256": (configs.make_format(2, 2, k_mode=1, v_mode=1, k_group=128, v_group=32), 256),
          "k2v4": (configs.make_format(2, 4, k_group=32, v_group=128), 128),
          "affine2_meta16_d256": (configs.make_format(2, 2, k_group=32, v_group=256, meta_fp16=1), 256),
          "sym2_key_affine_value": (configs.make_format(2, 2, k_mode=1, k_group=64, v_group=32), 64)}


def compare(name, got, ref):
    for i in range(10):
        part = slice(ref.offsets[i], ref.offsets[i] + ref.lengths[i])
        diff = np.flatnonzero(got[part] != ref.image[part])
        assert not diff.size, f"{name}: section {i} is not the oracle's at {diff.size} bytes, first at {diff[0]}"


@pytest.mark.parametrize("cuts", list(CUTS))
@pytest.mark.parametrize("name", list(LARGE))
def test_append(name, cuts):
    from paper_2609_04263_amd import kvq
    fmt, D = LARGE[name]
    B, n, H = 2, 420, 3
    K, V = (large_tokens(s + D, B, n, H, D) for s in (3000, 4000))
    ref = oracle.Cache(fmt, B, H, D, n)
    ref.append(K, V)
    c = kvq.Cache(fmt, B, H, D, n)
    for a, b in zip(CUTS[cuts][:-1], CUTS[cuts][1:]):
        c.append(dev_bf16(K[:, a:b]), dev_bf16(V[:, a:b]))
    compare(name, image(c), ref)


@pytest.mark.parametrize("name", [k for k in LARGE if LARGE[k][0]["rotate"] == 0])
def test_fused_append(name):
    # weights that copy the hidden states: K from channel 0 on, V from channel 256 on
    from paper_2609_04263_amd import kvq
    fmt, D = LARGE[name]
    B, n, d_kv = 2, 160, 256
    H = d_kv // D
    K, V = (large_tokens(s + D, B, n, H, D) for s in (5000, 6000))
    x = dev_bf16(np.concatenate([K.reshape(B * n, d_kv), V.reshape(B * n, d_kv)], 1))
    W = torch.zeros((256 + 2 * d_kv, 2 * d_kv), dtype=torch.bfloat16, device="cuda")
    W[256:] = torch.eye(2 * d_kv)
    ref = oracle.Cache(fmt, B, H, D, n)
    ref.append(K, V)
    c = kvq.Cache(fmt, B, H, D, n)
    Q = torch.empty((B * n, 256), dtype=torch.bfloat16, device="cuda")
    kvq.project_append(x, W, None, None, 0, 0.0, 256, d_kv, Q, c, n, None)
    compare(name, image(c), ref)
