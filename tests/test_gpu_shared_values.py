"""Shared-prefix attention of values whose sizes differ from token to token:
every product keeps its bits, whatever other tokens hold and however little
weight they have.

Bound.  The tokens that carry an output have scores of at most about 5 natural
units here (no part of theirs is larger unless a test says so), for which
test_gpu_shared.py derives 5e-6 of a score and as much again of the sums: 1e-5
of the output's norm.  2^-15 = 3e-5 (half of that file's 2^-14) leaves a
factor of three, and 8 times that is accepted of a single row, as there.
"""
import numpy as np
import pytest

from paper_2609_04263_amd import configs, synth

from test_gpu_append import CASES
from test_gpu_shared import Pair, call, close, reference

pytestmark = pytest.mark.gpu

# (one format per kind of key, code width, metadata, rotation and fp16 tokens)
NAMES = ["tiny_b1", "tiny_b16", "kivi", "gqa12b", "hadamard", "perch_k4v2_window64", "had_affine_window", "affine8",
         "kvarn_sink", "sink32_window", "sink64"]
MORE = {
    "g32_d128": (configs.make_format(4, 4, k_group=32, v_group=32), 128),
    "g32_d256": (configs.make_format(2, 2, k_group=32, v_group=32), 256),
    "g128_d256_8": (configs.make_format(8, 8, k_group=128, v_group=256), 256),
}


def unit(D):
    return np.where(np.arange(D) % 2 == 0, 1.0, -1.0).astype(np.float32)


def tokens(fmt, U, H, D, n, seed, lower=None, size=None):
    """K, V of n tokens: K of token t minus lower[t] (natural units of a query along unit(D)), V times size[t]."""
    K, V = synth.kv_tokens(seed, U, n, H, D)
    if lower is not None:
        k = synth.bf16_bits_to_f32(K) - (lower / np.sqrt(D))[None, :, None, None] * unit(D)
        K = synth.to_bf16_bits(k.astype(np.float32))
    if size is not None:
        V = synth.to_bf16_bits(synth.bf16_bits_to_f32(V) * size[None, :, None, None].astype(np.float32))
    return Pair(fmt, U, H, D, n).append(K, V)


def along(seed, B, C, H_q, D):
    """Queries along unit(D): a key's part along it is a score of its own."""
    q = synth.bf16_bits_to_f32(synth.queries(seed, B * C, H_q, D)).reshape(B, C, H_q, D)
    return synth.to_bf16_bits(q * np.float32(0.25) + unit(D))


def where(n, lo, hi, inside, outside):
    t = np.arange(n)
    return np.where((t >= lo) & (t < hi), inside, outside).astype(np.float64)


def bounded(fmt, power):
    """A power of two that the format can hold: a window's tokens pass through fp16 before they are coded."""
    return 2.0 ** (min(power, 13) if fmt["flush"] else power)


def check(prefix, suffix, first, Q, factor=0.5, chunk=None, rows=slice(None)):
    D = Q.shape[-1]
    want = reference(prefix, suffix, first, Q, D ** -0.5)[:, rows]
    for k in range(3):
        got = call(prefix, suffix, first, Q, D ** -0.5, chunk=chunk, kernels=k)[:, rows]
        close(got, want, factor, f"kernels={k}")


@pytest.mark.parametrize("first", [[0, 3], [0, 33]])
@pytest.mark.parametrize("power", [12, 20, 30])
@pytest.mark.parametrize("name", NAMES + list(MORE))
def test_large_values_of_no_weight(name, power, first):
    """64 coded tokens of the prefix 2^power times the others' size, 60 natural units below them."""
    fmt, D = {**CASES, **MORE}[name]
    n, H, B = 500, 2, first[-1]
    prefix = tokens(fmt, 1, H, D, n, 60, where(n, 160, 224, 60, 0), where(n, 160, 224, bounded(fmt, power), 1))
    suffix = tokens(fmt, B, H, D, 40, 61)
    check(prefix, suffix, first, along(62, B, 1, 2 * H, D))


@pytest.mark.parametrize("power", [13, 24, 40])
@pytest.mark.parametrize("name", NAMES + list(MORE))
def test_large_and_small_blocks_in_turn(name, power):
    """1024 rows over 3000 tokens, so that every wave meets large blocks (of no weight) before small ones and after."""
    fmt, D = {**CASES, **MORE}[name]
    n, B = 3000, 64
    large = (np.arange(n) // 128 % 2 == 1) & (np.arange(n) < 2700)
    prefix = tokens(fmt, 1, 1, D, n, 58, np.where(large, 60.0, 0.0), np.where(large, bounded(fmt, power), 1.0))
    suffix = tokens(fmt, B, 1, D, 5, 59)
    check(prefix, suffix, [0, B], along(57, B, 1, 16, D))


@pytest.mark.parametrize("first", [[0, 3], [0, 33]])
@pytest.mark.parametrize("name", NAMES + list(MORE))
def test_one_large_token_of_no_weight_in_every_block(name, first):
    """Every 32nd token, so that no block is without one."""
    fmt, D = {**CASES, **MORE}[name]
    n, H, B = 500, 2, first[-1]
    here = (np.arange(n) % 32 == 5) & (np.arange(n) > 130) & (np.arange(n) < 320)  # (coded in every format)
    prefix = tokens(fmt, 1, H, D, n, 63, np.where(here, 60.0, 0.0),
                    np.where(here, bounded(fmt, 24), 1.0))
    suffix = tokens(fmt, B, H, D, 40, 64)
    # per-channel groups of 32 tokens share the large keys' scale: every key of a block is coarse, and its own
    # block's scores spread to twice the 5 units
    check(prefix, suffix, first, along(65, B, 1, 2 * H, D), 1.0 if fmt["k_axis"] else 0.5)


@pytest.mark.parametrize("name", ["tiny_b1", "tiny_b16", "gqa12b", "hadamard", "affine8"] + list(MORE))
@pytest.mark.parametrize("B,C,n_s", [(2, 5, 37), (1, 40, 60)])
def test_tokens_that_a_query_does_not_see(name, B, C, n_s):
    """The newest token of each suffix is 2^30 times the others' size; the queries before it are compared."""
    fmt, D = {**CASES, **MORE}[name]
    H = 2
    prefix = tokens(fmt, 1, H, D, 200, 66)
    suffix = tokens(fmt, B, H, D, n_s, 67, size=where(n_s, n_s - 1, n_s, 2.0 ** 30, 1))
    check(prefix, suffix, [0, B], along(68, B, C, 2 * H, D), chunk=True, rows=slice(0, C - 1))


@pytest.mark.parametrize("first", [[0, 3], [0, 33]])
@pytest.mark.parametrize("power", [-12, -6, 6, 12])
@pytest.mark.parametrize("name", NAMES)
def test_values_of_one_size(name, power, first):
    """All values small or large: fp16 tokens (windows, sinks) beside coded ones of the same size."""
    fmt, D = CASES[name]
    n, H, B = 420, 2, first[-1]
    prefix = tokens(fmt, 1, H, D, n, 69, size=np.full(n, 2.0 ** power))
    suffix = tokens(fmt, B, H, D, 170, 70, size=np.full(170, 2.0 ** power))
    check(prefix, suffix, first, along(71, B, 1, 2 * H, D))


@pytest.mark.parametrize("first", [[0, 3], [0, 33]])
@pytest.mark.parametrize("name", ["kivi", "sym4_window", "had_affine_window", "kvarn_sink", "sink32_window", "sink64"])
def test_fp16_tokens_of_all_sizes(name, first):
    """Window and sink tokens from 2^-14 to 2^12 of the others' size, the large ones without weight; the small
    ones' own outputs are in the sum."""
    fmt, D = CASES[name]
    n, H, B = 260, 2, first[-1]
    size = 2.0 ** (np.arange(n) * 7 % 27 - 14.0)
    prefix = tokens(fmt, 1, H, D, n, 72, np.where(size > 0.1, 60.0, 0.0), size)
    suffix = tokens(fmt, B, H, D, 100, 73, np.full(100, 60.0), np.full(100, 2.0 ** 10))
    # (per-channel groups mix keys 60 units apart, as above)
    check(prefix, suffix, first, along(74, B, 1, 2 * H, D), 1.0 if fmt["k_axis"] else 0.5)


@pytest.mark.parametrize("first", [[0, 3], [0, 33]])
@pytest.mark.parametrize("name", ["tiny_b1", "tiny_b16", "gqa12b", "hadamard", "affine8"] + list(MORE))
def test_large_values_of_little_weight_that_dominate(name, first):
    """Values of 2^56 at 35 natural units below the others: weights of 2^-50, outputs of 2^6."""
    fmt, D = {**CASES, **MORE}[name]
    n, H, B = 500, 2, first[-1]
    prefix = tokens(fmt, 1, H, D, n, 75, where(n, 160, 224, 35, 0), where(n, 160, 224, 2.0 ** 56, 1))
    suffix = tokens(fmt, B, H, D, 40, 76)
    # (what dominates has scores of 35 + 5 units: eight times the bound's)
    check(prefix, suffix, first, along(77, B, 1, 2 * H, D), 8.0)
