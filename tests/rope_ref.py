"""Rotary positions and per-head norms in numpy (tests only): in the steps that
the library documents, and in 64 bits."""
import numpy as np

from paper_2609_04263_amd import synth


def angles(turns, pos):
    """Fractions of a turn: 31 bits of position times 24 and times 29 bits of the turns are exact in 64."""
    t, turns = pos.astype(np.longdouble)[..., None], np.asarray(turns, np.float64)
    high = turns.astype(np.float32).astype(np.float64)
    a = t * high.astype(np.longdouble)
    f = (a - np.rint(a)) + t * (turns - high).astype(np.longdouble)
    return f - np.rint(f)


def pairs(x, rot, interleaved):
    return (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])


def joined(a, b, rest, interleaved):
    z = np.stack([a, b], -1).reshape(a.shape[:-1] + (-1,)) if interleaved else np.concatenate([a, b], -1)
    return np.concatenate([z, rest], -1)


def steps(bits, weight, eps, turns, rot, interleaved, pos, scale=1.0):
    """bf16 bits [B, n, H, D] (weight: bits [D] or None) -> bf16 bits, in the documented binary32 steps."""
    x = synth.bf16_bits_to_f32(bits).astype(np.float32)
    D = x.shape[-1]
    if weight is not None:
        total = (x.astype(np.float64) ** 2).sum(-1, keepdims=True)
        r = (1.0 / np.sqrt(total / D + np.float64(np.float32(eps)))).astype(np.float32)
        x = (x * r) * synth.bf16_bits_to_f32(weight).astype(np.float32)
    f = (2 * np.pi * angles(turns, pos)[:, :, None, :].astype(np.float64))
    c = (np.float64(np.float32(scale)) * np.cos(f)).astype(np.float32)
    s = (np.float64(np.float32(scale)) * np.sin(f)).astype(np.float32)
    a, b = pairs(x, rot, interleaved)
    a, b = a * c - b * s, b * c + a * s
    assert a.dtype == np.float32
    return synth.to_bf16_bits(joined(a, b, x[..., rot:], interleaved))


def wide(bits, weight, eps, turns, rot, interleaved, pos, scale=1.0):
    """The definition in 64 bits: values and, per value, the size of what it is summed from."""
    x = synth.bf16_bits_to_f32(bits).astype(np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + float(np.float32(eps)))
        x = x * synth.bf16_bits_to_f32(weight).astype(np.float64)
    f = 2 * np.pi * angles(turns, pos)[:, :, None, :].astype(np.float64)
    c, s = float(np.float32(scale)) * np.cos(f), float(np.float32(scale)) * np.sin(f)
    a, b = pairs(x, rot, interleaved)
    size = np.abs(a) * np.abs(c) + np.abs(b) * np.abs(s), np.abs(b) * np.abs(c) + np.abs(a) * np.abs(s)
    return (joined(a * c - b * s, b * c + a * s, x[..., rot:], interleaved),
            joined(*size, np.abs(x[..., rot:]), interleaved))
