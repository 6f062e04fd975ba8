"""Host side of positions and of appends with positions, without a GPU:
frequencies against their formulas, refusals before anything is enqueued."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from paper_2609_04263_amd import configs

from test_gather_plan import cache, status
from test_host_abi import FAKE, FakeStorage, kvq  # noqa: F401  (kvq: the fixture)


def turns(rope):
    return np.array(rope.c.turns[:rope.c.rot // 2])


def plain(rot, base=10000.0):
    return np.array([base ** (-2.0 * i / rot) / (2 * math.pi) for i in range(rot // 2)])


# (frequencies are powers and quotients in 64 bits, a few roundings: 1e-14)
CLOSE = dict(rtol=1e-14, atol=0)


@pytest.mark.parametrize("rot", [16, 64, 96, 128, 256])
def test_frequencies(kvq, rot):
    np.testing.assert_allclose(turns(kvq.Rope(rot)), plain(rot), **CLOSE)
    np.testing.assert_allclose(turns(kvq.Rope(rot, base=500000.0)), plain(rot, 500000.0), **CLOSE)
    np.testing.assert_allclose(turns(kvq.Rope(rot, scaling="linear", factor=4.0)), plain(rot) / 4, **CLOSE)
    t = turns(kvq.Rope(rot, scaling="base", factor=8.0))
    np.testing.assert_allclose(t, plain(rot, 10000.0 * 8.0 ** (rot / (rot - 2))), **CLOSE)
    np.testing.assert_allclose([t[0], t[-1]], [plain(rot)[0], plain(rot)[-1] / 8], rtol=1e-12)
    assert kvq.Rope(rot).c.scale == 1.0 and kvq.Rope(rot).c.eps == np.float32(1e-6)


def test_scaling_by_bands(kvq):
    L, low, high, factor, rot = 2048.0, 1.0, 4.0, 8.0, 128
    got, f = turns(kvq.Rope(rot, 500000.0, scaling="bands", factor=factor, original=L, low=low, high=high)), plain(rot, 500000.0)
    for i in range(rot // 2):
        waves = L * f[i]
        keep = min(1.0, max(0.0, (waves - low) / (high - low)))
        want = f[i] if waves > high else f[i] / factor if waves < low else f[i] * (keep + (1 - keep) / factor)
        assert abs(got[i] - want) <= 1e-14 * want
    assert (got == f).any() or np.allclose(got[0], f[0], **CLOSE)
    np.testing.assert_allclose(got[-1], f[-1] / factor, **CLOSE)


def test_scaling_of_yarn(kvq):
    L, factor, rot, base = 4096.0, 4.0, 128, 10000.0
    r = kvq.Rope(rot, base, scaling="yarn", factor=factor, original=L, low=1.0, high=32.0)
    f = plain(rot, base)
    pair = lambda w: rot * math.log(L / (2 * math.pi * w)) / (2 * math.log(base))  # noqa: E731
    a, b = math.floor(pair(32.0)), math.ceil(pair(1.0))
    # (the pair of w waves makes w waves)
    assert math.isclose(L * base ** (-2 * pair(32.0) / rot) / (2 * math.pi), 32.0, rel_tol=1e-12)
    keep = np.clip((b - np.arange(rot // 2)) / (b - a), 0, 1)
    np.testing.assert_allclose(turns(r), f * (keep + (1 - keep) / factor), rtol=1e-13)
    assert r.c.scale == np.float32(0.1 * math.log(factor) + 1)
    assert turns(r)[0] == turns(kvq.Rope(rot, base))[0]


def test_frequencies_of_ones_own(kvq):
    r = kvq.Rope(32, turns=[0.25] * 16, scale=2.0, eps=1e-5, interleaved=True)
    assert list(r.c.turns[:17]) == [0.25] * 16 + [0.0]
    assert (r.c.layout, r.c.scale, r.c.eps) == (1, 2.0, np.float32(1e-5))
    with pytest.raises(ValueError):
        kvq.Rope(32, turns=[0.25] * 15)
    with pytest.raises(ValueError):
        kvq.Rope(32, scaling="other")


@pytest.mark.parametrize("kw", [
    dict(rot=8), dict(rot=-16), dict(rot=272), dict(rot=24), dict(rot=64, base=1.0), dict(rot=64, base=float("nan")),
    dict(rot=64, base=float("inf")), dict(rot=64, scaling="linear", factor=0.5),
    dict(rot=64, scaling="base", factor=float("inf")), dict(rot=64, scaling="bands", factor=8.0),
    dict(rot=64, scaling="bands", factor=8.0, original=2048.0, low=4.0, high=4.0),
    dict(rot=64, scaling="yarn", factor=8.0, original=2048.0, low=0.0, high=4.0),
    dict(rot=64, scaling="yarn", factor=float("nan"), original=2048.0)])
def test_refused_frequencies(kvq, kw):
    assert status(kvq, lambda: kvq.Rope(**kw)) == kvq.ERR_ARG


def test_init_refuses_unknown_layouts(kvq):
    f, r = kvq.lib().kvq_rope_init, kvq._Rope()
    for layout, scaling in ((2, 0), (-1, 0), (0, 5), (0, -1)):
        assert f(C.byref(r), 64, layout, 1e4, scaling, 1.0, 0.0, 1.0, 2.0) == kvq.ERR_ARG
    assert f(None, 64, 0, 1e4, 0, 1.0, 0.0, 1.0, 2.0) == kvq.ERR_ARG
    assert f(C.byref(r), 0, 0, 1e4, 2, 8.0, 0.0, 1.0, 2.0) == kvq.OK and r.rot == 0


class Shaped(FakeStorage):
    def __init__(self, *shape, addr=FAKE):
        super().__init__(0, addr)
        self.shape = shape

    def dim(self):
        return len(self.shape)

    def get_device(self):
        return self.device_index

    device_index = -1


def ints(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def qk(kvq, rope, Q=Shaped(2, 3, 4, 64), K=Shaped(2, 3, 2, 64, addr=2 * FAKE), **kw):
    return status(kvq, lambda: rope.qk(Q, K, stream=0, **kw))


def test_rope_refusals(kvq):
    rope = kvq.Rope(64)
    assert qk(kvq, rope, Q=Shaped(2, 3, 4, 32), K=None) == kvq.ERR_ARG     # head size
    assert qk(kvq, kvq.Rope(128)) == kvq.ERR_ARG                           # more rotated channels than there are
    assert qk(kvq, rope, Q=Shaped(2, 3, 4, 64, addr=FAKE + 8)) == kvq.ERR_ARG
    assert qk(kvq, rope, q_norm=Shaped(64, addr=FAKE + 2)) == kvq.ERR_ARG
    assert qk(kvq, rope, k_norm=Shaped(64, addr=FAKE + 2)) == kvq.ERR_ARG
    assert qk(kvq, rope, pos0=2 ** 31 - 2) == kvq.ERR_ARG                  # the third token is at 2^31
    assert qk(kvq, rope, Q=Shaped(0, 3, 4, 64), K=None) == kvq.ERR_ARG
    assert qk(kvq, rope, Q=Shaped(2 ** 16, 2 ** 14, 2, 64), K=None) == kvq.ERR_ARG
    assert qk(kvq, rope, Q=Shaped(2 ** 17, 2 ** 14, 1, 64), K=None) == kvq.ERR_ARG
    rope.qk(Shaped(2, 0, 4, 64), None, stream=0)                           # no tokens: nothing to do
    f, r = kvq.lib().kvq_rope_qk, C.byref(rope.c)
    assert f(r, FAKE, None, 1, 1, 4, 0, 64, None, None, FAKE + 2, 0, FAKE, None, 0) == kvq.ERR_ARG
    call = lambda *a: f(*a, None, None, None, 0, FAKE, None, 0)  # noqa: E731
    assert call(None, FAKE, None, 1, 1, 4, 0, 64) == kvq.ERR_ARG
    assert call(r, None, None, 1, 1, 0, 0, 64) == kvq.ERR_ARG              # neither queries nor keys
    assert call(r, None, None, 1, 1, 4, 0, 64) == kvq.ERR_ARG
    assert call(r, FAKE, None, 1, 1, 0, 0, 64) == kvq.ERR_ARG
    assert call(r, FAKE, None, 1, 1, -4, 0, 64) == kvq.ERR_ARG
    assert call(r, FAKE, None, 1, 1, 4, 2, 64) == kvq.ERR_ARG
    assert call(r, FAKE, None, 1, -1, 4, 0, 64) == kvq.ERR_ARG
    assert f(r, FAKE, None, 1, 1, 4, 0, 64, None, None, None, 0, None, None, 0) == kvq.ERR_ARG


@pytest.mark.parametrize("field,value", [("rot", 8), ("rot", -16), ("layout", 2), ("scale", float("inf")),
                                         ("eps", -1.0), ("eps", float("nan"))])
def test_a_bad_table_is_refused(kvq, field, value):
    rope = kvq.Rope(64)
    setattr(rope.c, field, value)
    assert qk(kvq, rope, q_norm=Shaped(64), k_norm=Shaped(64)) == kvq.ERR_ARG
    for bad in (float("nan"), 1.5, -2.0):
        rope = kvq.Rope(64)
        rope.c.turns[31] = bad
        assert qk(kvq, rope) == kvq.ERR_ARG


def test_rope_shapes(kvq):
    rope = kvq.Rope(64)
    for bad in (ints(2, 4), torch.zeros(2, 3, dtype=torch.int64), ints(2, 6)[:, ::2]):
        with pytest.raises(ValueError):
            rope.qk(Shaped(2, 3, 4, 64), Shaped(2, 3, 2, 64), pos=bad, stream=0)
    with pytest.raises(ValueError):
        rope.qk(None, None, stream=0)
    with pytest.raises(ValueError):
        rope.qk(Shaped(2, 3, 4, 64), Shaped(2, 4, 2, 64), stream=0)


def append(kvq, c, rope=None, K=Shaped(3, 8, 2, 64), V=Shaped(3, 8, 2, 64, addr=2 * FAKE), **kw):
    return status(kvq, lambda: c.append_rope(rope or kvq.Rope(64), K, V, stream=0, **kw))


def test_append_refusals(kvq):
    f = configs.make_format()
    c = cache(kvq, f, 3, 2, 64, 100, n=95)
    q = Shaped(3, 4, 8, 64, addr=3 * FAKE)
    assert append(kvq, c) == kvq.ERR_CAPACITY
    assert append(kvq, c, n_new=-1) == kvq.ERR_ARG
    assert append(kvq, c, K=Shaped(3, 8, 2, 64, addr=0), n_new=1) == kvq.ERR_ARG
    assert append(kvq, c, V=Shaped(3, 8, 2, 64, addr=FAKE + 8), n_new=1) == kvq.ERR_ARG
    assert append(kvq, c, K=Shaped(3, 4, 2, 64), n_new=5) == kvq.ERR_ARG          # five of four rows
    assert append(kvq, c, K=Shaped(3, 0, 2, 64), rows=ints(3, 2)) == kvq.ERR_ARG  # chosen from none
    assert append(kvq, c, n_new=4, Q=q) == kvq.ERR_ARG                            # no place for them
    assert append(kvq, c, n_new=4, Qo=q) == kvq.ERR_ARG
    assert append(kvq, c, rows=ints(3, 4), Q=q, Qo=q) == kvq.ERR_ARG              # queries beside chosen rows
    assert append(kvq, c, rope=kvq.Rope(128), n_new=4) == kvq.ERR_ARG
    assert append(kvq, c, n_new=4, k_norm=Shaped(64, addr=FAKE + 4)) == kvq.ERR_ARG
    assert append(kvq, c, n_new=4, pos0=2 ** 31 - 3) == kvq.ERR_ARG
    assert append(kvq, c, n_new=4, fmt=dict(f, k_bits=2, v_bits=2)) == kvq.ERR_FORMAT
    for kw in (dict(rows=ints(3, 5), n_new=4), dict(pos=ints(3, 5), n_new=4), dict(pos=ints(2, 4).long(), n_new=4)):
        with pytest.raises(ValueError):
            append(kvq, c, **kw)
    c.append_rope(kvq.Rope(64), Shaped(3, 8, 2, 64), Shaped(3, 8, 2, 64), n_new=0, stream=0)
    assert append(kvq, c, n_new=0, rope=kvq.Rope(128)) == kvq.ERR_ARG
    lib = kvq.lib()
    assert lib.kvq_append_rope(c.handle, C.byref(kvq.Rope(64).c), FAKE, FAKE, 4, FAKE + 2, 4, None, 0, None, None, None, 0,
                               None, c._fmt_ref, 0) == kvq.ERR_ARG
    bad = lib.kvq_append_rope(c.handle, None, FAKE, FAKE, 4, None, 4, None, 0, None, None, None, 0, None, c._fmt_ref, 0)
    assert bad == kvq.ERR_ARG
    assert c.n == 95


class OnDevice(Shaped):
    device_index = 0


def test_host_indices_beside_device_tensors(kvq):
    # (an address of host memory would be read on the GPU)
    c = cache(kvq, configs.make_format(), 3, 2, 64, 100, n=4)
    k, q = OnDevice(3, 8, 2, 64), OnDevice(3, 2, 8, 64, addr=3 * FAKE)
    for call in (lambda: kvq.Rope(64).qk(q, None, pos=ints(3, 2), stream=0),
                 lambda: kvq.Rope(64).qk(None, k, pos=ints(3, 8), stream=0),
                 lambda: c.append_rope(kvq.Rope(64), k, k, pos=ints(3, 8), stream=0),
                 lambda: c.append_rope(kvq.Rope(64), k, k, rows=ints(3, 2), stream=0),
                 lambda: c.tree_attn_shared(c, q, 2, 8, 0.125, ints(3, 2, 1), q, q, stream=0)):
        with pytest.raises(ValueError, match="device"):
            call()
    assert c.n == 4


def test_queries_of_other_tokens(kvq):
    c = cache(kvq, configs.make_format(), 3, 2, 64, 100, n=4)
    k = Shaped(3, 8, 2, 64)
    for q, kw in ((Shaped(3, 8, 8, 64), dict(n_new=4)), (Shaped(3, 8, 64), {}), (Shaped(3, 4, 8, 64), {})):
        with pytest.raises(ValueError, match="tokens"):
            c.append_rope(kvq.Rope(64), k, k, Q=q, Qo=q, stream=0, **kw)
    assert c.n == 4
