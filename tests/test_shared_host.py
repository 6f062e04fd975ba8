"""Host side of the shared-prefix calls, without a GPU: refusals before
anything is enqueued, and workspace sizes."""
import ctypes as C

import pytest

from paper_2609_04263_amd import configs

from test_gather_plan import cache, status
from test_host_abi import FAKE, FakeStorage, kvq  # noqa: F401  (kvq: the fixture)

FAR = FAKE + (1 << 34)


def pair(kvq, f=None, P=2, B=4, H=2, D=64, n_p=50, n_s=10, f2=None):
    f = f or configs.make_format()
    return cache(kvq, f, P, H, D, 100, n=n_p), cache(kvq, f2 or f, B, H, D, 100, n=n_s, addr=FAR)


def calls(kvq, p, s, H_q=8, C_len=2, first=None, Q=FAKE, O=FAKE, ws=FAKE, nbytes=1 << 30, sm=0.125):
    """Both entry points' statuses, or the one they share."""
    q, o, w = FakeStorage(0, Q), FakeStorage(0, O), FakeStorage(nbytes, ws)
    a = status(kvq, lambda: s.decode_attn_shared(p, q, H_q, sm, o, w, first=first, stream=0))
    b = status(kvq, lambda: s.prefill_attn_shared(p, q, C_len, H_q, sm, o, w, first=first, stream=0))
    return a if a == b else (a, b)


def test_refusals(kvq):
    p, s = pair(kvq)
    assert calls(kvq, p, s, H_q=3) == kvq.ERR_ARG
    assert calls(kvq, p, s, H_q=34) == kvq.ERR_ARG      # 17 query heads per KV head
    assert calls(kvq, p, s, H_q=0) == kvq.ERR_ARG
    for bad in ([1, 2, 4], [0, 2, 3], [0, 2, 5], [0, 5, 4], [0, -1, 4]):
        assert calls(kvq, p, s, first=bad) == kvq.ERR_ARG
    for bad in ([0, 4], [0, 1, 2, 4], [0, 2.0, 4]):
        with pytest.raises(ValueError):
            s.decode_attn_shared(p, FakeStorage(0), 8, 0.125, FakeStorage(0), FakeStorage(1 << 30), first=bad, stream=0)
    for kw in (dict(Q=0), dict(O=0), dict(ws=0), dict(Q=FAKE + 8), dict(O=FAKE + 4), dict(ws=FAKE + 8),
               dict(sm=float("nan")), dict(sm=float("inf"))):
        assert calls(kvq, p, s, **kw) == kvq.ERR_ARG, kw
    p3, _ = pair(kvq, P=3)
    assert calls(kvq, p3, s) == kvq.ERR_ARG               # four sequences in three equal groups
    many = cache(kvq, configs.make_format(), 257, 2, 64, 100, n=5)
    assert calls(kvq, many, s, first=[0] * 257 + [4]) == kvq.ERR_ARG
    assert (p.n, s.n) == (50, 10)


def test_caches_of_different_layers(kvq):
    p, s = pair(kvq)
    other = configs.make_format(4, 4, k_group=32)
    assert calls(kvq, p, pair(kvq, f2=other)[1]) == kvq.ERR_FORMAT
    assert calls(kvq, p, pair(kvq, H=4)[1]) == kvq.ERR_ARG
    assert calls(kvq, p, pair(kvq, D=128)[1]) == kvq.ERR_ARG
    lib, n = kvq.lib(), C.c_size_t()
    assert lib.kvq_shared_workspace_bytes(None, s.handle, 1, 8, C.byref(n)) == kvq.ERR_ARG
    assert lib.kvq_shared_workspace_bytes(p.handle, None, 1, 8, C.byref(n)) == kvq.ERR_ARG
    assert lib.kvq_shared_workspace_bytes(p.handle, s.handle, 1, 8, None) == kvq.ERR_ARG


def test_lengths(kvq):
    # nothing to attend to; a chunk longer than the suffix; a chunk of nothing
    p, s = pair(kvq, n_p=0, n_s=0)
    assert calls(kvq, p, s) == kvq.ERR_ARG
    p, s = pair(kvq, n_p=50, n_s=3)
    q, w = FakeStorage(0), FakeStorage(1 << 30)
    for C_len in (4, 0, -1):
        assert status(kvq, lambda: s.prefill_attn_shared(p, q, C_len, 8, 0.125, q, w, stream=0)) == kvq.ERR_ARG
    p, s = pair(kvq, n_p=50, n_s=0)
    assert status(kvq, lambda: s.prefill_attn_shared(p, q, 1, 8, 0.125, q, w, stream=0)) == kvq.ERR_ARG
    # B C H_q is held in 32 bits
    assert status(kvq, lambda: s.shared_workspace_bytes(p, 8, 1 << 27)) == kvq.ERR_ARG


def test_workspace(kvq):
    for D in (64, 128, 256):
        p, s = pair(kvq, D=D, f=configs.make_format(k_group=64))
        for C_len in (1, 2, 10):
            need = s.shared_workspace_bytes(p, 8, C_len)
            rows = 4 * C_len * 8
            assert need >= rows * (D + 2) * 4 * 2 and need % 8 == 0
            q = FakeStorage(0)
            assert status(kvq, lambda: s.prefill_attn_shared(p, q, C_len, 8, 0.125, q, FakeStorage(need - 1),
                                                             stream=0)) == kvq.ERR_WORKSPACE
        # it does not depend on the lengths
        p.restore(0), s.restore(100)
        assert s.shared_workspace_bytes(p, 8, 10) == need


def test_a_workspace_serves_every_smaller_call(kvq):
    # (up to C queries: what a call of fewer needs is never more)
    for D, B, H_q in ((64, 1, 2), (64, 4, 8), (128, 1, 4), (128, 3, 32), (256, 2, 4)):
        p, s = pair(kvq, D=D, P=1, B=B, f=configs.make_format(k_group=64))
        need = [s.shared_workspace_bytes(p, H_q, c) for c in range(1, 400)]
        assert need == sorted(need)
