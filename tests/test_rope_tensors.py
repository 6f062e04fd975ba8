"""The binding refuses tensors that are not what a call with positions reads and
writes: the library sees addresses alone, so another shape, type, layout or device
would be read as if it were right, or out of range."""
import pytest
import torch

from paper_2609_04263_amd import configs

from test_gather_plan import cache
from test_host_abi import kvq  # noqa: F401  (the fixture)
from test_rope_host import OnDevice, Shaped

B, N, H_Q, H, D = 3, 4, 8, 2, 64


def bf16(*shape, device="cpu"):
    return torch.zeros(shape, dtype=torch.bfloat16, device=device)


def wrong(*shape, device="cpu"):
    """Tensors in the place of one of this shape: another type, not in one piece, fewer and more numbers."""
    yield torch.zeros(shape, dtype=torch.float32, device=device)
    yield torch.zeros(shape, dtype=torch.float16, device=device)
    yield bf16(*shape[:-1], 2 * shape[-1], device=device)[..., ::2]
    yield bf16(*shape, 2, device=device)[..., 0]
    if len(shape) > 1:
        yield bf16(shape[0], shape[2], shape[1], *shape[3:], device=device).transpose(1, 2)


def counts(*shape, device="cpu"):
    yield bf16(*shape[:-1], shape[-1] - 8, device=device)
    yield bf16(2 * shape[0], *shape[1:], device=device)


def refused(call, match="expected"):
    with pytest.raises(ValueError, match=match):
        call()


def check_qk(kvq, device):
    rope = kvq.Rope(D)
    q, k = (B, N, H_Q, D), (B, N, H, D)
    Q, K = bf16(*q, device=device), bf16(*k, device=device)
    for t in wrong(*q, device=device):
        refused(lambda: rope.qk(t, K, stream=0))
        refused(lambda: rope.qk(t, None, stream=0))
    for t in wrong(*k, device=device):
        refused(lambda: rope.qk(Q, t, stream=0))
        refused(lambda: rope.qk(None, t, stream=0))
    for t in (*wrong(*q, device=device), *counts(*q, device=device)):
        refused(lambda: rope.qk(Q, K, Qo=t, stream=0))
    for t in (*wrong(*k, device=device), *counts(*k, device=device)):
        refused(lambda: rope.qk(Q, K, Ko=t, stream=0))
    for t in (*wrong(D, device=device), *counts(D, device=device)):
        refused(lambda: rope.qk(Q, K, q_norm=t, stream=0))
        refused(lambda: rope.qk(Q, K, k_norm=t, stream=0))


def check_append(kvq, c, device):
    rope = kvq.Rope(D)
    q, k = (B, N, H_Q, D), (B, N, H, D)
    Q, K, V = (bf16(*s, device=device) for s in (q, k, k))

    def append(K=K, V=V, **kw):
        c.append_rope(rope, K, V, stream=0, **kw)
    for s in ((B + 1, N, H, D), (B, N, H + 1, D), (B, N, H, 2 * D), (B, H + 1, D), (B, H, 2 * D), (2 * B, H, D),
              (B, H * D + 8), (B + 1, H * D)):
        t = bf16(*s, device=device)
        refused(lambda: append(K=t, V=t))
    for t in wrong(*k, device=device):
        refused(lambda: append(K=t))
        refused(lambda: append(V=t))
    for t in counts(*k, device=device):
        refused(lambda: append(V=t))
    refused(lambda: append(V=bf16(B, N + 1, H, D, device=device)))
    for t in (*wrong(*q, device=device), *counts(*q, device=device)):
        refused(lambda: append(Q=t, Qo=Q))
        refused(lambda: append(Q=Q, Qo=t))
    for s in ((B - 1, N, H_Q, D), (B, N, H_Q, D // 2)):
        t = bf16(*s, device=device)
        refused(lambda: append(Q=t, Qo=t))
    t = bf16(B - 1, H_Q, D, device=device)  # (one token, without its axis)
    refused(lambda: append(K=K[:, :1].contiguous(), V=V[:, :1].contiguous(), Q=t, Qo=t))
    for t in (*wrong(D, device=device), *counts(D, device=device)):
        refused(lambda: append(k_norm=t))
        refused(lambda: append(Q=Q, Qo=Q, q_norm=t))
    assert c.n == 4


def test_qk(kvq):
    check_qk(kvq, "cpu")


def test_append(kvq):
    check_append(kvq, cache(kvq, configs.make_format(), B, H, D, 100, n=4), "cpu")


def test_weights_of_the_host(kvq):
    c = cache(kvq, configs.make_format(), B, H, D, 100, n=4)
    q, k, w = OnDevice(B, N, H_Q, D), OnDevice(B, N, H, D), bf16(D)
    for call in (lambda: kvq.Rope(D).qk(q, k, q_norm=w, stream=0), lambda: kvq.Rope(D).qk(None, k, k_norm=w, stream=0),
                 lambda: c.append_rope(kvq.Rope(D), k, k, k_norm=w, stream=0),
                 lambda: c.append_rope(kvq.Rope(D), k, k, Q=q, Qo=q, q_norm=w, stream=0)):
        refused(call, "device")
    assert c.n == 4


def test_positions_beyond_32_bits(kvq):
    c = cache(kvq, configs.make_format(), B, H, D, 100, n=4)
    k = Shaped(B, N, H, D)
    for pos0 in (2 ** 31, -2 ** 31 - 1, 2 ** 32, 2 ** 40):
        for call in (lambda: kvq.Rope(D).qk(None, k, pos0=pos0, stream=0),
                     lambda: c.append_rope(kvq.Rope(D), k, k, pos0=pos0, stream=0)):
            with pytest.raises(kvq.KvqError) as e:
                call()
            assert e.value.status == kvq.ERR_ARG
    assert c.n == 4


def test_no_tokens(kvq):
    # (torch has no address for a tensor without elements)
    rope, none = kvq.Rope(D), bf16(B, 0, H_Q, D)
    assert none.data_ptr() == 0
    rope.qk(none, bf16(B, 0, H, D), stream=0)
    rope.qk(none, None, Qo=bf16(B, 0, H_Q, D), q_norm=bf16(D), stream=0)
    rope.qk(None, bf16(B, 0, H, D), pos=torch.zeros((B, 0), dtype=torch.int32), stream=0)
    c = cache(kvq, configs.make_format(), B, H, D, 100, n=4)
    k = bf16(B, 0, H, D)
    c.append_rope(rope, k, k, stream=0)
    c.append_rope(rope, k, k, Q=none, Qo=none, q_norm=bf16(D), k_norm=bf16(D), stream=0)
    some = bf16(B, N, H, D)
    c.append_rope(rope, some, some, rows=torch.zeros((B, 0), dtype=torch.int32), stream=0)
    assert c.n == 4
    f = kvq.lib().kvq_rope_qk
    for heads in ((0, 0), (-1, 1), (1, -1)):
        assert f(rope._ref, None, None, B, 0, *heads, D, None, None, None, 0, None, None, 0) == kvq.ERR_ARG


@pytest.mark.gpu
def test_on_the_device():
    from paper_2609_04263_amd import kvq
    c = kvq.Cache(configs.make_format(), B, H, D, 100)
    k, v, q = bf16(B, N, H, D, device="cuda"), bf16(B, N, H, D, device="cuda"), bf16(B, N, H_Q, D, device="cuda")
    w = bf16(D, device="cuda")
    c.append_rope(kvq.Rope(D), k, v, Q=q, Qo=torch.empty_like(q), q_norm=w, k_norm=w)
    check_qk(kvq, "cuda")
    check_append(kvq, c, "cuda")
    host = bf16(B, N, H_Q, D)
    for call in (lambda: kvq.Rope(D).qk(q, bf16(B, N, H, D)), lambda: kvq.Rope(D).qk(q, k, Qo=host),
                 lambda: kvq.Rope(D).qk(q, k, k_norm=bf16(D)),
                 lambda: c.append_rope(kvq.Rope(D), k, bf16(B, N, H, D)), lambda: c.append_rope(kvq.Rope(D), k, v, Q=host, Qo=q),
                 lambda: c.append_rope(kvq.Rope(D), k, v, Q=q, Qo=host),
                 lambda: c.append_rope(kvq.Rope(D), k, v, Q=q, Qo=q, q_norm=bf16(D))):
        refused(call, "device")
    # slices of a fused projection's rows are refused, its parts made contiguous are not
    qkv = bf16(B, N, H_Q + 2 * H, D, device="cuda")
    parts = qkv.split((H_Q, H, H), 2)
    refused(lambda: c.append_rope(kvq.Rope(D), parts[1], parts[2]))
    c.append_rope(kvq.Rope(D), parts[1].contiguous(), parts[2].contiguous())
    # one token in the projection's own shape
    c.append_rope(kvq.Rope(D), bf16(B, H * D, device="cuda"), bf16(B, H * D, device="cuda"))
    assert c.n == 2 * N + 1
