"""Drafted tokens as a serving loop handles them: projection, append with
positions into a draft cache, attention of the tree over the committed cache
and the drafts, append of the accepted path, the next step.

A node's output is compared with decode attention over a cache that holds its
path alone, and the committed cache with one that was appended to token by
token, byte for byte.
"""
import numpy as np
import pytest
import torch

from paper_2609_04263_amd import synth

from gpu_util import ATOL, RTOL, assert_close, dev_bf16
from test_gpu_append import CASES

pytestmark = pytest.mark.gpu

B, H, G, C, D_IN = 3, 2, 4, 13, 256


class Layer:
    """One layer's projection, norms and positions."""

    def __init__(self, name, seed):
        from paper_2609_04263_amd import kvq
        self.kvq, (self.fmt, self.D) = kvq, CASES[name]
        d_q, d_kv = H * G * self.D, H * self.D
        self.d_q, self.d_kv = d_q, d_kv
        self.W = dev_bf16(synth.normal_bf16(seed, "W", (d_q + 2 * d_kv, D_IN), std=D_IN ** -0.5))
        self.norms = {k: dev_bf16(synth.to_bf16_bits(1 + 0.2 * synth.stream(seed, k).standard_normal(self.D).astype(np.float32)))
                      for k in ("q_norm", "k_norm")}
        self.rope = kvq.Rope(self.D, 500000.0)
        self.sm = self.D ** -0.5

    def project(self, x):
        n = x.shape[1]
        Q, K, V = (torch.empty((B, n, h, self.D), dtype=torch.bfloat16, device="cuda") for h in (H * G, H, H))
        self.kvq.project_qkv(x.view(B * n, D_IN), self.W, None, None, 0, 0.0, self.d_q, self.d_kv, Q, K, V, None)
        return Q, K, V

    def cache(self, T):
        return self.kvq.Cache(self.fmt, B, H, self.D, T)


def hidden(seed, name, n):
    return dev_bf16(synth.normal_bf16(seed, name, (B, n, D_IN)))


def tree(seed):
    """Parents [B, C] and depths of a random tree."""
    rng = synth.stream(seed, "tree")
    parents = np.array([[int(rng.integers(max(-1, i - 4), i)) if i else -1 for i in range(C)] for _ in range(B)])
    depth = np.zeros((B, C), np.int64)
    for i in range(C):
        for b in range(B):
            depth[b, i] = depth[b, parents[b, i]] + 1 if parents[b, i] >= 0 else 0
    return parents, depth


def path(parents, i):
    out = []
    while i >= 0:
        out.append(i)
        i = int(parents[i])
    return out[::-1]


# (lengths that leave the KIVI window's oldest tokens where they are for a path of C)
@pytest.mark.parametrize("name,n", [("tiny_b16", 97), ("gqa12b", 64), ("hadamard", 130), ("kivi", 130), ("affine8", 33),
                                    ("sink64", 70)])
def test_steps_of_a_drafting_loop(name, n):
    L = Layer(name, 60)
    committed, alone = L.cache(n + 200), L.cache(n + 200)
    _, K, V = L.project(hidden(60, "prompt", n))
    for c in (committed, alone):
        c.append_rope(L.rope, K, V, k_norm=L.norms["k_norm"])
    draft = L.cache(C)
    O = torch.empty((B, C, H * G, L.D), dtype=torch.float32, device="cuda")
    ws = draft.shared_workspace(committed, H * G, C)
    for step in range(2):
        n = committed.n
        parents, depth = tree(61 + step)
        pos = torch.from_numpy(n + depth).int().cuda()
        Q, K, V = L.project(hidden(61 + step, "drafts", C))
        draft.reset()
        draft.append_rope(L.rope, K, V, Q=Q, Qo=Q, pos=pos, **L.norms)
        draft.tree_attn_shared(committed, Q, C, H * G, L.sm, L.kvq.tree_words(torch.from_numpy(parents)).cuda(), O, ws)
        # every sequence's deepest node, and its path alone
        last = depth.argmax(1)
        paths = [path(parents[b], int(last[b])) for b in range(B)]
        m = min(map(len, paths))
        kr = torch.empty_like(K)
        L.rope.qk(None, K, None, kr, k_norm=L.norms["k_norm"], pos=pos)
        out = torch.empty((B, H * G, L.D), dtype=torch.float32, device="cuda")
        for j in range(m):
            at = torch.tensor([p[j] for p in paths], device="cuda")
            seq = torch.arange(B, device="cuda")
            alone.append(kr[seq, at][:, None].contiguous(), V[seq, at][:, None].contiguous())
            alone.decode_attn(Q[seq, at].contiguous(), H * G, L.sm, out, alone.decode_workspace(H * G))
            torch.cuda.synchronize()
            if L.fmt["sink"]:  # (drafts are the first tokens of their cache, so it holds them as fp16 sink rows)
                continue
            assert_close(O[seq, at].cpu().numpy(), out.cpu().numpy(), f"{name} step {step} depth {j}", ATOL, RTOL)
        # the accepted path
        rows = torch.tensor([p[:m] for p in paths], dtype=torch.int32, device="cuda")
        committed.append_rope(L.rope, K, V, rows=rows, k_norm=L.norms["k_norm"], pos0=n)
        assert committed.length() == alone.length()
        assert torch.equal(committed.storage, alone.storage), f"{name} step {step}"


@pytest.mark.parametrize("name", ["tiny_b16", "kivi", "hadamard"])
def test_a_captured_step(name):
    n = 130
    L = Layer(name, 70)
    committed = L.cache(n + 20)
    _, K, V = L.project(hidden(70, "prompt", n))
    committed.append_rope(L.rope, K, V)
    draft, parents = L.cache(C), tree(71)
    x = hidden(71, "drafts", C)
    pos = torch.from_numpy(n + parents[1]).int().cuda()
    words = L.kvq.tree_words(torch.from_numpy(parents[0])).cuda()
    O, ws = torch.empty((B, C, H * G, L.D), dtype=torch.float32, device="cuda"), draft.shared_workspace(committed, H * G, C)
    Q, K, V = (torch.empty((B, C, h, L.D), dtype=torch.bfloat16, device="cuda") for h in (H * G, H, H))

    def step():
        draft.reset()
        L.kvq.project_qkv(x.view(B * C, D_IN), L.W, None, None, 0, 0.0, L.d_q, L.d_kv, Q, K, V, None)
        draft.append_rope(L.rope, K, V, Q=Q, Qo=Q, pos=pos, **L.norms)
        draft.tree_attn_shared(committed, Q, C, H * G, L.sm, words, O, ws)
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for k in range(4):  # other drafts, positions and trees each time
        x.copy_(hidden(80 + k, "drafts", C))
        p, d = tree(80 + k)
        pos.copy_(torch.from_numpy(n + d).int())
        words.copy_(L.kvq.tree_words(torch.from_numpy(p)))
        O.zero_()
        g.replay()
        torch.cuda.synchronize()
        got, image = O.clone(), draft.storage.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, O) and torch.equal(image, draft.storage)
