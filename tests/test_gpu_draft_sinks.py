"""A drafting step over caches with fp16 sink tokens: the draft cache's first tokens,
which all drafts are, stay as fp16 rows there.  The tree's output against 64-bit
attention over the oracle's caches of the same keys, as in test_gpu_tree.py."""
import numpy as np
import pytest
import torch

import oracle
from paper_2609_04263_amd import synth

from gpu_util import host_bits
from test_gpu_drafts import B, C, G, H, Layer, hidden, tree
from test_gpu_shared import close
from test_gpu_tree import reference

pytestmark = pytest.mark.gpu


class Pair:
    """A cache on the GPU, and in the oracle with the keys that kvq_rope_qk makes."""

    def __init__(self, L, T):
        self.L, self.gpu, self.ref = L, L.cache(T), oracle.Cache(L.fmt, B, H, L.D, T)

    def append(self, K, V, **kw):
        turned = torch.empty_like(K)
        self.L.rope.qk(None, K, None, turned, k_norm=self.L.norms["k_norm"], **kw)
        self.ref.append(host_bits(turned), host_bits(V))

    def dequant(self):
        return self.ref.dequant()


@pytest.mark.parametrize("name,n", [("sink64", 70), ("sink64", 40), ("kvarn_sink", 130), ("sink32_window", 150)])
def test_a_step(name, n):
    L = Layer(name, 160)
    committed, draft = Pair(L, n + 20), Pair(L, C)
    _, K, V = L.project(hidden(160, "prompt", n))
    committed.gpu.append_rope(L.rope, K, V, k_norm=L.norms["k_norm"])
    committed.append(K, V)
    parents, depth = tree(161)
    pos = torch.from_numpy(n + depth).int().cuda()
    Q, K, V = L.project(hidden(161, "drafts", C))
    draft.gpu.append_rope(L.rope, K, V, Q=Q, Qo=Q, pos=pos, **L.norms)
    draft.append(K, V, pos=pos)
    for pair in (committed, draft):
        torch.cuda.synchronize()
        assert np.array_equal(pair.gpu.storage.cpu().numpy(), pair.ref.image)
    sees = np.zeros((B, C, C), bool)
    for b in range(B):
        for i in range(C):
            j = i
            while j >= 0:
                sees[b, i, j] = True
                j = int(parents[b, j])
    O = torch.empty((B, C, H * G, L.D), dtype=torch.float32, device="cuda")
    draft.gpu.tree_attn_shared(committed.gpu, Q, C, H * G, L.sm, L.kvq.tree_words(torch.from_numpy(parents)).cuda(), O,
                               draft.gpu.shared_workspace(committed.gpu, H * G, C))
    torch.cuda.synchronize()
    want = reference(committed, draft, list(range(B + 1)), host_bits(Q), L.sm, sees)
    assert np.isfinite(synth.bf16_bits_to_f32(host_bits(Q))).all()
    close(O, want, 1.0, name)
