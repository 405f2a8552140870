"""Drafted tokens in a block with a window and in a cache that tracks weights (decode.py), against float64 computations from the
block's own 8-bit weights and the cache it left; bounds as in tests/test_gpu_decode_more.py."""
import numpy as np
import pytest
import torch

from oracle import block as ob
from oracle import drafts, serve
from paper_2412_09282_amd import decode

from gpu_util import say
from test_gpu_decode_more import host

pytestmark = pytest.mark.gpu


class Block:
    """One block of 8 bits over a cache, and what its rows have to be."""

    def __init__(self, lengths, heads=4, kv_heads=2, D=32, N=100, page=16, window=0, track=0, seed=0):
        self.g = np.random.default_rng(seed)
        self.heads, self.kv_heads, self.D, self.N, self.window = heads, kv_heads, D, N, window
        self.cache = decode.PagedCache(60, kv_heads, D, page=page, track=track)
        self.angles = decode.rotary_angles(300, D)
        W = [self.rand((heads + 2 * kv_heads) * D, N) * 0.1, self.rand(N, heads * D) * 0.1]
        self.block = decode.AttentionBlock(*W, heads, kv_heads, self.cache, *self.angles, window=window, bits=8)
        for _ in lengths:
            self.cache.add_sequence()
        self.block(self.rand(sum(lengths), N), self.cache.grow(lengths))

    def rand(self, *s):
        return torch.from_numpy(self.g.standard_normal(s).astype(np.float32)).cuda()

    def queries(self, x, places):
        """The rotated queries of rows x, to the bit."""
        m = self.block.qkv
        qkv = ob.w8_product(host(m.codes), host(m.scales), *ob.w8_quantize(host(x)), self.N, False)
        q = qkv[:, :self.heads * self.D].reshape(-1, self.heads, self.D)
        return serve.rotate(q, np.array(places, int), host(self.angles[0]), host(self.angles[1]), False)

    def check(self, y, batch, q, sees):
        """The rows y of a batch; returns what their attention's log-sum-exps are."""
        held = [host(t) for t in self.cache.tensors]
        o, lse = drafts.attention(held, host(batch.table), host(batch.start), host(batch.kv_len), q, self.D ** -0.5, sees)[:2]
        o = o.reshape(len(q), -1)
        W = host(self.block.out.codes)[:, :o.shape[1]].astype(np.float64) * host(self.block.out.scales)[:, None]
        most = np.abs(o).max(1, keepdims=True)
        tol = (most / 254 + 1e-4 * most) * np.abs(W).sum(1)[None] * (1 + 2.0 ** -10)
        assert (np.abs(host(y).astype(np.float64) - o @ W.T) <= tol).all()
        return lse


@pytest.mark.parametrize("window", [1, 8, 19, 40])
def test_a_chain_of_drafts_in_a_window(window):
    """Chains of drafts longer and shorter than the window see what the same tokens see decoded as plain rows."""
    say(f"chains of drafts, window {window}")
    t = Block([30, 3, 50], window=window)
    context, counts = [30, 3, 50], [20, 7, 1]
    x = t.rand(sum(counts), t.N)
    batch = t.cache.grow(counts, [[i - 1 for i in range(n)] for n in counts])
    y = t.block(x, batch)
    places = [c + i for c, n in zip(context, counts) for i in range(n)]
    t.check(y, batch, t.queries(x, places), [drafts.sees_causal(n, c + n, True, window) for c, n in zip(context, counts)])
