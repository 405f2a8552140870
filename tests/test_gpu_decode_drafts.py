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


def parents_of(g, n):
    return [-1 if i == 0 else int(g.integers(max(-1, i - 4), i)) for i in range(n)]


@pytest.mark.parametrize("heads,kv_heads,D,page,window", [(4, 2, 32, 16, 0), (3, 3, 16, 32, 6)])
def test_refused_drafts_do_not_count(heads, kv_heads, D, page, window):
    """Of the accepted drafts alone a cache's weights are what 64 bits make of them, token by token; the log-sum-exps that they are
    relative to are the kernel's, which move a weight by less than 1e-4 of itself."""
    say(f"weights of accepted drafts, {heads}/{kv_heads} x {D}, pages of {page}, window {window}")
    t = Block([30, 7, 60], heads, kv_heads, D, page=page, window=window, track=150, seed=D)
    for counts in ([9, 20, 1], [6, 0, 33]):
        trees = [parents_of(t.g, n) for n in counts]
        context = list(t.cache.lengths)
        x, base = t.rand(sum(counts), t.N), host(t.cache.weights).copy()
        batch = t.cache.grow(counts, trees)
        y = t.block(x, batch)
        q = t.queries(x, host(batch.places))
        words = batch.mask.shape[1]
        masks = [drafts.tree(p, c + n, words, window) for p, c, n in zip(trees, context, counts)]
        sees = [drafts.sees_mask(m, n, c + n, p, window) for (m, p), c, n in zip(masks, context, counts)]
        lse = t.check(y, batch, q, sees)
        accepted, start = [], host(batch.start)
        for b, p in enumerate(trees):
            path, i = [], len(p) // 2
            while p and i >= 0:
                path.insert(0, i)
                i = p[i]
            accepted.append(path)
            refused = np.setdiff1d(np.arange(len(p)), path)
            lse[start[b] + refused] = np.inf
        assert np.isinf(lse).any()
        held, table, lens = [host(a) for a in t.cache.tensors], host(batch.table), host(batch.kv_len)
        exp, tol = drafts.weights(held, table, start, lens, q, D ** -0.5, lse, sees, base, base, 1.0)
        if counts[0] == 9:  # while they wait: all of them
            every = host(t.cache.weights)[0].astype(np.float64)
            every[:, :30] -= base[0, :, :30]
            assert np.allclose(every[:, :39].sum(1), 9 * heads / kv_heads, rtol=1e-4, atol=1e-4)
        t.cache.accept(accepted)
        got = host(t.cache.weights)
        for b, (c, a) in enumerate(zip(context, accepted)):
            now = list(range(c)) + [c + i for i in a]
            e, old = exp[b][:, now], np.concatenate([base[b, :, :c], np.zeros((kv_heads, len(a)))], 1)
            assert (np.abs(got[b, :, :len(now)] - e) <= tol[b][:, now] + 1e-4 * np.abs(e - old)).all()
            # a row's weights add up to 1
            assert np.allclose((e - old).sum(1), len(a) * heads / kv_heads, rtol=1e-6)
