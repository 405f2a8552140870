"""The attention block on quantized data (decode.py): a batch of prompts, a mixed batch, then single tokens, each call's
output against a float64 computation from the block's own 4-bit weights and the cache it left.

The block runs in fp32: each of its two products is exact up to (N/32 + 64) 2^-24 of its terms' magnitude (N <= 128
columns: 2^-18), rotation and attention up to a few 2^-22, so an output row is within 1e-4 of its norm."""
import numpy as np
import pytest
import torch

from oracle import serve
from paper_2412_09282_amd import crvq as C
from paper_2412_09282_amd import decode

from gpu_util import say

pytestmark = pytest.mark.gpu


def values(w, N):
    out = torch.empty(w.codes.shape[0], N, device="cuda")
    C.crvq_w4_dequant(w.codes, w.scales, w.group, out, zeros=w.zeros)
    return out.double().cpu().numpy()


@pytest.mark.parametrize("heads,kv_heads,D,zeros,window", [(4, 4, 32, False, 0), (6, 2, 16, True, 20)])
def test_block(heads, kv_heads, D, zeros, window):
    say(f"attention block {heads}/{kv_heads} x {D}")
    N = 100
    g = np.random.default_rng(heads)
    rand = lambda *s: torch.from_numpy(g.standard_normal(s).astype(np.float32)).cuda()  # noqa: E731
    cache = decode.PagedCache(20, kv_heads, D, page=16)
    cos, sin = decode.rotary_angles(80, D)
    block = decode.AttentionBlock(rand((heads + 2 * kv_heads) * D, N) * 0.1, rand(N, heads * D) * 0.1, heads, kv_heads, cache,
                                  cos, sin, group=32, zeros=zeros, window=window)
    W, Wo = values(block.qkv, N), values(block.out, heads * D)
    for _ in range(3):
        cache.add_sequence()
    for counts in ([30, 7, 0], [1, 20, 5], [1, 1, 1], [1, 1, 1], [1, 0, 1]):
        x = rand(sum(counts), N)
        batch = cache.grow(counts)
        y = block(x, batch).double().cpu().numpy()
        start, lens, table = (t.cpu().numpy() for t in (batch.start, batch.kv_len, batch.table))
        q = (x.double().cpu().numpy() @ W.T)[:, :heads * D].reshape(-1, heads, D).astype(np.float32)
        place = np.concatenate([np.arange(k - n, k) for n, k in zip(counts, lens)]).astype(int)
        q = serve.rotate(q, place, cos.cpu().numpy(), sin.cpu().numpy(), False)
        held = [t.cpu().numpy() for t in cache.tensors]
        o = serve.attention(held, table, start, lens, q, D ** -0.5, True, window)[0]
        e = o.reshape(len(o), -1) @ Wo.T
        assert (np.linalg.norm(y - e, axis=1) <= 1e-4 * np.linalg.norm(e, axis=1)).all()
        # keys and values are stored within a step of their page's scale
        K = (x.double().cpu().numpy() @ W.T)[:, heads * D:(heads + kv_heads) * D].reshape(-1, kv_heads, D).astype(np.float32)
        K = serve.rotate(K, place, cos.cpu().numpy(), sin.cpu().numpy(), False)
        for b, n in enumerate(counts):
            got, _ = serve.values(held, table[b], lens[b])
            step = max((held[2][p].max() for p in table[b, :-(-lens[b] // 16)]), default=0)
            assert n == 0 or np.abs(got[lens[b] - n:] - K[start[b]:start[b + 1]]).max() <= step
    cache.drop_sequence(1)
    assert len(cache.free) == 20 - len(cache.pages[0]) - len(cache.pages[2])
    with pytest.raises(RuntimeError):
        cache.grow([1000, 0, 0])


def test_program():
    say("decode program")
    decode.main(["--channels", "512", "--heads", "8", "--kv-heads", "4", "--seqs", "2", "--prompt", "70", "--steps", "6"])
