"""The forms of the cache within a budget that sizes choose: moves of 256 heads of pages and more, selections with 16 tokens a thread
and of several rounds a workgroup, accumulated weights of either type in and out of registers; against oracle/drafts.py."""
import numpy as np
import pytest
import torch

from paper_2412_09282_amd import crvq as C

from gpu_util import say
from test_gpu_evict import check_gather, check_select, check_weights, normal, strange, ties
from test_gpu_kv import dev, same_bits

pytestmark = pytest.mark.gpu


def heads_of_pages(kept, Hkv, page):
    return max(-(-n // page) for n in kept) * len(kept) * Hkv


@pytest.mark.parametrize("lens,kept,Hkv,D,page", [
    ([700] * 8, [650, 700, 1, 0, 64, 65, 699, 300], 4, 64, 64),   # neighbours: whole rows pass through LDS
    ([4000] * 3, [1600, 1500, 40], 4, 128, 64),                   # runs of a token or two
    ([9000] * 2, [2111, 2100], 8, 80, 128),
    ([30000, 5], [5000, 5], 7, 64, 256),                          # more runs than fit: byte by byte
    ([400] * 9, [399, 300, 17, 16, 15, 400, 0, 31, 33], 2, 96, 16),
    ([500] * 16, [290] * 16, 2, 48, 32),
])
def test_moves_of_many_pages(lens, kept, Hkv, D, page):
    assert heads_of_pages(kept, Hkv, page) >= 256
    check_gather(lens, kept, Hkv, D, page)
    check_gather(lens, kept, Hkv, D, page, heads=1, seed=1)


@pytest.mark.parametrize("make_w", [normal, ties, strange], ids=["normal", "ties", "strange"])
@pytest.mark.parametrize("lens,budget,sinks,recent", [
    ([12000, 9001, 8192, 3], 4000, 4, 100), ([16384, 16383], 16000, 0, 0), ([8193], 1, 0, 1), ([16384, 100], 5000, 2000, 3000)])
def test_select_of_16_tokens_a_thread(lens, budget, sinks, recent, make_w):
    assert 8192 < max(lens) <= 16384
    check_select(lens, 2, max(lens), budget, sinks, recent, make_w)


def kept_of(w, length, budget, sinks, recent):
    """As oracle/drafts.py's select, by a sort of arrays."""
    n = min(length, budget)
    if n == length:
        return np.arange(length)
    t = np.arange(sinks, length - recent)
    x = w[t].astype(np.float64)
    order = np.lexsort((t, np.where(np.isnan(x), 0.0, -x), np.isnan(x)))
    return np.sort(np.concatenate([np.arange(sinks), t[order[:n - sinks - recent]], np.arange(length - recent, length)]))


@pytest.mark.parametrize("make_w", [normal, ties, strange], ids=["normal", "ties", "strange"])
@pytest.mark.parametrize("B,Hkv,ld,budget,sinks,recent", [(64, 2, 70001, 9000, 4, 500), (130, 4, 20001, 15000, 0, 64), (257, 4, 17000, 3000, 4, 0)])
def test_select_in_several_rounds(B, Hkv, ld, budget, sinks, recent, make_w):
    """So many heads that a workgroup's share of a long one is more than its threads take at once."""
    heads = B * Hkv
    chunks = min(-(-1024 // heads), -(-ld // 8192))
    assert -(-ld // chunks) > 8192
    say(f"select {budget} of up to {ld}, {heads} heads in {chunks} parts")
    g = np.random.default_rng(ld)
    lens = g.integers(0, 300, B).astype(np.int32)
    long = g.permutation(B)[:6]
    lens[long] = [ld, ld - 1, 16385, 9217, budget, budget + 1]
    w = make_w(g, (B, Hkv, ld)).astype(np.float32)
    keep, n = torch.full((B, Hkv, budget), -9, dtype=torch.int32, device="cuda"), torch.full((B,), -9, dtype=torch.int32, device="cuda")
    kept_w = torch.full((B, Hkv, budget), -9.0, device="cuda")
    C.crvq_kv_select(dev(w), dev(lens), budget, keep, n, kept_weights=kept_w, sinks=sinks, recent=recent)
    keep, kept_w = keep.cpu().numpy(), kept_w.cpu().numpy()
    assert (n.cpu().numpy() == np.minimum(lens, budget)).all()
    for b in range(B):
        for h in range(Hkv):
            exp = kept_of(w[b, h], int(lens[b]), budget, sinks, recent)
            assert (keep[b, h, :len(exp)] == exp).all() and (keep[b, h, len(exp):] == -9).all(), (b, h)
            same_bits(kept_w[b, h, :len(exp)], w[b, h][exp], "kept weights")
            assert (kept_w[b, h, len(exp):] == -9).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("new,kv,Hq,Hkv,D,page,kind,window", [
    ([16, 9], [500, 64], 2, 2, 256, 64, None, 0), ([17, 30], [300, 700], 2, 2, 192, 32, None, 0), ([60, 33], [400, 90], 2, 2, 256, 256, None, 50),
    ([64, 20], [900, 300], 2, 2, 128, 64, "tree", 0), ([13, 7], [257, 300], 4, 2, 64, 16, "tree", 9),
    ([65, 66], [900, 66], 1, 1, 64, 64, None, 0), ([200, 70], [300, 70], 3, 1, 256, 128, "tree", 0), ([90, 130], [700, 200], 4, 4, 128, 32, None, 64),
    ([130], [3000], 5, 1, 80, 64, "tree", 200)])
def test_weights_in_and_out_of_registers(new, kv, Hq, Hkv, D, page, kind, window, dtype):
    check_weights(new, kv, Hq, Hkv, D, page, dtype, window=window, kind=kind, seed=11)
