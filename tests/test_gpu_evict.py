"""GPU parity of the cache within a budget: accumulated weights against oracle/drafts.py in 64 bits (with its bound), the kept
tokens and the moved codes and scales bit for bit."""
import numpy as np
import pytest
import torch

from oracle import drafts
from paper_2412_09282_amd import crvq as C

from gpu_util import say
from test_gpu_drafts import random_parents, words_of
from test_gpu_kv import dev, make, same_bits, values_of

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------
# weights
# ------------------------------------------------------------------------------------------------

def check_weights(new, kv, Hq, Hkv, D, page, dtype, causal=True, window=0, seed=0, scale=None, kind=None, decay=1.0, with_before=True,
                  strided=False):
    g, cache, table, start, kv_len = make(seed + D, new, kv, Hkv, D, page)
    T, B = int(start[-1]), len(new)
    q = values_of(g, T, Hq, D, dtype=dtype)
    sc = D ** -0.5 if scale is None else scale
    mask = places = None
    if kind:
        words = -(-max(new) // 64)
        trees = [drafts.tree(random_parents(g, n), k, words) for n, k in zip(new, kv)]
        mask, places = np.concatenate([t[0] for t in trees]), np.concatenate([t[1] for t in trees])
        sees = [drafts.sees_mask(t[0], n, k, t[1], window) for t, n, k in zip(trees, new, kv)]
    else:
        sees = [drafts.sees_causal(n, k, causal, window) for n, k in zip(new, kv)]
    lse = drafts.attention(cache, table, start, kv_len, q, sc, sees)[1].astype(np.float32)
    if T > 3:
        lse[1] = np.nan  # rows that add nothing
        lse[2, 0] = np.inf
    ld = max(kv) + 5
    before = np.exp(g.standard_normal((B, Hkv, ld))).astype(np.float32)
    after = np.full((B, Hkv, ld), 7.0, np.float32)
    exp, tol = drafts.weights(cache, table, start, kv_len, q, sc, lse, sees, before if with_before else None, after, decay)
    qt = dev(q, dtype)
    if strided:
        store = torch.zeros(Hq, T, D + 1, dtype=qt.dtype, device="cuda")[:, :, 1:].transpose(0, 1)
        store.copy_(qt)
        qt = store
    got, d, batch = dev(after), [dev(a) for a in cache], (dev(table), dev(start), dev(kv_len), max(new), max(kv))
    old = dev(before) if with_before else None
    say(f"weights {new} of {kv} heads {Hq}/{Hkv} x {D} page {page} {dtype} causal {causal} window {window} {kind}")
    args = dict(scale=scale, causal=causal, window=window, mask=None if mask is None else words_of(mask),
                places=None if places is None else dev(places), decay=decay)
    C.crvq_kv_weights(qt, dev(lse), old, got, d[0], d[2], *batch, **args)
    err = np.abs(got.cpu().numpy().astype(np.float64) - exp)
    assert (err <= tol).all(), f"{int((err > tol).sum())} off, worst {np.max(err / np.maximum(tol, 1e-300)):.3g} of the bound " \
                               f"at {np.unravel_index((err - tol).argmax(), err.shape)}"
    if with_before:  # in place; what the call leaves alone stays as it was
        C.crvq_kv_weights(qt, dev(lse), old, old, d[0], d[2], *batch, **args)
        touched = np.zeros(after.shape, bool)
        for b, (n, k) in enumerate(zip(new, kv)):
            touched[b, :, :k if n else 0] = True
        same_bits(old.cpu().numpy(), np.where(touched, got.cpu().numpy(), before), "in place")
    return got


@pytest.mark.parametrize("new,kv,Hq,Hkv,D,page,dtype,causal,window", [
    ([1], [1], 1, 1, 16, 16, "f32", True, 0),
    ([1, 1, 0, 1], [38, 700, 20, 64], 8, 2, 64, 16, "f32", True, 0),
    ([1] * 9, [300, 1, 65, 64, 63, 17, 200, 257, 511], 4, 4, 128, 64, "bf16", True, 0),
    ([4, 1, 4], [1000, 999, 4], 8, 8, 80, 32, "bf16", True, 0),
    ([70, 3, 64], [90, 300, 64], 6, 2, 96, 64, "bf16", True, 0),
    ([300], [300], 3, 3, 256, 256, "f32", True, 0),
    ([300, 17], [700, 300], 16, 2, 128, 128, "bf16", True, 0),
    ([100, 1, 50], [260, 259, 50], 4, 2, 48, 32, "bf16", True, 37),
    ([40, 20], [90, 20], 4, 4, 64, 64, "f32", True, 1),
    ([33, 7], [100, 7], 4, 2, 192, 64, "f32", False, 0),
    ([20, 6], [7, 3], 2, 2, 32, 16, "bf16", True, 0),
    ([1, 1], [3000, 2500], 24, 1, 128, 64, "bf16", True, 800),
])
def test_weights(new, kv, Hq, Hkv, D, page, dtype, causal, window):
    check_weights(new, kv, Hq, Hkv, D, page, dtype, causal, window)


def test_weights_variants():
    check_weights([5, 1], [400, 90], 4, 2, 64, 32, "bf16", with_before=False)
    check_weights([5, 1], [400, 90], 4, 2, 64, 32, "f32", decay=0.5)
    check_weights([5, 40], [400, 90], 4, 2, 64, 32, "bf16", scale=1.5)
    check_weights([5, 40], [400, 90], 4, 2, 64, 32, "f32", scale=-0.2, strided=True)
    check_weights([5, 40], [400, 90], 4, 2, 64, 32, "bf16", strided=True)
    for window in (0, 30):
        check_weights([9, 70, 1], [400, 90, 300], 4, 2, 64, 32, "bf16", kind="tree", window=window)
        check_weights([24, 30], [600, 31], 3, 3, 128, 64, "f32", kind="tree", window=window)


def test_weights_of_many_rows_are_shared_out():
    check_weights([1100], [1500], 4, 1, 64, 64, "bf16")
    check_weights([700, 30], [700, 900], 8, 1, 128, 64, "f32", window=600)


def test_weights_sum_to_the_rows():
    """Every row's weights add up to 1: over all tokens and a key head they are its rows times its query heads."""
    new, kv = [33, 2], [500, 130]
    g, cache, table, start, kv_len = make(1, new, kv, 2, 64, 32)
    d, q = [dev(a) for a in cache], dev(values_of(g, 35, 6, 64))
    batch = (dev(table), dev(start), dev(kv_len), 33, 500)
    lse, w = torch.empty(35, 6, device="cuda"), torch.zeros(2, 2, 500, device="cuda")
    C.crvq_kv_attention(q, torch.empty_like(q), *d, *batch, lse=lse)
    C.crvq_kv_weights(q, lse, None, w, d[0], d[2], *batch)
    total = w.double().sum(-1)
    # every weight is off by some 2^-20 of itself at these scores (|s| < 8, lse < 12, 64 elements)
    assert torch.allclose(total, torch.tensor([[99.0], [6.0]], device="cuda", dtype=torch.float64).expand(2, 2), rtol=2.0 ** -18)


def test_weights_leave_bad_sequences_and_pages_alone():
    new, kv = [1, 1, 1, 1], [40, 200, 30, 36]
    g, cache, table, start, kv_len = make(2, new, kv, 2, 32, 16, garbage=False)
    cache[2][table[3, 1], 0] = np.nan
    table[3, 0] = -5
    d, q = [dev(a) for a in cache], dev(values_of(g, 4, 2, 32))
    kv_len[2] = -1
    w = torch.full((4, 2, 60), 7.0, device="cuda")
    C.crvq_kv_weights(q, torch.zeros(4, 2, device="cuda"), None, w, d[0], d[2], dev(table), dev(start), dev(kv_len), 1, 60)
    assert (w[1] == 7).all() and (w[2] == 7).all()                 # longer than max_kv; a negative length
    assert torch.isfinite(w).all() and (w[3, :, :16] == 0).all() and (w[3, 0, 16:32] == 0).all() and (w[3, 1, 16:36] > 0).all()
    assert (w[3, :, 36:] == 7).all() and (w[0, :, :40] > 0).all()


def test_weights_captured_and_replayed():
    for new, kv in (([1, 1], [3000, 90]), ([600], [900])):
        g, cache, table, start, kv_len = make(5, new, kv, 2, 64, 32)
        T = int(start[-1])
        d, batch = [dev(a) for a in cache], (dev(table), dev(start), dev(kv_len), max(new), max(kv))
        q, lse = torch.zeros(T, 4, 64, device="cuda"), torch.full((T, 4), 5.0, device="cuda")
        w = torch.zeros(len(new), 2, max(kv), device="cuda")
        call = lambda w: C.crvq_kv_weights(q, lse, w, w, d[0], d[2], *batch)  # noqa: E731
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call(w)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call(w)
        eager = w.clone()
        for _ in range(3):
            q.normal_()
            graph.replay()
            call(eager)
            torch.cuda.synchronize()
            assert torch.equal(w, eager)


# ------------------------------------------------------------------------------------------------
# selection
# ------------------------------------------------------------------------------------------------

def check_select(lens, Hkv, ld, budget, sinks, recent, make_w, room=0, seed=0):
    g = np.random.default_rng(seed)
    B = len(lens)
    w = make_w(g, (B, Hkv, ld)).astype(np.float32)
    cap = min(budget, ld) + room
    keep, kept_w = torch.full((B, Hkv, cap), -9, dtype=torch.int32, device="cuda"), torch.full((B, Hkv, cap), -9.0, device="cuda")
    n = torch.full((B,), -9, dtype=torch.int32, device="cuda")
    say(f"select {budget} of {lens[:6]}, {Hkv} heads, sinks {sinks}, recent {recent}")
    C.crvq_kv_select(dev(w), dev(np.array(lens, np.int32)), budget, keep, n, kept_weights=kept_w, sinks=sinks, recent=recent)
    keep, kept_w = keep.cpu().numpy(), kept_w.cpu().numpy()
    for b, length in enumerate(lens):
        length = length if 0 <= length <= ld else 0
        assert int(n[b]) == min(length, budget)
        for h in range(Hkv):
            exp = drafts.select(w[b, h], length, budget, sinks, recent)
            assert keep[b, h, :len(exp)].tolist() == exp, (b, h)
            same_bits(kept_w[b, h, :len(exp)], w[b, h][exp], "kept weights")
            assert (keep[b, h, len(exp):] == -9).all() and (kept_w[b, h, len(exp):] == -9).all()


def normal(g, s):
    return np.exp(2 * g.standard_normal(s))


def ties(g, s):
    return np.round(4 * g.random(s)) / 4


def strange(g, s):
    w = g.standard_normal(s) * np.exp2(g.integers(-140, 120, s).astype(np.float64))
    for x in (np.nan, np.inf, -np.inf, 0.0, -0.0, -np.nan):
        w[g.random(s) < 0.05] = x
    return w


@pytest.mark.parametrize("make_w", [normal, ties, strange, lambda g, s: np.zeros(s)], ids=["normal", "ties", "strange", "zeros"])
@pytest.mark.parametrize("lens,budget,sinks,recent", [
    ([1], 1, 0, 0), ([0, 5, 16], 4, 1, 2), ([100, 64, 63, 17], 16, 4, 4), ([1000, 1024, 1025, 2048], 300, 0, 0),
    ([1500, 10], 1500, 3, 7), ([3000], 1, 0, 0), ([700], 699, 0, 699), ([5000, 4999], 2000, 64, 500), ([90, -3, 70000], 10, 0, 0),
    ([400], 0, 0, 0)])
def test_select(lens, budget, sinks, recent, make_w):
    check_select(lens, 3, max(1, max(x for x in lens if x < 60000)), budget, sinks, recent, make_w)


def test_select_long():
    check_select([131001, 70000], 2, 131002, 9000, 4, 1000, ties, room=3)
    check_select([131001], 2, 131002, 130000, 4, 1000, normal)
    check_select([40000, 30000], 1, 40000, 39999, 0, 0, strange)


def test_select_many_heads():
    check_select([300] * 65, 5, 300, 77, 2, 30, ties)


# ------------------------------------------------------------------------------------------------
# the move
# ------------------------------------------------------------------------------------------------

def check_gather(lens, kept, Hkv, D, page, heads=None, seed=0, spoil=None):
    g, cache, table, _, kv_len = make(seed + D, [0] * len(lens), lens, Hkv, D, page, spare=0, garbage=False)
    B, to_pages = len(lens), max(1, -(-max(kept) // page))
    heads = Hkv if heads is None else heads
    n_old = cache[0].shape[0]
    cache = [np.concatenate([a, np.full((B * to_pages + 2, *a.shape[1:]), 99 if a.dtype == np.int8 else 7.0, a.dtype)]) for a in cache]
    cache[2] = np.where(g.random(cache[2].shape) < 0.3, cache[2], cache[2][:1])  # some pages of a head share their scale
    to = (n_old + g.permutation(B * to_pages)).reshape(B, to_pages).astype(np.int32)
    keep = np.full((B, heads, max(kept) + 3), -1, np.int32)
    for b, n in enumerate(kept):
        for h in range(heads):
            keep[b, h, :n] = np.sort(g.permutation(lens[b])[:n])
    n = np.array(kept, np.int32)
    if spoil:
        spoil(cache, table, keep, n, to)
    d = [dev(a) for a in cache]
    say(f"gather {kept} of {lens}, {Hkv} heads x {D}, page {page}, keep of {heads}")
    C.crvq_kv_gather(*d, dev(table), dev(kv_len), dev(keep), dev(n), dev(to))
    exp = drafts.gather(cache, table, kv_len, keep, n, to)
    for x, e, name in zip(d, exp, ("keys", "values", "key scales", "value scales")):
        same_bits(x.cpu().numpy(), e, name)
    return d, to


@pytest.mark.parametrize("lens,kept,Hkv,D,page", [
    ([1], [1], 1, 16, 16), ([40, 100], [16, 17], 2, 64, 16), ([200, 65, 0, 64], [64, 65, 0, 1], 3, 128, 64),
    ([700, 500], [129, 300], 2, 80, 32), ([300], [300], 4, 96, 64), ([1000, 1000], [999, 500], 1, 256, 256), ([600], [130], 2, 192, 128)])
def test_gather(lens, kept, Hkv, D, page):
    check_gather(lens, kept, Hkv, D, page)
    check_gather(lens, kept, Hkv, D, page, heads=1, seed=1)


def test_gather_of_what_is_not_there():
    def spoil(cache, table, keep, n, to):
        keep[0, 0, 3], keep[0, 1, 20] = 300, -1            # past the length; below 0
        table[1, 2] = 10 ** 6                               # a page that is not there
        cache[2][table[2, 0], 1] = np.nan                   # scales that cannot be used
        cache[3][table[2, 1], 0] = -1.0
        cache[2][table[3, 0], :] = 0.0                      # a page of zeros
        to[4, 0], to[5, 1] = -1, 10 ** 6                    # new pages that are not there
        n[6], n[7] = 10 ** 6, -4                            # counts that cannot be
    check_gather([300] * 8, [40] * 8, 2, 32, 16, spoil=spoil)


def test_kept_whole_is_the_same_attention():
    """Everything kept in order: codes, scales and so attention stay as they were, bit for bit."""
    lens, Hkv, D, page = [200, 65], 2, 64, 32
    g, cache, table, start, kv_len = make(3, [2, 1], lens, Hkv, D, page, spare=20, garbage=False)
    free = np.setdiff1d(np.arange(cache[0].shape[0]), table)[:14].reshape(2, 7).astype(np.int32)
    keep = np.tile(np.arange(200, dtype=np.int32), (2, 1, 1))
    d, q = [dev(a) for a in cache], dev(values_of(g, 3, 4, D))
    C.crvq_kv_gather(*d, dev(table), dev(kv_len), dev(keep), dev(kv_len), dev(free))
    a, b = torch.empty_like(q), torch.empty_like(q)
    C.crvq_kv_attention(q, a, *d, dev(table), dev(start), dev(kv_len), 2, 200)
    C.crvq_kv_attention(q, b, *d, dev(free), dev(start), dev(kv_len), 2, 200)
    assert torch.equal(a, b)


def test_evict_captured_and_replayed():
    lens, Hkv, D, page, budget = [500, 90, 700], 2, 64, 32, 96
    g, cache, table, _, kv_len = make(4, [0] * 3, lens, Hkv, D, page, spare=12, garbage=False)
    free = np.setdiff1d(np.arange(cache[0].shape[0]), table)[:9].reshape(3, 3).astype(np.int32)
    d, t, l, to = [dev(a) for a in cache], dev(table), dev(kv_len), dev(free)
    w = torch.zeros(3, Hkv, 700, device="cuda")
    keep, n = torch.zeros(3, Hkv, budget, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")

    def call(d, keep, n):
        C.crvq_kv_select(w, l, budget, keep, n, sinks=2, recent=10)
        C.crvq_kv_gather(*d, t, l, keep, n, to)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(d, keep, n)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(d, keep, n)
    for _ in range(3):
        w.normal_()
        graph.replay()
        d2, k2, n2 = [x.clone() for x in d], torch.zeros_like(keep), torch.zeros_like(n)
        call(d2, k2, n2)
        torch.cuda.synchronize()
        assert torch.equal(n, n2) and torch.equal(keep[:, :, :90], k2[:, :, :90])
        for x, y in zip(d, d2):
            assert torch.equal(x, y)
