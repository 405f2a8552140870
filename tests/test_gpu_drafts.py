"""GPU parity of attention for trees of drafted tokens against the numpy definition in oracle/drafts.py; the bounds are those of
tests/test_gpu_kv.py (the arithmetic is the same), masks and places are compared bit for bit."""
import numpy as np
import pytest
import torch

from oracle import drafts
from paper_2412_09282_amd import crvq as C

from gpu_util import say
from test_gpu_kv import DT, dev, host, make, values_of

pytestmark = pytest.mark.gpu


def random_parents(g, n):
    return np.array([-1 if i == 0 or g.random() < 0.1 else int(g.integers(max(0, i - 4), i)) for i in range(n)], np.int32)


def words_of(mask):
    return torch.from_numpy(mask.view(np.int64)).cuda()


@pytest.mark.parametrize("new,window", [([1], 0), ([5, 0, 3], 0), ([64, 1, 65], 0), ([130, 7], 0), ([300], 0), ([70, 40], 3), ([9], 1)])
def test_tree_mask(new, window):
    g = np.random.default_rng(sum(new))
    kv = [n + int(g.integers(0, 500)) for n in new]
    start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    parents = np.concatenate([random_parents(g, n) for n in new] + [np.zeros(0, np.int32)]).astype(np.int32)
    if new[0] == 64:  # a parent that comes later, and one below -1: the tokens and their children are out
        parents[10], parents[20] = 10, -2
    words = -(-max(new) // 64) + 1
    mask = torch.full((len(parents) + 1, words), 5, dtype=torch.int64, device="cuda")
    places = torch.full((len(parents) + 1,), 77, dtype=torch.int32, device="cuda")
    C.crvq_tree_mask(dev(parents), dev(start), dev(np.array(kv, np.int32)), max(new), mask[:-1], places[:-1], window=window)
    exp = [drafts.tree(parents[start[b]:start[b + 1]], kv[b], words, window) for b in range(len(new))]
    assert (mask.cpu().numpy().view(np.uint64)[:-1] == np.concatenate([e[0] for e in exp])).all()
    assert (places.cpu().numpy()[:-1] == np.concatenate([e[1] for e in exp])).all()
    assert (mask[-1] == 5).all() and int(places[-1]) == 77


def test_tree_mask_leaves_bad_sequences_out():
    start, kv = np.array([0, 3, 9, 40], np.int32), np.array([5, 9, 99], np.int32)  # too many rows; past the last row
    parents = np.array([-1, 0, 0, -1, 0, 1, 2, 3, 4], np.int32)
    mask, places = torch.full((9, 1), 5, dtype=torch.int64, device="cuda"), torch.full((9,), 77, dtype=torch.int32, device="cuda")
    C.crvq_tree_mask(dev(parents), dev(start), dev(kv), 4, mask, places)
    assert mask.flatten().tolist() == [1, 3, 5] + [5] * 6 and places.tolist() == [2, 3, 3] + [77] * 6


def check(new, kv, Hq, Hkv, D, page, dtype, window=0, seed=0, scale=None, kind="tree", inplace=False, strided=False):
    g, cache, table, start, kv_len = make(seed + D, new, kv, Hkv, D, page)
    T = int(start[-1])
    q = values_of(g, T, Hq, D, dtype=dtype)
    sc = D ** -0.5 if scale is None else scale
    words = -(-max(max(new), 1) // 64)
    sees, masks, places = [], [], []
    for n, k in zip(new, kv):
        m, p = drafts.tree(random_parents(g, n), k, words)
        if kind == "any":  # any bits, those past the last token among them, rows of none
            m = g.integers(0, 2 ** 63, (n, words)).astype(np.uint64) * np.uint64(2) + g.integers(0, 2, (n, words)).astype(np.uint64)
            m[::3] = 0
        masks.append(m)
        places.append(p)
        sees.append(drafts.sees_mask(m, n, k, p if kind == "tree" else None, window))
    exp, lse_exp, size, top, norm = drafts.attention(cache, table, start, kv_len, q, sc, sees)
    if strided:
        qt = torch.zeros(Hq, T, D + 1, dtype=DT[dtype], device="cuda")[:, :, 1:].transpose(0, 1)
        qt.copy_(dev(q))
    else:
        qt = dev(q, dtype)
    out = qt if inplace else torch.full_like(qt, 7.0)
    lse = torch.full((T, Hq), 7.0, device="cuda")
    say(f"tree {new} of {kv} heads {Hq}/{Hkv} x {D} page {page} {dtype} window {window} {kind}")
    C.crvq_kv_tree_attention(qt, out, *[dev(a) for a in cache], dev(table), dev(start), dev(kv_len), max(new), max(kv),
                             words_of(np.concatenate(masks)), scale=scale, window=window,
                             places=dev(np.concatenate(places)) if kind == "tree" else None, lse=lse)
    torch.cuda.synchronize()
    bits, p16, o16 = (2.0 ** -16, 2.0 ** -11, 2.0 ** -8) if dtype == "bf16" else (2.0 ** -24, 2.0 ** -21, 2.0 ** -23)
    delta = abs(sc) * np.abs(q).max(-1) * bits * norm
    move = 2 * delta + (8 + 2 * top) * 2.0 ** -23 + max(kv) * 2.0 ** -24
    tol = o16 * np.abs(exp) + (p16 + move)[..., None] * size
    got = host(out).astype(np.float64)
    err = np.abs(got - exp)
    assert np.isfinite(got).all()
    assert (err <= tol).all(), f"worst {np.max(err / np.maximum(tol, 1e-300)):.3g} of the bound"
    l = lse.cpu().numpy().astype(np.float64)
    empty = np.isneginf(lse_exp)
    assert (np.isneginf(l) == empty).all() and (got[empty] == 0).all()
    assert (np.abs(l - lse_exp)[~empty] <= (move + 2.0 ** -22 * (1 + np.abs(np.where(empty, 0, lse_exp))))[~empty]).all()
    return out


CASES = [
    # new, kv, Hq, Hkv, D, page, dtype, window
    ([1], [1], 1, 1, 16, 16, "f32", 0),
    ([8], [46], 8, 8, 64, 16, "f32", 0),
    ([3, 5, 0, 1], [3, 69, 40, 300], 8, 8, 128, 64, "bf16", 0),
    ([16, 2], [700, 33], 2, 2, 80, 16, "bf16", 0),
    ([17, 9], [1000, 64], 4, 4, 128, 64, "bf16", 0),       # more than one tile of columns
    ([24, 24, 7], [90, 24, 513], 6, 6, 96, 32, "f32", 0),
    ([40, 13], [200, 80], 16, 2, 128, 128, "bf16", 0),
    ([64, 30], [127, 640], 4, 1, 64, 64, "bf16", 0),
    ([65, 1], [65, 64], 2, 2, 48, 16, "f32", 0),            # a second word of the mask, no context
    ([130, 77], [400, 1000], 3, 3, 128, 64, "bf16", 0),
    ([61], [2300], 8, 1, 128, 128, "bf16", 0),
    ([33, 8], [500, 200], 4, 2, 256, 256, "bf16", 0),
    ([20, 31], [300, 40], 2, 2, 192, 64, "f32", 0),
    ([12, 30], [600, 35], 4, 4, 64, 32, "bf16", 100),       # windows into the context, and into the drafts
    ([30, 3], [64, 2000], 4, 4, 128, 64, "f32", 2),
    ([6, 20], [4, 0], 2, 2, 32, 16, "bf16", 0),             # more new tokens than the cache has
    ([20, 6], [7, 3], 2, 2, 32, 16, "f32", 5),
]


@pytest.mark.parametrize("kind", ["tree", "any"])
@pytest.mark.parametrize("new,kv,Hq,Hkv,D,page,dtype,window", CASES)
def test_tree_attention(new, kv, Hq, Hkv, D, page, dtype, window, kind):
    check(new, kv, Hq, Hkv, D, page, dtype, window, kind=kind)


@pytest.mark.parametrize("new,Hq,Hkv,dtype", [([5], 8, 8, "bf16"), ([24], 4, 4, "bf16"), ([60], 8, 2, "bf16"), ([7, 30], 4, 4, "f32")])
def test_long_context(new, Hq, Hkv, dtype):
    check(new, [9001 - 600 * i for i in range(len(new))], Hq, Hkv, 64, 64, dtype, seed=3)


def test_many_sequences_and_scores_far_apart():
    g = np.random.default_rng(9)
    new = [int(x) for x in g.integers(0, 30, 70)]
    check(new, [n + int(g.integers(0, 300)) for n in new], 4, 4, 64, 32, "bf16", seed=5)
    for dtype in ("bf16", "f32"):
        check([9, 20], [400, 1000], 4, 2, 64, 32, dtype, seed=4, scale=2.0)
        check([30, 2], [300, 600], 4, 4, 64, 32, dtype, seed=5, scale=-0.3)


def test_in_place_and_strided():
    a = check([30, 12], [300, 200], 6, 3, 64, 64, "bf16", seed=8)
    b = check([30, 12], [300, 200], 6, 3, 64, 64, "bf16", seed=8, inplace=True)
    c = check([30, 12], [300, 200], 6, 3, 64, 64, "bf16", seed=8, strided=True)
    assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("new", [[6, 9], [40, 33]])
def test_a_chain_is_causal_attention(new):
    """A draft without branches sees what crvq_kv_attention's rows see."""
    kv = [700, 90]
    g, cache, table, start, kv_len = make(3, new, kv, 4, 64, 32)
    T = int(start[-1])
    d, q = [dev(a) for a in cache], dev(values_of(g, T, 4, 64))
    parents = np.concatenate([np.arange(n) - 1 for n in new]).astype(np.int32)
    mask, places = torch.zeros(T, 1, dtype=torch.int64, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda")
    C.crvq_tree_mask(dev(parents), dev(start), dev(kv_len), max(new), mask, places)
    for window in (0, 64):
        a, b, la, lb = torch.zeros_like(q), torch.zeros_like(q), torch.zeros(T, 4, device="cuda"), torch.zeros(T, 4, device="cuda")
        where = (*d, dev(table), dev(start), dev(kv_len), max(new), max(kv))
        C.crvq_kv_attention(q, a, *where, window=window, lse=la)
        C.crvq_kv_tree_attention(q, b, *where, mask, window=window, places=places, lse=lb)
        # fp32 to the last few bits, whatever the order of the sums: 2^-24 each of scores, weights and up to 700 terms
        assert torch.allclose(a, b, rtol=0, atol=2.0 ** -12 * float(a.abs().max())) and torch.allclose(la, lb, rtol=0, atol=2.0 ** -12)


def test_bad_pages_rows_and_queries():
    """What a row does not see may be broken; what it sees makes it NaN; rows out of range are left alone."""
    g, cache, table, start, kv_len = make(4, [3, 2], [40, 36], 2, 32, 16, garbage=False)
    table[0, 2] = 10 ** 6  # the page of the first sequence's drafts (tokens 37 .. 39)
    d = [dev(a) for a in cache]
    q = dev(values_of(g, 5, 2, 32))
    mask = torch.tensor([[0], [2], [0], [3], [3]], dtype=torch.int64, device="cuda")
    out = torch.full_like(q, 7.0)
    C.crvq_kv_tree_attention(q, out, *d, dev(table), dev(start), dev(kv_len), 3, 40, mask)
    # tokens 32 .. 36 of the context lie in that page too: every row of the first sequence sees it
    assert torch.isnan(out[:3]).all() and torch.isfinite(out[3:]).all()
    kv_len[0] = 35  # drafts at 32 .. 34, context in the good pages
    C.crvq_kv_tree_attention(q, out, *d, dev(table), dev(start), dev(kv_len), 3, 40, mask)
    assert torch.isfinite(out[[0, 2, 3, 4]]).all() and torch.isnan(out[1]).all()
    q[4, 1, 3] = float("nan")
    out.fill_(7.0)
    start[2] = 6  # the second sequence's rows pass the last one
    C.crvq_kv_tree_attention(q, out, *d, dev(table), dev(start), dev(kv_len), 3, 40, mask)
    assert (out[3:] == 7).all()
    start[2] = 5
    C.crvq_kv_tree_attention(q, out, *d, dev(table), dev(start), dev(kv_len), 3, 40, mask)
    assert torch.isnan(out[4, 1]).all() and torch.isfinite(out[4, 0]).all() and torch.isfinite(out[3]).all()


@pytest.mark.parametrize("new,kv", [([6, 9], [700, 90]), ([40, 33], [3000, 1500])])
def test_captured_and_replayed(new, kv):
    g, cache, table, start, kv_len = make(5, new, kv, 4, 64, 32)
    T = int(start[-1])
    d = [dev(a) for a in cache] + [dev(table), dev(start), dev(kv_len)]
    parents = dev(np.concatenate([random_parents(g, n) for n in new]))
    q, mask = torch.zeros(T, 8, 64, device="cuda", dtype=torch.bfloat16), torch.zeros(T, 1, dtype=torch.int64, device="cuda")
    places = torch.zeros(T, dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)

    def call(out, mask, places):
        C.crvq_tree_mask(parents, d[5], d[6], max(new), mask, places)
        C.crvq_kv_tree_attention(q, out, *d, max(new), max(kv), mask, window=500, places=places)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(out, mask, places)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out, mask, places)
    for k in range(3):
        q.normal_()
        parents.copy_(dev(np.concatenate([random_parents(g, n) for n in new])))
        graph.replay()
        again = torch.empty_like(q)
        call(again, torch.zeros_like(mask), torch.zeros_like(places))
        torch.cuda.synchronize()
        assert torch.equal(out, again)
