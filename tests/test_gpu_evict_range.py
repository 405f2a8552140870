"""The cache within a budget at the ends of what its arrays may hold, against oracle/drafts.py."""
import numpy as np
import pytest

from oracle import drafts
from paper_2412_09282_amd import crvq as C

from gpu_util import say
from test_gpu_drafts import random_parents, words_of
from test_gpu_evict import check_gather
from test_gpu_kv import dev, make, values_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page,Hkv,D", [(16, 2, 32), (64, 3, 64), (128, 1, 128)])
def test_gather_of_scales_of_minus_zero(page, Hkv, D):
    """A page whose scale is -0 holds zeros, as one with 0 does: it neither replaces other pages' scales nor stands above NaN."""
    def spoil(cache, table, keep, n, to):
        for side in (2, 3):
            cache[side][table[0, 0], :] = -0.0        # beside pages with scales
            cache[side][table[1, :], :] = -0.0        # nothing else
            cache[side][table[2, 0], :] = -0.0        # beside one that cannot be used
            cache[side][table[2, 1], :] = np.nan
            cache[side][table[3, 0], :] = -0.0        # beside 0
            cache[side][table[3, 1:], :] = 0.0
    d, to = check_gather([3 * page] * 4, [2 * page + 3] * 4, Hkv, D, page, spoil=spoil)
    for scales in d[2:]:
        s = scales.cpu().numpy()[to]
        assert not np.signbit(s[~np.isnan(s)]).any() and (s[0] > 0).all() and (s[1] == 0).all() and (s[3] == 0).all()


def weights_of_scaled(new, kv, Hq, Hkv, D, page, dtype, by, window=0, seed=0, some=False, kind=None):
    """Weights of queries `by` times and key scales 1 / `by` times the usual ones; some: every second row's are 2^-20 of that."""
    g, cache, table, start, kv_len = make(seed + D, new, kv, Hkv, D, page)
    T, B = int(start[-1]), len(new)
    q = values_of(g, T, Hq, D, dtype=dtype)
    q = (q * np.float32(by)).astype(np.float32)
    if some:
        q[::2] *= np.float32(2.0 ** -20)
    cache[2] = (cache[2] / np.float32(by)).astype(np.float32)
    sc = D ** -0.5
    mask = places = None
    if kind:
        words = -(-max(new) // 64)
        trees = [drafts.tree(random_parents(g, n), k, words) for n, k in zip(new, kv)]
        mask, places = np.concatenate([t[0] for t in trees]), np.concatenate([t[1] for t in trees])
        sees = [drafts.sees_mask(t[0], n, k, t[1], window) for t, n, k in zip(trees, new, kv)]
    else:
        sees = [drafts.sees_causal(n, k, True, window) for n, k in zip(new, kv)]
    lse = drafts.attention(cache, table, start, kv_len, q, sc, sees)[1].astype(np.float32)
    assert np.isfinite(lse).all()
    after = np.full((B, Hkv, max(kv) + 2), 7.0, np.float32)
    exp, tol = drafts.weights(cache, table, start, kv_len, q, sc, lse, sees, None, after, 1.0)
    got, d = dev(after), [dev(a) for a in cache]
    say(f"weights {new} of {kv} heads {Hq}/{Hkv} x {D} page {page} {dtype}, queries {by:.3g} times")
    C.crvq_kv_weights(dev(q, dtype), dev(lse), None, got, d[0], d[2], dev(table), dev(start), dev(kv_len), max(new), max(kv), window=window,
                      mask=None if mask is None else words_of(mask), places=None if places is None else dev(places))
    got = got.cpu().numpy().astype(np.float64)
    assert np.isfinite(got).all()
    err = np.abs(got - exp)
    assert (err <= tol).all(), f"{int((err > tol).sum())} off, worst {np.max(err / np.maximum(tol, 1e-300)):.3g} of the bound"


# few columns, a wave's registers full of them, and those that are walked; with masks and without
SCALED = [([1, 1], [300, 700], 4, 4, 128, 64, 0, None), ([9, 3], [700, 90], 2, 2, 64, 32, 0, None), ([16], [500], 4, 2, 256, 64, 0, None),
          ([40, 8], [300, 90], 4, 4, 96, 16, 0, "tree"), ([64, 5], [900, 5], 3, 3, 64, 64, 40, None), ([300, 70], [700, 600], 6, 2, 128, 64, 0, None),
          ([200], [1500], 2, 1, 256, 128, 0, None), ([90, 33], [200, 300], 4, 2, 64, 32, 0, "tree")]


@pytest.mark.parametrize("some", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("new,kv,Hq,Hkv,D,page,window,kind", SCALED)
def test_weights_of_queries_near_the_end_of_fp32(new, kv, Hq, Hkv, D, page, window, kind, dtype, some):
    """Sums of codes times queries beyond fp32, scores of the usual size."""
    weights_of_scaled(new, kv, Hq, Hkv, D, page, dtype, 2.0 ** 118, window, seed=1, some=some, kind=kind)


@pytest.mark.parametrize("by", [2.0 ** -105, 2.0 ** -60, 2.0 ** 60, 2.0 ** 99])
@pytest.mark.parametrize("new,kv,Hq,Hkv,D,page,window,kind", SCALED[:3] + SCALED[5:])
def test_weights_of_queries_of_any_size(new, kv, Hq, Hkv, D, page, window, kind, by):
    for dtype in ("f32", "bf16"):
        weights_of_scaled(new, kv, Hq, Hkv, D, page, dtype, by, window, seed=2, kind=kind)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 30, 100])
def test_weights_of_a_key_of_zeros_among_scores_beyond_fp32(n, dtype):
    """The rows' one token whose score is finite (0) has all of their weight."""
    g, cache, table, start, kv_len = make(3, [n], [200], 1, 64, 64, garbage=False)
    cache[0][:] = -np.abs(cache[0].astype(np.int32) | 1).clip(1, 127)
    page, slot = divmod(37, 64)
    cache[0][table[0, page], 0, slot] = 0
    cache[2][:] = 2.0 ** 112
    q = np.full((n, 2, 64), 2.0 ** 118, np.float32)
    got, d = dev(np.zeros((1, 1, 200), np.float32)), [dev(a) for a in cache]
    C.crvq_kv_weights(dev(q, dtype), dev(np.zeros((n, 2), np.float32)), None, got, d[0], d[2], dev(table), dev(start), dev(kv_len), n, 200)
    exp = np.zeros(200)
    exp[37] = 2 * n
    assert got.cpu().numpy()[0, 0].tolist() == exp.tolist()
