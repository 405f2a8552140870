"""GPU attention over the paged 8-bit cache at the ends of its range, against float64: weights' bits, masked pages, scales that
lie far apart.

Bounds, for a row with probabilities p, S = sum_t p_t |V_t| and N = max_t ||K_t||_1 over what it sees.  A query element
is held to half a step of max|q| / 8355711 (three digits), below max|q| 2^-24, which moves a score by at most
delta = |scale| max|q| 2^-24 N and a weight by 2 delta relatively (bf16 prompts hold every bf16 element down to 2^-31 of max|q|:
less).  Scores, exp and sums in fp32 move a weight by (8 + 2 |s|_max) 2^-23 + n 2^-24, as in test_gpu_kv.py.  The weights in the
product with the values: fp32 24 bits (2^-23); bf16 prompts 11 bits (2^-11); bf16 single tokens two fp16 terms: the second is off
by at most 2^-24 of the weight or, where it is subnormal, by 2^-25, and the row's largest weight is at least 2^6, so p_t is off
by 2^-24 p_t + 2^-31 max p.  The output is rounded by 2^-8 (bf16) or 2^-23 (fp32) of itself.  Numbers below fp32's normal ones may
be 0: weights below 2^-126 of the row's largest, and results below 2^-126."""
import numpy as np
import pytest
import torch

from oracle import serve
from paper_2412_09282_amd import crvq as C

from gpu_util import say

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(DT[dtype])


def is_step(new, Hq, Hkv):
    return max(new) * (Hq // Hkv) <= 16


def reference(cache, table, start, kv_len, q, scale, causal, window, dtype, step):
    """(out, lse, bound of out, bound of lse) in float64, row by row."""
    kc, vc = [a.astype(np.float64) for a in cache[:2]]
    ks, vs = [a.astype(np.float64) for a in cache[2:]]
    T, Hq, D = q.shape
    G, P = Hq // kc.shape[1], kc.shape[2]
    out, tol = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    lse, lse_tol = np.full((T, Hq), -np.inf), np.zeros((T, Hq))
    rounding, weight = (2.0 ** -8, 2.0 ** -24 if step else 2.0 ** -11) if dtype == "bf16" else (2.0 ** -23, 2.0 ** -23)
    for b in range(len(kv_len)):
        n, length = int(start[b + 1] - start[b]), int(kv_len[b])
        pages = table[b, :-(-length // P)]
        K = (kc[pages] * ks[pages][:, :, None, None]).transpose(1, 0, 2, 3).reshape(kc.shape[1], -1, D)
        V = (vc[pages] * vs[pages][:, :, None, None]).transpose(1, 0, 3, 2).reshape(kc.shape[1], -1, D)
        for i in range(n):
            place = length - n + i
            hi = min(length, place + 1) if causal else length
            lo = max(0, place + 1 - window) if window else 0
            for h in range(Hq):
                row, Kh, Vh = (start[b] + i, h), K[h // G, lo:hi], V[h // G, lo:hi]
                s = Kh @ q[row].astype(np.float64) * scale
                p = np.exp(s - s.max())
                lse[row] = np.log(p.sum()) + s.max()
                p /= p.sum()
                out[row] = p @ Vh
                size, most = p @ np.abs(Vh), p.max() * np.abs(Vh).sum(0)
                move = 2 * abs(scale) * np.abs(q[row]).max() * 2.0 ** -24 * np.abs(Kh).sum(1).max() + \
                    (8 + 2 * np.abs(s).max()) * 2.0 ** -23 + length * 2.0 ** -24
                tol[row] = rounding * np.abs(out[row]) + (weight + move) * size + 2.0 ** -126 * (1 + np.abs(Vh).sum(0))
                if dtype == "bf16" and step:
                    tol[row] += 2.0 ** -31 * most
                lse_tol[row] = move + 2.0 ** -22 * (1 + abs(lse[row]))
    return out, lse, tol, lse_tol


def check(cache, table, new, kv, q, scale, dtype, causal=True, window=0, what=""):
    start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    kv_len = np.array(kv, np.int32)
    step = is_step(new, q.shape[1], cache[0].shape[1])
    exp, lse_exp, tol, lse_tol = reference(cache, table, start, kv_len, q, scale, causal, window, dtype, step)
    qt = dev(q, dtype)
    out, lse = torch.full_like(qt, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    C.crvq_kv_attention(qt, out, *[dev(a) for a in cache], dev(table), dev(start), dev(kv_len), max(new), max(kv), scale=scale,
                        causal=causal, window=window, lse=lse)
    torch.cuda.synchronize()
    got, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
    err = np.abs(got - exp)
    say(f"{what} {new} of {kv} {q.shape[1:]} {dtype} window {window} {'step' if step else 'prompt'}: "
        f"{np.max(err / np.maximum(tol, 1e-300)):.3g} of the bound")
    assert (err <= tol).all() and (np.abs(l - lse_exp) <= lse_tol).all()


def random_cache(g, pages, Hkv, D, page):
    return [g.integers(-127, 128, (pages, Hkv, page, D)).astype(np.int8),
            g.integers(-127, 128, (pages, Hkv, D, page)).astype(np.int8),
            np.exp2(g.uniform(-1, 1, (pages, Hkv)) - 6).astype(np.float32),
            np.exp2(g.uniform(-1, 1, (pages, Hkv)) - 6).astype(np.float32)]


def queries(g, dtype, *shape):
    q = g.standard_normal(shape).astype(np.float32)
    return serve.bf16_round(q) if dtype == "bf16" else q


@pytest.mark.parametrize("D,page", [(64, 16), (128, 64), (96, 32), (192, 64), (256, 16), (256, 256)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_single_tokens_keep_the_weights_bits(D, page, dtype):
    """Many outputs are small sums of large terms, so that a weight's rounding shows past the output's own."""
    g = np.random.default_rng(D + page)
    new, kv, Hq, Hkv = [1, 2, 1, 1], [2, 40, 3, 700], 8, 2
    per = -(-max(kv) // page)
    cache = random_cache(g, 4 * per, Hkv, D, page)
    table = g.permutation(4 * per).reshape(4, per).astype(np.int32)
    check(cache, table, new, kv, queries(g, dtype, sum(new), Hq, D), D ** -0.5, dtype, what="weights' bits")


@pytest.mark.parametrize("window", [0, 3])
@pytest.mark.parametrize("new", [4, 40])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pages_that_a_row_does_not_see(dtype, page, new, window):
    """Scores of about -150 wherever a row looks, and next to them a page that some rows do not see, whose keys are nothing: scale 0,
    or 2^-100 as an append of zeros leaves it.  It is the last page, which the mask hides from the first rows, or the first, which
    the window hides from the last ones."""
    for key_scale in (0.0, 2.0 ** -100):
        g = np.random.default_rng(page + new)
        D, Hq, Hkv = 64, 8, 2
        kv = (page + 5 if new == 4 else page + 35) if window else (2 * page + 2 if new == 4 else 2 * page + 20)
        per = -(-kv // page)
        cache = random_cache(g, per + 1, Hkv, D, page)
        cache[0] = g.integers(-127, -89, cache[0].shape).astype(np.int8)
        cache[2][:] = g.uniform(0.15, 0.17, cache[2].shape)
        table = g.permutation(per + 1)[:per].reshape(1, per).astype(np.int32)
        hidden = [p for p in range(per) if (p * page < 64 and p == 0 if window else p >= 2)]
        for p in hidden:
            cache[2][table[0, p]] = key_scale
        q = (1 + np.abs(queries(g, dtype, new, Hq, D)) / 8).astype(np.float32)
        q = serve.bf16_round(q) if dtype == "bf16" else q
        check(cache, table, [new], [kv], q, D ** -0.5, dtype, window=window, what=f"hidden pages of scale {key_scale:g},")


def paged(g, D, Hq, Hkv, page, n_pages, dtype, n, scores, value_scales):
    """A sequence of n_pages whole pages: score about scores[p] in page p (queries near 1, codes of keys 90 to 127), values of random
    codes with value_scales[p]."""
    cache = random_cache(g, n_pages, Hkv, D, page)
    cache[0] = g.integers(90, 128, cache[0].shape).astype(np.int8)
    table = g.permutation(n_pages).reshape(1, n_pages).astype(np.int32)
    for p in range(n_pages):
        cache[2][table[0, p]] = scores[p] / (D ** 0.5 * 108.5 * 1.1)
        cache[3][table[0, p]] = value_scales[p]
    q = (1 + np.abs(queries(g, dtype, n, Hq, D)) / 8).astype(np.float32)
    return cache, table, serve.bf16_round(q) if dtype == "bf16" else q


# The scales of the first and of the other pages, and by how much the pages with the larger ones score less: nothing of them is
# left (200, 300), or as much as of the others, the sums then holding both (2^60 = e^41.6, 2^100 = e^69.3).
SPREADS = [(0, -60, 200), (-60, 0, 200), (-60, 0, 41.6), (0, -60, 41.6), (50, -50, 69.3), (-50, 50, 69.3), (100, -100, 300),
           (-100, 100, 300), (60, 0, 0), (0, 60, 0)]


@pytest.mark.parametrize("first,second,less", SPREADS)
@pytest.mark.parametrize("page,new", [(64, 1), (16, 1), (64, 40), (16, 40)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_value_scales_far_apart(dtype, page, new, first, second, less):
    """512 tokens, the first half with one magnitude of value scales and the second with another: a wave meets both."""
    g = np.random.default_rng(page + new)
    pages = 512 // page
    half = [p < pages // 2 for p in range(pages)]
    big_first = first > second
    scores = [0.1 if f == big_first else less + 0.1 for f in half]
    cache, table, q = paged(g, 64, 8, 2, page, pages, dtype, new, scores, [2.0 ** (first if f else second) for f in half])
    check(cache, table, [new], [512], q, 64 ** -0.5, dtype, causal=False, what=f"value scales 2^{first}, 2^{second}, scores {less},")


@pytest.mark.parametrize("window", [0, 20])
@pytest.mark.parametrize("page,new", [(64, 4), (16, 4), (64, 40), (16, 40)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_value_scales_of_pages_that_a_row_does_not_see(dtype, page, new, window):
    """Next to pages of value scale 2^-60 one of 2^60 that some rows of a tile do not see: the last one under the mask, or the first
    one under the window."""
    g = np.random.default_rng(page + new)
    n_pages = -(-(page + 40) // page) if window else 3
    kv = page + 18 + new // 2 if window else 2 * page + new // 2
    scales = [2.0 ** (60 if (p == 0 if window else p == 2) else -60) for p in range(max(n_pages, -(-kv // page)))]
    cache, table, q = paged(g, 64, 8, 2, page, len(scales), dtype, new, [0.5] * len(scales), scales)
    check(cache, table, [new], [kv], q, 64 ** -0.5, dtype, window=window, what="hidden value scales,")


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_value_scales_of_zero(dtype, new):
    """A page whose value scale is 0 adds nothing, whatever its codes are."""
    g = np.random.default_rng(new)
    for scales in ([0.0] * 8, [1.0, 0.0, 0.0, 2.0 ** -60] * 2, [0.0, 2.0 ** -60, 1.0, 0.0] * 2):
        scores = [300.0 if s < 1 else 0.1 for s in scales]
        cache, table, q = paged(g, 64, 8, 2, 64, 8, dtype, new, scores, scales)
        check(cache, table, [new], [512], q, 64 ** -0.5, dtype, causal=False, what=f"value scales {scales[:4]},")


@pytest.mark.parametrize("value_log", [-40, 0, 40])
@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_past_2_24(dtype, new, value_log):
    """Scores so large that an exponent added to them is lost in their rounding.  All keys are the same, so the weights are equal
    whatever a score's rounding is, and an output is the mean of the values, up to the weights' own bits and n sums in fp32."""
    g = np.random.default_rng(new)
    D, Hq, Hkv, page, n = 64, 8, 2, 64, 300
    cache = random_cache(g, 5, Hkv, D, page)
    cache[0][:] = 100
    cache[2][:], cache[3][:] = 2.0 ** 10, 2.0 ** value_log
    table = np.array([[3, 0, 4, 1, 2]], np.int32)
    q = np.full((new, Hq, D), 2.0 ** 12, np.float32)
    start, kv_len = np.array([0, new], np.int32), np.array([n], np.int32)
    out = torch.full((new, Hq, D), 7.0, device="cuda").to(DT[dtype])
    C.crvq_kv_attention(dev(q, dtype), out, *[dev(a) for a in cache], dev(table), dev(start), dev(kv_len), new, n, causal=False)
    V = cache[1][table[0]].astype(np.float64).transpose(1, 0, 3, 2).reshape(Hkv, -1, D)[:, :n] * 2.0 ** value_log
    exp, size = np.repeat(V.mean(1), Hq // Hkv, 0)[None], np.repeat(np.abs(V).mean(1), Hq // Hkv, 0)[None]
    rounding, weight = (2.0 ** -8, 2.0 ** -11) if dtype == "bf16" else (2.0 ** -23, 2.0 ** -23)
    err = np.abs(out.double().cpu().numpy() - exp)
    assert (err <= rounding * np.abs(exp) + (weight + n * 2.0 ** -24) * size).all()
