"""GPU parity of the paged 8-bit cache: append (rotation, quantization, storage), read-back and attention,
against the plain numpy definitions in oracle/serve.py.

Append and read round every operation on its own in fp32, so codes, scales and values are compared bit for
bit.  Attention, with A = sum_t p_t |V_t| of a row: a query held in 16 (24) bits below its largest element moves a
score by at most delta = scale * max|q| * 2^-16 (2^-24) * max_t ||K_t||_1 and a weight by 2 delta relatively; scores, exp
and sums in fp32 move it by (8 + 2 |s|_max) 2^-23 + n 2^-24; fp16 weights by 2^-11 (their pairs by 2^-21); the output is
rounded by 2^-8 (2^-23) of itself."""
import numpy as np
import pytest
import torch

from oracle import serve
from paper_2412_09282_amd import crvq as C

from gpu_util import say

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def host(t):
    return t.detach().float().cpu().numpy()


def values_of(g, *shape, dtype="f32", by=1.0):
    x = (g.standard_normal(shape) * by).astype(np.float32)
    return serve.bf16_round(x) if dtype == "bf16" else x


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(DT[dtype])


def make(seed, new, kv, Hkv, D, page, spare=3, garbage=True):
    """A cache of random codes whose pages lie in any order, and the batch arrays."""
    g = np.random.default_rng(seed)
    B = len(new)
    per = max(1, max(-(-k // page) for k in kv))
    n_pages = B * per + spare
    table = g.permutation(n_pages)[:B * per].reshape(B, per).astype(np.int32)
    cache = [g.integers(-127, 128, (n_pages, Hkv, page, D)).astype(np.int8),
             g.integers(-127, 128, (n_pages, Hkv, D, page)).astype(np.int8),
             np.exp2(g.uniform(-1, 1, (n_pages, Hkv)) - 6).astype(np.float32),
             np.exp2(g.uniform(-1, 1, (n_pages, Hkv)) - 6).astype(np.float32)]
    if garbage:  # what no sequence holds must not matter: pages past a length, and their table entries
        for b, k in enumerate(kv):
            for p in range(-(-k // page), per):
                cache[2][table[b, p]] = np.nan
                cache[3][table[b, p]] = np.inf
                table[b, p] = [-1, 1 << 30, table[b, p]][p % 3]
    start = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    return g, cache, table, start, np.array(kv, np.int32)


def angle_table(n, rot):
    a = np.arange(n)[:, None] * 10000.0 ** (-np.arange(rot // 2) * 2 / rot)
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def same_bits(got, exp, what):
    got, exp = np.asarray(got), np.asarray(exp)
    assert got.shape == exp.shape, what
    ok = (got == exp) | (np.isnan(got) & np.isnan(exp)) if got.dtype.kind == "f" else got == exp
    assert ok.all(), f"{what}: {int((~ok).sum())} of {ok.size} differ, first at {np.argwhere(~ok)[0]}: " \
                     f"{got[~ok][0]} for {exp[~ok][0]}"


# ------------------------------------------------------------------------------------------------
# append and read
# ------------------------------------------------------------------------------------------------

APPENDS = [
    # new, kv, Hq, Hkv, D, page, rot, interleaved, dtype
    ([1], [1], 1, 1, 16, 16, 16, False, "f32"),
    ([1], [38], 8, 8, 64, 16, 32, True, "f32"),
    ([1, 1, 1, 0, 1], [64, 65, 1, 0, 200], 8, 2, 128, 64, 128, False, "bf16"),
    ([3, 4, 2], [66, 4, 131], 4, 4, 80, 64, 40, False, "bf16"),      # half of the rotation not a multiple of eight
    ([70, 1, 0, 130], [75, 300, 40, 130], 6, 3, 96, 32, 96, False, "f32"),
    ([300, 17], [513, 17], 2, 1, 256, 256, 64, True, "bf16"),
    ([257], [1000], 5, 5, 112, 128, 0, False, "f32"),
    ([33, 2], [49, 31], 2, 2, 48, 16, 2, False, "f32"),
]


@pytest.mark.parametrize("new,kv,Hq,Hkv,D,page,rot,interleaved,dtype", APPENDS)
@pytest.mark.parametrize("strided", [False, True])
def test_append_and_read(new, kv, Hq, Hkv, D, page, rot, interleaved, dtype, strided):
    say(f"append {new} of {kv} heads {Hq}/{Hkv} x {D} page {page} rot {rot} {dtype} strided {strided}")
    g, cache, table, start, kv_len = make(len(new) + D, new, kv, Hkv, D, page, garbage=False)
    T = int(start[-1])
    qkv = [values_of(g, T, h, D, dtype=dtype, by=by) for h, by in ((Hq, 1.0), (Hkv, 3.0), (Hkv, 0.3))]
    cos, sin = angle_table(max(kv) + 1, rot) if rot else (None, None)
    exp, q_exp = serve.append(cache, table, start, kv_len, qkv[1], qkv[2], cos, sin, None, interleaved, qkv[0])
    if strided:  # one tensor of all heads with an odd row length: no row is 16-byte aligned
        rows = torch.zeros(T, (Hq + 2 * Hkv) * D + 1, dtype=DT[dtype], device="cuda")
        parts = rows[:, 1:].split([Hq * D, Hkv * D, Hkv * D], 1)
        q, k, v = [p.unflatten(1, (-1, D)) for p in parts]
        for t, a in zip((q, k, v), qkv):
            t.copy_(dev(a))
        q_out = q
    else:
        q, k, v = [dev(a, dtype) for a in qkv]
        q_out = torch.empty_like(q)
    d = [dev(a) for a in cache]
    batch = (dev(table), dev(start), dev(kv_len), max(new))
    angles = dict(cos=None if cos is None else dev(cos), sin=None if sin is None else dev(sin))
    C.crvq_kv_append(k, v, *d, *batch, interleaved=interleaved, q=q, q_out=q_out, **angles)
    torch.cuda.synchronize()
    for name, a, e in zip(("k codes", "v codes", "k scales", "v scales"), d, exp):
        a = a.cpu().numpy()
        if "codes" in name:  # slots past a sequence's length hold nothing
            for b in range(len(new)):
                for s in range(kv[b], -(-kv[b] // page) * page):
                    page_of = table[b, s // page]
                    for x in (a, e):
                        if name[0] == "k":
                            x[page_of, :, s % page] = 0
                        else:
                            x[page_of, :, :, s % page] = 0
        same_bits(a, e, name)
    rounded = serve.bf16_round(q_exp) if dtype == "bf16" else q_exp
    same_bits(host(q_out), rounded, "q")
    # the same call again changes nothing
    before = [t.clone() for t in d]
    if not strided:
        C.crvq_kv_append(k, v, *d, *batch, interleaved=interleaved, q=q, q_out=q_out, **angles)
        for x, y in zip(before, d):
            assert torch.equal(x, y)
    # read back: the whole of every sequence, then its last tokens only
    got = [t.cpu().numpy() for t in d]
    for counts in (kv, new):
        st = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        total = int(st[-1])
        if strided:
            ko = torch.zeros(Hkv, total, D + 3, dtype=DT[dtype], device="cuda")[:, :, 1:D + 1].transpose(0, 1)
        else:
            ko = torch.empty(total, Hkv, D, dtype=DT[dtype], device="cuda")
        vo = torch.empty_like(ko)
        C.crvq_kv_read(ko, vo, *d, dev(table), dev(st), dev(kv_len), max(counts))
        for b in range(len(new)):
            K, V = serve.values(got, table[b], kv[b])
            part = slice(kv[b] - counts[b], kv[b])
            for o, e, what in ((ko, K, "k read"), (vo, V, "v read")):
                e = serve.bf16_round(e[part]) if dtype == "bf16" else e[part]
                same_bits(host(o[st[b]:st[b + 1]]), e, what)


def test_append_token_by_token():
    """A sequence that grows one token at a time, its scales with it, then is read by attention."""
    say("append token by token")
    Hkv, D, page, n = 2, 64, 16, 37
    g, cache, table, _, _ = make(5, [n], [n], Hkv, D, page)
    k = values_of(g, n, Hkv, D) * np.exp(g.uniform(-2, 2, (n, 1, 1))).astype(np.float32)
    v = values_of(g, n, Hkv, D)
    cos, sin = angle_table(n, D)
    d, exp = [dev(a) for a in cache], cache
    for t in range(n):
        start, kv_len = np.array([0, 1], np.int32), np.array([t + 1], np.int32)
        exp, _ = serve.append(exp, table, start, kv_len, k[t:t + 1], v[t:t + 1], cos, sin)
        C.crvq_kv_append(dev(k[t:t + 1]), dev(v[t:t + 1]), *d, dev(table), dev(start), dev(kv_len), 1, cos=dev(cos), sin=dev(sin))
        for p in range(t // page + 1):
            same_bits(d[2][table[0, p]].cpu().numpy(), exp[2][table[0, p]], f"k scale after {t + 1}")
        K, V = serve.values([a.cpu().numpy() for a in d], table[0], t + 1)
        Ke, Ve = serve.values(exp, table[0], t + 1)
        same_bits(K, Ke, f"keys after {t + 1}")
        same_bits(V, Ve, f"values after {t + 1}")


def test_append_positions_and_bad_indices():
    """Given places, places outside the table, pages that do not exist, and sequences left out."""
    say("append: positions, bad indices")
    Hq, Hkv, D, page = 2, 2, 32, 16
    new, kv = [2, 3, 4, 2], [20, 5, 40, 2]
    g, cache, table, start, kv_len = make(11, new, kv, Hkv, D, page, garbage=False)
    T = sum(new)
    q, k, v = values_of(g, T, Hq, D), values_of(g, T, Hkv, D), values_of(g, T, Hkv, D)
    cos, sin = angle_table(50, 16)
    places = g.integers(0, 50, T).astype(np.int32)
    places[3], places[10] = 50, -1            # rows of sequence 1 and 3: rotated elements NaN
    table[2, 2] = len(cache[0])               # sequence 2's new tokens have no page
    exp, q_exp = serve.append(cache, table, start, kv_len, k, v, cos, sin, places, False, q)
    d = [dev(a) for a in cache]
    qo = torch.zeros(T, Hq, D, device="cuda")
    C.crvq_kv_append(dev(k), dev(v), *d, dev(table), dev(start), dev(kv_len), max(new), cos=dev(cos), sin=dev(sin),
                     positions=dev(places), q=dev(q), q_out=qo)
    same_bits(host(qo), q_exp, "q")
    assert np.isnan(q_exp).sum() == 2 * Hq * 16
    for b in (0, 1, 3):
        for i, (x, e) in enumerate(zip(d, exp)):
            for p in range(-(-kv[b] // page)):
                if i > 1:
                    same_bits(x[table[b, p]].cpu().numpy(), e[table[b, p]], f"scales of sequence {b}")
    assert torch.isnan(d[2][int(table[1, 0])]).all() and not torch.isnan(d[3][int(table[1, 0])]).any()
    for i in range(4):
        same_bits(d[i][int(table[2, 1])].cpu().numpy(), cache[i][int(table[2, 1])], "a page not written to")
    # sequences left out: more tokens than max_new, than the length, a length past the table, rows past the end
    for bad in (dict(max_new=1), dict(kv_len=[1, 2, 3, 1]), dict(kv_len=[999, 999, 999, 999]),
                dict(start=[-3, -2, 20, 30, 40]), dict(start=[5, 3, 2, 1, 0])):
        d = [dev(a) for a in cache]
        C.crvq_kv_append(dev(k), dev(v), *d, dev(table), dev(np.array(bad.get("start", start), np.int32)),
                         dev(np.array(bad.get("kv_len", kv_len), np.int32)), bad.get("max_new", max(new)))
        for x, a in zip(d, cache):
            same_bits(x.cpu().numpy(), a, f"left out {bad}")


def test_append_not_finite():
    say("append: NaN and infinity")
    Hkv, D, page = 2, 32, 16
    g, cache, table, start, kv_len = make(12, [2], [10], Hkv, D, page)
    k, v = values_of(g, 2, Hkv, D), values_of(g, 2, Hkv, D)
    k[1, 0, 3], v[0, 1, 7] = np.inf, np.nan
    exp, _ = serve.append(cache, table, start, kv_len, k, v)
    d = [dev(a) for a in cache]
    C.crvq_kv_append(dev(k), dev(v), *d, dev(table), dev(start), dev(kv_len), 2)
    for x, e in zip(d[2:], exp[2:]):
        same_bits(x.cpu().numpy(), e, "scales")
    assert torch.isnan(d[2][int(table[0, 0]), 0]) and torch.isnan(d[3][int(table[0, 0]), 1])
    out = torch.empty(2, Hkv, D, device="cuda")
    C.crvq_kv_attention(dev(values_of(g, 2, Hkv, D)), out, *d, dev(table), dev(start), dev(kv_len), 2, 10)
    assert torch.isnan(out).all()                     # both heads see a page that is not finite
    zero = torch.zeros(2, Hkv, D, device="cuda")      # nothing but zeros: the smallest scale, zeros come back
    g, cache, table, start, kv_len = make(13, [2], [2], Hkv, D, page)
    d = [dev(a) for a in cache]
    C.crvq_kv_append(zero, zero, *d, dev(table), dev(start), dev(kv_len), 2)
    ko = torch.ones(2, Hkv, D, device="cuda")
    C.crvq_kv_read(ko, None, *d, dev(table), dev(start), dev(kv_len), 2)
    assert (ko == 0).all() and float(d[2][int(table[0, 0]), 0]) == 2.0 ** -100


# ------------------------------------------------------------------------------------------------
# attention
# ------------------------------------------------------------------------------------------------

def check_attention(new, kv, Hq, Hkv, D, page, dtype, causal=True, window=0, seed=0, scale=None, inplace=False,
                    q_by=1.0, strided=False):
    g, cache, table, start, kv_len = make(seed + D, new, kv, Hkv, D, page)
    T = int(start[-1])
    q = values_of(g, T, Hq, D, dtype=dtype, by=q_by)
    sc = D ** -0.5 if scale is None else scale
    exp, lse_exp, size, top, norm = serve.attention(cache, table, start, kv_len, q, sc, causal, window)
    if strided:
        qt = torch.zeros(Hq, T, D + 1, dtype=DT[dtype], device="cuda")[:, :, 1:].transpose(0, 1)
        qt.copy_(dev(q))
    else:
        qt = dev(q, dtype)
    out = qt if inplace else torch.full_like(qt, 7.0)
    lse = torch.full((T, Hq), 7.0, device="cuda")
    C.crvq_kv_attention(qt, out, *[dev(a) for a in cache], dev(table), dev(start), dev(kv_len), max(new), max(kv),
                        scale=scale, causal=causal, window=window, lse=lse)
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
    used = float(np.max(err[size > 0] / tol[size > 0])) if (size > 0).any() else 0.0
    say(f"attention {new} of {kv} heads {Hq}/{Hkv} x {D} page {page} {dtype} causal {causal} window {window}: {used:.2f} of the bound")
    return out


@pytest.mark.parametrize("new,kv,Hq,Hkv,D,page,dtype,causal,window", [
    ([1], [1], 1, 1, 16, 16, "f32", True, 0),
    ([1], [38], 8, 8, 64, 16, "f32", True, 0),
    ([1, 1, 1, 1], [1, 64, 65, 300], 32, 8, 128, 64, "bf16", True, 0),
    ([1, 0, 1, 1], [17, 5, 0, 129], 8, 1, 96, 32, "bf16", True, 0),        # an empty cache: zeros
    ([1, 1], [700, 33], 24, 1, 80, 16, "f32", True, 0),                    # more heads a key head than a tile has
    ([5, 1, 0, 33], [5, 70, 9, 100], 6, 2, 112, 16, "f32", True, 0),
    ([70, 64, 3], [70, 200, 130], 4, 2, 128, 128, "bf16", True, 0),
    ([129], [300], 3, 3, 256, 256, "bf16", True, 0),
    ([40, 20], [90, 20], 4, 4, 64, 64, "f32", True, 1),                    # every token sees itself alone
    ([100, 1, 50], [260, 259, 50], 4, 2, 48, 32, "bf16", True, 37),
    ([33, 7], [100, 7], 4, 2, 192, 64, "f32", False, 0),
    ([20, 6], [7, 0], 2, 2, 32, 16, "bf16", False, 0),                     # more queries than keys, and no keys
    ([20, 6], [7, 3], 2, 2, 32, 16, "f32", True, 0),                       # places below 0 see nothing
    ([2, 3], [1500, 1400], 4, 4, 128, 64, "bf16", True, 500),
])
def test_attention(new, kv, Hq, Hkv, D, page, dtype, causal, window):
    check_attention(new, kv, Hq, Hkv, D, page, dtype, causal, window)


@pytest.mark.parametrize("kv,Hq,Hkv,dtype", [([9001], 8, 1, "bf16"), ([5000, 3, 2049], 4, 2, "f32"), ([4097], 1, 1, "bf16")])
def test_attention_long(kv, Hq, Hkv, dtype):
    """Few rows and long caches: the work is divided along the cache and joined."""
    check_attention([1] * len(kv), kv, Hq, Hkv, 64, 64, dtype, seed=3)


def test_attention_scores_far_apart():
    """Scores of magnitude some hundreds: the running maximum moves, weights vanish."""
    for dtype in ("bf16", "f32"):
        check_attention([3, 1], [400, 1000], 4, 2, 64, 32, dtype, seed=4, scale=2.0)
        check_attention([1, 2], [300, 600], 4, 2, 64, 32, dtype, seed=5, scale=-0.3)
        check_attention([2], [200], 2, 2, 64, 32, dtype, seed=6, q_by=1e-30)
        check_attention([2], [200], 2, 2, 64, 32, dtype, seed=7, q_by=0.0)


@pytest.mark.parametrize("new,kv", [([1, 1], [3000, 100]), ([65, 3], [200, 40])])
def test_attention_in_place_and_strided(new, kv):
    check_attention(new, kv, 8, 2, 64, 32, "bf16", seed=8, inplace=True)
    check_attention(new, kv, 8, 2, 64, 32, "f32", seed=8, inplace=True)
    check_attention(new, kv, 8, 2, 64, 32, "bf16", seed=9, strided=True)
    check_attention(new, kv, 8, 2, 64, 32, "f32", seed=9, strided=True, inplace=True)


@pytest.mark.parametrize("spread", [2.0 ** 60, 2.0 ** -60])
def test_attention_scales_far_apart(spread):
    """Pages of values whose scales differ by 2^60, the large ones first or last."""
    Hkv, D, page, n = 2, 64, 16, 100
    g, cache, table, start, kv_len = make(21, [1], [n], Hkv, D, page)
    for p in range(4, 7):
        cache[3][table[0, p]] *= np.float32(spread)
    q = values_of(g, 1, Hkv, D)
    exp, _, size, top, norm = serve.attention(cache, table, start, kv_len, q, D ** -0.5)
    out = torch.empty(1, Hkv, D, device="cuda")
    C.crvq_kv_attention(dev(q), out, *[dev(a) for a in cache], dev(table), dev(start), dev(kv_len), 1, n)
    move = 2 * D ** -0.5 * np.abs(q).max(-1) * 2.0 ** -24 * norm + (8 + 2 * top) * 2.0 ** -23 + n * 2.0 ** -24
    tol = 2.0 ** -23 * np.abs(exp) + (2.0 ** -21 + move)[..., None] * size
    assert (np.abs(host(out) - exp) <= tol).all()


def test_attention_not_finite_and_bad_indices():
    say("attention: rows and sequences that cannot be computed")
    Hq, Hkv, D, page = 4, 2, 32, 16
    new, kv = [3, 2, 2, 2], [40, 30, 50, 20]
    g, cache, table, start, kv_len = make(31, new, kv, Hkv, D, page)
    T = sum(new)
    q = values_of(g, T, Hq, D)
    args = lambda: (*[dev(a) for a in cache], dev(table), dev(start))  # noqa: E731
    exp = serve.attention(cache, table, start, kv_len, q, D ** -0.5)[0]
    # a NaN and an infinity in queries: that row and head alone
    bad = q.copy()
    bad[1, 2, 5], bad[4, 0, 31] = np.nan, -np.inf
    out = torch.empty(T, Hq, D, device="cuda")
    C.crvq_kv_attention(dev(bad), out, *args(), dev(kv_len), max(new), max(kv))
    nan = np.zeros((T, Hq), bool)
    nan[1, 2] = nan[4, 0] = True
    got = host(out)
    assert np.isnan(got[nan]).all() and np.allclose(got[~nan], exp[~nan], rtol=1e-4, atol=1e-5)
    # a page outside the cache: the rows that see it; with a window that hides it, none
    keep = table.copy()
    table[0, 0], table[2, 1] = -1, len(cache[0])
    C.crvq_kv_attention(dev(q), out, *args(), dev(kv_len), max(new), max(kv))
    got = host(out)
    assert np.isnan(got[[0, 1, 2, 5, 6]]).all() and np.allclose(got[[3, 4, 7, 8]], exp[[3, 4, 7, 8]], rtol=1e-4, atol=1e-5)
    C.crvq_kv_attention(dev(q), out, *args(), dev(kv_len), max(new), max(kv), window=8)
    assert torch.isfinite(out).all()
    table[:] = keep
    # a length past the table, a negative one, more rows than max_new, rows past the end
    lens = kv_len.copy()
    lens[1], lens[3] = 10 ** 6, -1
    C.crvq_kv_attention(dev(q), out, *args(), dev(lens), max(new), max(kv))
    got = host(out)
    assert np.isnan(got[[3, 4, 7, 8]]).all() and np.isfinite(got[[0, 1, 2, 5, 6]]).all()
    out.fill_(7)
    C.crvq_kv_attention(dev(q), out, *args(), dev(kv_len), 2, max(kv))
    got = host(out)
    assert np.isnan(got[:2]).all() and (got[2] == 7).all() and np.isfinite(got[3:]).all()
    out.fill_(7)
    start[4] = T + 5
    C.crvq_kv_attention(dev(q), out, *args(), dev(kv_len), max(new), max(kv))
    got = host(out)
    assert (got[7:] == 7).all() and np.isfinite(got[:7]).all()


def test_attention_is_deterministic_and_follows_its_stream():
    say("attention on a side stream, twice")
    new, kv, Hq, Hkv, D, page = [1] * 5, [3000, 1, 700, 64, 2999], 8, 2, 128, 64
    g, cache, table, start, kv_len = make(41, new, kv, Hkv, D, page)
    q = dev(values_of(g, 5, Hq, D, dtype="bf16"), "bf16")
    a = [*[dev(x) for x in cache], dev(table), dev(start), dev(kv_len), 1, max(kv)]
    one, two = torch.empty_like(q), torch.empty_like(q)
    C.crvq_kv_attention(q, one, *a)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        C.crvq_kv_attention(q, two, *a)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(one, two)
    # what the cache holds past the lengths does not matter
    for b in range(5):
        last = int(table[b, (kv[b] - 1) // page])
        a[0][last, :, kv[b] % page or page:] = -128
        a[1][last, :, :, kv[b] % page or page:] = 127
    C.crvq_kv_attention(q, two, *a)
    assert torch.equal(one, two)


def test_attention_in_a_graph():
    say("attention and append replayed in a graph")
    new, kv, Hq, Hkv, D, page = [1, 1, 1], [500, 64, 2000], 4, 2, 64, 32
    g, cache, table, start, kv_len = make(51, new, kv, Hkv, D, page, garbage=False)
    d = [dev(x) for x in cache]
    q, k, v = [dev(values_of(g, 3, h, D)) for h in (Hq, Hkv, Hkv)]
    out = torch.empty_like(q)
    batch = (dev(table), dev(start), dev(kv_len))

    def step():
        C.crvq_kv_append(k, v, *d, *batch, 1)
        C.crvq_kv_attention(q, out, *d, *batch, 1, max(kv))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        q.copy_(dev(values_of(g, 3, Hq, D)))
        k.mul_(1.25)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        step()
        assert torch.equal(got, out), i


def test_attention_on_a_given_stream():
    """The stream argument, as a stream and as a handle; the workspace is not handed on before the call is done."""
    say("attention on a given stream")
    kv, Hq, Hkv, D, page = [9000], 8, 2, 128, 64
    g, cache, table, start, kv_len = make(61, [1], kv, Hkv, D, page)
    q = dev(values_of(g, 1, Hq, D, dtype="bf16"), "bf16")
    a = [*[dev(x) for x in cache], dev(table), dev(start), dev(kv_len), 1, max(kv)]
    one = torch.empty_like(q)
    C.crvq_kv_attention(q, one, *a)
    torch.cuda.synchronize()
    size = C.lib().crvq_kv_attention_workspace_size(1, Hq, Hkv, D, 1, max(kv))
    assert size > 0
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        outs = []
        for _ in range(20):
            out = torch.empty_like(q)
            C.crvq_kv_attention(q, out, *a, stream=stream)
            torch.full((size,), 255, dtype=torch.uint8, device="cuda")  # would take a freed workspace
            outs.append(out)
        torch.cuda.synchronize()
        assert all(torch.equal(o, one) for o in outs)


@pytest.mark.parametrize("B", [2, 63, 64, 65, 70])
def test_attention_many_sequences(B):
    """Prompts of many sequences of different lengths, empty ones among them: whatever order they are taken in."""
    g = np.random.default_rng(B)
    new = [int(n) for n in g.integers(0, 5, B)]
    new[0] = 4
    kv = [n + int(k) for n, k in zip(new, g.integers(0, 90, B))]
    check_attention(new, kv, 8, 1, 32, 16, "bf16", seed=B)
    check_attention(new, kv, 6, 1, 32, 64, "f32", seed=B)
