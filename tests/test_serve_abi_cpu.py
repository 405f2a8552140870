"""CPU-only: the calls of the quantized attention block reject bad arguments on the host, before anything is
enqueued, and the numpy definitions in oracle/serve.py agree with closed forms."""
import ctypes

import numpy as np
import pytest

from oracle import serve


@pytest.fixture(scope="module")
def L():
    from paper_2412_09282_amd import crvq
    return crvq.lib()


def P(n):
    return ctypes.c_void_p(n << 32)  # never dereferenced


def err(L):
    return L.crvq_last_error().decode()


CACHE = dict(B=2, Hq=8, Hkv=4, D=64, page=32, n_pages=10, k=P(1), v=P(2), ks=P(3), vs=P(4), table=P(5), ld=5, start=P(6),
             kv_len=P(7), max_new=1, n=2, dt=1)


def append(L, **kw):
    a = dict(CACHE, nk=P(8), nv=P(9), q=P(10), qo=P(11), q_tok=512, qo_tok=512, cos=P(12), sin=P(13), angles=100, rot=64)
    a.update(kw)
    return L.crvq_kv_append(a["B"], a["Hq"], a["Hkv"], a["D"], a["page"], a["n_pages"], a["k"], a["v"], a["ks"], a["vs"],
                            a["table"], a["ld"], a["start"], a["kv_len"], a["max_new"], a["n"], a["dt"], a["nk"], 256, 64,
                            a["nv"], 256, 64, a["q"], a["q_tok"], 64, a["qo"], a["qo_tok"], 64, a["cos"], a["sin"],
                            a["angles"], a["rot"], None, 0, None)


def read(L, **kw):
    a = dict(CACHE, ko=P(8), vo=P(9), tok=256)
    a.update(kw)
    return L.crvq_kv_read(a["B"], a["Hkv"], a["D"], a["page"], a["n_pages"], a["k"], a["v"], a["ks"], a["vs"], a["table"],
                          a["ld"], a["start"], a["kv_len"], a["max_new"], a["n"], a["dt"], a["ko"], a["tok"], 64, a["vo"],
                          256, 64, None)


def attend(L, **kw):
    a = dict(CACHE, max_kv=160, q=P(8), q_tok=512, out=P(9), o_tok=512, scale=0.125, causal=1, window=0, lse=None,
             ws=P(20), wsb=1 << 30)
    a.update(kw)
    return L.crvq_kv_attention(a["B"], a["Hq"], a["Hkv"], a["D"], a["page"], a["n_pages"], a["k"], a["v"], a["ks"], a["vs"],
                               a["table"], a["ld"], a["start"], a["kv_len"], a["max_new"], a["max_kv"], a["n"], a["dt"],
                               a["q"], a["q_tok"], 64, a["out"], a["o_tok"], 64, a["scale"], a["causal"], a["window"],
                               a["lse"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("call", [append, read, attend])
def test_cache_arguments(L, call):
    for bad, status, text in [
            (dict(dt=2), 1, "dtype"), (dict(D=8), 2, "D ="), (dict(D=272), 2, "D ="), (dict(D=72), 2, "D ="),
            (dict(page=24), 2, "page"), (dict(page=512), 2, "page"), (dict(page=0), 2, "page"), (dict(Hkv=0), 1, "Hkv"),
            (dict(B=-1), 1, "negative"), (dict(max_new=-1), 1, "negative"), (dict(n=-1), 1, "negative"),
            (dict(n=1 << 31), 2, "rows"), (dict(n_pages=1 << 31), 2, "pages"), (dict(n_pages=-1), 1, "negative"),
            (dict(start=None), 1, "start"), (dict(kv_len=None), 1, "kv_len"), (dict(table=None), 1, "block_table"),
            (dict(k=None), 1, "cache"), (dict(vs=None), 1, "cache"),
            (dict(k=ctypes.c_void_p((1 << 32) + 8)), 1, "aligned"), (dict(v=ctypes.c_void_p((2 << 32) + 4)), 1, "aligned")]:
        assert call(L, **bad) == status, bad
        assert text in err(L), (bad, err(L))
    for nothing in (dict(B=0), dict(max_new=0), dict(n=0)):
        assert call(L, start=None, kv_len=None, **nothing) == 0


def test_append_arguments(L):
    for bad in (dict(nk=None), dict(nv=None), dict(q=None), dict(qo=None), dict(cos=None), dict(sin=None), dict(rot=63),
                dict(rot=66), dict(rot=0), dict(angles=-1), dict(Hq=6), dict(qo_tok=500), dict(q_tok=-1),
                dict(nk=ctypes.c_void_p((8 << 32) + 1)), dict(qo=ctypes.c_void_p((10 << 32) + 64)), dict(v=P(1)),
                dict(qo=P(10), qo_tok=513)):
        assert append(L, **bad) == 1, bad


def test_read_arguments(L):
    assert read(L, ko=None, vo=None) == 0
    assert read(L, tok=200) == 1 and "overlap" in err(L)
    assert read(L, ko=ctypes.c_void_p((8 << 32) + 1)) == 1


def test_attention_arguments(L):
    for bad in (dict(q=None), dict(out=None), dict(Hq=6), dict(Hq=0), dict(max_kv=-1), dict(scale=float("nan")),
                dict(scale=float("inf")), dict(window=-1), dict(window=4, causal=0), dict(o_tok=100),
                dict(out=ctypes.c_void_p((8 << 32) + 128)), dict(lse=P(8)), dict(lse=P(9)), dict(out=P(8), o_tok=1024)):
        assert attend(L, **bad) == 1, bad
    need = L.crvq_kv_attention_workspace_size(1, 64, 8, 128, 1, 131072)
    assert need == L.crvq_workspace_size(10, 1, 1, 0, 0, 128, None, 64, 8, 131072)
    need = L.crvq_kv_attention_workspace_size(1, 64, 8, 64, 1, 131072)  # the helper's heads are 64 elements apart
    assert need > 0 and attend(L, B=1, Hq=64, Hkv=8, max_kv=131072, q_tok=1 << 14, o_tok=1 << 14, wsb=need - 1) == 3
    assert attend(L, B=1, Hq=64, Hkv=8, max_kv=131072, q_tok=1 << 14, o_tok=1 << 14, wsb=need, ws=None) == 3
    assert L.crvq_kv_attention_workspace_size(1, 6, 4, 64, 1, 100) == 0
    assert L.crvq_kv_attention_workspace_size(1, 8, 4, 65, 1, 100) == 0


def test_w4_arguments(L):
    W = dict(M=32, N=100, group=32, codes=P(1), ld=64, s=P(2), sdt=0, lds=4, z=P(3), ldz=4)

    def product(**kw):
        a = dict(W, T=2, x=P(4), ldx=100, xdt=1, y=P(5), ldy=32, ydt=1, ws=P(6), wsb=1 << 30)
        a.update(kw)
        return L.crvq_w4_gemv(a["M"], a["N"], a["T"], a["group"], a["codes"], a["ld"], a["s"], a["sdt"], a["lds"], a["z"],
                              a["ldz"], a["x"], a["ldx"], a["xdt"], a["y"], a["ldy"], a["ydt"], a["ws"], a["wsb"], None)

    def quantize(**kw):
        a = dict(W, W=P(4), ldw=100, dt=0)
        a.update(kw)
        return L.crvq_w4_quantize(a["M"], a["N"], a["group"], a["W"], a["ldw"], a["dt"], a["codes"], a["ld"], a["s"],
                                  a["sdt"], a["lds"], a["z"], a["ldz"], None)

    def dequant(**kw):
        a = dict(W, W=P(4), ldw=100, dt=0)
        a.update(kw)
        return L.crvq_w4_dequant(a["M"], a["N"], a["group"], a["codes"], a["ld"], a["s"], a["sdt"], a["lds"], a["z"],
                                 a["ldz"], a["W"], a["ldw"], a["dt"], None)

    for call in (product, quantize, dequant):
        for bad, status in [(dict(M=-1), 1), (dict(N=0), 1), (dict(group=48), 2), (dict(group=16), 2), (dict(sdt=2), 1),
                            (dict(codes=None), 1), (dict(s=None), 1), (dict(ld=56), 1), (dict(ld=48), 1),
                            (dict(codes=ctypes.c_void_p((1 << 32) + 8)), 1), (dict(lds=3), 1), (dict(ldz=3), 1),
                            (dict(s=ctypes.c_void_p((2 << 32) + 2)), 1), (dict(M=1 << 31), 2)]:
            assert call(**bad) == status, (call.__name__, bad)
        assert call(M=0, codes=None, s=None, z=None) == 0
    for bad in (dict(W=None), dict(ldw=99), dict(dt=2), dict(W=P(1))):
        assert quantize(**bad) == 1 and dequant(**bad) == 1, bad
    assert quantize(s=P(3)) == 1 and "overlap" in err(L)
    for bad in (dict(T=-1), dict(x=None), dict(y=None), dict(ldx=99), dict(ldy=31), dict(xdt=2), dict(ydt=7), dict(y=P(4)),
                dict(y=P(1)), dict(y=P(2))):
        assert product(**bad) == 1, bad
    assert product(T=0, x=None, y=None) == 0
    assert L.crvq_workspace_size(11, 0, 2, 0, 0, 0, None, 32, 100, 0) == L.crvq_w4_gemv_workspace_size(32, 100, 2)


# ---- the definitions against closed forms ----------------------------------------------------------------

def test_definitions():
    g = np.random.default_rng(1)
    x = g.standard_normal((3, 2, 16)).astype(np.float32)
    a = np.array([0.0, np.pi / 2, 1.0])[:, None] * np.ones(4)
    cos, sin = np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)
    y = serve.rotate(x, [0, 1, 2], cos, sin, False)
    np.testing.assert_array_equal(y[0], x[0])                                     # no angle: the same
    np.testing.assert_allclose(y[1][:, :4], -x[1][:, 4:8], atol=1e-6)             # a quarter turn
    np.testing.assert_allclose(np.hypot(y[2][:, :4], y[2][:, 4:8]), np.hypot(x[2][:, :4], x[2][:, 4:8]), rtol=1e-6)
    np.testing.assert_array_equal(y[:, :, 8:], x[:, :, 8:])
    z = serve.rotate(x, [0, 1, 2], cos, sin, True)
    np.testing.assert_allclose(z[1][:, 0:8:2], -x[1][:, 1:8:2], atol=1e-6)
    # a page: codes within half a step, after a growth within one
    codes, scale = serve.append_page(np.zeros((16, 8), np.int8), np.float32(0), 0, x[0, :, :8])
    assert np.abs(codes[:2] * scale - x[0, :, :8]).max() <= scale / 2 * 1.0001
    more, larger = serve.append_page(codes, scale, 2, 5 * x[1, :, :8])
    assert larger > scale and np.abs(more[:2] * larger - x[0, :, :8]).max() <= (scale + larger) / 2 * 1.0001
    kept, same = serve.append_page(more, larger, 4, 0.01 * x[2, :, :8])
    assert same == larger and (kept[:4] == more[:4]).all()
    # attention over equal keys is the mean of the values, over one key the value
    cache = [np.ones((2, 1, 16, 16), np.int8), g.integers(-9, 9, (2, 1, 16, 16)).astype(np.int8), np.ones((2, 1), np.float32),
             np.ones((2, 1), np.float32)]
    q = g.standard_normal((3, 1, 16)).astype(np.float32)
    out, lse, _, _, _ = serve.attention(cache, np.array([[1, 0]]), np.array([0, 3]), np.array([20]), q, 0.5)
    V = np.concatenate([cache[1][1, 0].T, cache[1][0, 0].T]).astype(float)
    for i in range(3):
        np.testing.assert_allclose(out[i, 0], V[:18 + i].mean(0), atol=1e-13)
        np.testing.assert_allclose(lse[i, 0], 0.5 * q[i, 0].sum() + np.log(18 + i))
    out = serve.attention(cache, np.array([[1, 0]]), np.array([0, 3]), np.array([20]), q, 0.5, True, 1)[0]
    np.testing.assert_allclose(out[2, 0], V[19])
    # four bits: within half a step of the weights, zeros exact, codes back to back
    W = g.standard_normal((5, 100)).astype(np.float32)
    W[:, ::7] = 0
    for zeros in (False, True):
        codes, s, z = serve.w4_quantize(W, 32, zeros, False)
        V = serve.w4_values(codes, s, z, 32)
        assert (V[:, ::7] == 0).all()
        assert np.abs(V - W).max() <= s.max() * (1.0 if zeros else 0.5) * 1.0001
        p = serve.w4_pack(codes, 64)
        np.testing.assert_array_equal(np.stack([p & 15, p >> 4], -1).reshape(5, -1)[:, :100], codes)
