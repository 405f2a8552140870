"""CPU-only: the 8-bit product's and the norms' calls reject bad arguments on the host, before anything is enqueued, and the
numpy definitions in oracle/block.py agree with closed forms."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import block
from paper_2412_09282_amd import crvq as C


@pytest.fixture(scope="module")
def L():
    return C.lib()


def P(n, off=0):
    return ctypes.c_void_p((n << 40) + off)  # never dereferenced


def err(L):
    return L.crvq_last_error().decode()


def quantize(L, **kw):
    a = dict(rows=4, N=100, X=P(1), ldx=100, dt=0, codes=P(2), ld=112, scales=P(3))
    a.update(kw)
    return L.crvq_w8_quantize(*a.values(), None)


def gemm(L, **kw):
    a = dict(M=64, N=100, T=8, codes=P(1), ld=112, scales=P(2), x=P(3), ldx=112, xs=P(4), y=P(5), ldy=64, dt=1, ws=P(6), wsb=1 << 40)
    a.update(kw)
    return L.crvq_w8_gemm(*a.values(), None)


def norm(L, **kw):
    a = dict(T=4, N=96, kind=0, x=P(1), ldx=96, dt=1, post=1, w_post=P(2), b_post=P(3), gate=P(4), ldg=96, alpha=1.0, r=P(5), ldr=96,
             r_out=P(6), ldro=96, rdt=0, w_pre=P(7), b_pre=P(8), wdt=0, eps=1e-5, h=P(9), ldh=96, hs=None)
    a.update(kw)
    return L.crvq_norm(*a.values(), None)


def test_quantize_arguments(L):
    for bad, status in [(dict(rows=-1), 1), (dict(N=0), 1), (dict(N=65537, ldx=70000, ld=70016), 2), (dict(rows=1 << 31), 2),
                        (dict(X=None), 1), (dict(codes=None), 1), (dict(scales=None), 1), (dict(dt=2), 1), (dict(ldx=99), 1),
                        (dict(ld=104), 1), (dict(ld=96), 1), (dict(codes=P(2, 8)), 1), (dict(scales=P(3, 2)), 1),
                        (dict(X=P(1, 2)), 1), (dict(codes=P(1, 64)), 1), (dict(scales=P(2, 16)), 1), (dict(scales=P(1, 4)), 1)]:
        assert quantize(L, **bad) == status, (bad, err(L))
        assert "crvq_w8_quantize" in err(L)
    assert quantize(L, rows=0, X=None, codes=None, scales=None) == 0


def test_gemm_arguments(L):
    for bad, status in [(dict(M=-1), 1), (dict(T=-1), 1), (dict(N=0), 1), (dict(N=65537, ld=70016, ldx=70016), 2), (dict(M=1 << 31), 2),
                        (dict(T=1 << 31), 2), (dict(codes=None), 1), (dict(x=None), 1), (dict(scales=None), 1), (dict(xs=None), 1),
                        (dict(y=None), 1), (dict(dt=2), 1), (dict(ld=100), 1), (dict(ldx=96), 1), (dict(ldy=63), 1),
                        (dict(codes=P(1, 4)), 1), (dict(x=P(3, 8)), 1), (dict(y=P(5, 1)), 1), (dict(y=P(1, 32)), 1),
                        (dict(y=P(2)), 1), (dict(y=P(3)), 1), (dict(y=P(4)), 1)]:
        assert gemm(L, **bad) == status, (bad, err(L))
        assert "crvq_w8_gemm" in err(L)
    for nothing in (dict(M=0, ldy=0), dict(T=0)):
        assert gemm(L, codes=P(1), y=None, **nothing) == 0


def test_gemm_workspace(L):
    for M, N, T in [(64, 100, 8), (1031, 3000, 1), (4096, 4096, 300), (100, 65536, 100), (28672, 8192, 4096)]:
        need = L.crvq_w8_gemm_workspace_size(M, N, T)
        assert need % 256 == 0 and need == L.crvq_workspace_size(12, 0, T, 0, 0, 0, None, M, N, 0)
        if need:
            args = dict(M=M, N=N, T=T, ld=65536, ldx=65536, ldy=M)
            assert gemm(L, ws=None, wsb=0, **args) == 3 and gemm(L, wsb=need - 1, **args) == 3 and gemm(L, ws=P(6, 64), **args) == 3
    for none in [(0, 8, 8), (8, 0, 8), (8, 8, 0), (1 << 31, 8, 8), (8, 65537, 8)]:
        assert L.crvq_w8_gemm_workspace_size(*none) == 0


def test_norm_arguments(L):
    for bad, status in [(dict(kind=2), 1), (dict(T=-1), 1), (dict(N=0), 1), (dict(N=65537), 2), (dict(T=1 << 31), 2), (dict(dt=2), 1),
                        (dict(rdt=2), 1), (dict(wdt=5), 1), (dict(alpha=float("nan")), 1), (dict(alpha=float("inf")), 1),
                        (dict(eps=-1e-9), 1), (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1), (dict(post=0), 1),
                        (dict(h=None), 1), (dict(h=None, w_pre=None, b_pre=None, r_out=None), 1), (dict(x=None), 1), (dict(ldx=95), 1),
                        (dict(ldg=95), 1), (dict(ldg=-96), 1), (dict(ldr=90), 1), (dict(ldro=90), 1), (dict(ldh=90), 1), (dict(x=P(1, 1)), 1),
                        (dict(r=P(5, 2)), 1), (dict(r_out=P(6, 2)), 1), (dict(w_pre=P(7, 2)), 1), (dict(hs=P(10), ldh=100), 1),
                        (dict(hs=P(10), h=P(9, 8)), 1), (dict(r_out=P(5, 64)), 1), (dict(r_out=P(1)), 1), (dict(h=P(1, 32)), 1),
                        (dict(h=P(5)), 1), (dict(h=P(6)), 1), (dict(h=P(4)), 1), (dict(h=P(2)), 1), (dict(r_out=P(8)), 1),
                        (dict(hs=P(9)), 1), (dict(hs=P(1)), 1), (dict(h=P(1), hs=P(10)), 1), (dict(r_out=P(5), ldro=100), 1)]:
        assert norm(L, **bad) == status, (bad, err(L))
        assert "crvq_norm" in err(L)
    assert norm(L, T=0, x=None) == 0 and norm(L, T=0, x=None, h=None, w_pre=None, b_pre=None, r_out=None) == 0


def test_alpha_of_fp64_only(L):
    assert norm(L, alpha=1e300) == 1 and "alpha" in err(L)


def test_definition_against_closed_forms():
    c, s = block.w8_quantize(np.array([[127, -254, 1, 0.5], [0, 0, 0, 0]], np.float32))
    assert s.tolist() == [2, 2.0 ** -100] and c[0, :5].tolist() == [64, -127, 0, 0, 0] and not c[1].any()
    y = block.w8_product(np.array([[1, 2, 3]], np.int8), np.array([0.5], np.float32), np.array([[4, 5, 6]], np.int8),
                         np.array([2.0], np.float32), 2, False)
    assert y.tolist() == [[14.0]]
    r, _, h, _ = block.norm(np.array([[3.0, -4.0]]), r=np.array([[0.0, 8.0]]), eps=0.0)
    assert np.allclose(r, [[3, 4]]) and np.allclose(h, np.array([[3, 4]]) / np.sqrt(12.5))
    _, _, h, _ = block.norm(np.array([[1.0, 3.0]]), eps=0.0, layer=True, w_pre=np.array([2.0, 2.0]), b_pre=np.array([1.0, 0.0]))
    assert np.allclose(h, [[-1, 2]])


def test_binding_refusals():
    f, i8 = torch.zeros(2, 32), torch.zeros(2, 32, dtype=torch.int8)
    for call in (lambda: C.crvq_w8_quantize(f, i8, torch.zeros(2)), lambda: C.crvq_w8_gemm(i8, torch.zeros(2), i8, torch.zeros(2), torch.zeros(2, 2)),
                 lambda: C.crvq_norm(f, f.clone())):
        with pytest.raises(ValueError, match="host memory"):
            call()
    with pytest.raises(ValueError, match="kind"):
        C.crvq_norm(f, f.clone(), kind="mean")
    for call in (lambda: C.crvq_w8_quantize(torch.zeros(2, 33), i8, torch.zeros(2)), lambda: C.crvq_w8_quantize(f, i8, torch.zeros(3)),
                 lambda: C.crvq_w8_quantize(f, i8.float(), torch.zeros(2)),
                 lambda: C.crvq_w8_gemm(i8, torch.zeros(2), i8, torch.zeros(2), torch.zeros(2, 3)),
                 lambda: C.crvq_w8_gemm(i8, torch.zeros(2), i8, torch.zeros(2), torch.zeros(2, 2), n_cols=33),
                 lambda: C.crvq_w8_gemm(i8, torch.zeros(2), torch.zeros(2, 48, dtype=torch.int8), torch.zeros(2), torch.zeros(2, 2)),
                 lambda: C.crvq_norm(f, f.clone().bfloat16()), lambda: C.crvq_norm(f, torch.zeros(2, 31)),
                 lambda: C.crvq_norm(f, i8, h_scales=torch.zeros(3)), lambda: C.crvq_norm(f, f.clone(), w_pre=torch.zeros(31)),
                 lambda: C.crvq_norm(f, f.clone(), gate=torch.zeros(3, 32)),
                 lambda: C.crvq_norm(f, f.clone(), w_pre=torch.zeros(32), b_pre=torch.zeros(32).bfloat16()),
                 lambda: C.crvq_norm(f, f.clone(), residual=f.clone(), residual_out=f.clone().bfloat16())):
        with pytest.raises(AssertionError):
            call()
