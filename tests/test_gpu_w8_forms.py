"""Every form that the 8-bit product takes, at sizes that end inside its tiles, bit for bit against the definition of
oracle/block.py (its sums, exact in fp64 as well: they stay below 2^53)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle.serve import bf16_round
from paper_2412_09282_amd import crvq as C

from gpu_util import say
from test_gpu_w8 import DT, host, matrices, same_bits

FORMS = ["few1", "few2", "few12", "few22", "tile64x32", "tile128x64", "tile64", "tile128", "tile256x128", "tile256"]


class Plan(ctypes.Structure):
    """crvq::W8Plan (crvq_internal.h)."""
    _fields_ = [("form", ctypes.c_int), ("splits", ctypes.c_int)]


def plan(M, N, T, far=False):
    f = C.lib()._ZN4crvq7plan_w8Elllb
    f.argtypes, f.restype = [ctypes.c_int64] * 3 + [ctypes.c_bool], Plan
    p = f(M, N, T, far)
    return FORMS[p.form], p.splits


# form, M, N, T, splits
CASES = [
    ("few1", 37, 4097, 16, 1), ("few1", 6143, 300, 9, 1), ("few2", 6147, 1031, 9, 1), ("few2", 12287, 255, 16, 1),
    ("few12", 6143, 513, 31, 1), ("few12", 33, 2049, 17, 1), ("few22", 6147, 700, 17, 1), ("few22", 12287, 129, 32, 1),
    ("few22", 6143, 511, 63, 1),
    ("tile64x32", 12301, 531, 17, 1), ("tile64x32", 12289, 1, 9, 1), ("tile64x32", 12337, 128, 32, 1), ("tile64x32", 28673, 1000, 31, 1),
    ("tile128x64", 20497, 333, 50, 1), ("tile128x64", 20481, 1030, 33, 1), ("tile128x64", 20607, 17, 64, 1),
    ("tile64", 6147, 500, 64, 1), ("tile64", 65, 2065, 129, 2), ("tile64", 200, 20600, 65, 20), ("tile64", 1, 8193, 200, 8),
    ("tile128", 16403, 129, 67, 1), ("tile128", 1029, 700, 3001, 1), ("tile128", 8193, 16, 301, 1),
    ("tile256x128", 4099, 531, 1100, 1), ("tile256x128", 8209, 128, 515, 1), ("tile256x128", 22289, 15, 129, 1),
    ("tile256", 2049, 700, 4097, 1), ("tile256", 4100, 1, 2050, 1), ("tile256", 5000, 145, 1601, 1),
]


@pytest.mark.parametrize("form,M,N,T,splits", CASES)
def test_sizes_take_the_forms(form, M, N, T, splits):
    assert plan(M, N, T) == (form, splits)


def test_every_form_is_there():
    assert {c[0] for c in CASES} == set(FORMS)


def expected(c, sw, x, sx, N, dtype):
    acc = x[:, :N].astype(np.float64) @ c[:, :N].astype(np.float64).T
    y = acc.astype(np.float32) * (sx[:, None] * sw[None])
    return bf16_round(y) if dtype == "bf16" else y


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form,M,N,T,splits", CASES)
def test_product(form, M, N, T, splits, dtype):
    c, sw, x, sx = matrices(M, N, T, M + N + T)
    say(f"product {M} x {N}, {T} tokens, {dtype}: {form}")
    exp = expected(c, sw, x, sx, N, dtype)
    for pad in (3, 4):  # rows of y that stores of four elements fit, and others
        store = torch.full((T + 1, -(-M // 4) * 4 + pad), 3.0, dtype=DT[dtype], device="cuda")
        C.crvq_w8_gemm(*(torch.from_numpy(a).cuda() for a in (c, sw, x, sx)), store[:T, :M], n_cols=N)
        assert bool((store[T:] == 3).all()) and bool((store[:, M:] == 3).all()), "written outside y"
        same_bits(host(store[:T, :M]), exp, "y")


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["matrix", "x", "both"])
@pytest.mark.parametrize("T", [5, 17, 100])
def test_rows_far_apart(T, which):
    """Rows 2^22 bytes and more apart."""
    M, N, far = 35, 1003, (1 << 22) + 48
    say(f"product {M} x {N}, {T} tokens, rows of {which} far apart")
    assert plan(M, N, T, True) == ("few1" if T <= 16 else "few22", 1)
    c, sw, x, sx = matrices(M, N, T, T)

    def at(a, wide):
        ld = far if wide else a.shape[1]
        store = torch.full((len(a) * ld,), 77, dtype=torch.int8, device="cuda")
        t = torch.as_strided(store, a.shape, (ld, 1))
        t.copy_(torch.from_numpy(a))
        return t

    y = torch.empty(T, M, device="cuda")
    C.crvq_w8_gemm(at(c, which != "x"), torch.from_numpy(sw).cuda(), at(x, which != "matrix"), torch.from_numpy(sx).cuda(), y, n_cols=N)
    same_bits(host(y), expected(c, sw, x, sx, N, "f32"), "y")
