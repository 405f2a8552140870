"""CPU-only: how the 4-bit product divides its rows over workgroups."""
import ctypes

import pytest


class Plan(ctypes.Structure):
    """crvq::W4Plan (crvq_internal.h)."""
    _fields_ = [(f, ctypes.c_int) for f in ("tb", "nb", "per_pass", "waves", "batches", "chunks")] + [("groups", ctypes.c_int64)]


@pytest.fixture(scope="module")
def library():
    from paper_2412_09282_amd import crvq
    L = crvq.lib()
    plan, lds = L._ZN4crvq12plan_w4_gemvElllbi, L._ZN4crvq11w4_gemv_ldsERKNS_6W4PlanElbi
    plan.argtypes, plan.restype = [ctypes.c_int64] * 3 + [ctypes.c_bool, ctypes.c_int], Plan
    lds.argtypes, lds.restype = [ctypes.POINTER(Plan), ctypes.c_int64, ctypes.c_bool, ctypes.c_int], ctypes.c_size_t
    return plan, lds


@pytest.mark.parametrize("M,N,T,f32,group", [
    (4096, 4096, 16, False, 32), (9001, 4100, 16, False, 32), (9001, 4100, 32, False, 128), (5120, 13824, 11, False, 128),
    (5120, 13824, 11, False, 64), (5125, 8200, 5, True, 32), (20001, 4100, 5, True, 32), (8192, 8192, 5, True, 32)])
def test_one_round_where_one_fills_the_chip(library, M, N, T, f32, group):
    """256 CUs hold 160 KB of LDS each: one pass's workgroups all fit at once, by the LDS they are launched with."""
    plan, lds = library
    p = plan(M, N, T, f32, group.bit_length() - 1)
    per_cu = (160 << 10) // lds(ctypes.byref(p), T, f32, group.bit_length() - 1)
    assert per_cu >= 1 and p.groups * p.chunks * -(-T // p.per_pass) <= 256 * per_cu


def test_every_workgroup_fits(library):
    """Over the range of shapes: LDS within a CU's, every block of rows taken, every column in a chunk."""
    plan, lds = library
    for M in (1, 16, 17, 300, 4096, 28672, 1 << 20):
        for N in (1, 128, 129, 3000, 8192, 14336, 1 << 20):
            for T in (1, 2, 3, 5, 8, 11, 16, 17, 32, 33, 300, 5000):
                for f32 in (False, True):
                    for log2 in (5, 6, 7, 8):
                        p = plan(M, N, T, f32, log2)
                        assert lds(ctypes.byref(p), T, f32, log2) <= 160 << 10
                        assert 1 <= p.groups <= -(-M // 16) and 1 <= p.waves <= 16 and p.batches >= 1
                        steps = p.waves * p.batches * (4 if p.nb == 1 else 2)
                        assert p.chunks * steps * 128 >= N > (p.chunks - 1) * steps * 128


def test_workspace_of_many_vectors():
    """A prompt's workspace does not grow with its length."""
    from paper_2412_09282_amd import crvq
    size = crvq.lib().crvq_w4_gemv_workspace_size
    for M, N in ((12288, 4096), (5120, 13824), (28672, 8192), (4096, 14336)):
        for T in (64, 300, 1200, 2049, 8192, 100000, 3000000):
            one_pass = max(size(M, N, t) for t in (5, 10, 16, 32))
            assert size(M, N, T) <= max(64 << 20, one_pass), (M, N, T)
