"""GPU 4-bit product at sizes where a workgroup walks several blocks of rows and, in some, several batches of columns: the loop that
the small shapes of test_gpu_w4.py leave after one turn.  Sampled rows against float64, with the bound of that file: (N/32 + 64)
2^-24 A of the terms' magnitude A = sum_g s_g (24 + z_g) sum_k |x_k|, and the rounding to the output's type.

Each shape states by the library's own plan that it gets there, so that a change of the plan cannot take the coverage away."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2412_09282_amd import crvq as C

from gpu_util import say

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


class Plan(ctypes.Structure):
    """crvq::W4Plan (crvq_internal.h): how a product is divided."""
    _fields_ = [(f, ctypes.c_int) for f in ("tb", "nb", "per_pass", "waves", "batches", "chunks")] + [("groups", ctypes.c_int64)]


def plan_of(M, N, T, xdt, group):
    f = C.lib()._ZN4crvq12plan_w4_gemvElllbi  # W4Plan crvq::plan_w4_gemv(int64_t, int64_t, int64_t, bool, int)
    f.argtypes, f.restype = [ctypes.c_int64] * 3 + [ctypes.c_bool, ctypes.c_int], Plan
    return f(M, N, T, xdt == "f32", group.bit_length() - 1)


@pytest.mark.parametrize("M,N,T,group,zeros,sdt,xdt,batches", [
    (28679, 8192, 1, 128, False, "bf16", "bf16", 2), (28679, 8192, 1, 32, True, "bf16", "bf16", 2),
    (28679, 8192, 1, 64, True, "f32", "bf16", 2), (40001, 8300, 1, 32, True, "f32", "f32", 1),
    (40001, 8300, 1, 256, False, "bf16", "f32", 1), (30001, 8200, 2, 32, True, "bf16", "bf16", 2),
    (30001, 9000, 3, 64, True, "f32", "bf16", 1), (30001, 8200, 4, 128, False, "bf16", "bf16", 1),
    (20001, 4100, 6, 64, True, "bf16", "bf16", 1), (9001, 14000, 5, 64, True, "f32", "bf16", 1),
    (9001, 8200, 7, 32, True, "bf16", "bf16", 2), (9001, 8200, 12, 32, False, "f32", "bf16", 1),
    (9001, 4100, 16, 32, True, "bf16", "bf16", 1), (5120, 13824, 11, 64, True, "bf16", "bf16", 1),
    (5125, 13824, 11, 128, True, "bf16", "bf16", 1), (9001, 4100, 32, 128, False, "f32", "bf16", 1),
    (9001, 4100, 29, 256, True, "bf16", "bf16", 1), (5125, 8200, 2, 32, True, "f32", "f32", 2),
    (5125, 8200, 3, 32, True, "bf16", "f32", 2), (5125, 8200, 5, 32, False, "f32", "f32", 1),
    (5125, 8200, 2, 64, True, "bf16", "f32", 1), (5125, 8200, 4, 64, True, "f32", "f32", 1),
    (5125, 8200, 5, 128, True, "bf16", "f32", 1), (9001, 2100, 10, 128, False, "f32", "f32", 1)])
def test_product_over_many_blocks(M, N, T, group, zeros, sdt, xdt, batches):
    p = plan_of(M, N, T, xdt, group)
    walk = -(-(-(-M // 16)) // p.groups)
    assert walk >= 3 and p.batches >= batches, (walk, p.batches)
    g = torch.Generator(device="cuda").manual_seed(M + N + T)
    G, ld = -(-N // group), -(-N // 32) * 16
    codes = torch.randint(0, 256, (M, ld), generator=g, device="cuda", dtype=torch.uint8)
    scales = (torch.rand(M, G, generator=g, device="cuda") * 0.01 + 0.001).to(DT[sdt])
    zp = torch.randint(0, 16, (M, G), generator=g, device="cuda", dtype=torch.uint8) if zeros else None
    x = torch.randn(T, N, generator=g, device="cuda").to(DT[xdt])
    y = torch.full((T, M), 7.0, device="cuda")
    C.crvq_w4_gemv(codes, scales, group, x, y, zeros=zp)
    torch.cuda.synchronize()
    # the first and last rows, and one of every seven blocks between them: 16 p.groups rows further a workgroup is at its next block
    rows = torch.unique(torch.cat((torch.arange(40), torch.arange(M - 40, M), torch.arange(0, M, 7 * 16 + 1))))
    c = codes.cpu()[rows].numpy()
    c = np.stack((c & 15, c >> 4), -1).reshape(len(rows), -1)[:, :N].astype(np.float64)
    s = scales.float().cpu()[rows].numpy().astype(np.float64)
    z = zp.cpu()[rows].numpy().astype(np.float64) if zeros else np.full(s.shape, 8.0)
    each = lambda a: np.repeat(a, group, 1)[:, :N]  # noqa: E731
    x = x.float().cpu().numpy().astype(np.float64)
    exp = x @ ((c - each(z)) * each(s)).T
    A = np.add.reduceat(np.abs(x), np.arange(0, N, group), axis=1) @ (s * (24 + z)).T
    err = np.abs(y.cpu()[:, rows].numpy().astype(np.float64) - exp)
    tol = (N / 32 + 64) * 2.0 ** -24 * A + 2.0 ** -23 * np.abs(exp)
    say(f"w4 product {M}x{N} x {T} group {group} {sdt} {xdt}: walk {walk}, {p.batches} batches, {p.chunks} chunks: {np.max(err / tol):.3f} of the bound")
    assert (err <= tol).all()
    assert torch.isfinite(y).all()


@pytest.mark.parametrize("M,N,T,group,zeros,xdt", [
    (12288, 4096, 1200, 128, False, "bf16"), (5120, 13824, 333, 64, True, "bf16"), (4100, 4096, 1025, 32, True, "f32"),
    (28672, 8192, 130, 128, True, "bf16"), (1031, 3000, 301, 32, True, "f32"), (16, 96, 70000, 32, False, "bf16")])
def test_product_of_a_prompt(M, N, T, group, zeros, xdt):
    """As many vectors as a prompt has, in more than one launch where their parts are large: sampled rows and vectors, all written."""
    g = torch.Generator(device="cuda").manual_seed(M + T)
    G, ld = -(-N // group), -(-N // 32) * 16
    codes = torch.randint(0, 256, (M, ld), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.rand(M, G, generator=g, device="cuda") * 0.01 + 0.001
    zp = torch.randint(0, 16, (M, G), generator=g, device="cuda", dtype=torch.uint8) if zeros else None
    x = torch.randn(T, N, generator=g, device="cuda").to(DT[xdt])
    wide = torch.full((T, M + 3), float("nan"), device="cuda")
    y = wide[:, 1:M + 1]
    C.crvq_w4_gemv(codes, scales, group, x, y, zeros=zp)
    torch.cuda.synchronize()
    assert torch.isfinite(y).all() and torch.isnan(wide[:, 0]).all() and torch.isnan(wide[:, M + 1:]).all()
    rows = torch.unique(torch.cat((torch.arange(min(M, 20)), torch.arange(max(0, M - 20), M), torch.arange(0, M, 97))))
    at = torch.unique(torch.cat((torch.arange(T - 40, T), torch.arange(0, T, max(1, T // 200)))))
    c = codes.cpu()[rows].numpy()
    c = np.stack((c & 15, c >> 4), -1).reshape(len(rows), -1)[:, :N].astype(np.float64)
    s = scales.cpu()[rows].numpy().astype(np.float64)
    z = zp.cpu()[rows].numpy().astype(np.float64) if zeros else np.full(s.shape, 8.0)
    each = lambda a: np.repeat(a, group, 1)[:, :N]  # noqa: E731
    x = x[at.cuda()].float().cpu().numpy().astype(np.float64)
    exp = x @ ((c - each(z)) * each(s)).T
    A = np.add.reduceat(np.abs(x), np.arange(0, N, group), axis=1) @ (s * (24 + z)).T
    err = np.abs(y.cpu()[at][:, rows].numpy().astype(np.float64) - exp)
    tol = (N / 32 + 64) * 2.0 ** -24 * A + 2.0 ** -23 * np.abs(exp)
    say(f"w4 product {M}x{N} x {T} group {group} {xdt}: {np.max(err / tol):.4f} of the bound")
    assert (err <= tol).all()
