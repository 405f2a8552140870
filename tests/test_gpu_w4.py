"""GPU parity of the 4-bit matrices with group scales (quantize, dequantize, product) with the plain numpy
definitions in oracle/serve.py.

Quantization and reconstruction round every operation on its own in fp32: compared bit for bit.  The product:
with A = sum_g s_g (24 + z_g) sum_k |x_k| of a row, every partial sum is at most A, a chain has at most N/32 + 64 fp32
additions, so |y - W x| <= (N/32 + 64) 2^-24 A, and the rounding to the output's type."""
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


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(DT[dtype])


def row_bytes(N):
    return -(-N // 32) * 16


@pytest.mark.parametrize("M,N,group,zeros,sdt,dtype", [
    (1, 1, 32, False, "f32", "f32"), (3, 31, 32, True, "bf16", "bf16"), (17, 33, 64, True, "f32", "bf16"),
    (5, 300, 256, False, "bf16", "f32"), (64, 1000, 128, True, "f32", "f32"), (130, 257, 32, False, "bf16", "bf16"),
    (33, 4096, 128, False, "bf16", "bf16")])
def test_quantize_and_back(M, N, group, zeros, sdt, dtype):
    say(f"w4 quantize {M}x{N} group {group} zeros {zeros} scales {sdt} from {dtype}")
    g = np.random.default_rng(M * N)
    W = (g.standard_normal((M, N)) * 0.02 + 0.01).astype(np.float32)
    W[0, : N // 2] = 0                                   # groups of nothing but zeros
    W[-1] = np.abs(W[-1])                                # groups of one sign
    if dtype == "bf16":
        W = serve.bf16_round(W)
    codes, scales, zp = serve.w4_quantize(W, group, zeros, sdt == "bf16")
    G, ld = scales.shape[1], row_bytes(N)
    wide = torch.zeros(M, N + 5, dtype=DT[dtype], device="cuda")
    wide[:, 1:N + 1] = dev(W)
    out = torch.full((M, ld + 16), 0xEE, dtype=torch.uint8, device="cuda")
    s = torch.zeros(M, G + 1, dtype=DT[sdt], device="cuda")[:, :G]
    z = torch.zeros(M, G + 2, dtype=torch.uint8, device="cuda")[:, :G] if zeros else None
    C.crvq_w4_quantize(wide[:, 1:N + 1], out, s, group, zeros=z)
    np.testing.assert_array_equal(out[:, :ld].cpu().numpy(), serve.w4_pack(codes, ld))
    assert (out[:, ld:] == 0xEE).all()                   # nothing past the padded row
    np.testing.assert_array_equal(host(s), scales)
    if zeros:
        np.testing.assert_array_equal(z.cpu().numpy(), zp)
    for odt in ("f32", "bf16"):
        back = torch.full((M, N + 3), 7.0, dtype=DT[odt], device="cuda")
        C.crvq_w4_dequant(out, s, group, back[:, 2:N + 2], zeros=z)
        e = serve.w4_values(codes, scales, zp, group).astype(np.float32)
        np.testing.assert_array_equal(host(back[:, 2:N + 2]), serve.bf16_round(e) if odt == "bf16" else e)
        assert (back[:, :2] == 7).all() and (back[:, N + 2:] == 7).all()


def test_quantize_not_finite():
    say("w4 quantize: NaN and infinity")
    W = torch.randn(4, 96, device="cuda")
    W[1, 40], W[2, 70] = float("nan"), float("-inf")
    for zeros in (False, True):
        codes = torch.zeros(4, 48, dtype=torch.uint8, device="cuda")
        s = torch.zeros(4, 3, device="cuda")
        z = torch.zeros(4, 3, dtype=torch.uint8, device="cuda") if zeros else None
        C.crvq_w4_quantize(W, codes, s, 32, zeros=z)
        bad = torch.zeros(4, 3, dtype=torch.bool)
        bad[1, 1] = bad[2, 2] = True
        assert torch.equal(torch.isnan(s).cpu(), bad)
        assert (codes.view(4, 3, 16)[1, 1] == 0).all() and (codes.view(4, 3, 16)[2, 2] == 0).all()


def check_product(M, N, T, group, zeros, sdt, xdt, ydt, seed=0, odd=False, scale=1.0):
    g = np.random.default_rng(seed + M + N + T)
    G, ld = -(-N // group), row_bytes(N) + (32 if odd else 0)
    codes = g.integers(0, 16, (M, N)).astype(np.uint8)
    packed = serve.w4_pack(codes, ld)
    if N % 2:
        packed[:, N // 2] |= 0xF0                       # what lies past column N must not matter
    packed[:, (N + 1) // 2:] = 0xAB
    scales = (g.random((M, G)) * 0.01 + 0.001).astype(np.float32)
    if sdt == "bf16":
        scales = serve.bf16_round(scales)
    zp = g.integers(0, 16, (M, G)).astype(np.uint8) if zeros else np.full((M, G), 8, np.uint8)
    x = (g.standard_normal((T, N)) * scale).astype(np.float32)
    if xdt == "bf16":
        x = serve.bf16_round(x)
    W = serve.w4_values(codes, scales, zp, group)
    exp = x.astype(np.float64) @ W.T
    ax = np.add.reduceat(np.abs(x.astype(np.float64)), np.arange(0, N, group), axis=1)
    A = ax @ (scales.astype(np.float64) * (24.0 + zp)).T
    if odd:
        xt = torch.zeros(T, N + 7, dtype=DT[xdt], device="cuda")[:, 3:N + 3]
        yt = torch.full((T, M + 5), 7.0, dtype=DT[ydt], device="cuda")[:, 2:M + 2]
        st = torch.zeros(M, G + 1, dtype=DT[sdt], device="cuda")[:, 1:]
        zt = torch.zeros(M, G + 3, dtype=torch.uint8, device="cuda")[:, 1:G + 1] if zeros else None
        xt.copy_(dev(x))
        st.copy_(dev(scales))
        if zeros:
            zt.copy_(dev(zp))
    else:
        xt, yt, st = dev(x, xdt), torch.full((T, M), 7.0, dtype=DT[ydt], device="cuda"), dev(scales, sdt)
        zt = dev(zp) if zeros else None
    C.crvq_w4_gemv(dev(packed), st, group, xt, yt, zeros=zt)
    torch.cuda.synchronize()
    got = host(yt).astype(np.float64)
    tol = (N / 32 + 64) * 2.0 ** -24 * A + (2.0 ** -8 if ydt == "bf16" else 2.0 ** -23) * np.abs(exp)
    err = np.abs(got - exp)
    assert np.isfinite(got).all() and (err <= tol).all(), f"worst {np.max(err / tol):.3g} of the bound"
    say(f"w4 product {M}x{N} x {T} group {group} zeros {zeros} {sdt} {xdt}->{ydt}: {np.max(err / tol):.3f} of the bound")


@pytest.mark.parametrize("M,N,T,group,zeros,sdt,xdt,ydt", [
    (1, 1, 1, 32, False, "f32", "f32", "f32"), (16, 128, 1, 128, False, "bf16", "bf16", "bf16"),
    (15, 33, 1, 32, True, "f32", "bf16", "f32"), (100, 1000, 1, 64, True, "bf16", "f32", "f32"),
    (1031, 3000, 1, 32, True, "f32", "f32", "f32"), (257, 515, 2, 256, False, "f32", "bf16", "bf16"),
    (64, 4096, 4, 128, True, "bf16", "bf16", "bf16"), (333, 2049, 5, 32, True, "f32", "f32", "f32"),
    (48, 700, 8, 64, False, "bf16", "bf16", "f32"), (70, 1535, 11, 64, True, "bf16", "bf16", "bf16"),
    (129, 640, 16, 128, False, "f32", "bf16", "f32"), (65, 900, 17, 32, True, "f32", "bf16", "bf16"),
    (40, 2100, 23, 128, True, "bf16", "f32", "f32"), (31, 1200, 64, 64, False, "bf16", "bf16", "bf16"),
    (5, 14000, 3, 128, False, "bf16", "bf16", "f32"), (2, 30000, 1, 64, True, "f32", "f32", "f32"),
    (20, 96, 100, 32, True, "f32", "f32", "bf16"), (4096, 4096, 1, 128, False, "bf16", "bf16", "bf16"),
    (9000, 512, 1, 128, True, "bf16", "bf16", "bf16")])
def test_product(M, N, T, group, zeros, sdt, xdt, ydt):
    check_product(M, N, T, group, zeros, sdt, xdt, ydt)
    check_product(M, N, T, group, zeros, sdt, xdt, ydt, seed=1, odd=True)


def test_product_magnitudes():
    for scale in (1e30, 1e-30):
        for xdt in ("f32", "bf16"):
            check_product(50, 600, 2, 64, True, "f32", xdt, "f32", scale=scale)


def test_product_not_finite_is_its_own_vector_only():
    say("w4 product: NaN and infinity")
    for T in (3, 9, 20):
        for dt in (torch.float32, torch.bfloat16):
            codes = torch.randint(0, 256, (40, 160), dtype=torch.uint8, device="cuda")
            s = torch.rand(40, 10, device="cuda")
            x = torch.randn(T, 320, device="cuda").to(dt)
            y, e = torch.empty(T, 40, device="cuda"), torch.empty(T, 40, device="cuda")
            C.crvq_w4_gemv(codes, s, 32, x, e)
            x[1, 100], x[2, 319] = float("inf"), float("nan")
            C.crvq_w4_gemv(codes, s, 32, x, y)
            assert torch.isnan(y[1:3]).all() and torch.equal(y[0], e[0]) and torch.equal(y[3:], e[3:])


def test_product_of_nothing():
    codes = torch.zeros(8, 16, dtype=torch.uint8, device="cuda")
    s = torch.ones(8, 1, device="cuda")
    C.crvq_w4_gemv(codes, s, 32, torch.ones(0, 20, device="cuda"), torch.ones(0, 8, device="cuda"))
    C.crvq_w4_gemv(codes[:0], s[:0], 32, torch.ones(2, 20, device="cuda"), torch.ones(2, 0, device="cuda"))
