"""GPU 4-bit product with vectors at the ends of fp32's and bf16's range, against float64.

The bound of test_gpu_w4.py, (N/32 + 64) 2^-24 A with A = sum_g s_g (24 + z_g) sum_k |x_k|, and the rounding to fp32; sums are held
in units of 2^-12, so that each of them may also be off by fp32's smallest step, 2^-149, in that unit, times its scale: (N/32 + 64)
2^-137 sum_g s_g (products: 2^-149 each, N 2^-137 s)."""
import numpy as np
import pytest
import torch

from oracle import serve
from paper_2412_09282_amd import crvq as C

from gpu_util import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("low,high", [(125.0, 127.9), (118.0, 127.0), (-100.0, -90.0), (-120.0, -110.0), (-126.0, -120.0)])
@pytest.mark.parametrize("T,group,xdt", [(1, 128, "bf16"), (1, 32, "f32"), (3, 64, "f32"), (11, 64, "bf16"), (17, 128, "bf16"), (9, 256, "f32")])
def test_product_at_the_ends_of_the_range(T, group, xdt, low, high):
    """Magnitudes of 2^low to 2^high; the scales keep the results themselves finite."""
    M, N = 50, 600
    g = np.random.default_rng(T + group)
    x = (np.exp2(g.uniform(low, high, (T, N))) * g.choice([-1, 1], (T, N))).astype(np.float32)
    if xdt == "bf16":
        x = serve.bf16_round(x)
    x = np.clip(x, -3.38e38, 3.38e38)
    G = -(-N // group)
    codes = g.integers(0, 16, (M, N)).astype(np.uint8)
    scales = (g.random((M, G)) * 1e-5 + 1e-5).astype(np.float32) if high > 0 else (g.random((M, G)) + 1).astype(np.float32)
    zp = g.integers(0, 16, (M, G)).astype(np.uint8)
    exp = x.astype(np.float64) @ serve.w4_values(codes, scales, zp, group).T
    A = np.add.reduceat(np.abs(x.astype(np.float64)), np.arange(0, N, group), axis=1) @ (scales.astype(np.float64) * (24.0 + zp)).T
    dt = torch.bfloat16 if xdt == "bf16" else torch.float32
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    y = torch.full((T, M), 7.0, device="cuda")
    C.crvq_w4_gemv(dev(serve.w4_pack(codes, -(-N // 32) * 16)), dev(scales), group, dev(x).to(dt), y, zeros=dev(zp))
    got = y.double().cpu().numpy()
    tol = (N / 32 + 64) * 2.0 ** -24 * A + 2.0 ** -23 * np.abs(exp) + \
        (N / 32 + 64 + N) * 2.0 ** -137 * scales.astype(np.float64).sum(1)[None]
    err = np.abs(got - exp)
    say(f"w4 product of 2^{low} to 2^{high}, {T} x {group} {xdt}: {np.max(err / tol):.3g} of the bound")
    assert np.isfinite(got).all() and (err <= tol).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_quantize_weights_whose_spread_passes_fp32(dtype):
    """Finite weights from -3e38 to 3e38: 15 steps of 4e37 around a zero point, each weight within half a step and a rounding of it."""
    say(f"w4 quantize: a spread past fp32's range, {dtype}")
    W = (torch.linspace(-1, 1, 64, device="cuda") * 3e38).to(dtype).repeat(3, 1)
    W[1] = 0
    W[2] *= 0.4                                          # 2.4e38 wide: within the range
    codes = torch.zeros(3, 32, dtype=torch.uint8, device="cuda")
    s, z = torch.zeros(3, 2, device="cuda"), torch.zeros(3, 2, dtype=torch.uint8, device="cuda")
    C.crvq_w4_quantize(W, codes, s, 32, zeros=z)
    s64 = torch.zeros(3, 1, device="cuda")
    z64 = torch.zeros(3, 1, dtype=torch.uint8, device="cuda")
    C.crvq_w4_quantize(W, codes, s64, 64, zeros=z64)
    out = torch.empty(3, 64, device="cuda")
    C.crvq_w4_dequant(codes, s64, 64, out, zeros=z64)
    w = W.double()
    spread = (w.clamp(min=0).amax(1) - w.clamp(max=0).amin(1)).clamp(min=15 * 2.0 ** -100)
    assert ((s64[:, 0].double() - spread / 15).abs() <= 2.0 ** -23 * spread / 15).all()
    step = s64.double()
    assert torch.isfinite(s).all() and ((out.double() - w).abs() <= step * (1 + 2.0 ** -20)).all()
