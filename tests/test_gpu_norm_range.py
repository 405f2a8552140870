"""Norms of finite rows whose centred elements lie beyond fp32, against the fp64 definition in oracle/block.py and its bounds."""
import numpy as np
import pytest
import torch

from oracle import block
from oracle.serve import bf16_round
from paper_2412_09282_amd import crvq as C

from gpu_util import say
from test_gpu_norm import HALF, check, dev, host

pytestmark = pytest.mark.gpu


def far_apart(N, dtype):
    """Rows of 3e38 and -3e38: one of a kind among the others, either sign; halves; and ones of usual size between them."""
    g = np.random.default_rng(N)
    x = np.full((6, N), -3e38, np.float32)
    x[0, 0] = 3e38
    x[1], x[1, N // 2] = 3e38, -3e38
    x[2, ::2] = 3e38
    x[3] = g.uniform(-3.2e38, 3.2e38, N)
    x[4] = g.standard_normal(N)
    x[5] = g.standard_normal(N) * 1e-30
    return bf16_round(x) if dtype == "bf16" else x


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["layer", "rms"])
@pytest.mark.parametrize("N", [4, 17, 600, 1025, 4096, 8200, 30001, 65536])
def test_rows_at_the_end_of_fp32(N, kind, dtype):
    say(f"norm of rows of 3e38, {kind}, {N}, {dtype}")
    x = far_apart(N, dtype)
    w = np.random.default_rng(1).standard_normal(N).astype(np.float32)
    layer = kind == "layer"
    h = torch.empty(6, N, dtype=dev(x, dtype).dtype, device="cuda")
    C.crvq_norm(dev(x, dtype), h, w_pre=dev(w, "f32"), eps=0.0, kind=kind)
    _, _, exp, tol = block.norm(x, w_pre=w, eps=0.0, layer=layer)
    assert np.isfinite(exp).all()
    check(host(h), exp, tol + HALF[dtype] * (np.abs(exp) + tol), "h")
    # after a block: normed first, its gate and the residual sum behind it
    r = torch.ones(6, N, device="cuda")
    C.crvq_norm(dev(x, dtype), None, residual=r, residual_out=r, w_post=dev(w, "f32"), alpha=0.5, eps=0.0, kind=kind)
    exp, tol, _, _ = block.norm(x, np.ones((6, N)), None, 0.5, True, w, eps=0.0, layer=layer)
    check(host(r), exp, tol + 2.0 ** -24 * (np.abs(exp) + tol), "r")
