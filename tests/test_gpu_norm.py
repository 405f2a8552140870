"""GPU parity of the norms around a block against the fp64 definition in oracle/block.py, which also gives how far fp32
arithmetic may take each element; a result stored in bf16 may be off by 2^-8 of itself more."""
import itertools

import numpy as np
import pytest
import torch

from oracle import block
from oracle.serve import bf16_round
from paper_2412_09282_amd import crvq as C

from gpu_util import say

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def values(g, *shape, dtype="f32", by=1.0):
    x = (g.standard_normal(shape) * by).astype(np.float32)
    return bf16_round(x) if dtype == "bf16" else x


def dev(a, dtype, pad=0):
    if a is None:
        return None
    t = torch.from_numpy(a).cuda().to(DT[dtype])
    if pad and t.dim() == 2:
        store = torch.full((t.shape[0], t.shape[1] + pad), 7.0, dtype=t.dtype, device="cuda")
        store[:, :t.shape[1]] = t
        t = store[:, :t.shape[1]]
    return t


def host(t):
    return t.detach().double().cpu().numpy()


def check(got, exp, tol, what):
    off = np.abs(got - exp) - tol
    assert (off <= 0).all(), f"{what}: {int((off > 0).sum())} of {off.size} off, worst {off.max()} at {np.unravel_index(off.argmax(), off.shape)}"


CASES = [
    # T, N, kind, post, gate, residual, biases, dtype, r_dtype, w_dtype, pad
    (1, 1, "rms", False, None, True, False, "f32", "f32", "f32", 0),
    (3, 16, "rms", True, "full", True, False, "bf16", "f32", "f32", 0),
    (5, 17, "layer", True, "channel", True, True, "f32", "f32", "f32", 0),
    (2, 100, "layer", False, None, False, True, "bf16", "bf16", "bf16", 3),
    (7, 512, "rms", True, "channel", True, False, "bf16", "bf16", "f32", 8),
    (9, 1000, "rms", False, "full", True, False, "f32", "bf16", "bf16", 0),
    (4, 1024, "layer", True, "full", True, True, "bf16", "f32", "bf16", 0),
    (3, 1025, "rms", True, None, True, False, "bf16", "bf16", "f32", 0),
    (2, 2040, "layer", False, "channel", True, False, "f32", "f32", "f32", 1),
    (32, 4096, "rms", False, None, True, False, "bf16", "bf16", "bf16", 0),
    (3, 5120, "layer", True, "full", True, True, "f32", "f32", "f32", 0),
    (2, 8192, "rms", True, "full", True, False, "bf16", "f32", "f32", 0),
    (2, 11008, "rms", True, None, True, False, "f32", "bf16", "f32", 0),
    (2, 13831, "layer", True, "full", True, True, "bf16", "bf16", "f32", 2),
    (1, 28672, "rms", False, None, False, False, "bf16", "f32", "f32", 0),
    (1, 65536, "layer", True, "full", True, True, "f32", "f32", "f32", 0),
    (2, 65535, "rms", True, "full", True, False, "bf16", "f32", "f32", 0),
    (300, 24, "layer", True, "full", True, True, "bf16", "f32", "f32", 0),
]


def inputs(case, seed=0, mean=0.0):
    T, N, kind, post, gate, residual, biases, dt, rdt, wdt, pad = case
    g = np.random.default_rng(N + T + seed)
    a = dict(x=values(g, T, N, dtype=dt) + np.float32(mean), r=values(g, T, N, dtype=rdt, by=3) if residual else None,
             gate=None if gate is None else values(g, *((N,) if gate == "channel" else (T, N)), dtype=dt),
             w_post=values(g, N, dtype=wdt) if post else None, b_post=values(g, N, dtype=wdt) if post and biases else None,
             w_pre=values(g, N, dtype=wdt), b_pre=values(g, N, dtype=wdt) if biases else None)
    if mean:
        a["x"] = values(g, T, N) * np.float32(0.01) + np.float32(mean)
        a["x"] = bf16_round(a["x"]) if dt == "bf16" else a["x"]
    t = {k: dev(v, wdt if k[1:2] == "_" else rdt if k == "r" else dt, pad) for k, v in a.items()}
    return a, t


@pytest.mark.parametrize("alpha", [1.0, -0.375])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_norm(case, alpha):
    T, N, kind, post, gate, residual, biases, dt, rdt, wdt, pad = case
    a, t = inputs(case)
    r, r_tol, h, h_tol = block.norm(a["x"], a["r"], a["gate"], alpha, post, a["w_post"], a["b_post"], a["w_pre"], a["b_pre"],
                                    1e-5, kind == "layer")
    r_out = torch.full((T + 1, N + 2 * pad), 9.0, dtype=DT[rdt], device="cuda")
    h_out = torch.full((T + 1, N + pad), 9.0, dtype=DT[dt], device="cuda")
    say(f"norm {case} alpha {alpha}")
    args = dict(residual=t["r"], w_pre=t["w_pre"], b_pre=t["b_pre"], w_post=t["w_post"], b_post=t["b_post"], gate=t["gate"],
                alpha=alpha, eps=1e-5, kind=kind)
    C.crvq_norm(t["x"], h_out[:T, :N], residual_out=r_out[:T, :N], **args)
    check(host(r_out)[:T, :N], r, r_tol + HALF[rdt] * (np.abs(r) + r_tol), "r")
    check(host(h_out)[:T, :N], h, h_tol + HALF[dt] * (np.abs(h) + h_tol), "h")
    for o in (r_out, h_out):
        assert (host(o)[T:] == 9).all() and (host(o)[:, N:] == 9).all(), "written outside"
    # one of the two alone is the same
    only_r, only_h = torch.zeros(T, N, dtype=DT[rdt], device="cuda"), torch.zeros(T, N, dtype=DT[dt], device="cuda")
    C.crvq_norm(t["x"], None, residual_out=only_r, **{k: v for k, v in args.items() if k not in ("w_pre", "b_pre")})
    C.crvq_norm(t["x"], only_h, **args)
    assert torch.equal(only_r, r_out[:T, :N]) and torch.equal(only_h, h_out[:T, :N])
    # in 8 bits: the codes and scales that quantizing the unrounded h gives
    end = -(-N // 16) * 16
    codes, scales = torch.full((T, end), 55, dtype=torch.int8, device="cuda"), torch.zeros(T, device="cuda")
    C.crvq_norm(t["x"], codes, h_scales=scales, **args)
    c, s = host(codes), host(scales)[:, None]
    assert (c[:, N:] == 0).all() and (np.abs(c) <= 127).all()
    check(c[:, :N] * s, h, 0.5 * s * (1 + 2.0 ** -20) + h_tol, "h in 8 bits")
    check(s[:, 0], np.abs(h).max(1) / 127, h_tol.max(1) / 127 + 2.0 ** -23 * s[:, 0], "scale of h")
    if dt == "f32":
        again, s2 = torch.zeros_like(codes), torch.zeros_like(scales)
        C.crvq_w8_quantize(h_out[:T, :N], again, s2)
        assert torch.equal(again, codes) and torch.equal(s2, scales)


@pytest.mark.parametrize("kind,by", itertools.product(["rms", "layer"], [1e30, 1e-30]))
def test_rows_whose_squares_leave_fp32(kind, by):
    g = np.random.default_rng(5)
    x = (g.standard_normal((4, 600)) * by).astype(np.float32)
    h = torch.empty(4, 600, device="cuda")
    C.crvq_norm(dev(x, "f32"), h, eps=0.0, kind=kind)
    _, _, exp, tol = block.norm(x, eps=0.0, layer=kind == "layer")
    check(host(h), exp, tol, "h")


def test_small_spread_around_a_large_mean():
    a, t = inputs((3, 4096, "layer", False, None, False, False, "f32", "f32", "f32", 0), mean=1000.0)
    h = torch.empty(3, 4096, device="cuda")
    C.crvq_norm(t["x"], h, w_pre=t["w_pre"], eps=1e-5, kind="layer")
    x = a["x"].astype(np.float64)
    c = x - x.mean(1, keepdims=True)
    exp = c / np.sqrt((c * c).mean(1, keepdims=True) + 1e-5) * a["w_pre"]
    check(host(h), exp, 6 * 2.0 ** -24 * np.abs(exp), "h")  # x itself is exact: nothing is lost before the centre is taken off


def test_rows_with_a_nan_or_infinity_stay_alone():
    g = np.random.default_rng(6)
    x = g.standard_normal((4, 300)).astype(np.float32)
    clean = torch.empty(4, 300, device="cuda")
    C.crvq_norm(dev(x, "f32"), clean)
    x[1, 5], x[2, 299] = np.nan, np.inf
    h, codes, s = torch.empty(4, 300, device="cuda"), torch.ones(4, 304, dtype=torch.int8, device="cuda"), torch.zeros(4, device="cuda")
    C.crvq_norm(dev(x, "f32"), h)
    C.crvq_norm(dev(x, "f32"), codes, h_scales=s)
    assert torch.equal(h[[0, 3]], clean[[0, 3]]) and torch.isnan(h[1]).all() and torch.isnan(h[2, 299])
    assert torch.isnan(s[1:3]).all() and torch.isfinite(s[[0, 3]]).all() and (codes[1:3] == 0).all()


@pytest.mark.parametrize("N", [40, 700, 5120, 9001])
def test_outputs_in_the_place_of_inputs(N):
    case = (5, N, "rms", True, "full", True, False, "bf16", "bf16", "f32", 0)
    a, t = inputs(case)
    args = dict(w_pre=t["w_pre"], w_post=t["w_post"], gate=t["gate"], alpha=0.5)
    r, h = torch.empty_like(t["r"]), torch.empty_like(t["x"])
    C.crvq_norm(t["x"], h, residual=t["r"], residual_out=r, **args)
    x2, r2 = t["x"].clone(), t["r"].clone()
    C.crvq_norm(x2, x2, residual=r2, residual_out=r2, **args)
    assert torch.equal(r2, r) and torch.equal(x2, h)
    x3, r3 = t["x"].clone(), t["r"].clone()
    C.crvq_norm(x3, r3, residual=r3, residual_out=x3, **args)
    assert torch.equal(x3, r) and torch.equal(r3, h)


def test_captured_and_replayed_on_another_stream():
    case = (6, 5120, "layer", True, "full", True, True, "f32", "f32", "f32", 0)
    _, t = inputs(case)
    h, r = torch.empty_like(t["x"]), torch.empty_like(t["r"])
    call = lambda h, r: C.crvq_norm(t["x"], h, residual=t["r"], residual_out=r, w_pre=t["w_pre"], w_post=t["w_post"],  # noqa: E731
                                    gate=t["gate"], kind="layer")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(h, r)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(h, r)
    for k in range(3):
        t["x"].normal_()
        graph.replay()
        h2, r2 = torch.empty_like(h), torch.empty_like(r)
        call(h2, r2)
        torch.cuda.synchronize()
        assert torch.equal(h, h2) and torch.equal(r, r2)


def test_no_rows():
    C.crvq_norm(torch.zeros(0, 64, device="cuda"), torch.zeros(0, 64, device="cuda"))
    torch.cuda.synchronize()
