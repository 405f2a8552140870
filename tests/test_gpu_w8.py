"""GPU parity of the 8-bit matrices: quantization and product against the numpy definitions in oracle/block.py, bit for bit
(the sums are exact integers and every fp32 operation is rounded on its own)."""
import numpy as np
import pytest
import torch

from oracle import block
from oracle.serve import bf16_round
from paper_2412_09282_amd import crvq as C

from gpu_util import say

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def host(t):
    return t.detach().float().cpu().numpy() if t.is_floating_point() else t.detach().cpu().numpy()


def same_bits(got, exp, what):
    ok = (got == exp) | (np.isnan(got) & np.isnan(exp)) if got.dtype.kind == "f" else got == exp
    assert got.shape == exp.shape and ok.all(), f"{what}: {int((~ok).sum())} of {ok.size} differ, first at " \
        f"{np.argwhere(~ok)[0]}: {got[~ok][0]} for {exp[~ok][0]}"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,N,pad", [(1, 1, 0), (3, 15, 0), (5, 16, 8), (2, 17, 3), (9, 511, 0), (4, 512, 0), (7, 1000, 0),
                                        (3, 1024, 0), (2, 1025, 7), (3, 2048, 0), (2, 4088, 0), (33, 8192, 0), (2, 8200, 0),
                                        (2, 16384, 0), (1, 30001, 0), (1, 65536, 0)])
def test_quantize(rows, N, pad, dtype):
    g = np.random.default_rng(rows * 7 + N)
    x = (g.standard_normal((rows, N)) * np.exp2(g.integers(-20, 20, (rows, 1)))).astype(np.float32)
    if rows > 2:
        x[1] = 0
        x[2, N // 2] = np.nan if N % 2 else -np.inf
    if rows > 3:
        x[3] *= np.float32(2.0 ** -130)  # scales at their floor
    if dtype == "bf16":
        x = bf16_round(x)
    full = torch.full((rows, N + pad), 7.0, dtype=DT[dtype], device="cuda")
    full[:, :N] = torch.from_numpy(x).cuda()
    end = -(-N // 16) * 16
    store = torch.full((rows + 1, end + 16), 99, dtype=torch.int8, device="cuda")
    scales = torch.full((rows + 1,), 5.0, device="cuda")
    say(f"quantize {rows} x {N}, {dtype}")
    C.crvq_w8_quantize(full[:, :N], store[:rows, :end], scales[:rows])
    codes, s = block.w8_quantize(x)
    same_bits(host(scales)[:rows], s, "scales")
    same_bits(host(store)[:rows, :end], codes, "codes")
    assert (host(store)[:rows, end:] == 99).all() and (host(store)[rows:] == 99).all() and host(scales)[rows] == 5


def matrices(M, N, T, seed, extremes=False):
    g = np.random.default_rng(seed)
    end = -(-N // 16) * 16
    # past column N the rows hold anything: it may not matter
    c, x = g.integers(-127, 128, (M, end)).astype(np.int8), g.integers(-127, 128, (T, end)).astype(np.int8)
    if extremes:
        c[:], x[:] = -128, -128
    return c, np.exp2(g.uniform(-12, -8, M)).astype(np.float32), x, np.exp2(g.uniform(-8, -4, T)).astype(np.float32)


def product(c, sw, x, sx, N, dtype, pad=0):
    M, T = len(c), len(x)
    store = torch.full((T + 1, M + 3 + pad), 3.0, dtype=DT[dtype], device="cuda")
    C.crvq_w8_gemm(*(torch.from_numpy(a).cuda() for a in (c, sw, x, sx)), store[:T, :M], n_cols=N)
    got = host(store)
    assert (got[T:] == 3).all() and (got[:, M:] == 3).all(), "written outside y"
    return got[:T, :M]


SIZES = [(1, 1, 1), (16, 64, 16), (17, 63, 1), (1031, 3000, 1), (1031, 3000, 17), (100, 257, 5), (64, 16, 64), (300, 1000, 33),
         (255, 4096, 32), (513, 511, 65), (256, 256, 256), (257, 129, 255), (1000, 700, 300), (512, 1024, 513), (40, 100, 1500),
         (2050, 640, 130), (96, 20000, 40), (300, 8192, 700), (5, 65536, 3)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,T", SIZES)
def test_product(M, N, T, dtype):
    c, sw, x, sx = matrices(M, N, T, M + N + T)
    say(f"product {M} x {N}, {T} tokens, {dtype}")
    got = product(c, sw, x, sx, N, dtype)
    same_bits(got, block.w8_product(c, sw, x, sx, N, dtype == "bf16"), "y")


@pytest.mark.parametrize("T", [3, 300])
def test_product_largest_sums(T):
    """-128 in every place of the longest row: 2^30, an integer of 32 bits."""
    c, sw, x, sx = matrices(20, 65536, T, 1, extremes=True)
    same_bits(product(c, sw, x, sx, 65536, "f32"), block.w8_product(c, sw, x, sx, 65536, False), "y")


def test_product_bad_scales_stay_in_their_rows():
    c, sw, x, sx = matrices(200, 96, 70, 2)
    sw[7], sx[11], sx[12] = np.nan, np.inf, np.nan
    same_bits(product(c, sw, x, sx, 96, "f32"), block.w8_product(c, sw, x, sx, 96, False), "y")


def test_product_strided_rows_and_part_of_the_columns():
    c, sw, x, sx = matrices(130, 640, 90, 3)
    big = torch.from_numpy(c).cuda(), torch.from_numpy(x).cuda()
    y = torch.empty(90, 130, device="cuda")
    C.crvq_w8_gemm(big[0][::2], torch.from_numpy(sw).cuda()[:65].contiguous(), big[1][:, 64:], torch.from_numpy(sx).cuda(),
                   y[:, ::1][:, :65], n_cols=500)
    exp = block.w8_product(c[::2], sw[:65], x[:, 64:], sx, 500, False)
    same_bits(host(y)[:, :65], exp, "y")


def test_nothing_to_do():
    z = lambda *s, **k: torch.zeros(*s, device="cuda", **k)  # noqa: E731
    C.crvq_w8_quantize(z(0, 40), z(0, 48, dtype=torch.int8), z(0))
    C.crvq_w8_gemm(z(0, 48, dtype=torch.int8), z(0), z(3, 48, dtype=torch.int8), z(3), z(3, 0))
    C.crvq_w8_gemm(z(3, 48, dtype=torch.int8), z(3), z(0, 48, dtype=torch.int8), z(0), z(0, 3))
    torch.cuda.synchronize()


@pytest.mark.parametrize("T", [4, 40, 700])
def test_captured_and_replayed(T):
    """Replays of a captured call between eager ones, with new inputs in the same places."""
    c, sw, x, sx = (torch.from_numpy(a).cuda() for a in matrices(700, 1000, T, 4))
    raw, y = torch.randn(T, 1000, device="cuda"), torch.empty(T, 700, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        C.crvq_w8_quantize(raw, x, sx)
        C.crvq_w8_gemm(c, sw, x, sx, y, n_cols=1000)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        C.crvq_w8_quantize(raw, x, sx)
        C.crvq_w8_gemm(c, sw, x, sx, y, n_cols=1000)
    for k in range(4):
        raw.copy_(torch.randn(T, 1000, device="cuda") * (k + 1))
        graph.replay()
        got = y.clone()
        xe, se, ye = torch.zeros_like(x), torch.zeros_like(sx), torch.empty_like(y)
        C.crvq_w8_quantize(raw, xe, se)
        C.crvq_w8_gemm(c, sw, xe, se, ye, n_cols=1000)
        torch.cuda.synchronize()
        assert torch.equal(got, ye)


def test_one_row_of_any_stride():
    """A tensor of one row may have any stride between rows, 1 for instance."""
    row = torch.randn(40, device="cuda")
    one = torch.as_strided(row, (1, 40), (1, 1))
    store, s = torch.zeros(48, dtype=torch.int8, device="cuda"), torch.zeros(1, device="cuda")
    codes = torch.as_strided(store, (1, 48), (1, 1))
    C.crvq_w8_quantize(one, codes, s)
    c, sx = block.w8_quantize(host(one))
    same_bits(host(codes), c, "codes")
    y = torch.as_strided(torch.zeros(1, device="cuda"), (1, 1), (1, 1))
    C.crvq_w8_gemm(codes, s, codes, s, y)
    same_bits(host(y), block.w8_product(c, sx, c, sx, 40, False), "y")
    h, r = torch.as_strided(torch.zeros(40, device="cuda"), (1, 40), (1, 1)), torch.as_strided(row.clone(), (1, 40), (1, 1))
    C.crvq_norm(one, h, residual=r, residual_out=r)
    assert torch.equal(r, (one + one).clone()) and torch.isfinite(h).all()
