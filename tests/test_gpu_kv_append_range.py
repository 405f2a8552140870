"""GPU append to the paged 8-bit cache at the ends of its range: angle tables without rows, caches past 4 GiB."""
import pytest
import torch

from paper_2412_09282_amd import crvq as C

from gpu_util import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rot,interleaved", [(64, 0), (16, 0), (64, 1), (8, 0)])
def test_angle_table_without_rows(dtype, rot, interleaved):
    """Every place lies outside the table: the rotated elements are NaN, and so is a page's scale; nothing of the table is read."""
    say(f"append: no angles, rot {rot} interleaved {interleaved} {dtype}")
    Hq, Hkv, D, page, n = 4, 2, 64, 16, 3
    k, v, q = [torch.randn(n, h, D, device="cuda").to(dtype) for h in (Hkv, Hkv, Hq)]
    kc, vc = torch.zeros(1, Hkv, page, D, dtype=torch.int8, device="cuda"), torch.zeros(1, Hkv, D, page, dtype=torch.int8, device="cuda")
    ks, vs = torch.zeros(1, Hkv, device="cuda"), torch.zeros(1, Hkv, device="cuda")
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table, start, kv_len, q_out, one = ints(0), ints(0, n), ints(n), torch.zeros_like(q), torch.zeros(64, device="cuda")
    rows = lambda t, h: (t.data_ptr(), h * D, D)  # noqa: E731
    status = C.lib().crvq_kv_append(
        1, Hq, Hkv, D, page, 1, kc.data_ptr(), vc.data_ptr(), ks.data_ptr(), vs.data_ptr(), table.data_ptr(), 1, start.data_ptr(),
        kv_len.data_ptr(), n, n, C.dtype_code(k), *rows(k, Hkv), *rows(v, Hkv), *rows(q, Hq), *rows(q_out, Hq), one.data_ptr(),
        one.data_ptr(), 0, rot, None, interleaved, torch.cuda.current_stream().cuda_stream)
    assert status == 0
    assert torch.isnan(q_out[:, :, :rot]).all() and torch.equal(q_out[:, :, rot:], q[:, :, rot:])
    assert torch.isnan(ks).all() and torch.isfinite(vs).all() and (kc == 0).all()
    empty = torch.zeros(0, rot // 2, device="cuda")
    with pytest.raises(ValueError):
        C.crvq_kv_append(k, v, kc, vc, ks, vs, table.view(1, 1), start, kv_len, n, cos=empty, sin=empty)
    C.crvq_kv_append(k[:0], v[:0], kc, vc, ks, vs, table.view(1, 1), start * 0, kv_len * 0, 0, cos=empty, sin=empty)


@pytest.mark.parametrize("new", [1, 70])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_cache_past_4_gib(dtype, new):
    """Pages whose offsets pass 32 bits give what the same pages give in a small cache, bit for bit: append, read and attention."""
    say(f"cache past 4 GiB, {new} new tokens, {dtype}")
    Hq, Hkv, D, page, kv = 8, 2, 128, 256, 700
    here, far = [0, 1, 2], [40001, 65540, 32769]  # 64 KiB a page in each array
    n_pages = max(far) + 1
    assert n_pages * Hkv * page * D > 2 ** 32
    g = torch.Generator(device="cuda").manual_seed(new)
    codes = lambda *s: torch.randint(-127, 128, s, generator=g, device="cuda", dtype=torch.int8)  # noqa: E731
    small = [codes(3, Hkv, page, D), codes(3, Hkv, D, page), torch.rand(3, Hkv, generator=g, device="cuda") / 32,
             torch.rand(3, Hkv, generator=g, device="cuda") / 32]
    large = [torch.empty((n_pages, *t.shape[1:]), dtype=t.dtype, device="cuda") for t in small]
    for s, t in zip(small, large):
        t[far] = s
    k, v, q = [torch.randn(new, h, D, generator=g, device="cuda").to(dtype) for h in (Hkv, Hkv, Hq)]
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    start, kv_len, every = ints(0, new), ints(kv), ints(0, kv)
    got = []
    for cache, pages in ((small, here), (large, far)):
        table = ints(pages)
        C.crvq_kv_append(k, v, *cache, table, start, kv_len, new)
        out, lse = torch.empty_like(q), torch.empty(new, Hq, device="cuda")
        C.crvq_kv_attention(q, out, *cache, table, start, kv_len, new, kv, lse=lse)
        ko, vo = torch.empty(kv, Hkv, D, dtype=dtype, device="cuda"), torch.empty(kv, Hkv, D, dtype=dtype, device="cuda")
        C.crvq_kv_read(ko, vo, *cache, table, every, kv_len, kv)
        got.append([out, lse, ko, vo] + [t[pages] for t in cache])
    for x, y in zip(*got):
        assert torch.isfinite(x.float()).all() and torch.equal(x, y)
