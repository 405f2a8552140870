"""Drafts, weights and the move over a cache whose keys, and values, pass 4 GiB each: the same results as over a small cache that
holds the same pages, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2412_09282_amd import crvq as C

from gpu_util import say
from test_gpu_kv import dev, make, values_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [[3, 2], [20, 7], [140, 30]])
def test_far_pages(new):
    say(f"pages past 4 GiB, {new} new tokens")
    Hkv, D, page, n_pages = 8, 128, 64, 70000  # 4.6 GB of keys, as many of values
    kv = [700, 333]
    g, small, table, start, kv_len = make(7, new, kv, Hkv, D, page, spare=14, garbage=False)
    n = small[0].shape[0]
    far = torch.from_numpy(np.concatenate([np.arange(n_pages - n + 2, n_pages), [5, 35000]]).astype(np.int64)).cuda()  # page i of the small cache
    s = [dev(a) for a in small]
    big = [torch.empty(n_pages, *a.shape[1:], dtype=a.dtype, device="cuda") for a in s]
    for b, a in zip(big, s):
        b[far] = a
    where = far[dev(table).long()].to(torch.int32).contiguous()
    free = np.setdiff1d(np.arange(n), table)[:14].reshape(2, 7).astype(np.int32)
    to, far_to = dev(free), far[dev(free).long()].to(torch.int32).contiguous()
    T = int(start[-1])
    q = dev(values_of(g, T, 16, D, dtype="bf16"), "bf16")
    mask = torch.randint(-2 ** 62, 2 ** 62, (T, 3), device="cuda")
    results = []
    for cache, t, dest in ((s, dev(table), to), (big, where, far_to)):
        batch = (t, dev(start), dev(kv_len), max(new), max(kv))
        out, lse, w = torch.empty_like(q), torch.empty(T, 16, device="cuda"), torch.zeros(2, Hkv, max(kv), device="cuda")
        C.crvq_kv_tree_attention(q, out, *cache, *batch, mask, lse=lse)
        C.crvq_kv_weights(q, lse, None, w, cache[0], cache[2], *batch, mask=mask)
        keep, count = torch.zeros(2, Hkv, 400, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
        C.crvq_kv_select(w, dev(kv_len), 400, keep, count, sinks=3, recent=60)
        C.crvq_kv_gather(*cache, t, dev(kv_len), keep, count, dest)
        k, v = torch.empty(733, Hkv, D, device="cuda"), torch.empty(733, Hkv, D, device="cuda")
        C.crvq_kv_read(k, v, *cache, dest, dev(np.array([0, 400, 733], np.int32)), count, 400)
        results.append((out, lse, w, keep[0], keep[1, :, :333], count, k, v))
        torch.cuda.synchronize()
    for a, b in zip(*results):
        assert torch.equal(a, b)
