"""CPU-only: the calls of drafted tokens and of the cache within a budget reject bad arguments on the host, before anything is
enqueued, and the numpy definitions in oracle/drafts.py agree with closed forms."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import drafts, serve
from paper_2412_09282_amd import crvq as C


@pytest.fixture(scope="module")
def L():
    return C.lib()


def P(n, off=0):
    return ctypes.c_void_p((n << 40) + off)  # never dereferenced


def err(L):
    return L.crvq_last_error().decode()


def tree_mask(L, **kw):
    a = dict(B=2, parents=P(1), start=P(2), kv_len=P(3), max_new=70, n=100, window=0, mask=P(4), ld=2, places=P(5))
    a.update(kw)
    return L.crvq_tree_mask(*a.values(), None)


CACHE = dict(B=2, Hq=8, Hkv=4, D=64, page=32, n_pages=10, k=P(1), v=P(2), ks=P(3), vs=P(4), table=P(5), ld=5, start=P(6),
             kv_len=P(7), max_new=9, max_kv=160, n=12, dt=1)


def attend(L, **kw):
    a = dict(CACHE, q=P(8), q_tok=512, q_head=64, out=P(9), o_tok=512, o_head=64, scale=0.125, mask=P(10), ld_mask=1, window=0,
             places=P(11), lse=P(12), ws=P(20), wsb=1 << 40)
    a.update(kw)
    return L.crvq_kv_tree_attention(*a.values(), None)


def weights(L, **kw):
    a = dict({k: v for k, v in CACHE.items() if k not in ("v", "vs")}, q=P(8), q_tok=512, q_head=64, lse=P(12), scale=0.125, causal=1,
             window=0, mask=None, ld_mask=0, places=None, decay=1.0, before=P(13), after=P(14), ld_w=160, ws=P(20), wsb=1 << 40)
    a.update(kw)
    return L.crvq_kv_weights(*a.values(), None)


def select(L, **kw):
    a = dict(B=2, Hkv=4, kv_len=P(1), w=P(2), ld=1000, budget=100, sinks=4, recent=20, keep=P(3), ld_keep=100, n=P(4), kept=P(5), ws=P(20), wsb=1 << 40)
    a.update(kw)
    return L.crvq_kv_select(*a.values(), None)


def gather(L, **kw):
    a = dict(B=2, Hkv=4, D=64, page=32, n_pages=10, k=P(1), v=P(2), ks=P(3), vs=P(4), table=P(5), ld=5, kv_len=P(7), keep=P(8),
             ld_keep=100, heads=4, n=P(9), max_keep=100, to=P(10), ld_to=4)
    a.update(kw)
    return L.crvq_kv_gather(*a.values(), None)


def test_tree_mask_arguments(L):
    for bad, status in [(dict(B=-1), 1), (dict(max_new=-1), 1), (dict(n=-1), 1), (dict(window=-1), 1), (dict(B=65536), 2), (dict(n=1 << 31), 2),
                        (dict(parents=None), 1), (dict(start=None), 1), (dict(kv_len=None), 1), (dict(ld=1), 1), (dict(mask=P(4, 4)), 1),
                        (dict(places=P(5, 2)), 1), (dict(mask=P(1)), 1), (dict(places=P(1, 40)), 1), (dict(places=P(4, 64)), 1)]:
        assert tree_mask(L, **bad) == status and "crvq_tree_mask" in err(L), bad
    for nothing in (dict(B=0), dict(max_new=0), dict(n=0), dict(mask=None, places=None)):
        assert tree_mask(L, parents=None, **nothing) == 0


CACHE_BAD = [(dict(dt=2), 1, "dtype"), (dict(D=8), 2, "D ="), (dict(D=272), 2, "D ="), (dict(page=24), 2, "page"), (dict(Hkv=0), 1, "Hkv"),
             (dict(B=-1), 1, "negative"), (dict(n_pages=1 << 31), 2, "pages"), (dict(n_pages=-1), 1, "negative"),
             (dict(kv_len=None), 1, "kv_len"), (dict(table=None), 1, "block_table"), (dict(k=None), 1, "cache"), (dict(ks=None), 1, "cache"),
             (dict(k=P(1, 8)), 1, "aligned")]


@pytest.mark.parametrize("call", [attend, weights])
def test_cache_arguments(L, call):
    for bad, status, text in CACHE_BAD + [(dict(max_new=-1), 1, "negative"), (dict(n=-1), 1, "negative"), (dict(n=1 << 31), 2, "rows"),
                                          (dict(start=None), 1, "start"), (dict(Hq=6), 1, "Hq"), (dict(max_kv=-1), 1, "max_kv"),
                                          (dict(max_kv=(1 << 30) + 1, **({} if call is attend else dict(ld_w=1 << 31))), 1, "max_kv"),
                                          (dict(scale=float("inf")), 1, "scale"), (dict(window=-1), 1, "window"), (dict(q=None), 1, "q"),
                                          (dict(q_tok=-1), 1, "stride"), (dict(q=P(8, 1)), 1, "aligned"), (dict(mask=P(10, 4), ld_mask=1), 1, "aligned"),
                                          (dict(mask=P(10), ld_mask=0), 1, "ld_mask"), (dict(mask=P(10), ld_mask=1, places=P(11, 1)), 1, "places")]:
        assert call(L, **bad) == status, (bad, err(L))
        assert text in err(L), (bad, err(L))
    for nothing in (dict(B=0), dict(max_new=0), dict(n=0)):
        assert call(L, start=None, kv_len=None, **nothing) == 0


def test_tree_attention_arguments(L):
    for bad in (dict(mask=None), dict(out=None), dict(o_tok=500), dict(out=P(8, 64)), dict(lse=P(8)), dict(lse=P(9)), dict(out=P(10)),
                dict(out=P(11)), dict(lse=P(10)), dict(lse=P(11)), dict(v=None), dict(vs=None), dict(v=P(2, 4))):
        assert attend(L, **bad) == 1, bad
    assert attend(L, Hq=4 << 17, max_new=1) == 2 and attend(L, Hq=4 << 16, max_new=1 << 15, ld_mask=1 << 9) == 2
    need = L.crvq_kv_tree_attention_workspace_size(2, 8, 4, 64, 9, 100000)
    assert need and attend(L, max_kv=100000, wsb=need - 1) == 3 and attend(L, max_kv=100000, ws=None) == 3
    for none in [(0, 8, 4, 64, 9, 99), (2, 6, 4, 64, 9, 99), (2, 8, 4, 63, 9, 99), (2, 8, 4, 64, 0, 99), (2, 8, 4, 64, 9, -1)]:
        assert L.crvq_kv_tree_attention_workspace_size(*none) == 0


def test_weights_arguments(L):
    for bad, status in [(dict(causal=0, window=5), 1), (dict(decay=float("nan")), 1), (dict(ld_w=159), 1), (dict(lse=None), 1), (dict(after=None), 1),
                        (dict(lse=P(12, 2)), 1), (dict(before=P(13, 1)), 1), (dict(after=P(14, 2)), 1), (dict(after=P(13, 64)), 1),
                        (dict(after=P(8)), 1), (dict(after=P(12)), 1), (dict(mask=P(14, 8), ld_mask=1), 1),
                        (dict(mask=P(10), ld_mask=1, places=P(14)), 1), (dict(B=20000), 2), (dict(Hq=4 << 28, max_new=9), 2), (dict(Hq=4 << 16, max_new=1 << 15), 2),
                        (dict(Hq=4 << 17, max_new=1), 2)]:
        assert weights(L, **bad) == status, (bad, err(L))
    for fine in (dict(max_kv=0), dict(max_kv=0, after=None)):
        assert weights(L, **fine) == 0
    for shape in [(1, 64, 8, 128, 2048, 4000), (2, 8, 4, 64, 9, 160), (1, 8, 1, 64, 500, 600)]:
        need = L.crvq_kv_weights_workspace_size(*shape)
        B, Hq, Hkv, D, new, kv = shape
        assert need % 256 == 0 and need == L.crvq_workspace_size(13, B, new, 0, 0, D, None, Hq, Hkv, kv)
        if need:
            args = dict(B=B, Hq=Hq, Hkv=Hkv, D=D, max_new=new, max_kv=kv, n=new, q_tok=Hq * D, q_head=D, ld_w=kv, mask=None)
            assert weights(L, wsb=need - 1, **args) == 3 and weights(L, ws=None, **args) == 3


def test_select_arguments(L):
    for bad, status in [(dict(B=-1), 1), (dict(Hkv=0), 1), (dict(budget=-1, sinks=0, recent=0), 1), (dict(sinks=-1), 1), (dict(recent=-1), 1),
                        (dict(sinks=81), 1), (dict(sinks=(1 << 31) - 1, recent=1), 1), (dict(ld=-1), 1), (dict(ld=(1 << 30) + 1), 1), (dict(ld_keep=99), 1),
                        (dict(kv_len=None), 1), (dict(w=None), 1), (dict(keep=None), 1), (dict(n=None), 1), (dict(w=P(2, 2)), 1),
                        (dict(kept=P(5, 1)), 1), (dict(keep=P(2, 64)), 1), (dict(kept=P(3)), 1), (dict(kept=P(2)), 1), (dict(n=P(1)), 1),
                        (dict(B=1 << 30, Hkv=4), 2)]:
        assert select(L, **bad) == status and "crvq_kv_select" in err(L), (bad, err(L))
    assert select(L, B=0, kv_len=None) == 0
    need = L.crvq_kv_select_workspace_size(2, 4, 200000)
    assert need and need % 256 == 0 and need == L.crvq_workspace_size(15, 2, 0, 0, 0, 0, None, 0, 4, 200000)
    assert select(L, ld=200000, ws=None) == 3 and select(L, ld=200000, wsb=need - 1) == 3 and select(L, ld=200000, ws=P(20, 8)) == 3
    assert L.crvq_kv_select_workspace_size(2, 4, 1000) == 0 and L.crvq_kv_select_workspace_size(2, 4, -1) == 0


def test_gather_arguments(L):
    for bad, status, text in CACHE_BAD:
        if "dt" in bad:
            continue
        assert gather(L, **bad) == status, (bad, err(L))
        assert text in err(L) or "kv_len" in err(L), (bad, err(L))
    for bad in (dict(heads=2), dict(heads=0), dict(ld_to=-1), dict(ld_keep=99), dict(max_keep=-1), dict(keep=None), dict(n=None), dict(to=None),
                dict(v=P(1)), dict(vs=P(3)), dict(v=P(2, 8))):
        assert gather(L, **bad) == 1 and "crvq_kv_gather" in err(L), bad
    assert gather(L, B=0, keep=None) == 0 and gather(L, max_keep=0, keep=None) == 0


def test_definitions_against_closed_forms():
    mask, places = drafts.tree([-1, 0, 0, 2, -1], 12, 1)
    assert mask[:, 0].tolist() == [1, 3, 5, 13, 16] and places.tolist() == [7, 8, 8, 9, 7]
    assert drafts.tree([-1, 0, 1, 2], 4, 1, window=2)[0][:, 0].tolist() == [1, 3, 6, 12]
    assert drafts.tree([-1, 1, 1], 9, 1)[1].tolist() == [6, -1, -1]
    assert drafts.select(np.array([5., 1, 3, 3, 9, 0]), 6, 4, 1, 1) == [0, 2, 4, 5]
    assert drafts.select(np.array([np.nan, 1, -np.inf]), 3, 2, 0, 0) == [1, 2]
    # a chain's mask sees what causal attention sees, with the same results
    g = np.random.default_rng(0)
    cache = [g.integers(-127, 128, (6, 2, 16, 16)).astype(np.int8), g.integers(-127, 128, (6, 2, 16, 16)).astype(np.int8),
             np.full((6, 2), 0.01, np.float32), np.full((6, 2), 0.02, np.float32)]
    table, start, kv = np.array([[3, 1, 5]], np.int32), np.array([0, 4], np.int32), np.array([40], np.int32)
    q = g.standard_normal((4, 4, 16)).astype(np.float32)
    mask, places = drafts.tree([-1, 0, 1, 2], 40, 1)
    sees = drafts.sees_mask(mask, 4, 40, places)
    assert (sees == drafts.sees_causal(4, 40)).all()
    for a, b in zip(drafts.attention(cache, table, start, kv, q, 0.25, [sees]), serve.attention(cache, table, start, kv, q, 0.25)):
        assert np.allclose(a, b)
    lse = drafts.attention(cache, table, start, kv, q, 0.25, [sees])[1]
    w, _ = drafts.weights(cache, table, start, kv, q, 0.25, lse, [sees], None, np.zeros((1, 2, 40)), 1.0)
    assert np.allclose(w.sum(-1), 8)
    # tokens of one page keep their codes
    to = np.array([[0]], np.int32)
    k, v, ks, vs = drafts.gather(cache, table, kv, np.array([[[17, 20, 31]]]), [3], to)
    assert (k[0, :, :3] == cache[0][1][:, [1, 4, 15]]).all() and (v[0, :, :, :3] == cache[1][1][:, :, [1, 4, 15]]).all() and not k[0, :, 3:].any()


def test_binding_refusals():
    i32 = dict(dtype=torch.int32)
    kc, vc, sc = torch.zeros(1, 2, 16, 32, dtype=torch.int8), torch.zeros(1, 2, 32, 16, dtype=torch.int8), torch.zeros(1, 2)
    table, start, n = torch.zeros(1, 1, **i32), torch.tensor([0, 2], **i32), torch.tensor([2], **i32)
    q, lse, w, m = torch.zeros(2, 4, 32), torch.zeros(2, 4), torch.zeros(1, 2, 9), torch.zeros(2, 1, dtype=torch.int64)
    keep = torch.zeros(1, 2, 4, **i32)
    for call in (lambda: C.crvq_tree_mask(torch.zeros(2, **i32), start, n, 2, m),
                 lambda: C.crvq_kv_tree_attention(q, q.clone(), kc, vc, sc, sc.clone(), table, start, n, 2, 2, m),
                 lambda: C.crvq_kv_weights(q, lse, None, w, kc, sc, table, start, n, 2, 2),
                 lambda: C.crvq_kv_select(w, n, 4, keep, n.clone()),
                 lambda: C.crvq_kv_gather(kc, vc, sc, sc.clone(), table, n, keep, n, table)):
        with pytest.raises(ValueError, match="host memory"):
            call()
    for call in (lambda: C.crvq_tree_mask(torch.zeros(2, **i32), start, n, 65, m),
                 lambda: C.crvq_tree_mask(torch.zeros(2, **i32), start, n, 2, m.int()),
                 lambda: C.crvq_kv_tree_attention(q, q.clone(), kc, vc, sc, sc.clone(), table, start, n, 2, 2, m[:1]),
                 lambda: C.crvq_kv_tree_attention(q, q.clone(), kc, vc, sc, sc.clone(), table, start, n, 2, 2, m, places=n),
                 lambda: C.crvq_kv_weights(q, lse, w[:, :, :8], w, kc, sc, table, start, n, 2, 2),
                 lambda: C.crvq_kv_weights(q, lse[:, :3].contiguous(), None, w, kc, sc, table, start, n, 2, 2),
                 lambda: C.crvq_kv_select(w, n, 4, keep[:, :1], n.clone()),
                 lambda: C.crvq_kv_select(w, n, 4, keep, n.clone(), kept_weights=w),
                 lambda: C.crvq_kv_gather(kc, vc, sc, sc.clone(), table, n, keep.long(), n, table)):
        with pytest.raises(AssertionError):
            call()


class Somewhere:
    """What the binding asks a tensor about where it is."""

    def __init__(self, device, pinned=False):
        self.device, self.pinned = device, pinned

    is_cuda = property(lambda self: self.device >= 0)

    def get_device(self):
        return self.device

    def is_pinned(self):
        return self.pinned


def test_tensors_of_one_call_are_on_one_device():
    C._one_device(Somewhere(1), Somewhere(1), None, Somewhere(-1, True))
    C._one_device(Somewhere(-1, True), Somewhere(-1, True), Somewhere(0))
    for first, other, text in [(Somewhere(0), Somewhere(1), "tensors on"), (Somewhere(0), Somewhere(-1), "host memory"), (Somewhere(-1), Somewhere(0), "host memory")]:
        with pytest.raises(ValueError, match=text):
            C._one_device(first, Somewhere(first.device, True), other)
