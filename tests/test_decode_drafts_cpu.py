"""CPU-only: drafted tokens and stacks in decode.py, with the library's calls replaced by their definitions in oracle/drafts.py or noted
down."""
import numpy as np
import pytest
import torch

from oracle import drafts
from paper_2412_09282_amd import crvq as C
from paper_2412_09282_amd import decode


@pytest.fixture
def calls(monkeypatch):
    """Masks as oracle/drafts.py has them; what other calls got."""
    noted = []

    def tree_mask(parents, start, kv_len, max_new, mask=None, places=None, window=0, stream=None):
        for b in range(kv_len.numel()):
            r0, r1 = int(start[b]), int(start[b + 1])
            m, p = drafts.tree(parents[r0:r1].numpy(), int(kv_len[b]), mask.shape[1], window)
            mask[r0:r1] = torch.from_numpy(m.view(np.int64))
            places[r0:r1] = torch.from_numpy(p)

    monkeypatch.setattr(C, "crvq_tree_mask", tree_mask)
    for name in ("crvq_w8_quantize", "crvq_w8_gemm", "crvq_kv_append", "crvq_kv_attention", "crvq_kv_tree_attention", "crvq_kv_weights",
                 "crvq_kv_gather", "crvq_norm", "crvq_w4_quantize", "crvq_w4_gemv"):
        monkeypatch.setattr(C, name, lambda *a, _name=name, **k: noted.append((_name, a, k)))
    return noted


def block_of(cache, window=0, N=32, bits=8):
    heads, D = cache.k.shape[1], cache.k.shape[3]
    return decode.AttentionBlock(torch.zeros(3 * heads * D, N), torch.zeros(N, heads * D), heads, heads, cache, torch.ones(99, D // 2),
                                 torch.zeros(99, D // 2), window=window, bits=bits)


def cache_of(lengths, **kw):
    c = decode.PagedCache(24, 2, 16, page=16, device="cpu", **kw)
    for _ in lengths:
        c.add_sequence()
    c.grow(lengths)
    return c


@pytest.mark.parametrize("window", [1, 8, 20, 100])
def test_drafts_see_no_further_than_the_window(calls, window):
    """A chain of drafts sees what the same tokens see as plain rows."""
    c = cache_of([30, 3])
    block = block_of(c, window)
    batch = c.grow([20, 7], [[i - 1 for i in range(20)], [i - 1 for i in range(7)]])
    masks, places = batch.mask.numpy().view(np.uint64), batch.places.numpy()
    for rows, n, k in ((slice(0, 20), 20, 50), (slice(20, 27), 7, 10)):
        assert (drafts.sees_mask(masks[rows], n, k, places[rows], window) == drafts.sees_causal(n, k, True, window)).all()
    block(torch.zeros(27, 32), batch)
    assert [k["window"] for name, _, k in calls if name == "crvq_kv_tree_attention"] == [window]


def test_masks_of_another_window_are_refused(calls):
    c = cache_of([30])
    block = block_of(c, 8)
    batch = c.grow([4], [[-1, 0, 1, 2]])
    block.window = 3
    with pytest.raises(ValueError, match="window"):
        block(torch.zeros(4, 32), batch)
    batch.window = None  # a mask of the program's own
    block(torch.zeros(4, 32), batch)


def test_weights_are_of_the_accepted_drafts(calls):
    """Nothing is added before it is known which drafts stay; then the others' rows add nothing, and all of it before tokens
    move."""
    c = cache_of([30, 3, 9], track=90)
    block = block_of(c)
    trees = [[-1, 0, 0, 2, 1], [-1, -1, 1], [-1, 0]]
    for name in ("accept", "refuse"):
        lengths = list(c.lengths)
        batch = c.grow([5, 3, 2], trees)
        del calls[:]
        block(torch.zeros(10, 32), batch)
        assert not [x for x in calls if x[0] == "crvq_kv_weights"]
        lse = next(k["lse"] for n, _, k in calls if n == "crvq_kv_tree_attention")
        lse.copy_(torch.arange(20).view(10, 2))
        c.accept([[0, 2, 3], [], [0, 1]] if name == "accept" else [[], [], []])
        made = [n for n, _, _ in calls if n in ("crvq_kv_weights", "crvq_kv_gather")]
        if name == "refuse":
            assert made == [] and c.lengths == lengths
            continue
        assert made == ["crvq_kv_weights", "crvq_kv_gather"]
        _, (q, got, before, after, *where), k = next(x for x in calls if x[0] == "crvq_kv_weights")
        stay = [0, 2, 3, 8, 9]
        assert (got[stay] == lse[stay]).all() and torch.isinf(got).all(1).nonzero().flatten().tolist() == [1, 4, 5, 6, 7]
        assert after.data_ptr() == before.data_ptr() == c.weights.data_ptr() and k["mask"] is batch.mask and k["places"] is batch.places
        assert where[4] is batch.kv_len and where[2] is batch.table and c.lengths == [33, 3, 11]


def test_weights_while_drafts_wait_and_of_other_masks(calls):
    c = cache_of([30, 3], track=90)
    block = block_of(c)
    batch = c.grow([2, 1], [[-1, 0], [-1]])
    block(torch.zeros(3, 32), batch)
    del calls[:]
    held = c.weights  # as if all stayed: a copy
    assert [x[0] for x in calls] == ["crvq_kv_weights"] and calls[0][1][3].data_ptr() == held.data_ptr()
    c.add_sequence()  # not in the batch
    c.accept([[0, 1], []])
    assert c.weights.shape == (3, 2, 90) and calls[-1][1][3].shape == (2, 2, 90) and c.weights.data_ptr() != held.data_ptr()
    # a mask of the program's own: its rows are no drafts, and count at once
    plain = c.grow([1, 1, 0])
    plain.mask = torch.ones(2, 1, dtype=torch.int64)
    del calls[:]
    block(torch.zeros(2, 32), plain)
    assert [x[0] for x in calls].count("crvq_kv_weights") == 1


@pytest.mark.parametrize("bad", [[1], [3], [0, 3], [0, 2, 4], [0, 1, 2], [0, 5], [5, 6], [0, 1, 3, 6]])
def test_only_paths_of_the_tree_are_accepted(calls, bad):
    c = cache_of([10, 4])
    trees = [[-1, 0, 0, 1, 3, -1, 2], [-1, 0]]
    c.grow([7, 2], trees)
    before = [list(p) for p in c.pages], list(c.lengths), list(c.free), list(c.places)
    with pytest.raises(ValueError, match="path"):
        c.accept([bad, [0]])
    with pytest.raises(ValueError, match="path"):
        c.accept([[0], [1]])
    assert before == (c.pages, c.lengths, c.free, c.places) and c.drafts == [7, 2] and not calls
    c.accept([[0, 1, 3, 4], []])
    assert c.lengths == [14, 4] and c.drafts is None
    c.grow([1, 2], [[-1], [-1, -1]])  # two that follow the context themselves
    c.drop_sequence(0)
    with pytest.raises(ValueError, match="path"):
        c.accept([[], [0, 1]])
    c.accept([[], [1]])
    assert c.lengths == [0, 5]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [(8,), (8, 8), (4, 8, 4), (8, 4, 8)])
def test_a_stack_keeps_its_type(calls, dtype, bits):
    caches = [cache_of([0]) for _ in bits]
    stack = decode.Stack([block_of(c, bits=b) for c, b in zip(caches, bits)], [torch.ones(32) for _ in bits], dtype=dtype)
    del calls[:]
    stack(torch.zeros(3, 32), [c.grow([3]) for c in caches])
    for name, a, k in calls:
        if name in ("crvq_w8_gemm", "crvq_w4_gemv"):  # queries, keys and values, and the block's result
            assert a[4].dtype == dtype, name
        elif name == "crvq_norm":
            assert a[0].dtype == dtype and (a[1] is None or k.get("h_scales") is not None or a[1].dtype == dtype)
        elif name == "crvq_kv_attention":
            assert a[0].dtype == a[1].dtype == dtype
    assert sum(n == "crvq_kv_attention" for n, _, _ in calls) == len(bits)


def test_drafts_of_a_tracking_cache_are_not_captured(monkeypatch, calls):
    """Which of them count is known at accept, outside of any graph."""
    class OnTheGpu:
        is_cuda = True

    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    c = cache_of([10], track=60)
    with pytest.raises(RuntimeError, match="graph"):
        c.attended(OnTheGpu(), None, c.grow([2], [[-1, 0]]), 0)
    c.accept([[0]])
    c.attended(OnTheGpu(), None, c.grow([2]), 0)  # tokens that stay whatever comes
    assert calls[-1][0] == "crvq_kv_weights"
