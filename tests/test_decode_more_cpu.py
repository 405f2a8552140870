"""CPU-only: the pages and batches of decode.py with drafts and a budget, as far as they need no GPU."""
import pytest
import torch

from paper_2412_09282_amd import decode


def cache(**kw):
    c = decode.PagedCache(8, 2, 16, page=16, device="cpu", **kw)
    for _ in range(2):
        c.add_sequence()
    return c


def drafted(c, counts):
    """A batch of drafts without its mask, which the GPU makes."""
    c.grow(counts)
    c.places = [p - n for p, n in zip(c.places, counts)]
    c.drafts = list(counts)


def test_accepting_the_first_drafts_moves_nothing():
    c = cache()
    c.grow([14, 3])
    drafted(c, [5, 4])
    assert len(c.free) == 8 - 2 - 1 and c.lengths == [19, 7]
    with pytest.raises(RuntimeError, match="wait"):
        c.grow([1, 1])
    c.accept([[0], []])
    assert c.lengths == [15, 3] and c.places == [15, 3] and c.drafts is None
    assert len(c.free) == 8 - 1 - 1 and sorted(c.free + c.pages[0] + c.pages[1]) == list(range(8))
    b = c.grow([1, 1])
    assert b.places is None and b.mask is None and b.kv_len.tolist() == [16, 4]


@pytest.mark.parametrize("bad", [[[0]], [[5], []], [[-1], []], [[1, 0], []], [[1, 1], []]])
def test_what_cannot_be_accepted(bad):
    c = cache()
    drafted(c, [5, 4])
    with pytest.raises(ValueError):
        c.accept(bad)
    assert c.drafts == [5, 4]


def test_refusals():
    c = cache()
    with pytest.raises(RuntimeError, match="no drafted"):
        c.accept([[], []])
    with pytest.raises(RuntimeError, match="track"):
        c.evict(4)
    with pytest.raises(ValueError, match="parent"):
        c.grow([2, 1], [[-1], [-1]])
    t = cache(track=40)
    assert t.weights.shape == (2, 2, 40)
    with pytest.raises(RuntimeError, match="tracked"):
        t.grow([41, 0])
    for args in ((0,), (4, 5), (4, 1, -1), (4, 2, 3)):
        with pytest.raises(ValueError, match="budget"):
            t.evict(*args)
    t.evict(4)  # nothing to do
    drafted(t, [2, 2])
    with pytest.raises(RuntimeError, match="wait"):
        t.evict(4)
    t.drop_sequence(0)
    assert t.drafts == [0, 2]
    t.accept([[], [0, 1]])
    assert t.lengths == [0, 2] and t.places == [0, 2]
    block = object.__new__(decode.AttentionBlock)
    block.bits, block.window, block.cache = 4, 3, t
    with pytest.raises(ValueError, match="8-bit"):
        block(torch.zeros(2, 8), t.grow([1, 1]), torch.zeros(2))
    t.evicted = True
    with pytest.raises(ValueError, match="window"):
        block(torch.zeros(2, 8), t.grow([1, 1]))
    with pytest.raises(ValueError, match="norms"):
        decode.Stack([block], [])
    with pytest.raises(ValueError, match="batches"):
        decode.Stack([block], [torch.ones(8)])(torch.zeros(2, 8), [])


def test_places_after_an_eviction():
    c = cache()
    c.grow([20, 3])
    c.lengths[0], c.pages[0], c.evicted = 5, c.pages[0][:1], True  # as evict leaves it
    b = c.grow([2, 1])
    assert b.places.tolist() == [20, 21, 3] and b.kv_len.tolist() == [7, 4] and c.places == [22, 4]
    assert c.grow([0, 1]).places.tolist() == [4]
