"""CPU-only: the pages and batches of decode.py, and what it refuses."""
import pytest
import torch

from paper_2412_09282_amd import decode


def cache():
    c = decode.PagedCache(6, 2, 16, page=16, device="cpu")
    for _ in range(2):
        c.add_sequence()
    return c


def test_a_batch_knows_its_rows():
    c = cache()
    b = c.grow([20, 3])
    assert (b.tokens, b.max_new, b.max_kv) == (23, 20, 20) and b.start.tolist() == [0, 20, 23]
    block = object.__new__(decode.AttentionBlock)  # the rows are looked at before anything of the block is used
    block.heads, block.kv_heads, block.D = 2, 2, 16
    for rows in (22, 24, 0):
        with pytest.raises(ValueError, match="rows"):
            block(torch.zeros(rows, 8), b)


def test_negative_counts_change_nothing():
    c = cache()
    c.grow([20, 3])
    before = [list(p) for p in c.pages], list(c.lengths), list(c.free)
    with pytest.raises(ValueError, match="negative"):
        c.grow([1, -2])
    assert before == (c.pages, c.lengths, c.free)
