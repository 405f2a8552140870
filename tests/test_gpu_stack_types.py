"""Stacks of blocks of 4 and 8 bits with activations of either type (decode.py), call by call."""
import pytest
import torch

from paper_2412_09282_amd import crvq as C
from paper_2412_09282_amd import decode

from gpu_util import say

pytestmark = pytest.mark.gpu


def make(bits):
    g = torch.Generator(device="cuda").manual_seed(4)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    N, H, D = 96, 3, 32
    blocks = []
    for b in bits:
        c = decode.PagedCache(8, H, D, page=16)
        c.add_sequence()
        blocks.append(decode.AttentionBlock(rand(3 * H * D, N) * 0.1, rand(N, H * D) * 0.1, H, H, c, *decode.rotary_angles(64, D),
                                            group=32, bits=b))
    return blocks, [1 + 0.1 * rand(N) for _ in bits], [1 + 0.1 * rand(N) for _ in bits], rand


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [(8, 8), (4, 8, 4), (8, 4, 8)])
def test_stack(bits, dtype):
    say(f"stack of {bits} bits, {dtype}")
    (blocks, pre, post, rand), (again, _, _, _) = make(bits), make(bits)
    stack = decode.Stack(blocks, pre, post, alpha=0.5, dtype=dtype)
    for n in (20, 1):
        r = rand(n, 96)
        expect = r.clone()
        stack(r, [b.cache.grow([n]) for b in blocks])
        for b, w, p in zip(again, pre, post):
            zeros, h, s = torch.zeros(n, 96, device="cuda", dtype=dtype), torch.empty(n, 96, device="cuda", dtype=dtype), None
            if b.bits == 8:
                h, s = torch.empty(n, 96, device="cuda", dtype=torch.int8), torch.empty(n, device="cuda")
            C.crvq_norm(zeros, h, residual=expect, w_pre=w, eps=1e-5, h_scales=s)
            out = b(h, b.cache.grow([n])) if s is None else b(h, b.cache.grow([n]), s, dtype)
            assert out.dtype == dtype
            C.crvq_norm(out, None, residual=expect, residual_out=expect, w_post=p, alpha=0.5, eps=1e-5)
        # in the stack a block's norm is in one call with the sum before it: the same fp32 numbers
        assert torch.equal(r, expect)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_codes_are_as_good_as_what_they_are_of(dtype):
    """A block brings activations to the codes and scales that it may be given instead."""
    (a, b), _, _, rand = make((8, 8))
    b.qkv, b.out = a.qkv, a.out
    for n in (20, 1, 3):
        x = rand(n, 96).to(dtype)
        codes, scales = torch.empty(n, 96, device="cuda", dtype=torch.int8), torch.empty(n, device="cuda")
        C.crvq_w8_quantize(x, codes, scales)
        assert torch.equal(a(x, a.cache.grow([n])), b(codes, b.cache.grow([n]), scales, dtype))
