"""The attention block of a decoder on quantized data, as a sequence of libcrvq calls.

    python -m paper_2412_09282_amd.decode [--channels 4096 --heads 32 --kv-heads 32 --seqs 4 --prompt 300 --steps 32]

A block holds its projections in 4 bits with group scales (crvq_w4_quantize) and its keys and values in a paged
cache of 8 bits with a scale for each page and head.  One call of the block takes the activations of every
sequence's new tokens (prompts, single tokens, or both in one batch) through

    crvq_w4_gemv       queries, keys and values, one stacked matrix
    crvq_kv_append     rotation by the tokens' places, quantization and storage of keys and values
    crvq_kv_attention  attention of the new tokens over the cache
    crvq_w4_gemv       the output projection

Every arithmetic step runs in the library's kernels; this module allocates device tensors, hands out pages and
sequences the calls.  The program decodes with random weights and activations and prints the time of a step.
"""
from __future__ import annotations

import argparse
import dataclasses
from typing import List, Optional, Sequence

import torch

from . import crvq as C


class W4Matrix:
    """An M x N matrix in 4 bits: codes, group scales and (optionally) zero points."""

    def __init__(self, W: torch.Tensor, group: int = 128, zeros: bool = False, scale_dtype=torch.bfloat16):
        M, N = W.shape
        groups = -(-N // group)
        self.group = group
        self.codes = torch.empty(M, -(-N // 32) * 16, dtype=torch.uint8, device=W.device)
        self.scales = torch.empty(M, groups, dtype=scale_dtype, device=W.device)
        self.zeros = torch.empty(M, groups, dtype=torch.uint8, device=W.device) if zeros else None
        C.crvq_w4_quantize(W, self.codes, self.scales, group, zeros=self.zeros)

    def product(self, x: torch.Tensor, y: Optional[torch.Tensor] = None) -> torch.Tensor:
        """x (T x N) times the matrix transposed; y: T x M of x's type unless given."""
        if y is None:
            y = torch.empty(x.shape[0], self.codes.shape[0], dtype=x.dtype, device=x.device)
        C.crvq_w4_gemv(self.codes, self.scales, self.group, x, y, zeros=self.zeros)
        return y


class PagedCache:
    """Pages of keys and values in 8 bits and the sequences that own them."""

    def __init__(self, n_pages: int, kv_heads: int, head_dim: int, page: int = 64, device="cuda"):
        self.page = page
        self.k = torch.zeros(n_pages, kv_heads, page, head_dim, dtype=torch.int8, device=device)
        self.v = torch.zeros(n_pages, kv_heads, head_dim, page, dtype=torch.int8, device=device)
        self.k_scale = torch.zeros(n_pages, kv_heads, device=device)
        self.v_scale = torch.zeros(n_pages, kv_heads, device=device)
        self.free = list(range(n_pages - 1, -1, -1))
        self.pages: List[List[int]] = []
        self.lengths: List[int] = []

    def add_sequence(self) -> int:
        self.pages.append([])
        self.lengths.append(0)
        return len(self.lengths) - 1

    def drop_sequence(self, b: int) -> None:
        """The sequence's pages are free again; it stays in the batch with nothing in it."""
        self.free.extend(reversed(self.pages[b]))
        self.pages[b], self.lengths[b] = [], 0

    def grow(self, counts: Sequence[int]) -> "Batch":
        """Room for counts[b] more tokens of every sequence, and the batch arrays of the call that brings them."""
        if len(counts) != len(self.lengths):
            raise ValueError(f"{len(counts)} counts for {len(self.lengths)} sequences")
        if min(counts, default=0) < 0:
            raise ValueError("a sequence cannot bring a negative number of tokens")
        need = [max(0, -(-(n + k) // self.page) - len(p)) for n, k, p in zip(counts, self.lengths, self.pages)]
        if sum(need) > len(self.free):
            raise RuntimeError(f"the cache is full: {sum(need)} pages needed, {len(self.free)} free")
        for b, n in enumerate(need):
            self.pages[b].extend(self.free.pop() for _ in range(n))
            self.lengths[b] += counts[b]
        dev, width = self.k.device, max(1, max((len(p) for p in self.pages), default=1))
        starts = [0]
        for n in counts:
            starts.append(starts[-1] + n)
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
        table = ints([p + [0] * (width - len(p)) for p in self.pages]).view(len(self.pages), width)
        return Batch(table, ints(starts), ints(self.lengths), max(counts, default=0), max(self.lengths, default=0),
                     starts[-1])

    @property
    def tensors(self):
        return self.k, self.v, self.k_scale, self.v_scale


@dataclasses.dataclass
class Batch:
    """The new tokens of one call: block table, first rows, lengths with the new tokens, and their bounds."""
    table: torch.Tensor
    start: torch.Tensor
    kv_len: torch.Tensor
    max_new: int
    max_kv: int
    tokens: Optional[int] = None  # new tokens of all sequences


def rotary_angles(n: int, rot: int, base: float = 10000.0, device="cuda"):
    """cos and sin (n x rot / 2) of the usual rotary positions."""
    a = torch.arange(n, device=device, dtype=torch.float64)[:, None] * \
        base ** (-torch.arange(rot // 2, device=device, dtype=torch.float64) * 2 / rot)
    return a.cos().float(), a.sin().float()


class AttentionBlock:
    """Stacked query / key / value projection, cache and output projection of one decoder layer."""

    def __init__(self, W_qkv: torch.Tensor, W_out: torch.Tensor, heads: int, kv_heads: int, cache: PagedCache, cos, sin,
                 group: int = 128, zeros: bool = False, window: int = 0):
        D = cache.k.shape[3]
        if W_qkv.shape[0] != (heads + 2 * kv_heads) * D or W_out.shape[1] != heads * D:
            raise ValueError("the projections do not fit the heads")
        self.heads, self.kv_heads, self.D, self.window = heads, kv_heads, D, window
        self.qkv, self.out = W4Matrix(W_qkv, group, zeros), W4Matrix(W_out, group, zeros)
        self.cache, self.cos, self.sin = cache, cos, sin

    def __call__(self, x: torch.Tensor, batch: Batch) -> torch.Tensor:
        """x: the new tokens' activations, T x channels, sequence after sequence."""
        if batch.tokens is not None and x.shape[0] != batch.tokens:
            raise ValueError(f"{x.shape[0]} rows for a batch of {batch.tokens} new tokens")
        H, K, D = self.heads, self.kv_heads, self.D
        q, k, v = (t.unflatten(1, (-1, D)) for t in self.qkv.product(x).split([H * D, K * D, K * D], 1))
        where = (*self.cache.tensors, batch.table, batch.start, batch.kv_len)
        C.crvq_kv_append(k, v, *where, batch.max_new, cos=self.cos, sin=self.sin, q=q, q_out=q)
        o = torch.empty(x.shape[0], H, D, dtype=x.dtype, device=x.device)
        C.crvq_kv_attention(q, o, *where, batch.max_new, batch.max_kv, window=self.window)
        return self.out.product(o.flatten(1))


def main(argv=None):
    ap = argparse.ArgumentParser()
    ap.add_argument("--channels", type=int, default=4096)
    ap.add_argument("--heads", type=int, default=32)
    ap.add_argument("--kv-heads", type=int, default=32)
    ap.add_argument("--seqs", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=300)
    ap.add_argument("--steps", type=int, default=32)
    args = ap.parse_args(argv)
    D, total = args.channels // args.heads, args.prompt + args.steps
    g = torch.Generator(device="cuda").manual_seed(0)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    cache = PagedCache(args.seqs * (-(-total // 64)), args.kv_heads, D)
    W = rand((args.heads + 2 * args.kv_heads) * D, args.channels).mul_(0.02).bfloat16()
    Wo = rand(args.channels, args.heads * D).mul_(0.02).bfloat16()
    block = AttentionBlock(W, Wo, args.heads, args.kv_heads, cache, *rotary_angles(total, D))
    for _ in range(args.seqs):
        cache.add_sequence()
    y = block(rand(args.seqs * args.prompt, args.channels).bfloat16(), cache.grow([args.prompt] * args.seqs))
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    for i in range(args.steps):
        if i == min(4, args.steps - 1):
            start.record()
        y = block(rand(args.seqs, args.channels).bfloat16(), cache.grow([1] * args.seqs))
    end.record()
    torch.cuda.synchronize()
    n = args.steps - min(4, args.steps - 1)
    print(f"{args.seqs} sequences of {args.prompt} + {args.steps} tokens, {args.channels} channels, {args.heads} heads: "
          f"{start.elapsed_time(end) / n * 1e3:.1f} us a step; output finite: {bool(torch.isfinite(y).all())}", flush=True)


if __name__ == "__main__":
    main()
