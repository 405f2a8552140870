"""Drafts, a budget of tokens, 8-bit projections and norms together (decode.py), as a program uses them: each step of a block
against a float64 computation from its own 8-bit weights and the cache it left.

A block of 8 bits brings its fp32 activations to 8 bits exactly as oracle/block.py does, so its queries are known to the bit
(their rotation too).  The attention's rows are within 1e-4 of their largest element (as in tests/test_gpu_decode.py); the
output projection brings them to 8 bits with half a step of max|o| / 127 each, which moves an output by at most that times the
row's sum of |W|."""
import numpy as np
import pytest
import torch

from oracle import block as ob
from oracle import drafts, serve
from paper_2412_09282_amd import crvq as C
from paper_2412_09282_amd import decode

from gpu_util import say

pytestmark = pytest.mark.gpu


def host(t):
    return t.detach().cpu().numpy()


def trees(g, counts):
    return [[-1 if i == 0 else int(g.integers(-1, i)) for i in range(n)] for n in counts]


def path_to(parents, i):
    path = []
    while i >= 0:
        path.insert(0, i)
        i = parents[i]
    return path


class Check:
    def __init__(self, heads, kv_heads, D, N, n_pages, page, track, seed):
        self.g = np.random.default_rng(seed)
        rand = lambda *s: torch.from_numpy(self.g.standard_normal(s).astype(np.float32)).cuda()  # noqa: E731
        self.rand, self.heads, self.kv_heads, self.D, self.N = rand, heads, kv_heads, D, N
        self.cache = decode.PagedCache(n_pages, kv_heads, D, page=page, track=track)
        self.angles = decode.rotary_angles(200, D)
        self.block = decode.AttentionBlock(rand((heads + 2 * kv_heads) * D, N) * 0.1, rand(N, heads * D) * 0.1, heads, kv_heads,
                                           self.cache, *self.angles, bits=8)
        self.W = [(host(m.codes), host(m.scales)) for m in (self.block.qkv, self.block.out)]

    def step(self, counts, parents=None):
        x = self.rand(sum(counts), self.N)
        places = [p + i for p, n in zip(self.cache.places, counts) for i in range(n)]
        if parents is not None:
            places = [p + len(path_to(t, i)) - 1 for p, t in zip(self.cache.places, parents) for i in range(len(t))]
        batch = self.cache.grow(counts, parents)
        before = None if self.cache.weights is None else self.cache.weights.clone()
        y = host(self.block(x, batch)).astype(np.float64)
        start, lens, table = (host(t) for t in (batch.start, batch.kv_len, batch.table))
        qkv = ob.w8_product(*self.W[0], *ob.w8_quantize(host(x)), self.N, False)
        q = qkv[:, :self.heads * self.D].reshape(-1, self.heads, self.D)
        q = serve.rotate(q, np.array(places, int), host(self.angles[0]), host(self.angles[1]), False)
        held = [host(t) for t in self.cache.tensors]
        sees = [drafts.sees_causal(n, k) if parents is None else
                drafts.sees_mask(drafts.tree(parents[b], k, batch.mask.shape[1])[0], n, k) for b, (n, k) in enumerate(zip(counts, lens))]
        o = drafts.attention(held, table, start, lens, q, self.D ** -0.5, sees)[0].reshape(len(q), -1)
        Wo = self.W[1][0][:, :o.shape[1]].astype(np.float64) * self.W[1][1][:, None]
        most = np.abs(o).max(1, keepdims=True)
        tol = (most / 254 + 1e-4 * most) * np.abs(Wo).sum(1)[None] * (1 + 2.0 ** -10)
        assert (np.abs(y - o @ Wo.T) <= tol).all()
        if before is not None:  # every row's weights add up to 1
            for b, (n, k) in enumerate(zip(counts, lens)):
                old = before[b, :, :k - n].double().sum(1)
                got = self.cache.weights[b, :, :k].double().sum(1) - (old if n else self.cache.weights[b, :, :k].double().sum(1))
                assert torch.allclose(got, torch.full_like(got, n * self.heads / self.kv_heads), rtol=1e-4, atol=1e-4)
        keys = qkv[:, self.heads * self.D:(self.heads + self.kv_heads) * self.D].reshape(-1, self.kv_heads, self.D)
        return serve.rotate(keys, np.array(places, int), host(self.angles[0]), host(self.angles[1]), False), start

    def pages_are_whole(self):
        held = self.cache.free + [p for s in self.cache.pages for p in s]
        assert sorted(held) == list(range(self.cache.k.shape[0]))
        assert [len(p) for p in self.cache.pages] == [-(-n // self.cache.page) for n in self.cache.lengths]


@pytest.mark.parametrize("heads,kv_heads,D,page", [(4, 4, 32, 16), (6, 2, 16, 32)])
def test_drafts_and_budget(heads, kv_heads, D, page):
    say(f"drafts and budget, {heads}/{kv_heads} x {D}, pages of {page}")
    t = Check(heads, kv_heads, D, 100, 40, page, 150, heads)
    for _ in range(3):
        t.cache.add_sequence()
    t.step([30, 7, 1])
    for counts in ([9, 5, 0], [20, 33, 6], [3, 1, 17]):
        parents = trees(t.g, counts)
        keys, start = t.step(counts, parents)
        accepted = [path_to(p, len(p) - 1) if p else [] for p in parents]
        if counts[0] == 20:
            accepted[1] = []
        context = [n - k for n, k in zip(t.cache.lengths, counts)]
        t.cache.accept(accepted)
        t.pages_are_whole()
        assert t.cache.lengths == [c + len(a) for c, a in zip(context, accepted)] == t.cache.places
        held = [host(x) for x in t.cache.tensors]
        for b, a in enumerate(accepted):  # the accepted tokens' keys, within a step and a half of their page's scale
            got, _ = serve.values(held, t.cache.pages[b], t.cache.lengths[b])
            step = max((held[2][p].max() for p in t.cache.pages[b]), default=0)
            assert not a or np.abs(got[context[b]:] - keys[start[b]:start[b + 1]][a]).max() <= 1.5 * step
        t.step([1, 1, 1])
    lens = list(t.cache.lengths)
    w, pages, held = host(t.cache.weights), [list(p) for p in t.cache.pages], [host(x).copy() for x in t.cache.tensors]
    t.cache.evict(24, sinks=2, recent=6)
    t.pages_are_whole()
    assert t.cache.lengths == [min(n, 24) for n in lens] and t.cache.places == lens
    now = [host(x) for x in t.cache.tensors]
    for b, n in enumerate(lens):
        old, _ = serve.values(held, pages[b], n)
        new, _ = serve.values(now, t.cache.pages[b], t.cache.lengths[b])
        for h in range(kv_heads):
            keep = drafts.select(w[b, h], n, 24, 2, 6)
            step = max(now[2][p, h] for p in t.cache.pages[b])
            assert np.abs(new[:, h] - old[keep, h]).max() <= 0.5 * step * (1 + 2.0 ** -20)
            assert (host(t.cache.weights)[b, h, :min(n, 24)] == w[b, h, keep]).all()
    t.step([1, 1, 1])           # places go on where they were
    t.step([4, 0, 9], trees(t.g, [4, 0, 9]))
    t.cache.accept([[0], [], [0]])
    t.step([2, 1, 1])
    t.cache.drop_sequence(0)
    t.pages_are_whole()


def test_evict_in_turns_where_pages_are_few():
    """Six free pages of sixteen: sequences are brought down one after the other, each into pages that the ones before left."""
    t = Check(2, 2, 16, 40, 16, 16, 100, 1)
    for _ in range(2):
        t.cache.add_sequence()
    t.step([80, 76])
    assert len(t.cache.free) == 6
    t.cache.evict(70, recent=8)
    t.pages_are_whole()
    assert t.cache.lengths == [70, 70]
    t.step([1, 1])
    t.cache.free.clear()  # no page left to move to
    with pytest.raises(RuntimeError, match="full"):
        t.cache.evict(60)


@pytest.mark.parametrize("bits", [4, 8])
def test_stack(bits):
    """A stack is its blocks with the norms between them, call by call; the first norm is of the stream itself."""
    say(f"stack of {bits} bits")
    g = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    N, H, D = 96, 3, 32

    def make():
        g.manual_seed(4)
        blocks = []
        for _ in range(3):
            c = decode.PagedCache(8, H, D, page=16)
            c.add_sequence()
            blocks.append(decode.AttentionBlock(rand(3 * H * D, N) * 0.1, rand(N, H * D) * 0.1, H, H, c, *decode.rotary_angles(64, D),
                                                group=32, bits=bits))
        return blocks, [1 + 0.1 * rand(N) for _ in blocks], [1 + 0.1 * rand(N) for _ in blocks]

    (blocks, pre, post), (again, _, _) = make(), make()
    stack = decode.Stack(blocks, pre, post, alpha=0.5)
    for n in (20, 1):
        r = rand(n, N)
        expect, stream = r.clone(), r.double()
        got = stack(r, [b.cache.grow([n]) for b in blocks])
        assert got is r
        for b, w, p in zip(again, pre, post):
            h = torch.empty(n, N, device="cuda", dtype=torch.bfloat16)
            zeros = torch.zeros_like(h)
            if bits == 8:
                h, s = torch.empty(n, 96, device="cuda", dtype=torch.int8), torch.empty(n, device="cuda")
                C.crvq_norm(zeros, h, residual=expect, w_pre=w, eps=1e-5, h_scales=s)
                out = b(h, b.cache.grow([n]), s)
            else:
                C.crvq_norm(zeros, h, residual=expect, w_pre=w, eps=1e-5)
                out = b(h, b.cache.grow([n]))
            c = out.double()
            stream = expect.double() + 0.5 * c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) * p.double()
            C.crvq_norm(out, None, residual=expect, residual_out=expect, w_post=p, alpha=0.5, eps=1e-5)
            assert torch.allclose(expect.double(), stream, rtol=0, atol=float(stream.abs().max()) * 2.0 ** -20)
        # in the stack a block's norm is of the unrounded stream in one call with the sum before it: the same fp32 numbers
        assert torch.equal(got, expect)


def test_program():
    say("decode program with a stack")
    common = ["--channels", "512", "--heads", "8", "--kv-heads", "4", "--seqs", "2", "--prompt", "70", "--steps", "12"]
    decode.main(common + ["--layers", "2", "--bits", "8", "--draft", "7", "--budget", "64"])
    decode.main(common + ["--layers", "2", "--draft", "5"])
    decode.main(common + ["--layers", "1", "--bits", "8", "--budget", "64"])
