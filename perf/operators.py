"""Performance cases of the quantized decoder-block operators: the attention block of a decoder whose cache is held
in 8 bits and whose projections are held in 4 bits.

A case is a dict of plain values; "op" names the operator:

  append    new keys and values rotated, quantized and written to the paged cache, queries rotated in the same call;
            returns the values that the pages written to now stand for (read back through the cache) and the queries
  attend    attention of new tokens over the paged 8-bit cache; returns the outputs and log-sum-exps
  w4        the product of one or a few activation vectors with a 4-bit matrix with group scales
  quant     a matrix brought to 4 bits and back; returns the scales and the values the codes stand for

listed() gives the fixed cases, draw(rng) others of the same ranges.  Head counts and widths are those of the layers
that this package quantizes (4096, 5120, 8192 channels in heads of 128), or generic small ones.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
DEV = "cuda"
FLOOR = 2.0 ** -100  # smallest scale of a block of the cache or a group of weights


def listed():
    return [
        # one decoding step of 32 conversations on a 4096-channel block of 32 heads
        {"name": "append_step_4096", "op": "append", "B": 32, "new": 1, "kv": 4096, "Hq": 32, "Hkv": 32, "D": 128,
         "page": 64, "rot": 128, "interleaved": False, "dtype": "bf16"},
        # the prompts of three requests on an 8192-channel block of 64 heads that share 8 key heads
        {"name": "append_prompt_8192", "op": "append", "B": 3, "new": 2048, "kv": 4000, "Hq": 64, "Hkv": 8, "D": 128,
         "page": 64, "rot": 128, "interleaved": False, "dtype": "bf16"},
        # one short conversation's next token, fp32: latency
        {"name": "attend_one", "op": "attend", "B": 1, "new": 1, "kv": 38, "Hq": 8, "Hkv": 8, "D": 64, "page": 16,
         "causal": True, "window": 0, "dtype": "f32"},
        # one decoding step of 32 conversations of up to 4096 tokens, every head with its own keys
        {"name": "attend_step_4096", "op": "attend", "B": 32, "new": 1, "kv": 4096, "Hq": 32, "Hkv": 32, "D": 128,
         "page": 64, "causal": True, "window": 0, "dtype": "bf16"},
        # the next token of one very long document, 64 heads over 8 key heads
        {"name": "attend_long_8192", "op": "attend", "B": 1, "new": 1, "kv": 131001, "Hq": 64, "Hkv": 8, "D": 128,
         "page": 128, "causal": True, "window": 0, "dtype": "bf16"},
        # prompts of two requests, the second half of each read after the first one is in the cache
        {"name": "attend_prompt_8192", "op": "attend", "B": 2, "new": 2048, "kv": 4000, "Hq": 64, "Hkv": 8, "D": 128,
         "page": 64, "causal": True, "window": 0, "dtype": "bf16"},
        # a mixed batch (prompts of odd lengths, single tokens, an empty request), sliding window, heads of 96, fp32
        {"name": "attend_mixed_window", "op": "attend", "B": 9, "new": 301, "kv": 1500, "Hq": 12, "Hkv": 4, "D": 96,
         "page": 32, "causal": True, "window": 500, "dtype": "f32"},
        # one token through an odd layer with groups of 32 and zero points, fp32 activations: latency
        {"name": "w4_ragged", "op": "w4", "M": 1031, "N": 3000, "T": 1, "group": 32, "zeros": True, "scales": "f32",
         "dtype": "f32"},
        # one token through the largest projection here (28672 x 8192): memory
        {"name": "w4_mlp_8192", "op": "w4", "M": 28672, "N": 8192, "T": 1, "group": 128, "zeros": False,
         "scales": "bf16", "dtype": "bf16"},
        # eleven conversations' next tokens through a 13824-channel down projection
        {"name": "w4_down_13824", "op": "w4", "M": 5120, "N": 13824, "T": 11, "group": 64, "zeros": True,
         "scales": "bf16", "dtype": "bf16"},
        # an odd layer brought to 4 bits around zero in groups of 32, from fp32
        {"name": "quant_ragged", "op": "quant", "M": 1031, "N": 3000, "group": 32, "zeros": False, "scales": "f32",
         "dtype": "f32"},
        # a projection brought to 4 bits in groups with zero points, and back
        {"name": "quant_5120", "op": "quant", "M": 5120, "N": 5120, "group": 128, "zeros": True, "scales": "bf16",
         "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the ranges the listed ones stand for: sizes spread over their logarithm, odd ones among them."""
    op = rng.choice(("append", "attend", "attend", "attend", "w4", "w4", "quant"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    if op in ("append", "attend"):
        Hkv = rng.choice((1, 2, 4, 5, 8, 8, 32))
        Hq = Hkv * rng.choice((1, 1, 2, 3, 4, 8))
        D = rng.choice((64, 80, 96, 128, 128, 128, 192, 256))
        page = rng.choice((16, 32, 64, 64, 128, 256))
        new = rng.choice((1, 1, 1, 4, _log(rng, 2, 2048)))
        B = _log(rng, 1, 48)
        kv = new + _log(rng, 1, 16384)
        # within the largest listed cases: the cache, the new tokens and (for attention) the pairs of tokens
        while B > 1 and (B * kv * Hkv * D > 1.2e8 or B * new * Hq * D > 3e7 or B * new * kv * Hq * D > 1e11):
            B = (B + 1) // 2
        kv = min(kv, max(new, int(1.2e8 / (B * Hkv * D))))
        while new > 1 and (B * new * Hq * D > 3e7 or B * new * kv * Hq * D > 1e11):
            new = (new + 1) // 2
        case = {"op": op, "B": B, "new": new, "kv": kv, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page, "dtype": dtype}
        if op == "append":
            case["rot"] = rng.choice((D, D, D // 2, 0))
            case["interleaved"] = rng.random() < 0.3
        else:
            case["causal"] = rng.random() < 0.85
            case["window"] = rng.choice((0, 0, _log(rng, 16, 4096))) if case["causal"] else 0
        return case
    M, N = _log(rng, 64, 16384), _log(rng, 64, 14336)
    case = {"op": op, "M": M, "N": N, "group": rng.choice((32, 64, 128, 128)), "zeros": rng.random() < 0.5,
            "scales": rng.choice(("f32", "bf16")), "dtype": dtype}
    if op == "w4":
        case["T"] = rng.choice((1, 1, 2, 4, _log(rng, 1, 64)))
    return case


# ------------------------------------------------------------------------------------------------
# lengths: a function of the case alone
# ------------------------------------------------------------------------------------------------

def _lengths(case):
    """New tokens and tokens in the cache (the new ones among them) of every sequence.  The first has the case's own;
    the others have fewer: half of the sequences bring one token where the case brings many, and one in nine none."""
    r = random.Random("%(op)s %(B)d %(new)d %(kv)d %(Hq)d %(D)d" % case)
    new, kv = [case["new"]], [case["kv"]]
    for b in range(1, case["B"]):
        n = 0 if b % 9 == 8 else case["new"] if case["new"] == 1 or r.random() < 0.2 else r.randint(1, case["new"])
        if case["new"] > 64 and b % 2 == 0 and b > 2:
            n = min(n, 1)
        new.append(n)
        kv.append(0 if n == 0 and b % 18 == 8 else r.randint(max(n, case["kv"] // 2), case["kv"]))
    return new, kv


def _starts(counts):
    at = [0]
    at.extend(sum(counts[:i + 1]) for i in range(len(counts)))
    return at


def _held(case):
    """Tokens of every sequence that lie in the pages its new tokens are written to."""
    new, kv = _lengths(case)
    return [k - (k - n) // case["page"] * case["page"] if n else 0 for n, k in zip(new, kv)]


def _seen(case, n, k):
    """(query, key) pairs of one sequence that the mask leaves, and the keys that any of its queries sees."""
    if not case["causal"]:
        return n * k, k if n else 0
    w = case["window"] or k
    return sum(min(p + 1, w) for p in range(k - n, k)), min(k, n - 1 + w) if n else 0


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------

def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(int(seed) + 1)
    dt = DTYPES[case["dtype"]]
    if case["op"] in ("append", "attend"):
        return _prepare_cache(case, g, dt)
    M, N, G = case["M"], case["N"], -(-case["N"] // case["group"])
    s = {"case": case, "group": case["group"]}
    sdt = DTYPES[case["scales"]]
    ld = -(-N // 32) * 16  # bytes of a row of codes: two to a byte, rows padded to 16 bytes
    if case["op"] == "quant":
        s["W"] = _randn(g, M, N).mul_(0.02).to(dt)
        s["codes"] = torch.zeros(M, ld, dtype=torch.uint8, device=DEV)
        s["scales"] = torch.empty(M, G, dtype=sdt, device=DEV)
        s["zeros"] = torch.empty(M, G, dtype=torch.uint8, device=DEV) if case["zeros"] else None
        s["out"] = torch.empty(M, N, dtype=torch.float32, device=DEV)
        return s
    s["codes"] = torch.randint(0, 256, (M, ld), generator=g, device=DEV, dtype=torch.uint8)
    s["scales"] = (torch.rand(M, G, generator=g, device=DEV) * 0.004 + 0.004).to(sdt)
    s["zeros"] = torch.randint(5, 11, (M, G), generator=g, device=DEV, dtype=torch.uint8) if case["zeros"] else None
    s["x"] = _randn(g, case["T"], N).to(dt)
    s["y"] = torch.empty(case["T"], M, dtype=dt, device=DEV)
    return s


def _prepare_cache(case, g, dt):
    """A cache with its sequences' tokens in pages of any order, and the new tokens' queries (keys, values)."""
    B, Hq, Hkv, D, P = case["B"], case["Hq"], case["Hkv"], case["D"], case["page"]
    new, kv = _lengths(case)
    per = max(1, -(-max(kv) // P))
    total = sum(new)
    table = torch.randperm(B * per, generator=g, device=DEV).to(torch.int32).view(B, per)
    s = {"case": case, "table": table, "start": _ints(_starts(new)), "kv_len": _ints(kv), "max_new": max(new),
         "max_kv": max(kv), "q": _randn(g, total, Hq, D).to(dt)}
    for name, shape in (("k", (B * per, Hkv, P, D)), ("v", (B * per, Hkv, D, P))):
        codes = torch.empty(shape, dtype=torch.int8, device=DEV)
        for part in codes.split(max(1, (1 << 26) // (Hkv * P * D))):
            part.copy_(_randn(g, *part.shape).mul_(32).round_().clamp_(-127, 127))
        s[name + "_cache"] = codes
        s[name + "_scale"] = torch.exp2(torch.rand(B * per, Hkv, generator=g, device=DEV) - 0.5) / 32
    if case["op"] == "attend":
        s["out"] = torch.empty(total, Hq, D, dtype=dt, device=DEV)
        s["lse"] = torch.empty(total, Hq, device=DEV)
        return s
    # new keys with a few strong channels, as projections give them
    s["k"] = (_randn(g, total, Hkv, D) * (1 + 3 * (torch.rand(D, generator=g, device=DEV) < 0.05))).to(dt)
    s["v"] = _randn(g, total, Hkv, D).to(dt)
    s["cos"] = s["sin"] = None
    if case["rot"]:
        a = torch.arange(max(kv), device=DEV, dtype=torch.float64)[:, None] * \
            10000.0 ** (-torch.arange(case["rot"] // 2, device=DEV, dtype=torch.float64) * 2 / case["rot"])
        s["cos"], s["sin"] = a.cos().float(), a.sin().float()
    held = _held(case)
    s["read_start"], s["max_read"] = _ints(_starts(held)), max(held)
    s["q_out"] = torch.empty_like(s["q"])
    s["k_out"] = torch.empty(sum(held), Hkv, D, dtype=dt, device=DEV)
    s["v_out"] = torch.empty_like(s["k_out"])
    return s


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------

def run(s):
    if own:
        return _OWN[s["case"]["op"]](s)
    return _PLAIN[s["case"]["op"]](s)


def _own_append(s):
    from paper_2412_09282_amd import crvq
    cache = (s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["table"])
    crvq.crvq_kv_append(s["k"], s["v"], *cache, s["start"], s["kv_len"], s["max_new"], cos=s["cos"], sin=s["sin"],
                        interleaved=s["case"]["interleaved"], q=s["q"], q_out=s["q_out"])
    crvq.crvq_kv_read(s["k_out"], s["v_out"], *cache, s["read_start"], s["kv_len"], s["max_read"])
    return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}


def _own_attend(s):
    from paper_2412_09282_amd import crvq
    crvq.crvq_kv_attention(s["q"], s["out"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["table"],
                           s["start"], s["kv_len"], s["max_new"], s["max_kv"], causal=s["case"]["causal"],
                           window=s["case"]["window"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_w4(s):
    from paper_2412_09282_amd import crvq
    crvq.crvq_w4_gemv(s["codes"], s["scales"], s["group"], s["x"], s["y"], zeros=s["zeros"])
    return {"y": s["y"]}


def _own_quant(s):
    from paper_2412_09282_amd import crvq
    crvq.crvq_w4_quantize(s["W"], s["codes"], s["scales"], s["group"], zeros=s["zeros"])
    crvq.crvq_w4_dequant(s["codes"], s["scales"], s["group"], s["out"], zeros=s["zeros"])
    return {"W": s["out"], "scales": s["scales"]}


_OWN = {"append": _own_append, "attend": _own_attend, "w4": _own_w4, "quant": _own_quant}


# ---- the plain forms: elementary operations in 32 bits, rounded once at the end ------------------

def _rotate(x, cos, sin, interleaved):
    """Pairs (i, i + r) of the first 2 r elements, or (2 i, 2 i + 1), turned by the row's angles."""
    r = cos.shape[-1]
    a, b = (x[..., 0:2 * r:2], x[..., 1:2 * r:2]) if interleaved else (x[..., :r], x[..., r:2 * r])
    u, w = a * cos - b * sin, b * cos + a * sin
    u = torch.stack((u, w), -1).flatten(-2) if interleaved else torch.cat((u, w), -1)
    return torch.cat((u, x[..., 2 * r:]), -1)


def _over(x, n):
    """x / n rounded once: by a tensor, since a number would be replaced by its rounded reciprocal."""
    return x / torch.full((), float(n), device=DEV)


def _plain_append(s):
    case, P = s["case"], s["case"]["page"]
    Hkv, dt = case["Hkv"], s["q"].dtype
    total, count = s["q"].shape[0], s["k_out"].shape[0]
    start, read, kv = s["start"].long(), s["read_start"].long(), s["kv_len"].long()
    rows = torch.arange(total, device=DEV)
    seq = torch.searchsorted(start[1:], rows, right=True)
    pos = kv[seq] - start[seq + 1] + rows                        # place of every new token in its sequence
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    if s["cos"] is not None:
        cos, sin = s["cos"][pos][:, None], s["sin"][pos][:, None]
        q, k = _rotate(q, cos, sin, case["interleaved"]), _rotate(k, cos, sin, case["interleaved"])
    # every token of the pages written to: the old ones' codes, then the new ones' values in their places
    rows = torch.arange(count, device=DEV)
    rseq = torch.searchsorted(read[1:], rows, right=True)
    rpos = kv[rseq] - read[rseq + 1] + rows
    page = s["table"].long()[rseq, rpos // P]
    slot = rpos % P
    new_at = read[seq + 1] - start[seq + 1] + torch.arange(total, device=DEV)
    is_old = torch.ones(count, dtype=torch.bool, device=DEV)
    is_old[new_at] = False
    n_pages = s["k_cache"].shape[0]
    has_old = torch.zeros(n_pages, dtype=torch.bool, device=DEV)
    has_old[page[is_old]] = True

    def stored(x, codes, scale):
        most = torch.zeros(n_pages, Hkv, device=DEV)
        most.scatter_reduce_(0, page[new_at][:, None].expand(-1, Hkv), x.abs().amax(-1), "amax")
        fresh = _over(most, 127).clamp(min=FLOOR)
        new = torch.where(has_old[:, None], torch.maximum(scale, fresh), fresh)
        grown = codes.float() * (scale / new)[page][..., None]
        grown = torch.where((new > scale)[page][..., None], grown.round(), codes.float())
        grown[new_at] = (x / new[page[new_at]][..., None]).round().clamp(-127, 127)
        return (grown * new[page][..., None]).to(dt)

    return {"q": q.to(dt), "k": stored(k, s["k_cache"][page, :, slot], s["k_scale"]),
            "v": stored(v, s["v_cache"][page, :, :, slot], s["v_scale"])}


def _plain_attend(s):
    case, P = s["case"], s["case"]["page"]
    B, Hq, Hkv, D, n = case["B"], case["Hq"], case["Hkv"], case["D"], s["max_new"]
    G, total, per = Hq // Hkv, s["q"].shape[0], s["table"].shape[1]
    start, kv, table = s["start"].long(), s["kv_len"].long(), s["table"].long()
    counts = start[1:] - start[:-1]
    # keys [B, Hkv, D, tokens], values [B, Hkv, tokens, D]
    k = s["k_cache"][table].float() * s["k_scale"][table][..., None, None]
    k = k.permute(0, 2, 4, 1, 3).reshape(B, Hkv, D, per * P)
    rows = (start[:-1, None] + torch.arange(n, device=DEV)).clamp(max=total - 1)
    q = s["q"].float()[rows].view(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D)
    w = torch.matmul(q, k).mul_(D ** -0.5).view(B, Hkv, n, G, per * P)
    del k, q
    t = torch.arange(per * P, device=DEV)
    pos = (kv - counts)[:, None] + torch.arange(n, device=DEV)
    seen = (t < kv[:, None]).view(B, 1, -1).expand(B, n, per * P)
    if case["causal"]:
        seen = seen & (t <= pos[..., None])
        if case["window"]:
            seen = seen & (t > pos[..., None] - case["window"])
    w.masked_fill_(~seen[:, None, :, None], -math.inf)
    most = w.amax(-1, keepdim=True)
    some = most > -math.inf
    most = torch.where(some, most, 0.0)
    w.sub_(most).exp_()
    norm = w.sum(-1, keepdim=True)
    v = s["v_cache"][table].float() * s["v_scale"][table][..., None, None]
    v = v.permute(0, 2, 1, 4, 3).reshape(B, Hkv, per * P, D)
    o = torch.matmul(w.view(B, Hkv, n * G, per * P), v).view(B, Hkv, n, G, D)
    o = o / torch.where(some, norm, 1.0)
    lse = torch.where(some, norm.log() + most, -math.inf)[..., 0]
    at = torch.arange(total, device=DEV)
    seq = torch.searchsorted(start[1:], at, right=True)
    at = at - start[seq]
    return {"out": o[seq, :, at].reshape(total, Hq, D).to(s["q"].dtype), "lse": lse[seq, :, at].reshape(total, Hq)}


def _values(codes, scales, zeros, group, N):
    """The matrix that codes, scales and zero points stand for, in the scales' widened type."""
    M = codes.shape[0]
    c = torch.stack((codes & 15, codes >> 4), -1).view(M, -1)[:, :N]
    z = 8.0 if zeros is None else zeros.float().repeat_interleave(group, 1)[:, :N]
    return (c.float() - z) * scales.float().repeat_interleave(group, 1)[:, :N]


def _plain_w4(s):
    x = s["x"].float()
    W = _values(s["codes"], s["scales"], s["zeros"], s["group"], x.shape[1])
    return {"y": torch.matmul(x, W.t()).to(s["x"].dtype)}


def _plain_quant(s):
    W, group = s["W"].float(), s["group"]
    M, N = W.shape
    G = s["scales"].shape[1]
    w = torch.zeros(M, G * group, device=DEV)
    w[:, :N] = W
    w = w.view(M, G, group)
    if s["zeros"] is not None:
        lo, hi = w.amin(-1, keepdim=True).clamp(max=0), w.amax(-1, keepdim=True).clamp(min=0)
        scale = _over(hi - lo, 15)
    else:
        scale = _over(w.abs().amax(-1, keepdim=True), 7)
    scale = scale.clamp(min=FLOOR).to(s["scales"].dtype)
    step = scale.float()
    z = (-lo / step).round().clamp(0, 15) if s["zeros"] is not None else 8.0
    c = ((w / step).round() + z).clamp(0, 15)
    return {"W": ((c - z) * step).view(M, -1)[:, :N].contiguous(), "scales": scale.view(M, G)}


_PLAIN = {"append": _plain_append, "attend": _plain_attend, "w4": _plain_w4, "quant": _plain_quant}


# ------------------------------------------------------------------------------------------------
# what one pass cannot do without
# ------------------------------------------------------------------------------------------------

def work(case):
    if case["op"] in ("append", "attend"):
        es, new, kv = SIZE[case["dtype"]], *_lengths(case)
        Hq, Hkv, D, total = case["Hq"], case["Hkv"], case["D"], sum(new)
        if case["op"] == "attend":
            seen = [_seen(case, n, k) for n, k in zip(new, kv)]
            keys = sum(k for _, k in seen)
            return {"bytes": keys * Hkv * (2 * D + 8 / case["page"]) + total * Hq * (2 * D * es + 4),
                    "flops": 4 * D * Hq * sum(p for p, _ in seen)}
        # the new tokens in, their codes out, the queries in and out; the pages' codes in and their values out
        held = sum(_held(case))
        return {"bytes": total * Hkv * D * (2 * es + 2) + total * Hq * D * 2 * es + held * Hkv * D * (2 + 2 * es)
                + total * case["rot"] * 4, "flops": total * (Hq + 2 * Hkv) * D * 4 + held * Hkv * D * 2}
    M, N = case["M"], case["N"]
    G = -(-N // case["group"])
    held = M * ((N + 1) // 2) + M * G * (SIZE[case["scales"]] + case["zeros"])
    if case["op"] == "w4":
        return {"bytes": held + (M + N) * case["T"] * SIZE[case["dtype"]], "flops": 2 * M * N * case["T"]}
    # the weights in, codes and scales out; codes and scales in, values out
    return {"bytes": M * N * (SIZE[case["dtype"]] + 4) + 2 * held, "flops": 8 * M * N}


# ------------------------------------------------------------------------------------------------
# the same outputs in 64 bits, sequence by sequence and head by head
# ------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "w4": _exact_w4, "quant": _exact_quant}[case["op"]](case, s)


def _exact_turn(x, place, s, interleaved):
    """x (tokens, heads, D) in 64 bits with every pair turned as a complex number."""
    if s["cos"] is None:
        return x
    r = s["cos"].shape[1]
    turn = torch.complex(s["cos"][place].double(), s["sin"][place].double())[:, None]
    x = x.clone()
    first = torch.arange(r, device=DEV) * (2 if interleaved else 1)
    second = first + (1 if interleaved else r)
    y = torch.complex(x[..., first], x[..., second]) * turn
    x[..., first], x[..., second] = y.real, y.imag
    return x


def _exact_append(case, s):
    new, kv = _lengths(case)
    P = case["page"]
    q, k, v = [], [], []
    at = 0
    for b, (n, length) in enumerate(zip(new, kv)):
        if not n:
            continue
        place = torch.arange(length - n, length, device=DEV)
        q.append(_exact_turn(s["q"][at:at + n].double(), place, s, case["interleaved"]))
        xk = _exact_turn(s["k"][at:at + n].double(), place, s, case["interleaved"])
        xv = s["v"][at:at + n].double()
        at += n
        first = (length - n) // P
        for p in range(first, (length - 1) // P + 1):
            id = int(s["table"][b, p])
            lo, hi = max(length - n, p * P), min(length, (p + 1) * P)
            old = lo - p * P
            for x, codes, scales, out in ((xk, s["k_cache"][id], s["k_scale"][id], k),
                                          (xv, s["v_cache"][id].transpose(1, 2), s["v_scale"][id], v)):
                part = x[lo - (length - n):hi - (length - n)].transpose(0, 1)          # heads, tokens, D
                scale = part.abs().amax((1, 2)).div(127).clamp(min=FLOOR)
                before = codes[:, :old].double()
                if old:
                    was = scales.double()
                    scale = torch.maximum(was, scale)
                    before = torch.round(before * (was / scale)[:, None, None])
                after = torch.round(part / scale[:, None, None]).clamp(-127, 127)
                out.append((torch.cat((before, after), 1) * scale[:, None, None]).transpose(0, 1))
    return {"q": torch.cat(q), "k": torch.cat(k), "v": torch.cat(v)}


def _exact_attend(case, s):
    new, kv = _lengths(case)
    D, G = case["D"], case["Hq"] // case["Hkv"]
    out = torch.zeros(sum(new), case["Hq"], D, dtype=torch.float64, device=DEV)
    lse = torch.full((sum(new), case["Hq"]), -math.inf, dtype=torch.float64, device=DEV)
    at = 0
    for b, (n, length) in enumerate(zip(new, kv)):
        if n and length:
            pages = s["table"][b, :-(-length // case["page"])].long()
            i = torch.arange(length - n, length, device=DEV)[:, None]
            t = torch.arange(length, device=DEV)
            hidden = torch.zeros(n, length, dtype=torch.bool, device=DEV)
            if case["causal"]:
                hidden = t > i
                if case["window"]:
                    hidden = hidden | (t <= i - case["window"])
            for h in range(case["Hkv"]):
                k = (s["k_cache"][pages, h].double() * s["k_scale"][pages, h].double()[:, None, None]).reshape(-1, D)[:length]
                v = s["v_cache"][pages, h].double() * s["v_scale"][pages, h].double()[:, None, None]
                v = v.transpose(1, 2).reshape(-1, D)[:length]
                for j in range(h * G, h * G + G):
                    score = (s["q"][at:at + n, j].double() @ k.t()) / math.sqrt(D)
                    score = score.masked_fill(hidden, -math.inf)
                    lse[at:at + n, j] = torch.logsumexp(score, -1)
                    full = lse[at:at + n, j, None]
                    out[at:at + n, j] = torch.where(full > -math.inf, torch.exp(score - full), 0.0) @ v
        at += n
    return {"out": out, "lse": lse}


def _exact_w4(case, s):
    M, N, group = case["M"], case["N"], case["group"]
    y = torch.zeros(case["T"], M, dtype=torch.float64, device=DEV)
    for g in range(0, N, group):
        byte = s["codes"][:, g // 2:(min(N, g + group) + 1) // 2].double()
        high = torch.floor(byte / 16)
        z = 8.0 if s["zeros"] is None else s["zeros"][:, g // group, None].double()
        w = torch.empty(M, 2 * byte.shape[1], dtype=torch.float64, device=DEV)
        w[:, 0::2], w[:, 1::2] = byte - 16 * high - z, high - z
        w = w[:, :min(group, N - g)] * s["scales"][:, g // group, None].double()
        y += s["x"][:, g:g + group].double() @ w.t()
    return {"y": y}


def _exact_quant(case, s):
    N, group = case["N"], case["group"]
    values, scales = [], []
    for g in range(0, N, group):
        w = s["W"][:, g:g + group].double()
        if case["zeros"]:
            lo, hi = w.amin(1, keepdim=True).clamp(max=0), w.amax(1, keepdim=True).clamp(min=0)
            scale = ((hi - lo) / 15).clamp(min=FLOOR).to(s["scales"].dtype).double()
            zero = torch.round(-lo / scale).clamp(0, 15)
        else:
            scale = (w.abs().amax(1, keepdim=True) / 7).clamp(min=FLOOR).to(s["scales"].dtype).double()
            zero = torch.full_like(scale, 8)
        values.append((torch.clamp(torch.round(w / scale) + zero, 0, 15) - zero) * scale)
        scales.append(scale)
    return {"W": torch.cat(values, 1), "scales": torch.cat(scales, 1)}
