"""Plain numpy reference of the quantized attention block: the paged 8-bit cache, attention over it and the
4-bit matrices with group scales.

Quantities that the definitions round (rotated elements, scales, codes) follow them operation by operation
in float32; products, sums and softmax are float64.  Arrays are laid out as the definitions say: key codes
[page][head][slot][d], value codes [page][head][d][slot], scales [page][head].
"""
from __future__ import annotations

import numpy as np

F = np.float32
MIN_SCALE = F(2.0 ** -100)


def bf16_round(x):
    """float32 values rounded to bfloat16 (nearest, ties to even), as float32; NaN and infinities stay."""
    x = np.ascontiguousarray(x, dtype=F)
    u = x.view(np.uint32).astype(np.uint64)
    r = (((u + 0x7FFF + ((u >> 16) & 1)) >> 16) << 16).astype(np.uint32).view(F)
    return np.where(np.isfinite(x), r, x)


def rotate(x, place, cos, sin, interleaved):
    """x: rows x heads x D float32; place: row of the angle table for every row of x."""
    if cos is None:
        return x.copy()
    r = cos.shape[1]
    out = x.copy()
    for i in range(x.shape[0]):
        known = 0 <= place[i] < cos.shape[0]
        c, s = (cos[place[i]], sin[place[i]]) if known else (np.full(r, np.nan, F), np.zeros(r, F))
        first = np.arange(r) * 2 if interleaved else np.arange(r)
        second = first + (1 if interleaved else r)
        a, b = x[i][:, first], x[i][:, second]
        out[i][:, first] = a * c - b * s
        out[i][:, second] = b * c + a * s
    return out


def append_page(codes, scale, old, x):
    """codes: slots x D int8 of one head of a page; old: slots held before; x: new rows.  New codes and scale."""
    m = np.abs(x).max() if np.isfinite(x).all() else np.nan
    s = max(F(m) / F(127), MIN_SCALE) if np.isfinite(m) else F(np.nan)
    out = codes.copy()
    if old:
        if np.isfinite(s) and not s > scale:
            s = scale
        if s > scale:
            out[:old] = np.rint(codes[:old].astype(F) * F(scale / s)).astype(np.int8)
    with np.errstate(invalid="ignore"):
        q = np.clip(np.rint(x / s), -127, 127) if np.isfinite(s) else np.zeros_like(x)
    out[old:old + len(x)] = q.astype(np.int8)
    return out, F(s)


def append(cache, table, start, kv_len, k, v, cos=None, sin=None, positions=None, interleaved=False, q=None):
    """Updates the copies in cache = [k codes, v codes, k scales, v scales] and returns (cache, rotated q)."""
    kc, vc, ks, vs = [a.copy() for a in cache]
    P, q_out = kc.shape[2], None if q is None else q.copy()
    for b in range(len(kv_len)):
        rows = np.arange(start[b], start[b + 1])
        n, length = len(rows), int(kv_len[b])
        if not n:
            continue
        t = np.arange(length - n, length)
        place = t if positions is None else positions[rows]
        if q is not None:
            q_out[rows] = rotate(q[rows], place, cos, sin, interleaved)
        xk, xv = rotate(k[rows], place, cos, sin, interleaved), v[rows]
        for p in range(t[0] // P, t[-1] // P + 1):
            page = int(table[b, p])
            if not 0 <= page < kc.shape[0]:
                continue
            here = t // P == p
            old = int(t[here][0] % P)
            for h in range(kc.shape[1]):
                kc[page, h], ks[page, h] = append_page(kc[page, h], ks[page, h], old, xk[here][:, h])
                vt, vs[page, h] = append_page(vc[page, h].T, vs[page, h], old, xv[here][:, h])
                vc[page, h] = vt.T
    return [kc, vc, ks, vs], q_out


def values(cache, table_row, length):
    """(K, V) float32 [length][heads][D] that the cache holds for a sequence's first tokens; NaN for a missing page."""
    kc, vc, ks, vs = cache
    n_pages, H, P, D = kc.shape
    K, V = np.full((length, H, D), np.nan, F), np.full((length, H, D), np.nan, F)
    for p in range((length + P - 1) // P):
        page, hi = int(table_row[p]), min(P, length - p * P)
        if 0 <= page < n_pages:
            K[p * P:p * P + hi] = (kc[page].astype(F) * ks[page][:, None, None]).transpose(1, 0, 2)[:hi]
            V[p * P:p * P + hi] = (vc[page].astype(F) * vs[page][:, None, None]).transpose(2, 0, 1)[:hi]
    return K, V


def attention(cache, table, start, kv_len, q, scale, causal=True, window=0):
    """(out, lse, size) in float64; size = sum_t p_t |V_t|, the magnitude that rounding errors of the weights scale with,
    and the largest score and the largest 1-norm of a key that each row sees, for bounds."""
    kc = cache[0]
    T, Hq, D = q.shape
    G = Hq // kc.shape[1]
    out, size = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    lse = np.full((T, Hq), -np.inf)
    top, norm = np.zeros((T, Hq)), np.zeros((T, Hq))
    ks, vs = [a.astype(np.float64) for a in cache[2:]]
    for b in range(len(kv_len)):
        n, length = int(start[b + 1] - start[b]), int(kv_len[b])
        if not n or not length:
            continue
        P = kc.shape[2]
        pages = np.array(table[b, :(length + P - 1) // P])
        K = (kc[pages] * ks[pages][:, :, None, None]).transpose(1, 0, 2, 3).reshape(kc.shape[1], -1, D)[:, :length]
        V = (cache[1][pages] * vs[pages][:, :, None, None]).transpose(1, 0, 3, 2).reshape(kc.shape[1], -1, D)[:, :length]
        for i in range(n):
            place = length - n + i
            hi = min(length, place + 1) if causal else length
            lo = max(0, place + 1 - window) if window else 0
            if hi <= lo:
                continue
            for h in range(Hq):
                Kh, Vh = K[h // G, lo:hi], V[h // G, lo:hi]
                s = Kh @ q[start[b] + i, h].astype(np.float64) * scale
                p = np.exp(s - s.max())
                row = (start[b] + i, h)
                lse[row] = np.log(p.sum()) + s.max()
                p /= p.sum()
                out[row], size[row] = p @ Vh, p @ np.abs(Vh)
                top[row], norm[row] = np.abs(s).max(), np.abs(Kh).sum(1).max()
    return out, lse, size, top, norm


def w4_quantize(W, group, zeros, bf16_scales):
    """(codes M x N uint8 0..15, scales M x G float32, zero points M x G uint8) of float32 W."""
    M, N = W.shape
    G = -(-N // group)
    codes, scales, zp = np.zeros((M, N), np.uint8), np.zeros((M, G), F), np.full((M, G), 8, np.uint8)
    for g in range(G):
        w = W[:, g * group:(g + 1) * group]
        lo, hi = np.minimum(w.min(1), 0).astype(F), np.maximum(w.max(1), 0).astype(F)
        s = np.maximum((hi - lo) / F(15) if zeros else np.maximum(hi, -lo) / F(7), MIN_SCALE)
        s = bf16_round(s) if bf16_scales else s.astype(F)
        z = np.clip(np.rint(-lo / s), 0, 15) if zeros else np.full(M, 8, F)
        codes[:, g * group:(g + 1) * group] = np.clip(np.rint(w / s[:, None]) + z[:, None], 0, 15)
        scales[:, g], zp[:, g] = s, z
    return codes, scales, zp


def w4_pack(codes, ld):
    """Two codes a byte, the lower column in the low half; rows padded with zeros to ld bytes."""
    M, N = codes.shape
    full = np.zeros((M, 2 * ld), np.uint8)
    full[:, :N] = codes
    return full[:, 0::2] | (full[:, 1::2] << 4)


def w4_values(codes, scales, zeros, group):
    """float64 values of codes."""
    N = codes.shape[1]
    each = lambda a: np.repeat(a.astype(np.float64), group, 1)[:, :N]  # noqa: E731
    return (codes.astype(np.float64) - each(zeros)) * each(scales)
