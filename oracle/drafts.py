"""Plain numpy definitions of drafted tokens over the paged 8-bit cache and of the cache within a budget.  What rows see is
given as one boolean array (new tokens x tokens) for each sequence."""
import numpy as np


def tree(parents, length, words, window=0):
    """(mask rows uint64, places) of one sequence's drafted tokens."""
    n = len(parents)
    mask, places = np.zeros((n, words), np.uint64), np.full(n, -1, np.int64)
    for i in range(n):
        chain, j = [], i
        while j >= 0:
            chain.append(j)
            p = int(parents[j])
            if not -1 <= p < j:
                chain = None
                break
            j = p
        if chain is None:
            continue
        places[i] = max(length - n + len(chain) - 1, -1)
        for j in chain[:window or None]:
            mask[i, j // 64] |= np.uint64(1 << (j % 64))
    return mask, places.astype(np.int32)


def sees_causal(n, length, causal=True, window=0):
    place, t = np.arange(length - n, length)[:, None], np.arange(length)[None]
    s = np.ones((n, length), bool)
    if causal:
        s = t <= place
        if window:
            s &= t > place - window
    return s


def sees_mask(mask, n, length, places=None, window=0):
    """What the rows of a mask (uint64 words) see."""
    context = length - n
    place = np.asarray(places)[:, None] if places is not None else np.arange(context, length)[:, None]
    t = np.arange(length)
    s = np.ones((n, length), bool)
    if window:
        s &= t[None] > place - window
    for j in range(n):
        if context + j >= 0:
            s[:, context + j] = (mask[:, j // 64] >> np.uint64(j % 64)) & np.uint64(1) != 0
    return s


def attention(cache, table, start, kv_len, q, scale, sees):
    """(out, lse, size, top, norm) as serve.attention returns them."""
    T, Hq, D = q.shape
    G = Hq // cache[0].shape[1]
    out, size = np.zeros((T, Hq, D)), np.zeros((T, Hq, D))
    lse, top, norm = np.full((T, Hq), -np.inf), np.zeros((T, Hq)), np.zeros((T, Hq))
    for b, length in enumerate(int(k) for k in kv_len):
        r0, r1 = int(start[b]), int(start[b + 1])
        if r1 == r0 or not length:
            continue
        K, V = _values64(cache, table[b], length)
        for h in range(Hq):
            s = q[r0:r1, h].astype(np.float64) @ K[h // G].T * scale
            s[~sees[b]] = -np.inf
            m = s.max(1)
            some = np.isfinite(m)
            p = np.exp(s - np.where(some, m, 0.0)[:, None])
            l = p.sum(1)
            p /= np.where(some, l, 1.0)[:, None]
            lse[r0:r1, h] = np.where(some, np.log(np.where(some, l, 1.0)) + np.where(some, m, 0.0), -np.inf)
            out[r0:r1, h], size[r0:r1, h] = p @ V[h // G], p @ np.abs(V[h // G])
            top[r0:r1, h] = np.abs(np.where(sees[b], np.where(np.isfinite(s), s, 0.0), 0.0)).max(1)
            norm[r0:r1, h] = np.where(sees[b], np.abs(K[h // G]).sum(1)[None], 0.0).max(1)
    return out, lse, size, top, norm


def _values64(cache, row, length):
    """Keys and values of a sequence in 64 bits, Hkv x length x D."""
    P, Hkv, D = cache[0].shape[2], cache[0].shape[1], cache[0].shape[3]
    pages = np.array(row[:-(-length // P)])
    ks, vs = (a[pages].astype(np.float64)[:, :, None, None] for a in cache[2:])
    K = (cache[0][pages] * ks).transpose(1, 0, 2, 3).reshape(Hkv, -1, D)[:, :length]
    V = (cache[1][pages] * vs).transpose(1, 0, 3, 2).reshape(Hkv, -1, D)[:, :length]
    return K, V


def weights(cache, table, start, kv_len, q, scale, lse, sees, before, after, decay):
    """What crvq_kv_weights leaves in `after`, and a bound of what fp32 arithmetic may change of it.

    A score's products are exact and its at most 3 D of them added in fp32: off by 3 D 2^-24 of the sum of their
    magnitudes; its product with the key's scale, the log-sum-exp's and the difference are off by at most
    8 2^-24 (|s| + |lse| + 1), exp2 by 2^-22; a weight moves relatively by as much.  Sums add at most 32 + 16 + their
    number / 512 roundings in a row, decay one more."""
    u = 2.0 ** -24
    out, tol = after.astype(np.float64), np.zeros(after.shape)
    G, D = q.shape[1] // cache[0].shape[1], q.shape[2]
    for b, length in enumerate(int(k) for k in kv_len):
        r0, r1 = int(start[b]), int(start[b + 1])
        if r1 == r0:
            continue
        K, _ = _values64(cache, table[b], length)
        for h in range(K.shape[0]):
            total, wrong = np.zeros(length), np.zeros(length)
            for j in range(h * G, h * G + G):
                x, l = q[r0:r1, j].astype(np.float64), lse[r0:r1, j].astype(np.float64)
                fine = np.isfinite(l)
                x, l = np.where(fine[:, None], x, 0.0), np.where(fine, l, 0.0)[:, None]
                s = x @ K[h].T * scale
                w = np.where(sees[b] & fine[:, None], np.exp(s - l), 0.0)
                move = 3 * D * u * abs(scale) * (np.abs(x) @ np.abs(K[h]).T) + 8 * u * (np.abs(s) + np.abs(l) + 1) + 2.0 ** -22
                total += w.sum(0)
                wrong += (w * move).sum(0)
            wrong += total * u * (64 + (r1 - r0) * G / 512)
            if before is not None:
                old = decay * before[b, h, :length].astype(np.float64)
                old[max(length - (r1 - r0), 0):] = 0
                total = total + old
                wrong += u * np.abs(total)
            out[b, h, :length], tol[b, h, :length] = total, wrong
    return out, tol


def select(w, length, budget, sinks, recent):
    """The kept tokens of one head, in order."""
    n = min(length, budget)
    always = [t for t in range(length) if t < sinks or t >= length - recent]
    rest = sorted((t for t in range(length) if sinks <= t < length - recent),
                  key=lambda t: (np.isnan(w[t]), -w[t] if not np.isnan(w[t]) else 0.0, t))
    return sorted(always[:n] + rest[:n - len(always[:n])])


def gather(cache, table, kv_len, keep, kept_len, to):
    """The cache after the move (a copy)."""
    k, v, ks, vs = (a.copy() for a in cache)
    n_pages, Hkv, P, D = k.shape
    for b in range(len(kv_len)):
        count = int(kept_len[b])
        if count > keep.shape[2] or count > to.shape[1] * P:
            continue
        for p in range(-(-count // P) if count > 0 else 0):
            dest = int(to[b, p])
            if not 0 <= dest < n_pages:
                continue
            for h in range(Hkv):
                ts = [int(t) for t in keep[b, h if keep.shape[1] > 1 else 0, p * P:min(count, (p + 1) * P)]]
                pages = [int(table[b, t // P]) if 0 <= t < kv_len[b] else -1 for t in ts]
                for codes, scales, new_codes, new_scales in ((cache[0][:, h], cache[2], k[:, h], ks),
                                                             (cache[1][:, h].transpose(0, 2, 1), cache[3], v[:, h].transpose(0, 2, 1), vs)):
                    old = np.array([scales[g, h] if 0 <= g < n_pages else np.nan for g in pages], np.float32)
                    new_codes[dest] = 0
                    if not (np.isfinite(old) & (old >= 0)).all():
                        new_scales[dest, h] = np.nan
                        continue
                    new = old.max()
                    new_scales[dest, h] = new
                    for j, (t, g) in enumerate(zip(ts, pages)):
                        f = np.float32(1) if old[j] == new else np.float32(old[j] / new)
                        new_codes[dest, j] = np.rint(codes[g, t % P].astype(np.float32) * f)
    return k, v, ks, vs
