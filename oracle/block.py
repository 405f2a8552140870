"""Plain numpy definitions of what surrounds the attention block of a decoder on quantized data: 8-bit matrices with a scale
for each row and their product (rounded operation by operation in fp32 where the definition rounds, sums exact), and the
norms with gate and residual sum (fp64)."""
import numpy as np

from .serve import bf16_round

W8_FLOOR = np.float32(2.0 ** -100)


def w8_quantize(X):
    """Codes (int8, columns padded to a multiple of 16 with zeros) and scales of the rows of X (fp32)."""
    X = np.asarray(X, np.float32)
    rows, N = X.shape
    codes, scales = np.zeros((rows, -(-N // 16) * 16), np.int8), np.empty(rows, np.float32)
    for i, x in enumerate(X):
        if not np.isfinite(x).all():
            scales[i] = np.nan
            continue
        s = max(np.float32(np.abs(x).max() / np.float32(127)), W8_FLOOR)
        codes[i, :N] = np.clip(np.rint((x / s).astype(np.float32)), -127, 127)
        scales[i] = s
    return codes, scales


def w8_product(codes, scales, x_codes, x_scales, N, bf16):
    """y[t][r] of the first N columns: an exact sum as fp32, times the fp32 product of the scales."""
    acc = x_codes[:, :N].astype(np.int64) @ codes[:, :N].astype(np.int64).T
    with np.errstate(over="ignore", invalid="ignore"):
        y = acc.astype(np.float32) * (x_scales[:, None].astype(np.float32) * scales[None].astype(np.float32))
    return bf16_round(y) if bf16 else y


def _centred(x, layer):
    return x - x.mean(1, keepdims=True) if layer else x


def norm(x, r=None, gate=None, alpha=1.0, post=False, w_post=None, b_post=None, w_pre=None, b_pre=None, eps=1e-6, layer=False):
    """r' and h in 64 bits, and bounds of what fp32 arithmetic around fp64 sums may change of each.

    Every fp32 operation is off by at most 2^-24 of its result.  Up to r' there are at most seven on the way of x (its
    centre, the root's inverse, their product, w, b, gate, alpha), and the residual sum.  h inherits the error d of r':
    of its own element, of the mean (layer) and of the root, whose relative change is at most |d| / |c| in 2-norms, c
    the centred row; then at most five operations of its own (centre, inverse, product, w, b)."""
    u = 2.0 ** -24
    x = np.asarray(x, np.float64)
    one = lambda a, d: d if a is None else np.asarray(a, np.float64)  # noqa: E731
    if post:
        c = _centred(x, layer)
        y = c / np.sqrt((c * c).mean(1, keepdims=True) + eps) * one(w_post, 1.0)
        size, x = np.abs(y) + np.abs(one(b_post, 0.0)), y + one(b_post, 0.0)
    else:
        size = np.abs(x)
    g = alpha * one(gate, 1.0)
    out = one(r, 0.0) + g * x
    out_tol = 8 * u * np.abs(g) * size + u * np.abs(out)
    c = _centred(out, layer)
    d = out_tol + (out_tol.mean(1, keepdims=True) if layer else 0.0)
    inv = 1 / np.sqrt((c * c).mean(1, keepdims=True) + eps)
    length = np.sqrt((c * c).sum(1, keepdims=True))
    drift = np.sqrt((d * d).sum(1, keepdims=True)) / np.where(length > 0, length, 1.0)
    y = c * inv * one(w_pre, 1.0)
    h = y + one(b_pre, 0.0)
    h_tol = np.abs(one(w_pre, 1.0)) * inv * (d + np.abs(c) * drift) + 6 * u * (np.abs(y) + np.abs(h))
    return out, out_tol, h, h_tol
