"""The 8-bit row format and the sampling rule in 64 bits (numpy), for the tests of the operators that need no model."""
import math

import numpy as np


def quantize(x):
    """x [rows][K] float64 -> values [rows][Kp] (those the codes stand for), scale exponents [rows][blocks] of include/srm.h."""
    rows, K = x.shape
    kp = -(-K // 128) * 128
    blocks = np.zeros((rows, kp))
    blocks[:, :K] = x
    blocks = blocks.reshape(rows, -1, 128)
    finite = np.isfinite(blocks)
    top = np.where(finite, np.abs(blocks), 0.0).max(axis=-1)
    m, e = np.frexp(top)
    exp = np.where(top == 0, 0, np.maximum(e - 9 + (m > 0.875), -126))
    v = np.ldexp(np.where(finite, blocks, 0.0), -exp[..., None])
    _, e = np.frexp(v)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    q = np.where(finite, np.round(v / step) * step, np.nan)          # np.round: ties to even
    return q.reshape(rows, kp), exp


def scale_words(exp):
    """Scale exponents [rows][blocks] in the order of the scales' array: [ceil(blocks / 4)][rows][4] bytes."""
    rows, blocks = exp.shape
    out = np.full((rows, -(-blocks // 4) * 4), 127, dtype=np.uint8)
    out[:, :blocks] = exp + 127
    return out.reshape(rows, -1, 4).transpose(1, 0, 2).copy()


def scale_exponents(words, blocks):
    """The inverse: bytes [groups][rows][4] -> exponents [rows][blocks]."""
    rows = words.shape[1]
    return words.transpose(1, 0, 2).reshape(rows, -1)[:, :blocks].astype(np.int64) - 127


def dequantize(q, exp):
    rows, kp = q.shape
    return np.ldexp(q.reshape(rows, -1, 128), exp[..., None]).reshape(rows, kp)


def sample(row, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, u=0.0):
    """(token, log probability, distance of the draw and of the top-p cut to the next border) of one row of logits."""
    x = np.asarray(row, dtype=np.float64)
    x = np.where(np.isnan(x), -np.inf, x)
    most = x.max()
    if most == -np.inf:
        return -1, -math.inf, 1.0
    if not temperature > 0:
        return int(np.argmax(x)), 0.0, 1.0
    order = np.lexsort((np.arange(x.size), -x))
    with np.errstate(invalid="ignore", over="ignore"):
        arg = np.where(x == most, 0.0, (x - most) / np.float64(temperature))
        arg = np.where(x == -np.inf, -np.inf, arg)                    # (an infinite temperature)
        w = np.exp(arg)[order]
    n = int((w > 0).sum())
    if top_k > 0:
        n = min(n, top_k)
    if min_p > 0:
        n = min(n, int((w >= min(min_p, 1.0)).sum()))
    near = 1.0
    if top_p < 1:
        c = np.array([math.fsum(w[:n])]) if n == 1 else np.cumsum(w[:n])
        target = max(top_p, 0.0) * c[-1]
        n2 = 1 + int((c[:-1] < target).sum())
        if n > 1:
            d = np.abs(c[:-1] - target) / c[-1]
            near = min(near, float(d[d > 0].min()) if (d > 0).any() else 1.0)
        n = n2
    kept = np.sort(order[:n])
    wk = np.exp(arg[kept])
    c = np.cumsum(wk)
    t = (u if u > 0 else 0.0) * c[-1]
    at = min(int(np.searchsorted(c, t, side="right")), n - 1)
    d = np.abs(c - t) / c[-1]
    near = min(near, float(d[d > 0].min()) if (d > 0).any() else 1.0)
    return int(kept[at]), float(arg[kept[at]] - math.log(c[-1])), near
