"""fp64 CPU oracle of the operators around a block's attention, from their definitions (NumPy, one sample after the other).

residual: the gated residual with the norms before and after a block, forward and backward.
kept8: the values and scales of the 8-bit form. embedding, embedding_grad: lookup and its gradient.
"""
from __future__ import annotations

import numpy as np

TOP_SCALE = np.float32(float.fromhex("0x1.020406p+121"))  # the largest whose 127 fold is finite in fp32


def normed(t, kind, eps):
    """(normed t, mean, reciprocal deviation) over the last axis."""
    mean = t.mean(-1) if kind == "layer" else np.zeros(t.shape[:-1])
    d = t - mean[..., None]
    r = 1.0 / np.sqrt((d * d).mean(-1) + eps)
    return d * r[..., None], mean, r


def through(g, n, r, kind):
    """The gradient of a norm's input from that of its result, with the normed n and the reciprocal deviation r."""
    d = g - n * (g * n).mean(-1, keepdims=True)
    if kind == "layer":
        d = d - g.mean(-1, keepdims=True)
    return d * r[..., None]


def stream(x, a, gate, post_weight, c, post, eps):
    """h of one sample before its rounding: c x + gate P(a)."""
    if a is None:
        return c * x
    p = normed(a, post, eps)[0] if post else a
    if post_weight is not None:
        p = p * post_weight
    return c * x + (p if gate is None else gate * p)


def modulated(h, scale, shift, norm, eps, plus_one):
    y = normed(h, norm, eps)[0]
    if scale is not None:
        y = y * (scale + 1.0 if plus_one else scale)
    return y if shift is None else y + shift


def residual_grads(dh, dy, xh, r, xa, ra, gate, scale, post_weight, c, norm, post, plus_one):
    """dx, da and the sample's sums (A, dscale, dshift) from the normed h and a (a itself without a norm), which may be
    those of values kept in 8 bits, and the deviations."""
    H = np.zeros(xh.shape) if dh is None else dh.copy()
    if dy is not None:
        e = 1.0 if scale is None else scale + 1.0 if plus_one else scale
        H = H + through(dy * e, xh, r, norm)
    out = {"H": H, "dx": c * H, "dscale": np.zeros(H.shape[-1]), "dshift": np.zeros(H.shape[-1])}
    if dy is not None:
        out["dscale"], out["dshift"] = (dy * xh).sum(0), dy.sum(0)
    if xa is not None:
        K = H * (1.0 if gate is None else gate) * (1.0 if post_weight is None else post_weight)
        out["K"], out["da"], out["A"] = K, through(K, xa, ra, post) if post else K, (H * xa).sum(0)
    return out


def kept8(x):
    """(values, scales, whole numbers) of x [rows, columns] (float32 values) in 8 bits, in float32 arithmetic as defined."""
    f = np.float32
    x = np.asarray(x, f)
    rows, cols = x.shape
    blocks = -(-cols // 128)
    vals, scales, q = np.empty((rows, cols), f), np.empty((rows, blocks), f), np.zeros((rows, cols), np.int64)
    with np.errstate(invalid="ignore", over="ignore"):
        for b in range(blocks):
            part = x[:, 128 * b:128 * b + 128]
            good = np.isfinite(part).all(1)
            m = np.where(good, np.maximum(np.abs(np.where(np.isfinite(part), part, 0)).max(1), f(2.0 ** -100)), f(1)).astype(f)
            scale = np.where(good, np.minimum(m / f(127), TOP_SCALE), f(np.nan)).astype(f)
            w = np.where(good[:, None], np.rint(part * (f(127) / m)[:, None]), f(0)).astype(f)
            q[:, 128 * b:128 * b + 128] = w.astype(np.int64)
            scales[:, b] = scale
            vals[:, 128 * b:128 * b + 128] = w * scale[:, None]
    return vals, scales, q


def embedding(ids, table, scale, padding):
    out = np.zeros((len(ids), table.shape[1]))
    for t, i in enumerate(ids):
        if 0 <= i < table.shape[0] and i != padding:
            out[t] = scale * table[i]
    return out


def embedding_grad(ids, dout, vocab, scale, padding):
    """(gradient, sum of magnitudes, tokens of each id)"""
    g, mag, n = np.zeros((vocab, dout.shape[1])), np.zeros((vocab, dout.shape[1])), np.zeros(vocab, np.int64)
    for t, i in enumerate(ids):
        if 0 <= i < vocab and i != padding:
            g[i] += dout[t]
            mag[i] += np.abs(dout[t])
            n[i] += 1
    return g * scale, mag * abs(scale), n
