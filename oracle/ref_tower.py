"""fp64 NumPy oracle of the text tower's operators: packed attention with a bias per bucket of the relative
position, and layer norm, each with its analytic gradient. Shares no code with the HIP path.

Packed attention: sequence s has the query rows cu_q[s] .. and key rows cu_k[s] .. (len_q[s], len_k[s] of them,
or the whole slot). Query i stands at position p = i + n_k - n_q of the keys; pair (i, j) is valid for j < n_k and,
causal, j <= p. Its bias is bias[h][buckets[R + clamp(j - p, -R, R)]]; an entry below -65536 shuts the pair out
(probability 0), one above counts as 65536, a bucket outside the table adds 0.
"""
from __future__ import annotations

import numpy as np

BIAS_LIMIT = 65536.0


def _rows(cu, length, s):
    n = int(cu[s + 1]) - int(cu[s])
    return int(cu[s]), n, n if length is None else min(max(int(length[s]), 0), n)


def pair_terms(nq, nk, causal, bias=None, buckets=None):
    """(valid [nq, nk], additive bias [H, nq, nk] or None, bucket [nq, nk] with -1 for none or None)."""
    d = np.arange(nk)[None, :] - (np.arange(nq)[:, None] + nk - nq)
    valid = d <= 0 if causal else np.ones_like(d, dtype=bool)
    if bias is None:
        return valid, None, None
    R = (len(buckets) - 1) // 2
    u = np.asarray(buckets)[np.clip(d, -R, R) + R].astype(np.int64)
    none = (u < 0) | (u >= bias.shape[1])
    table = np.where(bias < -BIAS_LIMIT, -np.inf, np.where(bias > BIAS_LIMIT, BIAS_LIMIT, bias))
    add = np.where(none[None], 0.0, table[:, np.where(none, 0, u)])
    return valid, add, np.where(none, -1, u)


def packed_attention(q, k, v, cu_q, cu_k, len_q=None, len_k=None, causal=False, scale=None, bias=None, buckets=None,
                     dout=None, each=None):
    """Dict with o, lse and, given dout, dq, dk, dv (dbias with a bias). Rows that take no part: 0, lse -inf.
    q [Tq, H, D], k, v [Tk, Hkv, D], all float64. each(rows, keys, h, g, p, ds): called for every (sequence, head) with
    its row and key slices, its key head and the pairs' probabilities and score gradients."""
    Tq, H, D = q.shape
    Hkv = k.shape[1]
    c = 1.0 / np.sqrt(D) if scale is None else scale
    r = {"o": np.zeros_like(q), "lse": np.full((H, Tq), -np.inf)}
    if dout is not None:
        r.update(dq=np.zeros_like(q), dk=np.zeros_like(k), dv=np.zeros_like(v))
        if bias is not None:
            r["dbias"] = np.zeros(bias.shape)
    r["weight"] = None if bias is None else np.zeros((Tq, H, bias.shape[1]))  # probability of each bucket, per row
    for s in range(len(cu_q) - 1):
        q0, _, nq = _rows(cu_q, len_q, s)
        k0, _, nk = _rows(cu_k, len_k, s)
        if nq == 0 or nk == 0:
            continue
        valid, add, bucket = pair_terms(nq, nk, causal, bias, buckets)
        for h in range(H):
            g = h // (H // Hkv)
            Q, K, V = q[q0:q0 + nq, h], k[k0:k0 + nk, g], v[k0:k0 + nk, g]
            x = c * (Q @ K.T)
            if add is not None:
                x = x + add[h]
            x = np.where(valid, x, -np.inf)
            m = x.max(1, keepdims=True)
            m = np.where(np.isneginf(m), 0.0, m)
            e = np.exp(x - m)
            z = e.sum(1, keepdims=True)
            p = e / np.where(z > 0, z, 1.0)
            with np.errstate(divide="ignore"):
                r["lse"][h, q0:q0 + nq] = (np.log(z) + m)[:, 0]
            r["o"][q0:q0 + nq, h] = p @ V
            if bucket is not None:
                for u in range(bias.shape[1]):
                    r["weight"][q0:q0 + nq, h, u] = np.where(bucket == u, p, 0.0).sum(1)
            if dout is None:
                continue
            dO = dout[q0:q0 + nq, h]
            dp = dO @ V.T
            ds = p * (dp - (p * dp).sum(1, keepdims=True))
            r["dq"][q0:q0 + nq, h] = c * (ds @ K)
            r["dk"][k0:k0 + nk, g] += c * (ds.T @ Q)
            r["dv"][k0:k0 + nk, g] += p.T @ dO
            if bucket is not None:
                for u in range(bias.shape[1]):
                    r["dbias"][h, u] += ds[bucket == u].sum()
            if each is not None:
                each(slice(q0, q0 + nq), slice(k0, k0 + nk), h, g, p, ds)
    return r


def layer_norm(x, w=None, b=None, eps=1e-5, dout=None):
    """Dict with y, mean, rstd and, given dout, dx, dw, db. x [rows, columns], float64."""
    mean = x.mean(1)
    xc = x - mean[:, None]
    rstd = 1.0 / np.sqrt((xc * xc).mean(1) + eps)
    xh = xc * rstd[:, None]
    W = np.ones(x.shape[1]) if w is None else w
    r = {"y": xh * W + (0.0 if b is None else b), "mean": mean, "rstd": rstd}
    if dout is not None:
        g = dout * W
        r["dx"] = rstd[:, None] * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
        r["dw"], r["db"] = (dout * xh).sum(0), dout.sum(0)
    return r
