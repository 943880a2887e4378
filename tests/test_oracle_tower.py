"""Pins of the oracle of packed attention and layer norm, each independent of its formulas: torch in float64 with
autograd on dense masks, central differences, hand-made cases, planted mistakes (CPU)."""
import numpy as np
import pytest
import torch

from oracle import ref_tower as T


def _case(seed, lq, lk, H, Hkv, D, nb=0, R=0):
    g = np.random.default_rng(seed)
    cu_q, cu_k = np.cumsum([0] + lq), np.cumsum([0] + lk)
    q, k, v = (g.standard_normal((n, h, D)) for n, h in ((cu_q[-1], H), (cu_k[-1], Hkv), (cu_k[-1], Hkv)))
    x = dict(q=q, k=k, v=v, cu_q=cu_q, cu_k=cu_k, dout=g.standard_normal(q.shape))
    if nb:
        x.update(bias=g.standard_normal((H, nb)), buckets=g.integers(0, nb, 2 * R + 1))
    return x


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("nb", [0, 5])
def test_against_torch(causal, nb):
    lq, lk = [3, 7, 1, 4, 5], [3, 9, 6, 2, 5]  # fewer and more queries than keys
    x = _case(1, lq, lk, 4, 2, 8, nb, 3)
    r = T.packed_attention(causal=causal, **x)
    t = {n: torch.from_numpy(x[n]).requires_grad_(True) for n in ("q", "k", "v", "bias") if n in x}
    outs, total = [], 0.0
    for s in range(len(lq)):
        q, k, v = (t[n][x[c][s]:x[c][s + 1]].transpose(0, 1) for n, c in (("q", "cu_q"), ("k", "cu_k"), ("v", "cu_k")))
        k, v = k.repeat_interleave(2, 0), v.repeat_interleave(2, 0)
        mask = torch.zeros((4, lq[s], lk[s]), dtype=torch.float64)
        rel = torch.arange(lk[s])[None, :] - torch.arange(lk[s] - lq[s], lk[s])[:, None]
        if nb:
            mask = mask + t["bias"][:, torch.from_numpy(x["buckets"])[rel.clamp(-3, 3) + 3]]
        if causal:
            mask = mask.masked_fill(rel > 0, -torch.inf)
        some = ~torch.isinf(mask).all(-1)
        o = torch.nn.functional.scaled_dot_product_attention(q, k, v, attn_mask=torch.where(some[..., None], mask, torch.zeros_like(mask)))
        o = torch.where(some[..., None], o, torch.zeros_like(o)).transpose(0, 1)
        lse = torch.logsumexp(q @ k.transpose(1, 2) / 8 ** 0.5 + mask, -1)
        np.testing.assert_allclose(r["lse"][:, x["cu_q"][s]:x["cu_q"][s + 1]], lse.detach().numpy(), atol=1e-12)
        outs.append(o)
        total = total + (o * torch.from_numpy(x["dout"][x["cu_q"][s]:x["cu_q"][s + 1]])).sum()
    np.testing.assert_allclose(r["o"], torch.cat(outs).detach().numpy(), atol=1e-12)
    total.backward()
    for n in t:
        np.testing.assert_allclose(r["d" + n], t[n].grad.numpy(), atol=1e-11)


def test_against_differences():
    x = _case(2, [4, 3], [6, 3], 2, 1, 4, 4, 2)
    r = T.packed_attention(causal=True, **x)
    loss = lambda y: (T.packed_attention(causal=True, **y)["o"] * x["dout"]).sum()  # noqa: E731
    for n in ("q", "k", "v", "bias"):
        for at in np.ndindex(*x[n].shape):
            up, dn = ({**x, n: x[n].copy()} for _ in range(2))
            up[n][at] += 1e-5
            dn[n][at] -= 1e-5
            assert abs((loss(up) - loss(dn)) / 2e-5 - r["d" + n][at]) < 1e-8, (n, at)


def test_lengths_and_shut_out_pairs():
    x = _case(3, [5, 4], [5, 4], 1, 1, 4, 3, 2)
    ref = T.packed_attention(**x)
    # a slot's rows behind its length: the same as sequences of those lengths
    short = T.packed_attention(len_q=[3, 4], len_k=[2, 4], **x)
    y = dict(x, q=np.concatenate([x["q"][:3], x["q"][5:]]), k=np.concatenate([x["k"][:2], x["k"][5:]]),
             v=np.concatenate([x["v"][:2], x["v"][5:]]), dout=np.concatenate([x["dout"][:3], x["dout"][5:]]),
             cu_q=[0, 3, 7], cu_k=[0, 2, 6])
    cut = T.packed_attention(**y)
    np.testing.assert_array_equal(short["o"][[0, 1, 2, 5, 6, 7, 8]], cut["o"])
    assert (short["o"][3:5] == 0).all() and np.isneginf(short["lse"][:, 3:5]).all() and (short["dk"][2:5] == 0).all()
    np.testing.assert_array_equal(short["dbias"], cut["dbias"])
    # a shut-out bucket: probability 0, rows of it alone empty; a bucket outside the table adds nothing
    for low in (-np.inf, np.finfo(np.float32).min, -70000.0):
        shut = dict(x, bias=np.full((1, 3), low))
        r = T.packed_attention(**shut)
        assert (r["o"] == 0).all() and np.isneginf(r["lse"]).all() and (r["dbias"] == 0).all() and (r["dv"] == 0).all()
    r = T.packed_attention(**dict(x, buckets=np.array([-1, 3, 99, 3, 5])))
    plain = T.packed_attention(**{n: t for n, t in x.items() if n not in ("bias", "buckets")})
    np.testing.assert_array_equal(r["o"], plain["o"])
    assert (r["dbias"] == 0).all() and not np.allclose(ref["o"], plain["o"])


def test_planted_mistakes_fail():
    x = _case(4, [6], [6], 2, 1, 4, 4, 2)
    r = T.packed_attention(causal=True, **x)
    for wrong in (dict(x, buckets=x["buckets"][::-1].copy()), dict(x, k=x["k"][::-1].copy()), dict(x, bias=-x["bias"])):
        assert not np.allclose(T.packed_attention(causal=True, **wrong)["o"], r["o"], atol=1e-3)
    assert not np.allclose(T.packed_attention(causal=False, **x)["o"], r["o"], atol=1e-3)


def test_layer_norm_against_torch_and_differences():
    g = np.random.default_rng(5)
    x, w, b, dy = g.standard_normal((4, 7)) * 3 + 5, g.standard_normal(7), g.standard_normal(7), g.standard_normal((4, 7))
    r = T.layer_norm(x, w, b, 1e-3, dy)
    t = [torch.from_numpy(a).requires_grad_(True) for a in (x, w, b)]
    y = torch.nn.functional.layer_norm(t[0], (7,), t[1], t[2], 1e-3)
    y.backward(torch.from_numpy(dy))
    np.testing.assert_allclose(r["y"], y.detach().numpy(), atol=1e-12)
    for n, a in zip(("dx", "dw", "db"), t):
        np.testing.assert_allclose(r[n], a.grad.numpy(), atol=1e-12)
    loss = lambda z: (T.layer_norm(z, w, b, 1e-3)["y"] * dy).sum()  # noqa: E731
    for at in np.ndindex(4, 7):
        up, dn = x.copy(), x.copy()
        up[at] += 1e-5
        dn[at] -= 1e-5
        assert abs((loss(up) - loss(dn)) / 2e-5 - r["dx"][at]) < 1e-8
