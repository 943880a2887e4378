"""Pins of the oracle of the operators around a block's attention: closed forms, differences, identities."""
import numpy as np
import pytest

from oracle import ref_blocks as B

RNG = np.random.default_rng


def run(p, norm, post, c, plus_one, eps=1e-3):
    h = B.stream(p["x"], p["a"], p["gate"], p["wp"] if post else None, c, post, eps)
    return h, (B.modulated(h, p["scale"], p["shift"], norm, eps, plus_one) if norm else np.zeros_like(h))


@pytest.mark.parametrize("norm,post,c,plus_one", [("layer", None, 1.0, True), ("rms", None, 0.5, False), ("layer", "layer", 0.7, True),
                                                  ("rms", "rms", 1.0, True), ("layer", "rms", 1.0, False), (None, "layer", 1.0, True)])
def test_gradients_against_differences(norm, post, c, plus_one):
    g = RNG(3)
    n, k, eps = 5, 11, 1e-3
    p = {"x": g.standard_normal((n, k)), "a": g.standard_normal((n, k)) + 0.3}
    p |= {name: g.standard_normal(k) for name in ("gate", "scale", "shift", "wp")}
    dh, dy = g.standard_normal((n, k)), (g.standard_normal((n, k)) if norm else None)

    def loss():
        h, y = run(p, norm, post, c, plus_one, eps)
        return (dh * h).sum() + (0 if dy is None else (dy * y).sum())

    h = run(p, norm, post, c, plus_one, eps)[0]
    xh, _, r = B.normed(h, norm, eps) if norm else (h, None, None)
    xa, _, ra = B.normed(p["a"], post, eps) if post else (p["a"], None, None)
    got = B.residual_grads(dh, dy, xh, r, xa, ra, p["gate"], p["scale"] if norm else None, p["wp"] if post else None, c, norm, post, plus_one)
    want = {"x": got["dx"], "a": got["da"], "gate": got["A"] * (p["wp"] if post else 1)}
    if norm:
        want |= {"scale": got["dscale"], "shift": got["dshift"]}
    if post:
        want["wp"] = got["A"] * p["gate"]
    for name, grad in want.items():
        for at in np.ndindex(*p[name].shape):
            old, e = p[name][at], 1e-5
            p[name][at] = old + e
            up = loss()
            p[name][at] = old - e
            down = loss()
            p[name][at] = old
            assert abs((up - down) / (2 * e) - grad[at]) < 1e-6 * (1 + abs(grad[at])), (name, at)


def test_norms_closed_forms():
    t = np.array([[3.0, -1.0], [2.0, 2.0]])
    n, mean, r = B.normed(t, "layer", 1e-30)
    assert np.allclose(n[0], [1, -1]) and mean.tolist() == [1, 2] and np.isclose(r[0], 0.5) and (n[1] == 0).all()
    n, mean, r = B.normed(np.array([[3.0, 4.0]]), "rms", 0.0)
    assert np.allclose(n, [[3 / np.sqrt(12.5), 4 / np.sqrt(12.5)]]) and (mean == 0).all()
    # shifting and scaling a row changes no layer norm; scaling none of RMS
    t = RNG(1).standard_normal((4, 9))
    assert np.allclose(B.normed(5 * t + 3, "layer", 0)[0], B.normed(t, "layer", 0)[0])
    assert np.allclose(B.normed(5 * t, "rms", 0)[0], B.normed(t, "rms", 0)[0])


def test_kept8():
    x = np.zeros((5, 300), np.float32)
    x[0, :128] = np.arange(128)              # 127 steps of 1
    x[1, 128:256] = 2.0 ** -120              # under the least block size
    x[2, 299] = np.inf
    x[3, 5], x[3, 6] = np.nan, 7
    x[4, :3] = [254.0, 1.0, 3.0]             # steps of 2: 0.5 and 1.5 to even
    v, s, q = B.kept8(x)
    assert (v[0] == x[0]).all() and s[0, 0] == 1
    assert (v[1] == 0).all() and s[1, 1] == np.float32(2.0 ** -100) / np.float32(127)
    assert np.isnan(v[2, 256:]).all() and (v[2, :256] == 0).all()
    assert np.isnan(v[3, :128]).all() and (v[3, 128:] == 0).all()
    assert q[4, :3].tolist() == [127, 0, 2]
    g = RNG(2).standard_normal((50, 300)).astype(np.float32)
    v, s, q = B.kept8(g)
    step = np.repeat(s, 128, 1)[:, :300]
    assert np.abs(q).max() == 127 and (np.abs(v - g) <= step * (0.5 + 1e-4)).all()


def test_embedding_and_gradient():
    g = RNG(4)
    table, ids = g.standard_normal((7, 3)), np.array([2, 2, 0, 6, -1, 7, 5, 2])
    out = B.embedding(ids, table, 0.5, 0)
    assert (out[[2, 4, 5]] == 0).all() and np.allclose(out[0], 0.5 * table[2])
    dout = g.standard_normal((8, 3))
    grad, mag, n = B.embedding_grad(ids, dout, 7, 0.5, 0)
    assert n.tolist() == [0, 0, 3, 0, 0, 1, 1]
    # <dout, d out> = <gradient, d table>
    d = g.standard_normal((7, 3))
    assert np.isclose((dout * B.embedding(ids, d, 0.5, 0)).sum(), (grad * d).sum()) and (mag >= np.abs(grad) - 1e-12).all()


def test_top_scale_is_the_largest_of_a_finite_127_fold():
    f = np.float32
    with np.errstate(over="ignore"):
        assert np.isfinite(f(127) * B.TOP_SCALE) and np.isinf(f(127) * np.nextafter(B.TOP_SCALE, f(np.inf)))
    vals, _, _ = B.kept8(np.array([[np.finfo(f).max, 1.0, -np.finfo(f).max]], f))
    assert np.isfinite(vals).all()
