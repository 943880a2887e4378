"""Gated residual with the norms before and after a block on the GPU against the fp64 oracle, on every element.

Bounds, with u = 2^-24 (half a step of fp32 relative to the value): a row's sum is a chain of at most 40 additions (8 columns of a
thread, 4 steps and 2 levels within a wave, up to 16 waves), off by at most 40 u times the sum of the magnitudes; a column's
sum over rows is a chain of at most rows + 80 (a run's rows, the runs of a sample in up to 16 shares, these, the
samples likewise). Every result is rounded by at most half a step of its type. The stages are checked one by one: h against
the oracle's; y from the h that was returned, as its rounding is the definition's; the gradients from that h, or
from the values that the 8 bits hold, which themselves are compared bit by bit."""
import numpy as np
import pytest

from oracle import ref_blocks as B
from parity_util import log

pytestmark = pytest.mark.gpu

U, N = 2.0 ** -24, 40


def _vc():
    import paper_2501_08453_amd as vc
    return vc


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def half(t):
    return 2.0 ** -8 if t.element_size() == 2 else U


def make(rows, cols, samples=1, x="bf16", a="bf16", p="f32", post=None, norm="layer", shared=False, slices=False, with_a=True, gate=True,
         scale=True, shift=True, seed=1, mean=0.3, plus_one=True):
    """Inputs on the GPU; slices: the vectors of a sample lie in one longer row."""
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}
    new = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    t = {"x": (new(rows, cols) * 1.5 + mean).to(dt[x]), "a": (new(rows, cols) + mean).to(dt[a]) if with_a else None,
         "dh": new(rows, cols).to(dt[x]), "dy": new(rows, cols).to(dt[a]) if norm else None}
    if shared:
        vec = [(0.5 * new(cols) + o).to(dt[p]).cuda() for o in (0.3, 0.0 if plus_one else 1.0, 0.1)]
    elif slices:
        mod = (0.5 * new(samples, 5 * cols + 3) + 0.2).to(dt[p]).cuda()
        vec = [mod[:, k * cols + 1:(k + 1) * cols + 1] for k in range(3)]
    else:
        vec = [(0.5 * new(samples, cols) + 0.2).to(dt[p]).cuda() for _ in range(3)]
    t = {k: None if v is None else v.cuda() for k, v in t.items()}
    t["gate"] = vec[0] if gate and with_a else None
    t["scale"], t["shift"] = (vec[1] if scale and norm else None), (vec[2] if shift and norm else None)
    t["post_weight"] = (1 + 0.3 * new(cols)).to(dt[p]).cuda() if post == "weighted" else None
    return t


def _stats_err(t, kind, r):
    """Bounds of the errors of a norm's mean, and of 1 / deviation relative to it."""
    mag = np.abs(t).mean(1)
    e_mean = N * U * mag if kind == "layer" else 0 * mag
    d = np.abs(t - (t.mean(1, keepdims=True) if kind == "layer" else 0))
    # the sum of squares of differences to a mean that is off by e_mean, each difference rounded
    rel = (N + 6) * U + (e_mean * r) ** 2 + 4 * U * (np.abs(t) * d).mean(1) * r * r * (kind == "layer") + 2 * U * (mag * r) ** 2 * (kind == "layer")
    return e_mean, rel


def _normed_err(t, n, mean, r, e_mean, rel):
    """... of the normed value of t by these."""
    return e_mean[:, None] * r[:, None] + np.abs(n) * (rel[:, None] + 4 * U) + 2 * U * (np.abs(t) + np.abs(mean)[:, None]) * r[:, None]


def _near(name, got, want, tol, worst):
    got = _np(got) if not isinstance(got, np.ndarray) else got
    assert got.shape == want.shape, (name, got.shape, want.shape)
    assert np.isfinite(got).all(), name
    off = float((np.abs(got - want) / (tol + 1e-30)).max()) if got.size else 0.0
    worst[name] = max(worst.get(name, 0.0), off)
    assert off <= 1, (name, off)


def check(t, norm="layer", post=None, c=1.0, plus_one=True, eps=1e-5, slots=None, cu=None, lens=None, samples=1, checkpoint=False, y_dtype=None,
          without=(), api="call"):
    """slots: [(first row, rows that take part)] per sample."""
    import torch
    vc = _vc()
    x, a, dh, dy = t["x"], t["a"], t["dh"], t["dy"]
    rows, cols = x.shape
    S = samples
    slots = slots or [(s * (rows // S), rows // S) for s in range(S)]
    vec = {k: t[k] for k in ("gate", "scale", "shift", "post_weight")}
    desc = vc.make_residual_desc(rows, cols, S, norm=norm, post_norm=post, residual_scale=c, eps=eps, plus_one=plus_one, checkpoint=checkpoint)
    h, y, saved = vc.residual_norm_fwd(x, a, desc, **vec, cu=cu, lens=lens, y_dtype=y_dtype)
    grads = vc.residual_norm_bwd(None if "dh" in without else dh, None if "dy" in without else dy, saved)
    again = vc.residual_norm_bwd(None if "dh" in without else dh, None if "dy" in without else dy, saved)
    for p, q in zip(grads, again):
        assert (p is None) == (q is None) and (p is None or torch.equal(p, q))
    if a is None:
        assert h is x
    X, A, DH, DY = _np(x), _np(a), (None if "dh" in without else _np(dh)), (None if "dy" in without else _np(dy))
    V = {k: _np(v) for k, v in vec.items()}
    of = lambda k, s: None if V[k] is None else V[k] if V[k].ndim == 1 else V[k][s]  # noqa: E731
    Hn, Yn = _np(h), _np(y)
    if a is not None:
        live = np.zeros(rows, bool)
        for b, n in slots:
            live[b:b + n] = True
        for o in (h, y) + tuple(grads[:2]):
            assert o is None or (_np(o)[~live] == 0).all()
    if checkpoint:
        hk, ak = (None if k is None else vc.checkpoint_unpack(k, dtype=torch.float32).cpu().numpy() for k in (saved.h, saved.a))
    worst = {}
    hx, hy = half(x), (half(y) if y is not None else half(a))
    names = ("gate", "scale", "shift")
    sums = {k: np.zeros((S, cols)) for k in names}
    errs = {k: np.zeros((S, cols)) for k in names}
    dw, ew, dwm = (np.zeros(cols) for _ in range(3))
    mags = {k: np.zeros((S, cols)) for k in names}
    for s, (b, n) in enumerate(slots):
        if n == 0:
            continue
        r_ = slice(b, b + n)
        g, e_, f, w = of("gate", s), of("scale", s), of("shift", s), V["post_weight"]
        g1, w1 = (1.0 if g is None else g), (1.0 if w is None else w)
        e1 = 1.0 if e_ is None else e_ + 1 if plus_one else e_
        xs, as_ = X[r_], None if A is None else A[r_]
        xa = ra = e_xa = None
        if as_ is not None:
            xa, e_xa = as_, 0 * as_
            if post:
                xa, ma, ra = B.normed(as_, post, eps)
                ea, rela = _stats_err(as_, post, ra)
                e_xa = _normed_err(as_, xa, ma, ra, ea, rela)
            want = B.stream(xs, as_, g, w, c, post, eps)
            parts = np.abs(c * xs) + np.abs(g1 * w1 * xa)
            _near("h", Hn[r_], want, np.abs(g1 * w1) * e_xa + 4 * U * parts + hx * (np.abs(want) + 8 * U * parts), worst)
        hs = Hn[r_]
        if norm:
            nh, mh, rh = B.normed(hs, norm, eps)
            eh, relh = _stats_err(hs, norm, rh)
            if norm == "layer":
                _near("mean", saved.stats[0, r_], mh, eh, worst)
            _near("rstd", saved.stats[1, r_], rh, relh * rh, worst)
            e_nh = _normed_err(hs, nh, mh, rh, eh, relh)
            want = B.modulated(hs, e_, f, norm, eps, plus_one)
            tol = e_nh * np.abs(e1) + 4 * U * (np.abs(nh * e1) + np.abs(0 if f is None else f))
            _near("y", Yn[r_], want, tol + hy * (np.abs(want) + tol), worst)
        # backward, from what it was given
        nb, e_nb, xb, e_xb = (nh, e_nh, xa, e_xa) if norm else (hs, 0 * hs, xa, e_xa)
        if checkpoint:
            if norm:
                v, sc, q = B.kept8(hs)
                assert np.array_equal(v, hk[r_])
                nb = (v.astype(np.float64) - mh[:, None]) * rh[:, None]
                e_nb = _normed_err(v, nb, mh, rh, eh, relh)
            if as_ is not None:
                v, sc, q = B.kept8(as_)
                assert np.array_equal(v, ak[r_])
                v = v.astype(np.float64)
                xb, e_xb = v, 0 * v
                if post:
                    xb = (v - ma[:, None]) * ra[:, None]
                    e_xb = _normed_err(v, xb, ma, ra, ea, rela)
        dhs, dys = None if DH is None else DH[r_], None if DY is None else DY[r_]
        want = B.residual_grads(dhs, dys, nb, rh if norm else None, xb, ra, g, e_, w, c, norm, post, plus_one)
        e_H = 0 * nb
        if dys is not None:
            G = np.abs(dys * e1)
            m1 = G.mean(1, keepdims=True) * (norm == "layer")
            m2 = (G * (np.abs(nb) + e_nb)).mean(1, keepdims=True)
            e2 = (G * e_nb).mean(1, keepdims=True) + (N + 4) * U * m2
            mag = G + m1 + np.abs(nb) * m2
            e_H = rh[:, None] * ((N + 8) * U * mag + e_nb * m2 + np.abs(nb) * e2 + relh[:, None] * mag)
            errs["scale"][s] += (np.abs(dys) * e_nb).sum(0)
            mags["scale"][s] += np.abs(dys * nb).sum(0)
            mags["shift"][s] += np.abs(dys).sum(0)
        e_H = e_H + 2 * U * ((0 if dhs is None else np.abs(dhs)) + np.abs(want["H"]))
        if grads[0] is not None:
            tol = abs(c) * e_H + 2 * U * np.abs(want["dx"])
            _near("dx", _np(grads[0])[r_], want["dx"], tol + hx * (np.abs(want["dx"]) + tol), worst)
        if as_ is not None:
            e_K = np.abs(g1 * w1) * e_H + 4 * U * np.abs(want["K"])
            e_a = e_K
            if post:
                K = np.abs(want["K"])
                m1 = K.mean(1, keepdims=True) * (post == "layer")
                m2 = (K * np.abs(xb)).mean(1, keepdims=True)
                e1_ = (e_K.mean(1, keepdims=True) + (N + 4) * U * m1) * (post == "layer")
                e2 = (e_K * (np.abs(xb) + e_xb) + K * e_xb).mean(1, keepdims=True) + (N + 4) * U * m2
                mag = K + m1 + np.abs(xb) * m2
                e_a = ra[:, None] * (e_K + e1_ + np.abs(xb) * e2 + e_xb * (m2 + e2) + (rela[:, None] + 8 * U) * mag)
            _near("da", _np(grads[1])[r_], want["da"], e_a + hy * (np.abs(want["da"]) + e_a), worst)
            sums["gate"][s] = want["A"]
            errs["gate"][s] += (e_H * (np.abs(xb) + e_xb) + np.abs(want["H"]) * e_xb).sum(0)
            mags["gate"][s] += np.abs(want["H"] * xb).sum(0)
        sums["scale"][s], sums["shift"][s] = want["dscale"], want["dshift"]
    w = V["post_weight"]
    chain = (rows + 80) * U
    for k, got in zip(names, grads[2:5]):
        if got is None:
            assert V[k] is None
            continue
        v, e, m = sums[k], errs[k], mags[k]
        if V[k].ndim == 1:
            v, e, m = v.sum(0), e.sum(0), m.sum(0)
        if k == "gate" and w is not None:
            v, e, m = v * w, e * np.abs(w), m * np.abs(w)
        tol = e + chain * m
        _near("d" + k, got, v, tol + half(vec[k]) * (np.abs(v) + tol), worst)
    if w is not None:
        for s in range(S):
            g = of("gate", s)
            g = 1.0 if g is None else g
            dw, ew, dwm = dw + g * sums["gate"][s], ew + np.abs(g) * errs["gate"][s], dwm + np.abs(g) * mags["gate"][s]
        tol = ew + chain * dwm
        _near("dpost_weight", grads[5], dw, tol + half(vec["post_weight"]) * (np.abs(dw) + tol), worst)
    log("   off / bound:", ", ".join("%s %.2f" % kv for kv in worst.items()))
    return h, y, grads


SHAPES = [(1, 1), (3, 2), (1, 64), (7, 63), (33, 65), (5, 255), (64, 256), (129, 264), (31, 1000), (257, 1024), (16, 1155),
          (9, 2048), (40, 2056), (5, 4096), (6, 5001), (3, 8192)]
TYPES = [("bf16", "bf16", "bf16"), ("f32", "bf16", "f32"), ("f32", "f32", "f32"), ("bf16", "bf16", "f32")]


@pytest.mark.parametrize("x,a,p", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_shapes(rows, cols, x, a, p):
    check(make(rows, cols, x=x, a=a, p=p))


@pytest.mark.parametrize("norm", ["layer", "rms", None])
@pytest.mark.parametrize("post", [None, "layer", "rms"])
@pytest.mark.parametrize("ckpt", [False, True])
def test_norms(norm, post, ckpt):
    for seed, (rows, cols) in enumerate([(37, 200), (10, 1155), (5, 2304)]):
        t = make(rows, cols, norm=norm, post="weighted" if post and seed else None, seed=seed, p="bf16" if seed == 2 else "f32",
                 x="f32" if seed == 1 else "bf16")
        check(t, norm=norm, post=post, c=0.75, plus_one=bool(seed), checkpoint=ckpt)


@pytest.mark.parametrize("shared,slices", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("post", [None, "rms"])
def test_samples(shared, slices, post):
    """Equal slots, lengths in them, sequences one behind the other; empty ones; rows of no sample."""
    import torch
    dev = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    kw = dict(shared=shared, slices=slices, post="weighted" if post else None)
    check(make(60, 96, samples=5, **kw), post=post, samples=5)
    lens = [12, 0, 7, 1, 11]
    check(make(60, 96, samples=5, **kw), post=post, samples=5, lens=dev(lens), slots=[(12 * s, n) for s, n in enumerate(lens)])
    over = [99, -4, 7, 12, 2 ** 31 - 1]  # taken as the nearest within the slot
    check(make(60, 96, samples=5, **kw), post=post, samples=5, lens=dev(over),
          slots=[(12 * s, min(max(n, 0), 12)) for s, n in enumerate(over)])
    n = [0, 3, 0, 0, 41, 1, 7, 0]
    at = np.cumsum([0] + n)
    check(make(60, 520, samples=8, **kw), post=post, samples=8, cu=dev(at.tolist()), slots=list(zip(at, n)))
    at = at + 3  # rows before the first and behind the last
    check(make(60, 520, samples=8, **kw), post=post, samples=8, cu=dev(at.tolist()), slots=list(zip(at, n)))
    cut = [0, 2, 0, 0, 40, 1, 0, 0]
    check(make(60, 520, samples=8, **kw), post=post, samples=8, cu=dev(at.tolist()), lens=dev(cut), slots=list(zip(at, cut)))


@pytest.mark.parametrize("ckpt", [False, True])
def test_many_rows_and_samples(ckpt):
    """Runs of several rows, samples that begin and end within them, more samples than runs."""
    import torch
    rng = np.random.default_rng(5)
    rows, S = 20011, 700
    ends = np.sort(rng.integers(0, rows + 1, S - 1))
    at = np.concatenate([[0], ends, [rows]])
    cu = torch.tensor(at, dtype=torch.int32).cuda()
    check(make(rows, 72, samples=S, x="f32", a="bf16", post="weighted"), post="layer", samples=S, cu=cu, slots=list(zip(at[:-1], np.diff(at))), checkpoint=ckpt)
    check(make(20010, 40, samples=2001, shared=True), samples=2001, checkpoint=ckpt)
    check(make(20010, 136), checkpoint=ckpt)


def test_parts_left_out():
    for post in (None, "layer"):
        check(make(30, 200, gate=False, post=post and "weighted"), post=post)
        check(make(30, 200, scale=False, shift=False), post=post)
        check(make(30, 200, shift=False, plus_one=False, shared=True), post=post, plus_one=False)
        check(make(30, 200), post=post, without=("dh",))
        check(make(30, 200), post=post, without=("dy",))
    for ckpt in (False, True):
        check(make(30, 200, with_a=False), checkpoint=ckpt)
        check(make(30, 200, with_a=False, x="f32", a="f32"), checkpoint=ckpt, norm="rms")


def test_norm_alone_in_other_types():
    import torch
    vc = _vc()
    t = make(30, 200, with_a=False, x="f32", a="f32")
    h, y, _ = check({**t, "dy": t["dy"].to(torch.bfloat16)}, y_dtype=torch.bfloat16)
    assert y.dtype is torch.bfloat16 and h is t["x"]
    desc = vc.make_residual_desc(30, 200)
    full = vc.residual_norm_fwd(t["x"], None, desc, scale=t["scale"], shift=t["shift"])
    plain = vc.layer_norm_fwd(t["x"], 1 + t["scale"][0].float(), t["shift"][0].float())[0]
    assert torch.allclose(plain, full[1], rtol=1e-5, atol=1e-5)


def test_far_mean_no_variance_and_scales():
    t = make(50, 300, x="f32", a="f32", mean=300.0)
    check(t, post="layer")
    t = make(8, 128)
    t["x"][1], t["a"][1] = 2.0, 0.0  # no variance in either
    t["x"][2], t["a"][2] = 0.0, 0.0
    check(t, post="rms")
    check(t, post="layer", c=0.0)
    check(t, eps=0.5)


def test_masked_rows_may_hold_anything():
    import torch
    vc = _vc()
    t = make(40, 136, samples=4)
    lens = torch.tensor([3, 10, 0, 9], dtype=torch.int32).cuda()
    dead = torch.ones(40, dtype=torch.bool, device="cuda")
    for s, n in enumerate(lens.tolist()):
        dead[10 * s:10 * s + n] = False
    for ckpt in (False, True):
        desc = vc.make_residual_desc(40, 136, 4, post_norm="rms", checkpoint=ckpt)
        vec = {k: t[k] for k in ("gate", "scale", "shift")}
        outs = []
        for fill in (0.0, float("nan"), float("inf")):
            v = {k: t[k].clone() for k in ("x", "a", "dh", "dy")}
            for q in v.values():
                q[dead] = fill
            h, y, saved = vc.residual_norm_fwd(v["x"], v["a"], desc, lens=lens, **vec)
            outs.append((h, y) + vc.residual_norm_bwd(v["dh"], v["dy"], saved)[:5])
        for o in outs[1:]:
            assert all(torch.equal(p, q) and torch.isfinite(p).all() for p, q in zip(o, outs[0]))


def test_values_not_finite_stay_in_their_rows():
    import torch
    vc = _vc()
    t = make(20, 264)
    t["x"][3, 5], t["a"][11, 200] = float("nan"), float("inf")
    desc = vc.make_residual_desc(20, 264, checkpoint=True)
    h, y, saved = vc.residual_norm_fwd(t["x"], t["a"], desc, gate=t["gate"], scale=t["scale"], shift=t["shift"])
    bad = [3, 11]
    good = [r for r in range(20) if r not in bad]
    assert torch.isnan(y[bad]).all() and torch.isfinite(y[good]).all() and torch.isfinite(h[good]).all()
    dx = vc.residual_norm_bwd(t["dh"], t["dy"], saved)[0]
    assert torch.isnan(dx[bad]).all() and torch.isfinite(dx[good]).all()


def test_strides():
    import torch
    vc = _vc()
    for cols, off in ((256, 8), (256, 3), (101, 1)):
        t = make(30, cols, x="f32", a="bf16")
        want = check(t)
        wide = {}
        for k in ("x", "a", "dh", "dy"):
            w = torch.full((30, cols + 45), float("nan"), dtype=t[k].dtype, device="cuda")
            w[:, off:off + cols] = t[k]
            wide[k] = w[:, off:off + cols]
        got = check({**t, **wide})
        for p, q in zip(got[:2] + got[2], want[:2] + want[2]):
            assert (p is None and q is None) or torch.equal(p, q)
    none = vc.make_residual_desc(30, 101)
    with pytest.raises(ValueError, match="x must be contiguous"):
        vc.residual_norm_fwd(t["x"].t().contiguous().t(), t["a"], none)


def test_differentiable_streams_and_device():
    import torch
    vc = _vc()
    names = ("x", "a", "gate", "scale", "shift", "post_weight")
    for ckpt in (False, True):
        t = make(300, 520, samples=3, post="weighted", slices=True)
        desc = vc.make_residual_desc(300, 520, 3, post_norm="rms", checkpoint=ckpt)
        leaves = {k: t[k].detach().requires_grad_(True) for k in names}
        h, y = vc.residual_norm(leaves["x"], leaves["a"], desc, **{k: leaves[k] for k in names[2:]})
        grads = torch.autograd.grad((h, y), [leaves[k] for k in names], (t["dh"], t["dy"]))
        eh, ey, saved = vc.residual_norm_fwd(t["x"], t["a"], desc, **{k: t[k] for k in names[2:]})
        want = vc.residual_norm_bwd(t["dh"], t["dy"], saved)
        assert torch.equal(h, eh) and torch.equal(y, ey) and all(torch.equal(p, q) for p, q in zip(grads, want))
        # only one of the two results is used further, only some inputs want a gradient
        h, y = vc.residual_norm(leaves["x"], t["a"], desc, **{k: t[k] for k in names[2:]})
        g = torch.autograd.grad(y, leaves["x"], t["dy"])[0]
        assert torch.equal(g, vc.residual_norm_bwd(None, t["dy"], saved)[0])
        h, y = vc.residual_norm(t["x"], leaves["a"], desc, **{k: t[k] for k in names[2:]})
        g = torch.autograd.grad(h, leaves["a"], t["dh"])[0]
        assert torch.equal(g, vc.residual_norm_bwd(t["dh"], None, saved)[1])
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = vc.residual_norm_bwd(t["dh"], t["dy"], saved)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_graph_replays():
    import torch
    vc = _vc()
    t = make(700, 1032, samples=7, shared=True, post="weighted")
    cu = torch.tensor([0, 5, 5, 300, 301, 500, 640, 690], dtype=torch.int32).cuda()
    desc = vc.make_residual_desc(700, 1032, 7, post_norm="layer", checkpoint=True)
    vec = {k: t[k] for k in ("gate", "scale", "shift", "post_weight")}

    def step():
        h, y, saved = vc.residual_norm_fwd(t["x"], t["a"], desc, cu=cu, **vec)
        return (h, y) + vc.residual_norm_bwd(t["dh"], t["dy"], saved)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step()
    for k in range(3):
        for name in ("x", "a", "dh", "dy"):
            t[name].copy_(torch.randn(t[name].shape, device="cuda"))
        cu[2] = 7 + k  # the division is read on the device
        graph.replay()
        torch.cuda.synchronize()
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(kept, want))


def test_against_differences():
    """Gradients against differences of the kernels' own results, in fp32: the loss is a sum in fp64 of results off by at most some
    10 u relative, over steps of 2^-6; the parabola's term is taken out by the symmetric difference, the cubic one is of 2^-12."""
    import torch
    vc = _vc()
    t = make(6, 40, samples=2, x="f32", a="f32", post="weighted")
    desc = vc.make_residual_desc(6, 40, 2, norm="layer", post_norm="rms", residual_scale=0.5, eps=1e-2)
    names = ("x", "a", "gate", "scale", "shift", "post_weight")

    def loss(v):
        h, y, _ = vc.residual_norm_fwd(v["x"], v["a"], desc, **{k: v[k] for k in names[2:]})
        return float((h.double() * t["dh"].double()).sum() + (y.double() * t["dy"].double()).sum())

    saved = vc.residual_norm_fwd(t["x"], t["a"], desc, **{k: t[k] for k in names[2:]})[2]
    grads = dict(zip(names, vc.residual_norm_bwd(t["dh"], t["dy"], saved)))
    gen = torch.Generator().manual_seed(9)
    for k in names:
        d = torch.randn(t[k].shape, generator=gen).cuda()
        d /= d.norm()
        e = 2.0 ** -6
        diff = (loss({**t, k: t[k] + e * d}) - loss({**t, k: t[k] - e * d})) / (2 * e)
        want = float((grads[k].double() * d.double()).sum())
        assert abs(diff - want) <= 2e-3 * float(grads[k].double().norm()) + 1e-4, (k, diff, want)
