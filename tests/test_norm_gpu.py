"""Layer norm on the GPU against the fp64 oracle, on every element."""
import numpy as np
import pytest

from oracle import ref_tower as T
from parity_util import log

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (3, 2), (1, 64), (7, 63), (33, 65), (5, 255), (64, 256), (129, 264), (31, 1000), (257, 1024), (16, 1155),
          (9, 2048), (40, 2056), (5, 4096), (6, 5001), (3, 8192), (2, 16384), (3, 20001), (2, 65536), (2000, 40)]


def _vc():
    import paper_2501_08453_amd as vc
    return vc


def make(rows, cols, xd, pd, affine, seed=1, shift=0.5):
    import torch
    g = torch.Generator().manual_seed(seed)
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}
    x = (torch.randn((rows, cols), generator=g) * 2 + shift).to(dt[xd])
    dy = torch.randn((rows, cols), generator=g).to(dt[xd])
    w = (1 + 0.3 * torch.randn(cols, generator=g)).to(dt[pd]) if affine else None
    b = (0.3 * torch.randn(cols, generator=g)).to(dt[pd]) if affine else None
    return [None if t is None else t.cuda() for t in (x, w, b, dy)]


def _np(t):
    return None if t is None else t.double().cpu().numpy()


def check(x, w, b, dy, eps=1e-5):
    """Bounds, with u = 2^-24: a tree or run of n additions is off by at most n u times the sum of magnitudes; the runs
    here have at most cols / 64 + 16 (rows + 16 for the column sums) additions each; a result is rounded by at most half a
    step of its type."""
    vc = _vc()
    y, mean, rstd = vc.layer_norm_fwd(x, w, b, eps)
    dx, dw, db = vc.layer_norm_bwd(dy, x, w, b, mean, rstd)
    X, W, B, DY = _np(x), _np(w), _np(b), _np(dy)
    r = T.layer_norm(X, W, B, eps, DY)
    u = 2.0 ** -24
    half = {2: 2.0 ** -8, 4: u}
    n = X.shape[1] / 64 + 16
    a = np.abs(X).mean(1)
    e_mean = n * u * a
    xc = X - X.mean(1, keepdims=True)
    # the variance is of the differences to the rounded mean: off by that error squared, and by its own sum's rounding
    rel = n * u + 3 * u + (e_mean * r["rstd"]) ** 2 + 4 * u * a * r["rstd"]
    e_xh = (e_mean * r["rstd"])[:, None] + (np.abs(xc) * r["rstd"][:, None]) * (rel + 4 * u)[:, None] + 2 * u * (np.abs(X) * r["rstd"][:, None])
    Wm = np.ones(X.shape[1]) if W is None else np.abs(W)
    hx = half[x.element_size()]

    def near(name, got, want, tol):
        d = np.abs(_np(got) - want)
        log("   %-5s off / bound %.3f" % (name, float((d / tol).max())))
        assert np.isfinite(_np(got)).all() and (d <= tol).all(), name

    near("mean", mean, r["mean"], e_mean + 1e-30)
    near("rstd", rstd, r["rstd"], rel * r["rstd"] + 1e-30)
    near("y", y, r["y"], e_xh * Wm + (hx + 4 * u) * np.abs(r["y"]) + 4 * u * (0 if B is None else np.abs(B)) + 1e-30)
    g, xh = np.abs(DY) * Wm, np.abs(xc) * r["rstd"][:, None]
    m1, m2 = g.mean(1, keepdims=True), (g * (xh + e_xh)).mean(1, keepdims=True)
    e2 = (g * e_xh).mean(1, keepdims=True) + (n + 4) * u * m2
    mag = g + m1 + xh * m2
    near("dx", dx, r["dx"], r["rstd"][:, None] * ((n + 8) * u * mag + e_xh * m2 + xh * e2 + rel[:, None] * mag) + hx * np.abs(r["dx"]) + 1e-30)
    rows = X.shape[0] + 16
    if w is not None:
        hp = half[w.element_size()]
        near("dw", dw, r["dw"], (np.abs(DY) * (e_xh + rows * u * xh)).sum(0) + hp * np.abs(r["dw"]) + 1e-30)
        near("db", db, r["db"], rows * u * np.abs(DY).sum(0) + hp * np.abs(r["db"]) + 1e-30)
    else:
        assert dw is None and db is None


@pytest.mark.parametrize("xd,pd", [("bf16", "f32"), ("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_shapes(rows, cols, xd, pd):
    check(*make(rows, cols, xd, pd, True))


@pytest.mark.parametrize("xd", ["bf16", "f32"])
def test_no_weights_far_mean_and_zero_variance(xd):
    check(*make(50, 300, xd, "f32", False))
    check(*make(50, 1024, xd, "f32", True, shift=300.0))  # a mean of 150 times the deviation
    x, w, b, dy = make(4, 128, xd, "f32", True)
    x[1] = 2.0  # no variance: y = b, rstd = 1 / sqrt(eps)
    check(x, w, b, dy)


def test_many_rows():
    check(*make(20011, 96, "bf16", "f32", True))


def test_only_one_of_the_parameters():
    import torch
    vc = _vc()
    x, w, b, dy = make(40, 200, "bf16", "f32", True)
    y, mean, rstd = vc.layer_norm_fwd(x, w, None)
    dx, dw, db = vc.layer_norm_bwd(dy, x, w, None, mean, rstd)
    y2, m2, r2 = vc.layer_norm_fwd(x, w, torch.zeros_like(b))
    full = vc.layer_norm_bwd(dy, x, w, b, mean, rstd)
    assert torch.equal(y, y2) and db is None and torch.equal(dx, full[0]) and torch.equal(dw, full[1])
    y3, _, _ = vc.layer_norm_fwd(x, None, b)
    y4, _, _ = vc.layer_norm_fwd(x, torch.ones_like(w), b)
    dx3, dw3, db3 = vc.layer_norm_bwd(dy, x, None, b, mean, rstd)
    assert torch.equal(y3, y4) and dw3 is None and torch.equal(db3, full[2])


def test_strides_shapes_and_empty():
    import torch
    vc = _vc()
    x, w, b, dy = make(30, 256, "bf16", "f32", True)
    wide, dwide = (torch.full((30, 300), float("nan"), dtype=x.dtype, device="cuda") for _ in range(2))
    for off in (8, 3):  # 16-byte aligned rows or not
        wide[:, off:off + 256], dwide[:, off:off + 256] = x, dy
        a = vc.layer_norm_fwd(wide[:, off:off + 256], w, b)
        e = vc.layer_norm_fwd(x, w, b)
        for s, t in zip(a, e):
            assert torch.allclose(s.float(), t.float(), rtol=2.0 ** -7, atol=1e-6)
        check(wide[:, off:off + 256], w, b, dwide[:, off:off + 256])
    y, mean, rstd = vc.layer_norm_fwd(x.view(5, 6, 256), w, b)
    assert y.shape == (5, 6, 256) and mean.shape == (5, 6) and torch.equal(y.view(30, 256), vc.layer_norm_fwd(x, w, b)[0])
    none = torch.empty((0, 256), dtype=x.dtype, device="cuda")
    y, mean, rstd = vc.layer_norm_fwd(none, w, b)
    dx, dw, db = vc.layer_norm_bwd(none, none, w, b, mean, rstd)
    assert y.shape == dx.shape == (0, 256) and (dw == 0).all() and (db == 0).all()


def test_differentiable_stream_and_graph():
    import torch
    vc = _vc()
    x, w, b, dy = make(300, 520, "bf16", "f32", True)
    leaves = [t.clone().requires_grad_(True) for t in (x, w, b)]
    y = vc.layer_norm(*leaves)
    y.backward(dy)
    want_y, mean, rstd = vc.layer_norm_fwd(x, w, b)
    want = vc.layer_norm_bwd(dy, x, w, b, mean, rstd)
    assert torch.equal(y, want_y) and all(torch.equal(t.grad, g) for t, g in zip(leaves, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = vc.layer_norm_bwd(dy, x, w, b, mean, rstd)
    torch.cuda.synchronize()
    assert all(torch.equal(s, t) for s, t in zip(got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cy, cm, cr = vc.layer_norm_fwd(x, w, b)
        cg = vc.layer_norm_bwd(dy, x, w, b, cm, cr)
    for _ in range(3):
        x.copy_(torch.randn(x.shape, device="cuda"))
        g.replay()
        torch.cuda.synchronize()
        ey, em, er = vc.layer_norm_fwd(x, w, b)
        eg = vc.layer_norm_bwd(dy, x, w, b, em, er)
        torch.cuda.synchronize()
        assert torch.equal(cy, ey) and all(torch.equal(s, t) for s, t in zip(cg, eg))
