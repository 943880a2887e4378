"""Calls around a block's attention that only their memory makes special: strided inputs of a norm alone, saved tensors that come
back otherwise than they were, offsets past 32 bits, workspaces that two graphs share, views of leaves, the largest values."""
import pytest

from test_residual_gpu import check, make

pytestmark = pytest.mark.gpu


def _vc():
    import paper_2501_08453_amd as vc
    return vc


def _apart(t, more=37):
    """t with its rows further apart, NaN between them."""
    import torch
    w = torch.full((t.shape[0], t.shape[1] + more), float("nan"), dtype=t.dtype, device=t.device)
    w[:, 3:3 + t.shape[1]] = t
    return w[:, 3:3 + t.shape[1]]


@pytest.mark.parametrize("ckpt", [False, True])
@pytest.mark.parametrize("cols", [256, 101, 2500])
def test_norm_alone_of_strided_rows(cols, ckpt):
    """Without a block's output the backward reads x itself, whose rows lie apart."""
    import torch
    t = make(30, cols, x="f32", a="f32", with_a=False)
    want = check(t, checkpoint=ckpt)
    got = check({**t, "x": _apart(t["x"])}, checkpoint=ckpt)
    for p, q in zip(got[:2] + got[2], want[:2] + want[2]):
        assert (p is None and q is None) or torch.equal(p, q)


@pytest.mark.parametrize("with_a", [True, False])
def test_saved_tensors_that_come_back_elsewhere(with_a):
    """Tensors saved on the host come back contiguous, however they lay."""
    import torch
    vc = _vc()
    t = make(64, 136, samples=4, slices=True, with_a=with_a)
    names = ("x", "a", "gate", "scale", "shift") if with_a else ("x", "scale", "shift")
    base = {k: (_apart(t[k]) if k in "xa" else t[k]).detach() for k in names}
    desc = vc.make_residual_desc(64, 136, 4)
    grads = []
    for elsewhere in (False, True):
        v = {k: p.requires_grad_(True) for k, p in base.items()}
        with torch.autograd.graph.save_on_cpu() if elsewhere else torch.enable_grad():
            out = vc.residual_norm(v["x"], v.get("a"), desc, v.get("gate"), v["scale"], v["shift"])
        grads.append(torch.autograd.grad(out, list(v.values()), (t["dh"], t["dy"]) if with_a else t["dy"]))
    assert all(torch.equal(p, q) for p, q in zip(*grads))


def test_offsets_past_32_bits():
    """Rows that begin more than 2^31 elements in: as in a call of their own, whose form may sum a row in another order. Both are off by half
    a step of bf16, 2^-8, and some 40 u of magnitudes up to 30 (7e-5)."""
    import torch
    vc = _vc()
    cols, tail = 1536, 700
    rows = (1 << 31) // cols + 1000
    near = lambda p, q: torch.allclose(p.float(), q.float(), rtol=2.0 ** -7, atol=2e-4)  # noqa: E731
    new = lambda *s: torch.randn(s, device="cuda").to(torch.bfloat16)  # noqa: E731
    end = {k: new(tail, cols) for k in ("x", "a", "dh", "dy")}
    whole = {}
    for k, v in end.items():
        whole[k] = torch.zeros((rows, cols), dtype=v.dtype, device="cuda")
        whole[k][-tail:] = v
    vec = {k: torch.randn((2, cols), device="cuda") for k in ("gate", "scale", "shift")}
    cu = torch.tensor([0, rows - tail, rows], dtype=torch.int32, device="cuda")
    for ckpt in (False, True):
        desc = vc.make_residual_desc(rows, cols, 2, checkpoint=ckpt)
        h, y, saved = vc.residual_norm_fwd(whole["x"], whole["a"], desc, cu=cu, **vec)
        eh, ey, es = vc.residual_norm_fwd(end["x"], end["a"], vc.make_residual_desc(tail, cols, 1, checkpoint=ckpt),
                                          **{k: v[1] for k, v in vec.items()})
        assert torch.equal(h[-tail:], eh) and near(y[-tail:], ey)
        assert not h[0].any() and torch.equal(y[5], y[rows - tail - 1])
        dx, da = vc.residual_norm_bwd(whole["dh"], whole["dy"], saved, want=(True, True) + (False,) * 4)[:2]
        ex, ea = vc.residual_norm_bwd(end["dh"], end["dy"], es)[:2]
        assert near(dx[-tail:], ex) and near(da[-tail:], ea) and not dx[:-tail].any()
        del h, y, saved, dx, da


def test_graphs_that_share_a_workspace():
    """Two captured steps that are given the same workspace, replayed in turn."""
    import torch
    vc = _vc()
    t = make(400, 264, samples=4)
    vec = {k: t[k] for k in ("gate", "scale", "shift")}
    ids = torch.randint(0, 90, (9000,), device="cuda")
    dout = torch.randn((9000, 264), device="cuda")
    ws = torch.empty(1 << 25, dtype=torch.uint8, device="cuda")
    desc = vc.make_residual_desc(400, 264, 4)
    saved = vc.residual_norm_fwd(t["x"], t["a"], desc, **vec)[2]
    steps = (lambda w: vc.residual_norm_bwd(t["dh"], t["dy"], saved, ws=w),
             lambda w: (vc.embedding_bwd(dout, ids, 90, ws=w),))
    graphs = []
    for step in steps:
        step(ws)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            kept = step(ws)
        graphs.append((g, kept))
    for _ in range(3):
        for v in (t["dh"], t["dy"], dout):
            v.copy_(torch.randn(v.shape, device="cuda"))
        ids.random_(0, 90)
        for g, _ in graphs + graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        for step, (_, kept) in zip(steps, graphs):
            assert all(p is None and q is None or torch.equal(p, q) for p, q in zip(kept, step(None)))


def test_two_streams_at_once():
    """Calls on two streams, each with its own workspace, do not touch each other's."""
    import torch
    vc = _vc()
    work = []
    for k in range(2):
        ids = torch.randint(0, 500, (20000,), device="cuda")
        dout = torch.randn((20000, 128), device="cuda").to(torch.bfloat16)
        t = make(3000, 264, samples=5, seed=k)
        saved = vc.residual_norm_fwd(t["x"], t["a"], vc.make_residual_desc(3000, 264, 5), **{n: t[n] for n in ("gate", "scale", "shift")})[2]
        work.append((ids, dout, t, saved))
    run = lambda ids, dout, t, s: (vc.embedding_bwd(dout, ids, 500),) + vc.residual_norm_bwd(t["dh"], t["dy"], s)  # noqa: E731
    want = [run(*w) for w in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in work]
    got = [[], []]
    for _ in range(5):
        for k, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[k].append(run(*work[k]))
    torch.cuda.synchronize()
    for k in range(2):
        for g in got[k]:
            assert all(p is None and q is None or torch.equal(p, q) for p, q in zip(g, want[k]))


def test_views_of_leaves_stay_as_they_are():
    """Layers' weights in one parameter: an operation saves a view of it, whose gradient is that of the weight, not of its 8 bits."""
    import torch
    vc = _vc()
    w = torch.randn((3, 256, 256), device="cuda").to(torch.bfloat16).requires_grad_(True)
    x = torch.randn((300, 256), device="cuda").to(torch.bfloat16).requires_grad_(True)
    dy = torch.randn((300, 256), device="cuda").to(torch.bfloat16)
    want = torch.autograd.grad(x @ w[1], x, dy)[0]
    with vc.saved_in_8bit(min_elements=1):
        y = x @ w[1]
    assert torch.equal(torch.autograd.grad(y, x, dy)[0], want)


def test_largest_values_stay_finite():
    """127 steps of the largest fp32 number over 127, rounded, can be an infinity: the scale is a step smaller then."""
    import torch
    vc = _vc()
    top = torch.finfo(torch.float32).max
    x = torch.zeros((3, 200), device="cuda")
    x[0, 5], x[1, 190], x[2, 7] = top, -top, top * (1 - 2.0 ** -23)
    y = vc.checkpoint_unpack(vc.checkpoint_pack(x))
    assert torch.isfinite(y).all() and ((y - x).abs() <= top * 2.0 ** -23).all()


def test_more_columns_than_32_bits_hold():
    """Refused, not taken for the number's low bits."""
    import torch
    vc = _vc()
    wide = torch.empty((1, (1 << 32) + 128), dtype=torch.bfloat16, device="cuda")
    ids = torch.zeros(1, dtype=torch.int64, device="cuda")
    kept = vc.Packed8(torch.empty(wide.shape, dtype=torch.int8, device="cuda"),
                      torch.empty((1, (1 << 25) + 1), dtype=torch.float32, device="cuda"), wide.dtype)
    for f in (lambda: vc.checkpoint_pack(wide, out=kept), lambda: vc.checkpoint_unpack(kept, out=wide),
              lambda: vc.embedding_fwd(ids, wide, out=wide), lambda: vc.embedding_bwd(wide, ids, 1, into=wide)):
        with pytest.raises((ValueError, vc.JointAttnError), match="invalid descriptor|SHAPE|shape"):  # the backward asks for a workspace first
            f()


@pytest.mark.parametrize("cols,t,grad", [(4800, "f32", "f32"), (4801, "f32", "f32"), (4800, "bf16", "f32"), (4803, "bf16", "bf16"), (4800, "f32", "bf16")])
def test_embedding_of_more_than_the_caches_hold(cols, t, grad):
    """Lookups and gradients large enough to go past the caches: u = 2^-24, a row's sum of n tokens is off by (n + 18) u of the
    magnitudes, and half a step of its type."""
    import torch
    vc = _vc()
    dt = {"f32": torch.float32, "bf16": torch.bfloat16}
    T, V = (16001 if t == "f32" else 30001), 900
    ids = torch.randint(-1, V, (T,), device="cuda")
    ids[::7] = 3
    table, dout = torch.randn((V, cols), device="cuda").to(dt[t]), torch.randn((T, cols), device="cuda").to(dt[t])
    real = (ids >= 0) & (ids != 5)
    want = torch.where(real[:, None], table[ids.clamp(min=0)] * 0.5, torch.zeros((), dtype=dt[t], device="cuda"))
    assert torch.equal(vc.embedding_fwd(ids, table, 0.5, 5), want)  # a half is exact
    got = vc.embedding_bwd(dout, ids, V, 0.5, 5, dtype=dt[grad])
    n = torch.bincount(ids[real], minlength=V)[:, None]
    half = 2.0 ** -8 if grad == "bf16" else 2.0 ** -24
    for c in range(0, cols, 1601):
        d = dout[real][:, c:c + 1601].double()
        s, mag = (torch.zeros((V, d.shape[1]), dtype=torch.float64, device="cuda").index_add_(0, ids[real], 0.5 * p) for p in (d, d.abs()))
        tol = (n + 18) * 2.0 ** -24 * mag
        assert ((got[:, c:c + 1601].double() - s).abs() <= tol + half * (s.abs() + tol)).all()
    assert not got[5].any() and torch.equal(got, vc.embedding_bwd(dout, ids, V, 0.5, 5, dtype=dt[grad]))
