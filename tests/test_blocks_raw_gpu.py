"""Calls of the raw entry points around a block's attention that the tensor-level helpers never make."""
import pytest

from test_residual_gpu import U, half, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("post", [None, "rms"])
@pytest.mark.parametrize("others", ["none", "shared", "own"])
def test_gradient_of_a_gate_that_is_not_given(post, others):
    """gate NULL stands for 1; its gradient is still each sample's own, whichever other gradients are wanted. H and the products are
    those of a gate of ones, and so are the runs: the same sums bit by bit. Without norms they are sums of dh a over a sample's
    rows: chains of at most rows + 80 additions, each off by u = 2^-24 of the magnitudes, and half a step of fp32."""
    import torch
    import paper_2501_08453_amd as vc
    rows, cols, S = 60, 136, 5
    t = make(rows, cols, samples=S, p="f32", post="weighted" if post else None, shared=others == "shared")
    nan = lambda *s: torch.full(s, float("nan"), device="cuda")  # noqa: E731
    for norm in ("layer", None):
        vec = {"scale": t["scale"], "shift": t["shift"]} if norm else {}
        dy = t["dy"] if norm else None
        desc = vc.make_residual_desc(rows, cols, S, norm=norm, post_norm=post)
        one = torch.ones((S, cols), device="cuda")
        saved = vc.residual_norm_fwd(t["x"], t["a"], desc, gate=one, post_weight=t["post_weight"], **vec)[2]
        want = vc.residual_norm_bwd(t["dh"], dy, saved)
        d = saved.desc
        d.gate_stride = 0
        if norm and others == "shared":
            grads = [nan(cols), nan(cols)]
        elif norm and others == "own":
            grads = [nan(S, cols), nan(S, cols)]
        else:
            grads = [None, None]
        dgate, dwp = nan(S, cols), nan(cols) if post else None
        ws = vc.blocks._workspace(vc.vc_residualnorm_bwd_workspace_bytes(d), t["x"].device)
        stats = [s.contiguous() for s in saved.stats] if saved.stats is not None else [None] * 4
        vc.vc_residualnorm_bwd(d, t["dh"], dy, saved.h, saved.a, None, None, None, t["scale"] if norm else None, t["post_weight"], None, None,
                               *stats, None, None, dgate, *grads, dwp, ws, ws.numel())
        torch.cuda.synchronize()
        for got, w in zip([dgate, *grads, dwp], want[2:]):
            assert got is None or torch.equal(got, w)
        if norm is None and post is None:
            p = (t["dh"].double() * t["a"].double()).view(S, -1, cols)
            tol = (rows + 80) * U * p.abs().sum(1)
            assert ((dgate.double() - p.sum(1)).abs() <= tol + half(dgate) * (p.sum(1).abs() + tol)).all()
