"""8-bit checkpoints on the GPU: bit by bit against the definition in float32 arithmetic, and what autograd keeps in them."""
import numpy as np
import pytest

from oracle import ref_blocks as B

pytestmark = pytest.mark.gpu


def _vc():
    import paper_2501_08453_amd as vc
    return vc


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


def check(x, want=None):
    import torch
    vc = _vc()
    kept = vc.checkpoint_pack(x)
    vals, scales, q = B.kept8((x if want is None else want).float().cpu().numpy().reshape(-1, x.shape[-1]))
    assert kept.q.shape == x.shape and kept.dtype is x.dtype
    assert np.array_equal(kept.q.cpu().numpy().reshape(q.shape), q)
    assert same(kept.scales.cpu().numpy().reshape(scales.shape), scales)
    got = vc.checkpoint_unpack(kept, dtype=torch.float32)
    assert same(got.cpu().numpy().reshape(vals.shape), vals)
    low = vc.checkpoint_unpack(kept, dtype=torch.bfloat16)
    assert same(low.float().cpu().numpy(), got.to(torch.bfloat16).float().cpu().numpy())
    assert vc.checkpoint_unpack(kept).dtype is x.dtype
    return kept


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (2, 3), (5, 64), (7, 127), (3, 128), (9, 129), (4, 1000), (11, 1155), (3, 8200), (2, 20001),
                                       (5000, 128), (3001, 77)])
def test_shapes(rows, cols, dt):
    import torch
    g = torch.Generator().manual_seed(rows + cols)
    x = torch.randn((rows, cols), generator=g) * torch.exp(2 * torch.randn((rows, 1), generator=g))
    check(x.to(torch.bfloat16 if dt == "bf16" else torch.float32).cuda())


def test_edges():
    """Nothing but zeros, single large values, ties, the smallest and largest values, infinities and NaN."""
    import torch
    x = torch.zeros((9, 300))
    x[1, 7] = 1.0
    x[2, :128] = torch.arange(128) - 64.0
    x[2, 0] = 127.0  # steps of 1
    x[3, :4] = torch.tensor([254.0, 1.0, 3.0, -5.0])
    x[4] = 2.0 ** -126
    x[5] = 3.38e38
    x[6, 130], x[6, 290] = float("inf"), float("nan")
    x[7, 299] = -float("inf")
    x[8] = torch.randn(300) * 1e-41  # below the smallest normal number
    check(x.cuda())
    check(x.to(torch.bfloat16).cuda())


def test_shapes_strides_and_empty():
    import torch
    vc = _vc()
    x = torch.randn((4, 5, 6, 96), device="cuda").to(torch.bfloat16)
    check(x)
    wide = torch.full((30, 400), float("nan"), device="cuda")
    part = torch.randn((30, 211), device="cuda")
    wide[:, 7:218] = part
    check(wide[:, 7:218], part)
    none = vc.checkpoint_pack(torch.empty((0, 96), device="cuda"))
    assert none.q.shape == (0, 96) and none.scales.shape == (0, 1) and vc.checkpoint_unpack(none).shape == (0, 96)
    with pytest.raises(ValueError):
        vc.checkpoint_pack(x.transpose(0, 1))
    with pytest.raises(ValueError, match="scales has shape"):
        vc.checkpoint_unpack(vc.Packed8(none.q, none.scales[:, :0], none.dtype))
    kept = vc.checkpoint_pack(x)
    out = torch.empty_like(x)
    assert vc.checkpoint_unpack(kept, out=out) is out and torch.equal(out, vc.checkpoint_unpack(kept))


def test_offsets_past_32_bits():
    """2^31 + some elements in: the last rows are right."""
    import torch
    vc = _vc()
    rows, cols = (1 << 24) + 3, 129
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    tail = torch.randn((5, cols), device="cuda").to(torch.bfloat16)
    x[-5:] = tail
    kept = vc.checkpoint_pack(x)
    del x
    vals, scales, q = B.kept8(tail.float().cpu().numpy())
    assert np.array_equal(kept.q[-5:].cpu().numpy(), q) and np.array_equal(kept.scales[-5:].cpu().numpy(), scales)
    assert not kept.q[:-5].any()
    y = vc.checkpoint_unpack(kept)
    assert torch.equal(y[-5:].float().cpu(), torch.from_numpy(vals).to(torch.bfloat16).float()) and not y[:-5].any()


def test_kept_for_the_backward():
    """What autograd saves in the context is what pack and unpack leave of it; leaves, small and other tensors stay."""
    import torch
    vc = _vc()
    w = torch.randn((512, 512), device="cuda").to(torch.bfloat16).requires_grad_(True)
    x = torch.randn((600, 512), device="cuda").to(torch.bfloat16).requires_grad_(True)
    dy = torch.randn((600, 512), device="cuda").to(torch.bfloat16)
    through = lambda t: vc.checkpoint_unpack(vc.checkpoint_pack(t.detach()))  # noqa: E731
    with vc.saved_in_8bit():
        y = x * 1.5          # no leaf
        z = y * y            # saves y
        out = z @ w          # saves z and the leaf w
    gz, gw = dy @ w.detach().t(), through(z).t() @ dy
    gy = gz * through(y) + gz * through(y)
    got = torch.autograd.grad(out, (x, w), dy)
    assert torch.equal(got[1], gw)
    assert torch.allclose(got[0].float(), (gy * 1.5).float(), rtol=2.0 ** -6, atol=1e-3)
    with vc.saved_in_8bit(min_elements=1 << 24):
        y = x * 1.5
        out = (y * y) @ w
    keep = torch.autograd.grad(out, (x, w), dy)
    y = x * 1.5
    out = (y * y) @ w
    assert all(torch.equal(a, b) for a, b in zip(keep, torch.autograd.grad(out, (x, w), dy)))


def test_statistics_stay_as_they_are():
    """The attention's log-sum-exps and the norms' statistics are not packed; q, k, v and o are, where they are no leaves."""
    import torch
    vc = _vc()
    desc = vc.make_desc(1, 2, 64, 64, 2, 16, 16)
    n = 64 + 2 * 256
    leaves = [torch.randn((1, n, 2, 64), device="cuda").to(torch.bfloat16).requires_grad_(True) for _ in range(3)]
    do = torch.randn((1, n, 2, 64), device="cuda").to(torch.bfloat16)
    with vc.saved_in_8bit(min_elements=1):
        o = vc.joint_attention(*leaves, desc)
    with torch.no_grad():
        eo, lse = vc.fwd(*leaves, desc)
    ko = vc.checkpoint_unpack(vc.checkpoint_pack(eo))
    want = vc.bwd(*[t.detach() for t in leaves], ko, lse, do, desc)
    got = torch.autograd.grad(o, leaves, do)
    assert torch.equal(o, eo) and torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])


def test_graph_and_stream():
    import torch
    vc = _vc()
    x = torch.randn((301, 515), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = vc.checkpoint_unpack(vc.checkpoint_pack(x))
    torch.cuda.synchronize()
    assert torch.equal(y, vc.checkpoint_unpack(vc.checkpoint_pack(x)))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        kept = vc.checkpoint_pack(x)
        y = vc.checkpoint_unpack(kept)
    for _ in range(3):
        x.copy_(torch.randn_like(x))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, vc.checkpoint_unpack(vc.checkpoint_pack(x)))
