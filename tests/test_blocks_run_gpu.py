"""The operators around a block's attention as they are used: captions from their ids through two blocks (embedding, norm
with the caption's modulation, packed attention, gated residual with the norms before and after) and back, in bf16 with a fp32
oracle by autograd; the same with the activations kept in 8 bits; and stacked blocks whose outputs are packed."""
import numpy as np
import pytest

import workloads as W
from parity_util import log, to_gpu_bf16

pytestmark = pytest.mark.gpu

LENS, H, D, V = [5, 64, 1, 37], 4, 64, 300
C, R, S = H * D, sum(LENS), len(LENS)


def _params(torch):
    g = torch.Generator().manual_seed(7)
    p = {"table": torch.randn(V, C, generator=g) / C ** 0.5, "first": 0.2 * torch.randn(S, 2 * C, generator=g)}
    for i in range(2):
        p["qkv%d" % i] = torch.randn(C, 3 * C, generator=g) / C ** 0.5
        p["out%d" % i] = torch.randn(C, C, generator=g) / C ** 0.5
        p["mod%d" % i] = 0.3 * torch.randn(S, 3 * C, generator=g)
        p["post%d" % i] = 1 + 0.1 * torch.randn(C, generator=g)
    return p, torch.randint(0, V, (R,), generator=g), torch.randn(R, C, generator=g)


def _plain(torch, p, ids):
    """The same in fp32 torch operations."""
    def norm(t):
        return torch.nn.functional.layer_norm(t, (C,), eps=1e-5)

    def rms(t):
        return t / ((t * t).mean(-1, keepdim=True) + 1e-5).sqrt()

    which = torch.repeat_interleave(torch.arange(S), torch.tensor(LENS))
    x = p["table"][ids] * C ** 0.5
    first = p["first"][which]
    y = norm(x) * (1 + first[:, :C]) + first[:, C:]
    for i in range(2):
        q, k, v = (y @ p["qkv%d" % i]).view(R, 3, H, D).unbind(1)
        o, a = [], 0
        for n in LENS:
            s = torch.einsum("qhd,khd->hqk", q[a:a + n], k[a:a + n]) / D ** 0.5
            o.append(torch.einsum("hqk,khd->qhd", s.softmax(-1), v[a:a + n]))
            a += n
        a = torch.cat(o).reshape(R, C) @ p["out%d" % i]
        mod = p["mod%d" % i][which]
        x = x + mod[:, 2 * C:] * rms(a) * p["post%d" % i]
        y = norm(x) * (1 + mod[:, :C]) + mod[:, C:2 * C]
    return y


def _ours(torch, vc, p, ids, checkpoint):
    cu = torch.tensor(np.cumsum([0] + LENS), dtype=torch.int32).cuda()
    attn = vc.make_packed_desc(S, H, H, D, R, R, max(LENS), max(LENS))
    alone = vc.make_residual_desc(R, C, S, checkpoint=checkpoint)
    block = vc.make_residual_desc(R, C, S, post_norm="rms", checkpoint=checkpoint)
    x = vc.embedding(ids, p["table"], scale=C ** 0.5)
    y = vc.residual_norm(x, None, alone, scale=p["first"][:, :C], shift=p["first"][:, C:], cu=cu)
    for i in range(2):
        qkv = (y @ p["qkv%d" % i]).view(R, 3 * H, D)
        o = vc.packed_attention(qkv[:, :H], qkv[:, H:2 * H], qkv[:, 2 * H:], attn, cu, cu)
        mod = p["mod%d" % i]
        x, y = vc.residual_norm(x, o.view(R, C) @ p["out%d" % i], block, gate=mod[:, 2 * C:], scale=mod[:, :C], shift=mod[:, C:2 * C],
                                post_weight=p["post%d" % i], cu=cu)
    return y


@pytest.mark.parametrize("checkpoint", [False, True])
def test_captions_through_two_blocks(checkpoint):
    """Every rounding of an activation or gradient to bf16 is off by up to 2^-8 of its value; some 40 of them lie one behind
    the other each way, and errors of independent signs add as their squares: sqrt(40) 2^-9 (the root mean square of a
    rounding) is 1.2%, times 2 for how far norms and softmax spread them. In 8 bits, values of unit deviation come with a step
    of about 3 / 127, off by 0.7% in the root mean square, in two places of each block: below the same again, 5% in all."""
    import torch
    import paper_2501_08453_amd as vc
    params, ids, dy = _params(torch)
    leaves = {n: t.clone().requires_grad_(True) for n, t in params.items()}
    want = _plain(torch, leaves, ids)
    grads = torch.autograd.grad(want, list(leaves.values()), dy)
    low = {n: t.to(torch.bfloat16).cuda().requires_grad_(True) for n, t in params.items()}
    got = _ours(torch, vc, low, ids.cuda(), checkpoint)
    mine = torch.autograd.grad(got, list(low.values()), dy.to(torch.bfloat16).cuda())
    rel = lambda a, b: float((a.detach().float().cpu() - b).norm() / b.norm())  # noqa: E731
    off = {"y": rel(got, want.detach())} | {n: rel(a, b) for n, a, b in zip(low, mine, grads)}
    log("  ", ", ".join("%s %.4f" % kv for kv in off.items()))
    assert off.pop("y") <= 0.025 and all(torch.isfinite(t).all() for t in mine)
    assert max(off.values()) <= (0.05 if checkpoint else 0.025), off


def test_the_same_under_saved_in_8bit():
    """Forward results are those without the context bit by bit, gradients near them (bound as above)."""
    import torch
    import paper_2501_08453_amd as vc
    params, ids, dy = _params(torch)
    low = {n: t.to(torch.bfloat16).cuda().requires_grad_(True) for n, t in params.items()}
    dy = dy.to(torch.bfloat16).cuda()
    y = _ours(torch, vc, low, ids.cuda(), False)
    want = torch.autograd.grad(y, list(low.values()), dy)
    with vc.saved_in_8bit(min_elements=1):
        z = _ours(torch, vc, low, ids.cuda(), False)
    got = torch.autograd.grad(z, list(low.values()), dy)
    assert torch.equal(y, z)
    off = {n: float((a.float() - b.float()).norm() / b.float().norm()) for n, a, b in zip(low, got, want)}
    log("  ", ", ".join("%s %.4f" % kv for kv in off.items()))
    assert max(off.values()) <= 0.05 and max(off.values()) > 0, off


def test_packed_layers_of_a_stack():
    """Packed layers' gradients are those of the branch calls on the unpacked outputs, bit by bit; kept layers' those of keeping
    all; block outputs too; also when the backward runs twice, and beside recomputed and offloaded layers."""
    import torch
    import paper_2501_08453_amd as vc
    from paper_2501_08453_amd import memory as mem
    K = 4
    w = W.custom(1, 2, 128, 16, 4, 6, 8)
    desc = vc.desc_for(w, deterministic=True)
    inputs, douts = [], []
    for i in range(K):
        x = W.make_inputs(w, seed=5100 + i)
        inputs.append(tuple(to_gpu_bf16(x[n]) for n in ("q", "k", "v")))
        douts.append(to_gpu_bf16(x["do"]))

    def run(strategies, times=1):
        outs = [torch.full_like(inputs[0][0], float("nan")) for _ in range(K)]
        grads = [tuple(tuple(torch.full_like(inputs[0][0], float("nan")) for _ in range(3)) for _ in range(3)) for _ in range(K)]
        bs = mem.BlockStack(desc, inputs, strategies, outs, grads)
        bs.forward()
        for _ in range(times):
            bs.backward(douts)
        torch.cuda.synchronize()
        bs.close()
        return outs, grads

    keep = run(["keep"] * K)
    want = []
    for (q, k, v), do in zip(inputs, douts):
        through = lambda o: vc.checkpoint_unpack(vc.checkpoint_pack(o))  # noqa: E731
        (oj, lj), (os_, ls), (ot, lt) = vc.fwd(q, k, v, desc), vc.spatial_fwd(q, k, v, desc), vc.temporal_fwd(q, k, v, desc)
        want.append((vc.bwd(q, k, v, through(oj), lj, do, desc), vc.spatial_bwd(q, k, v, through(os_), ls, do, desc),
                     vc.temporal_bwd(q, k, v, through(ot), lt, do, desc)))
    for strategies, times in ((mem.plan(K, 1.0, "pack"), 1), (mem.plan(K, 0.5, "pack"), 2), (["offload", "pack", "recompute", "pack"], 1)):
        outs, grads = run(strategies, times)
        for i, s in enumerate(strategies):
            assert torch.equal(outs[i], keep[0][i]), (strategies, i)
            for br in range(3):
                ref = want[i][br] if s == "pack" else keep[1][i][br]
                assert all(torch.equal(a, b) for a, b in zip(grads[i][br], ref)), (strategies, i, br)
