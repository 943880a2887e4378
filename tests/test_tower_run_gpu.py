"""The text tower's operators as they are used: two layers over packed captions (norm, packed attention with the learned
bias, projections by torch), a last norm, and the caption tokens in the text slot of the joint attention."""
import numpy as np
import pytest

from parity_util import log

pytestmark = pytest.mark.gpu

LENS, H, HKV, D, T, F, GH, GW = [5, 64, 1, 37], 4, 2, 64, 64, 2, 6, 7
C = H * D


def _params(torch, gen):
    p = {}
    for i in range(2):
        p["w%d" % i], p["b%d" % i] = 1 + 0.1 * torch.randn(C, generator=gen), 0.1 * torch.randn(C, generator=gen)
        p["qkv%d" % i] = torch.randn(C, (H + 2 * HKV) * D, generator=gen) / C ** 0.5
        p["out%d" % i] = torch.randn(C, C, generator=gen) / C ** 0.5
        p["bias%d" % i] = 0.5 * torch.randn(H, 16, generator=gen)
    p["w2"], p["b2"] = 1 + 0.1 * torch.randn(C, generator=gen), 0.1 * torch.randn(C, generator=gen)
    return p


def _tower(p, x, norm, attend):
    for i in range(2):
        y = norm(x, p["w%d" % i], p["b%d" % i])
        qkv = (y @ p["qkv%d" % i]).view(-1, H + 2 * HKV, D)
        o = attend(qkv[:, :H], qkv[:, H:H + HKV], qkv[:, H + HKV:], p["bias%d" % i])
        x = x + o.reshape(-1, C) @ p["out%d" % i]
    return norm(x, p["w2"], p["b2"])


def _slots(torch, y, video):
    """Caption tokens in the text slot (zeros behind them), then the video tokens: [B, N, H, D]."""
    rows, a = [], 0
    for b, n in enumerate(LENS):
        rows.append(torch.cat([y[a:a + n].view(n, H, D), torch.zeros((T - n, H, D), dtype=y.dtype, device=y.device), video[b]]))
        a += n
    return torch.stack(rows)


def test_tower_feeds_the_joint_attention():
    import torch
    import paper_2501_08453_amd as vc
    gen = torch.Generator().manual_seed(3)
    params, x = _params(torch, gen), torch.randn(sum(LENS), C, generator=gen)
    video = torch.randn(len(LENS), F * GH * GW, H, D, generator=gen)
    dout = torch.randn(len(LENS), T + F * GH * GW, H, D, generator=gen)
    rnd = lambda t: t.to(torch.bfloat16)  # noqa: E731
    norms = [n for n in params if n[0] in "wb" and not n.startswith("bias")]  # kept in 32 bits, the rest in bf16
    buckets = vc.relative_buckets(16, 32)
    cu = torch.tensor(np.cumsum([0] + LENS), dtype=torch.int32).cuda()
    desc = vc.make_packed_desc(len(LENS), H, HKV, D, sum(LENS), sum(LENS), max(LENS), max(LENS), num_buckets=16, max_distance=32)
    joint = vc.make_desc(len(LENS), H, D, T, F, GH, GW, deterministic=True)
    leaves = {n: (t if n in norms else rnd(t)).cuda().requires_grad_(True) for n, t in params.items()}
    lx, lv = (rnd(t).cuda().requires_grad_(True) for t in (x, video))
    y = _tower(leaves, lx, vc.layer_norm, lambda q, k, v, b: vc.packed_attention(q, k, v, desc, cu, cu, bias=b, buckets=buckets))
    z = _slots(torch, y, lv)
    lens = torch.tensor(LENS, dtype=torch.int32).cuda()
    o = vc.joint_attention(z, z, z, joint, text_len=lens)
    o.backward(rnd(dout).cuda())

    # the same in 64 bits on the CPU, from the same rounded values
    ref = {n: t.detach().double().cpu().requires_grad_(True) for n, t in leaves.items()}
    rx, rv = (t.detach().double().cpu().requires_grad_(True) for t in (lx, lv))
    table = buckets.cpu().long()

    def attend(q, k, v, b):
        outs, a = [], 0
        for n in LENS:
            qq, kk, vv = (t[a:a + n].transpose(0, 1) for t in (q, k.repeat_interleave(H // HKV, 1), v.repeat_interleave(H // HKV, 1)))
            rel = torch.arange(n)[None, :] - torch.arange(n)[:, None]
            s = qq @ kk.transpose(1, 2) / D ** 0.5 + b[:, table[rel.clamp(-32, 32) + 32]]
            outs.append((s.softmax(-1) @ vv).transpose(0, 1))
            a += n
        return torch.cat(outs)

    ry = _tower(ref, rx, lambda t, w, b: torch.nn.functional.layer_norm(t, (C,), w, b), attend)
    rz = _slots(torch, ry, rv).transpose(1, 2)
    ok = (torch.arange(T + F * GH * GW)[None] >= T) | (torch.arange(T + F * GH * GW)[None] < torch.tensor(LENS)[:, None])
    s = (rz @ rz.transpose(2, 3) / D ** 0.5).masked_fill(~ok[:, None, None], -torch.inf)
    ro = (s.softmax(-1) @ rz).transpose(1, 2)
    ro.backward(rnd(dout).double())

    # Each of the about 16 stages of a way through the two layers and the joint attention rounds its tensor to bf16 once or
    # twice (relative rms at most 2^-8 / sqrt(3) a time), independently: sqrt(32) of them, and a factor 3 for what norms,
    # softmax and residual sums make of an error. 3 * sqrt(32) * 2^-8 / sqrt(3) = 0.038.
    for name, got, want in [("o", o, ro), ("x", lx.grad, rx.grad), ("video", lv.grad, rv.grad)] + [(n, leaves[n].grad, ref[n].grad) for n in params]:
        g, w = got.detach().double().cpu(), want.detach()
        off = float((g - w).norm() / w.norm())
        log("   %-6s relative error %.4f" % (name, off))
        assert torch.isfinite(g).all() and off <= 0.038, name
