"""Performance cases of the operators around a block's attention: the gated residual with the norms before and
after a block, activation checkpoints in 8 bits, and the embedding of tokens.

The residual stream x takes in a block's output a, h = c x + gate * P(a), and the next block reads
y = N(h) * (1 + scale) + shift, where gate, scale and shift belong to the row's sample (a clip, a caption) or
are learned. Checkpoints keep what a backward pass needs in 8 bits with a scale for each 128 columns of a row.
The embedding starts the text tower; its gradient sums the rows of equal tokens. `draw` spreads further cases
over the same ranges.
"""
from __future__ import annotations

import math

import torch

own = False  # False: the operators in elementary torch operations; True: the library's calls

DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}


def _res(name, mode, cols, rows=0, samples=1, lens="", slot=0, tail=0, x="bf16", a="bf16", p="bf16", norm="layer", post="",
         c=1.0, plus_one=True, gate=True, shared=False, ckpt=False, api="call"):
    """rows in `samples` equal slots; or, with lens (a text), sequences of those lengths one behind the other and
    `tail` rows behind the last, or at the head of slots of `slot` rows each. shared: one learned gate, scale
    and shift for all samples. ckpt: the backward's h and a kept in 8 bits."""
    if lens:
        n = _ints(lens)
        samples, rows = len(n), (slot * len(n) if slot else sum(n) + tail)
    return {"name": name, "op": "res", "mode": mode, "cols": cols, "rows": rows, "samples": samples, "lens": lens, "slot": slot,
            "tail": tail, "x": x, "a": a, "p": p, "norm": norm, "post": post, "c": c, "plus_one": plus_one, "gate": gate,
            "shared": shared, "ckpt": ckpt, "api": api}


def _pack(name, rows, cols, x="bf16"):
    return {"name": name, "op": "pack", "mode": "both", "rows": rows, "cols": cols, "x": x}


def _emb(name, mode, tokens, vocab, cols, t="bf16", out="bf16", grad="f32", scale=1.0, pad=-1, ids="i64"):
    """grad: the type of the table's gradient. pad: the id that stands for no token, -1: none."""
    return {"name": name, "op": "emb", "mode": mode, "tokens": tokens, "vocab": vocab, "cols": cols, "t": t, "out": out,
            "grad": grad, "scale": scale, "pad": pad, "ids": ids}


CAPTIONS = ("77,120,8,201,163,45,256,99,110,131,180,17,64,152,140,33,77,230,105,111,88,190,61,128,146,173,25,119,"
            "200,94,102,127")


def listed():
    return [
        # The smallest call: one token each of a batch of requests, every one with its own modulation.
        _res("residual-tokens", "fwd", 2048, rows=16, samples=16),
        # A training step of a block over a long clip's tokens, the modulation of its one sample.
        _res("residual-clip-train", "train", 1536, rows=57856),
        # The same with the backward's activations kept in 8 bits.
        _res("residual-clip-train-8bit", "train", 1536, rows=57856, ckpt=True),
        # Captions one behind the other, a norm on either side of each block, a stream in 32 bits, learned vectors.
        _res("residual-captions-train", "train", 1024, lens=CAPTIONS, x="f32", p="f32", norm="rms", post="rms", shared=True,
             api="autograd"),
        # Odd columns, padded slots of different lengths, everything in 32 bits, a scaled residual.
        _res("residual-odd-train", "train", 1155, lens="1700,903,4,1250", slot=1701, x="f32", a="f32", p="f32", post="layer",
             c=0.75),
        # The attention outputs of a long clip into 8 bits and back, as a layer's checkpoint is kept and used.
        _pack("checkpoint-outputs", 57856 * 24, 128),
        # One caption's activations: the launches decide.
        _pack("checkpoint-caption", 205, 1024),
        # A stream in 32 bits with odd columns.
        _pack("checkpoint-odd", 5001, 1155, x="f32"),
        # The tokens of one serving step.
        _emb("embed-tokens", "fwd", 16, 50000, 2048),
        # Captions of a batch of clips, scaled by the root of the columns, some of them padding.
        _emb("embed-captions-train", "train", 32 * 256, 32128, 1024, scale=32.0, pad=0),
        # A training step over long texts: the table's gradient in 32 bits.
        _emb("embed-long-train", "train", 65536, 50000, 1536),
        # Odd columns, a table in 32 bits.
        _emb("embed-odd-train", "train", 5000, 1999, 1155, t="f32", out="f32", scale=0.5, ids="i32"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["res", "res", "res", "pack", "emb", "emb"])
    cols = _log_uniform(rng, 64, 8192)
    if rng.random() < 0.7:
        cols = (cols + 7) // 8 * 8
    most = max(2, min(60000, 80_000_000 // cols))
    if kind == "pack":
        x = rng.choice(["bf16", "bf16", "f32"])
        return _pack("", _log_uniform(rng, 1, most * (2 if x == "bf16" else 1)), cols, x=x)
    if kind == "emb":
        table = max(3, min(60000, 70_000_000 // cols))
        t = rng.choice(["bf16", "bf16", "f32"])
        vocab = _log_uniform(rng, 3, table)
        return _emb("", rng.choice(["fwd", "train", "train"]), _log_uniform(rng, 1, most), vocab, cols, t=t, out=t,
                    grad=rng.choice(["f32", t]), scale=rng.choice([1.0, cols ** 0.5, 0.37]), pad=rng.choice([-1, 0, vocab - 1]),
                    ids=rng.choice(["i64", "i32"]))
    mode = rng.choice(["fwd", "train", "train"])
    x, a, p, ckpt = rng.choice([("bf16", "bf16", "bf16", False), ("bf16", "bf16", "bf16", True), ("f32", "bf16", "f32", False),
                                ("f32", "f32", "f32", False)])
    form = dict(x=x, a=a, p=p, ckpt=ckpt and mode == "train", norm=rng.choice(["layer", "layer", "rms"]), post=rng.choice(["", "", "layer", "rms"]),
                c=rng.choice([1.0, 1.0, 0.75]), plus_one=rng.random() < 0.7, gate=rng.random() < 0.8, shared=rng.random() < 0.3,
                api=rng.choice(["call", "autograd"]) if mode == "train" else "call")
    rows = _log_uniform(rng, 1, max(2, min(60000, 320_000_000 // (cols * (BYTES[x] + BYTES[a])))))
    samples = min(rows, _log_uniform(rng, 1, 64))
    slot = rows // samples
    if rng.random() < 0.4:
        return _res("", mode, cols, rows=slot * samples, samples=samples, **form)
    if rng.random() < 0.4:
        return _res("", mode, cols, lens=",".join(str(rng.randint(0 if k else 1, slot)) for k in range(samples)), slot=slot, **form)
    ends = sorted(rng.randint(0, rows) for _ in range(samples - 1)) + [rows]  # some of the sequences hold nothing
    n = [e - b for b, e in zip([0] + ends, ends)]
    return _res("", mode, cols, lens=",".join(map(str, n)), tail=rng.choice([0, 0, 7]), **form)


def _ints(text):
    return [int(t) for t in text.split(",")]


def _starts(c):
    """First row and length of each sample."""
    if not c["lens"]:
        per = c["rows"] // c["samples"]
        return [(s * per, per) for s in range(c["samples"])]
    out, at = [], 0
    for k, n in enumerate(_ints(c["lens"])):
        out.append((k * c["slot"] if c["slot"] else at, n))
        at += n
    return out


def _inputs(c, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    new = lambda *shape: torch.randn(shape, generator=gen, device=DEV)  # noqa: E731
    if c["op"] == "pack":
        # columns of different sizes, as activations have them, one in 64 far larger
        size = torch.exp(0.5 * new(c["cols"]))
        size[::64] *= 8
        return {"x": (new(c["rows"], c["cols"]) * size).to(DT[c["x"]])}
    if c["op"] == "emb":
        # frequent and rare tokens: the chance of an id falls as its inverse
        u = torch.rand(c["tokens"], generator=gen, device=DEV, dtype=torch.float64)
        ids = (torch.exp(u * math.log(c["vocab"] + 1.0)) - 1).long().clamp(max=c["vocab"] - 1)
        x = {"ids": ids.to(torch.int64 if c["ids"] == "i64" else torch.int32), "table": new(c["vocab"], c["cols"]).to(DT[c["t"]])}
        if c["mode"] == "train":
            x["dy"] = new(c["tokens"], c["cols"]).to(DT[c["out"]])
        return x
    rows, cols, S = c["rows"], c["cols"], c["samples"]
    x = {"x": (new(rows, cols) * 1.5 + 0.3).to(DT[c["x"]]), "a": new(rows, cols).to(DT[c["a"]]), "gate": None, "post_weight": None,
         "cu": None, "lens": None}
    if c["shared"]:
        x["scale"], x["shift"], x["gate"] = ((o + 0.2 * new(cols)).to(DT[c["p"]]) for o in (0.0 if c["plus_one"] else 1.0, 0.0, 0.5))
    else:
        # one projection of each sample's condition gives all of its vectors, and more for the block's other half
        mod = (0.3 * new(S, 6 * cols) + (0.0 if c["plus_one"] else 1.0)).to(DT[c["p"]])
        x["shift"], x["scale"], x["gate"] = mod[:, :cols], mod[:, cols:2 * cols], mod[:, 2 * cols:3 * cols]
    if not c["gate"]:
        x["gate"] = None
    if c["post"]:
        x["post_weight"] = (1 + 0.2 * new(cols)).to(DT[c["p"]])
    dev = lambda t: torch.tensor(t, dtype=torch.int32, device=DEV)  # noqa: E731
    if c["lens"]:
        n = _ints(c["lens"])
        if c["slot"]:
            x["lens"] = dev(n)
        else:
            x["cu"] = dev([sum(n[:k]) for k in range(S + 1)])
    if c["mode"] == "train":
        x["dh"], x["dy"] = new(rows, cols).to(DT[c["x"]]), new(rows, cols).to(DT[c["a"]])
    return x


def prepare(c, seed):
    s = {"case": c, **_inputs(c, seed)}
    if c["op"] == "res" and c["api"] == "autograd":
        for n in ("x", "a", "gate", "scale", "shift", "post_weight"):
            if s[n] is not None:
                s[n] = s[n].detach().requires_grad_(True)
    return s


# --- the operators in elementary operations, 32 bits -----------------------------------------

def _plain_blocks(x, cols):
    """x with its columns as blocks of 128, zeros behind the last."""
    return torch.nn.functional.pad(x.float(), (0, -cols % 128)).view(x.shape[0], -1, 128)


def _plain_8bit(x):
    """The values that x has in 8 bits, and the blocks' scales."""
    cols = x.shape[1]
    b = _plain_blocks(x, cols)
    top = b.abs().amax(-1).clamp(min=2.0 ** -100)
    scale = top / 127
    q = torch.round(b * (127 / top)[..., None])
    return (q * scale[..., None]).view(x.shape[0], -1)[:, :cols], scale


def _plain_pack(s):
    y, scale = _plain_8bit(s["x"])
    return y.to(torch.bfloat16), scale


def _plain_embedding(s):
    c = s["case"]
    ids, V = s["ids"].long(), c["vocab"]
    real = (ids != c["pad"])[:, None]
    y = (s["table"][ids].float() * c["scale"] * real).to(DT[c["out"]])
    if c["mode"] == "fwd":
        return y
    g = torch.zeros((V, c["cols"]), device=DEV).index_add_(0, ids, s["dy"].float() * real) * c["scale"]
    return y, g.to(DT[c["grad"]])


def _plain_normed(x, kind, eps=1e-5):
    """(normed x, 1 / deviation)"""
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + eps)
    return x * r, r


def _plain_norm_grad(g, n, r, kind):
    d = g - n * (g * n).mean(-1, keepdim=True)
    if kind == "layer":
        d = d - g.mean(-1, keepdim=True)
    return d * r


def _plain_residual(s):
    c = s["case"]
    S, cols, rows = c["samples"], c["cols"], c["rows"]
    at = torch.arange(rows, device=DEV)
    if s["cu"] is not None:
        which = torch.searchsorted(s["cu"][1:].contiguous(), at, right=True)
        real = (which < S)[:, None]
        which = which.clamp(max=S - 1)
    else:
        which = at // (rows // S)
        real = None if s["lens"] is None else (at % (rows // S) < s["lens"][which])[:, None]

    def of_rows(p):  # a parameter as the rows meet it
        p = p.detach().float()
        return p if p.dim() == 1 or S == 1 else p[which]

    only = lambda t: t if real is None else t.masked_fill(~real, 0)  # noqa: E731

    def over(t):  # sums over the rows of each sample
        if s["cu"] is None:
            return t.view(S, rows // S, cols).sum(1)
        hot = (which[None, :] == torch.arange(S, device=DEV)[:, None]) & real[:, 0]
        return torch.matmul(hot.float(), t)

    x, a = s["x"].detach(), s["a"].detach()
    gate = None if s["gate"] is None else of_rows(s["gate"])
    scale, wp = of_rows(s["scale"]) + (1 if c["plus_one"] else 0), None if s["post_weight"] is None else s["post_weight"].detach().float()
    an, ar = _plain_normed(a.float(), c["post"]) if c["post"] else (a.float(), None)
    p = an if wp is None else an * wp
    h = x.float() * c["c"] + (p if gate is None else p * gate)
    h = only(h).to(x.dtype)
    n, r = _plain_normed(h.float(), c["norm"])
    y = only(n * scale + of_rows(s["shift"])).to(a.dtype)
    if c["mode"] == "fwd":
        return h, y
    if c["ckpt"]:  # the backward's own: from the values kept in 8 bits, and the forward's statistics
        h8, a8 = _plain_8bit(h)[0], _plain_8bit(a)[0]
        n = (h8 - (h.float().mean(-1, keepdim=True) if c["norm"] == "layer" else 0)) * r
        an = a8 if not c["post"] else (a8 - (a.float().mean(-1, keepdim=True) if c["post"] == "layer" else 0)) * ar
    dh, dy = only(s["dh"].float()), only(s["dy"].float())
    H = dh + _plain_norm_grad(dy * scale, n, r, c["norm"])
    H = only(H)
    k = H if gate is None else H * gate
    da = k if ar is None else _plain_norm_grad(k * wp, an, ar, c["post"])
    A, E, F = over(H * an), over(dy * n), over(dy)
    out = {"dx": (H * c["c"]).to(x.dtype), "da": da.to(a.dtype)}
    g = torch.ones((1, cols), device=DEV) if s["gate"] is None else s["gate"].detach().float()
    if wp is not None:
        out["dpost_weight"] = (A * g).sum(0)
    if gate is not None:
        out["dgate"] = A if wp is None else A * wp
    out["dscale"], out["dshift"] = E, F
    for name in ("dgate", "dscale", "dshift", "dpost_weight"):
        if name in out:
            out[name] = (out[name].sum(0) if c["shared"] and name != "dpost_weight" else out[name]).to(DT[c["p"]])
    return {"h": h, "y": y, **out}


# --- one pass ----------------------------------------------------------------------------------

def _own_residual(s):
    import paper_2501_08453_amd as vc
    c = s["case"]
    if "desc" not in s:
        s["desc"] = vc.make_residual_desc(c["rows"], c["cols"], c["samples"], norm=c["norm"], post_norm=c["post"] or None,
                                          residual_scale=c["c"], plus_one=c["plus_one"], checkpoint=c["ckpt"])
    kw = {"gate": s["gate"], "scale": s["scale"], "shift": s["shift"], "post_weight": s["post_weight"], "cu": s["cu"], "lens": s["lens"]}
    if c["mode"] == "fwd":
        return vc.residual_norm_fwd(s["x"], s["a"], s["desc"], **kw)[:2]
    if c["api"] == "autograd":
        h, y = vc.residual_norm(s["x"], s["a"], s["desc"], **kw)
        names = [n for n in ("x", "a", "gate", "scale", "shift", "post_weight") if s[n] is not None]
        g = torch.autograd.grad((h, y), [s[n] for n in names], (s["dh"], s["dy"]))
        return {"h": h.detach(), "y": y.detach(), **{"d" + n: t for n, t in zip(names, g)}}
    h, y, saved = vc.residual_norm_fwd(s["x"], s["a"], s["desc"], **kw)
    g = vc.residual_norm_bwd(s["dh"], s["dy"], saved)
    return {"h": h, "y": y, **{"d" + n: t for n, t in zip(("x", "a", "gate", "scale", "shift", "post_weight"), g) if t is not None}}


def _own(s):
    import paper_2501_08453_amd as vc
    c = s["case"]
    if c["op"] == "res":
        return _own_residual(s)
    if c["op"] == "pack":
        kept = vc.checkpoint_pack(s["x"])
        return vc.checkpoint_unpack(kept, dtype=torch.bfloat16), kept.scales
    pad = None if c["pad"] < 0 else c["pad"]
    y = vc.embedding_fwd(s["ids"], s["table"], scale=c["scale"], padding_id=pad)
    if c["mode"] == "fwd":
        return y
    return y, vc.embedding_bwd(s["dy"], s["ids"], c["vocab"], scale=c["scale"], padding_id=pad, dtype=DT[c["grad"]])


def run(s):
    if own:
        return _own(s)
    op = s["case"]["op"]
    return _plain_residual(s) if op == "res" else _plain_pack(s) if op == "pack" else _plain_embedding(s)


def work(c):
    n = c["cols"] * (c["rows"] if "rows" in c else c["tokens"])
    if c["op"] == "pack":  # in and out, the 8 bits and the scales written and read between
        return {"bytes": n * (BYTES[c["x"]] + 2 + 2) + 8 * c["rows"] * (-(-c["cols"] // 128)), "flops": 6 * n}
    if c["op"] == "emb":
        # rows of the table that the tokens meet, as ids are spread: at most all, at most one a token
        met = min(c["vocab"], c["tokens"])
        b = met * c["cols"] * BYTES[c["t"]] + n * BYTES[c["out"]] + c["tokens"] * (8 if c["ids"] == "i64" else 4)
        if c["mode"] == "train":
            b += n * BYTES[c["out"]] + c["vocab"] * c["cols"] * BYTES[c["grad"]]
        return {"bytes": b, "flops": n * (2 if c["mode"] == "train" else 1)}
    train = c["mode"] == "train"
    params = c["cols"] * BYTES[c["p"]] * ((2 + c["gate"]) * (1 if c["shared"] else c["samples"]) + bool(c["post"]))
    b = 2 * n * (BYTES[c["x"]] + BYTES[c["a"]]) * (2 if train else 1) + params * (2 if train else 1)
    return {"bytes": b, "flops": n * (45 if train else 14)}


# --- the same results in 64 bits, from the definitions -----------------------------------------

def _kept(t):
    """What 8 bits hold of t (64 bits): whole steps of a 127th of each block's largest value."""
    out = torch.empty_like(t)
    scales = []
    for j in range(0, t.shape[1], 128):
        part = t[:, j:j + 128]
        step = part.abs().max(1, keepdim=True).values.clamp(min=2.0 ** -100) / 127
        out[:, j:j + 128] = (part / step).round() * step
        scales.append(step)
    return out, torch.cat(scales, 1)


def exact(c, seed):
    x = _inputs(c, seed)
    if c["op"] == "pack":
        return _kept(x["x"].double())
    if c["op"] == "emb":
        ids = x["ids"].long()
        shut = ids == c["pad"]
        y = x["table"].double()[ids] * c["scale"]
        y[shut] = 0
        if c["mode"] == "fwd":
            return y
        # tokens in the order of their ids; a run's sum is the difference of two running sums in 64 bits
        order = torch.argsort(ids, stable=True)
        g = torch.zeros((c["vocab"], c["cols"]), dtype=torch.float64, device=DEV)
        ends = torch.searchsorted(ids[order], torch.arange(c["vocab"] + 1, device=DEV))
        for j in range(0, c["cols"], 256):
            dy = x["dy"][:, j:j + 256].double()
            dy[shut] = 0
            run_ = torch.zeros((c["tokens"] + 1, dy.shape[1]), dtype=torch.float64, device=DEV)
            torch.cumsum(dy[order], 0, out=run_[1:])
            g[:, j:j + 256] += (run_[ends[1:]] - run_[ends[:-1]]) * c["scale"]
        return y, g
    rows, cols, S = c["rows"], c["cols"], c["samples"]
    f64 = lambda *shape: torch.zeros(shape, dtype=torch.float64, device=DEV)  # noqa: E731
    h, y, dx, da = (f64(rows, cols) for _ in range(4))
    dgate, dscale, dshift, dw = (f64(S, cols) for _ in range(4))
    low = DT[c["x"]]

    def norm(t, kind, stats=None):
        """The normed t and its deviation; with stats = (mean, deviation), by these."""
        if stats is None:
            m = t.mean(1, keepdim=True) if kind == "layer" else 0.0
            stats = m, (((t - m) ** 2).mean(1, keepdim=True) + 1e-5).sqrt()
        return (t - stats[0]) / stats[1], stats

    for k, (r0, n) in enumerate(_starts(c)):
        if n == 0:
            continue
        of = lambda name: x[name].double() if c["shared"] else x[name][k].double()  # noqa: E731
        g = of("gate") if c["gate"] else torch.ones(cols, dtype=torch.float64, device=DEV)
        e, f = of("scale") + (1.0 if c["plus_one"] else 0.0), of("shift")
        w = x["post_weight"].double() if c["post"] else torch.ones_like(g)
        for b0 in range(r0, r0 + n, 16384):
            b = slice(b0, min(b0 + 16384, r0 + n))
            a = x["a"][b].double()
            an, sa = norm(a, c["post"]) if c["post"] else (a, None)
            hb = (c["c"] * x["x"][b].double() + g * (an * w)).to(low).double()  # the stream as it is kept
            hn, sh = norm(hb, c["norm"])
            h[b], y[b] = hb, hn * e + f
            if c["mode"] == "fwd":
                continue
            if c["ckpt"]:
                hn = norm(_kept(hb)[0], c["norm"], sh)[0]
                an = norm(_kept(a)[0], c["post"], sa)[0] if c["post"] else _kept(a)[0]
            dy = x["dy"][b].double()

            def through(up, normed, stats, kind):  # the gradient of a norm's input
                up = up - normed * (up * normed).mean(1, keepdim=True) - (up.mean(1, keepdim=True) if kind == "layer" else 0.0)
                return up / stats[1]

            big = x["dh"][b].double() + through(dy * e, hn, sh, c["norm"])
            dx[b] = c["c"] * big
            da[b] = through(big * g * w, an, sa, c["post"]) if c["post"] else big * g
            dgate[k] += (big * an * w).sum(0)
            dw[k] += (big * g * an).sum(0)
            dscale[k] += (dy * hn).sum(0)
            dshift[k] += dy.sum(0)
    if c["mode"] == "fwd":
        return h, y
    total = lambda t: t.sum(0) if c["shared"] else t  # noqa: E731
    out = {"h": h, "y": y, "dx": dx, "da": da, "dscale": total(dscale), "dshift": total(dshift)}
    if c["gate"]:
        out["dgate"] = total(dgate)
    if c["post"]:
        out["dpost_weight"] = dw.sum(0)
    return out
