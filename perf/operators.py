"""Performance cases of the text tower's operators: packed attention, its learned relative position
bias, and layer norm.

Packed attention takes sequences of different lengths laid one behind the other, causal or not, with
several query heads to a key head: captions encoded or trained without padding, prompts, and single
tokens at the end of a long cache. The bias adds table[head][bucket(key - query)] to its scores. Layer norm
stands before each attention. `draw` spreads further cases over the same ranges.
"""
from __future__ import annotations

import math

import torch

own = False  # False: the operators in elementary torch operations; True: the library's calls

DEV = "cuda"


def _attn(name, mode, H, Hkv, D, lq, lk=None, causal=True, nb=0, R=0, slack=0, qkv=False, api="call"):
    """lq, lk: the sequences' numbers of queries and keys, as texts. slack: rows of each key slot that hold
    nothing yet. qkv: q, k and v are slices of one projection's output."""
    return {"name": name, "op": "attn", "mode": mode, "H": H, "Hkv": Hkv, "D": D, "lq": lq, "lk": lq if lk is None else lk,
            "causal": causal, "nb": nb, "R": R, "slack": slack, "qkv": qkv, "api": api}


def _norm(name, mode, rows, cols, x="bf16", w="f32", bias=True):
    return {"name": name, "op": "norm", "mode": mode, "rows": rows, "cols": cols, "x": x, "w": w, "bias": bias}


CAPTIONS = ("77,120,8,201,163,45,256,99,110,131,180,17,64,152,140,33,77,230,105,111,88,190,61,128,146,173,25,119,"
            "200,94,102,127")


def listed():
    return [
        # The smallest call: one token of one sequence, a short cache; the launches decide.
        _attn("decode-one", "fwd", 16, 4, 64, "1", "700", slack=68),
        # A serving step: single tokens of a batch of requests at different points of their caches.
        _attn("decode-batch", "fwd", 32, 8, 128, ",".join(["1"] * 16),
              "8000,1,511,4097,64,7300,2222,129,6001,3500,900,5555,333,4800,12,7777", slack=200),
        # Captions of a batch of clips encoded without padding, bidirectional, with the bias.
        _attn("captions-encode", "fwd", 16, 16, 64, CAPTIONS, causal=False, nb=32, R=128),
        # The same tower in training: every gradient, the table's too.
        _attn("captions-train", "train", 16, 16, 64, CAPTIONS, causal=False, nb=32, R=128),
        # Longer texts with the bias, causal, in training.
        _attn("texts-bias-train", "train", 12, 12, 64, "2500,1999", nb=32, R=128),
        # Prompts of different lengths, causal, grouped heads.
        _attn("prompts", "fwd", 32, 8, 128, "4096,2731,1023,517,64,1"),
        # A prompt continued in pieces: a few hundred queries at the end of long caches.
        _attn("prompt-continued", "fwd", 32, 8, 128, "512,300", "16384,9001", slack=100),
        # A packed training step through the differentiable form, q, k, v slices of one projection.
        _attn("packed-train", "train", 16, 4, 128, "2048,1500,777,130,33,1", qkv=True, api="autograd"),
        # One long text in training.
        _attn("long-train", "train", 16, 2, 128, "12000"),
        # The norm of one serving step's tokens.
        _norm("norm-tokens", "fwd", 16, 2048, w="bf16"),
        # The norm of a training step over a clip's tokens, weights kept in 32 bits.
        _norm("norm-train", "train", 57856, 1536),
        # Inputs in 32 bits with an odd number of columns.
        _norm("norm-train-odd", "train", 5001, 1155, x="f32"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.3:
        x = rng.choice(["bf16", "bf16", "f32"])
        cols = _log_uniform(rng, 64, 8192)
        if rng.random() < 0.7:
            cols = (cols + 7) // 8 * 8
        rows = _log_uniform(rng, 1, max(2, min(60000, 80_000_000 // cols)))
        return _norm("", rng.choice(["fwd", "train"]), rows, cols, x=x, w=rng.choice(["f32", x]), bias=rng.random() < 0.8)
    D = rng.choice([64, 128])
    Hkv = rng.choice([1, 2, 4, 8, 16])
    G = rng.choice([g for g in (1, 2, 3, 4, 8) if g * Hkv <= 32])
    kind = rng.choice(["decode", "train", "train", "fwd", "bias", "bias"])
    if kind == "decode":
        S = _log_uniform(rng, 1, 24)
        lk = [_log_uniform(rng, 1, 9000) for _ in range(S)]
        lq = [rng.choice([1, 1, 1, 2, 5]) if n > 5 else 1 for n in lk]
        return _attn("", "fwd", G * Hkv, Hkv, D, ",".join(map(str, lq)), ",".join(map(str, lk)), slack=rng.randint(0, 200))
    if kind == "bias":
        S = _log_uniform(rng, 1, 32)
        n = [_log_uniform(rng, 4, 2500 if S <= 2 else 300) for _ in range(S)]
        return _attn("", rng.choice(["fwd", "train"]), min(G * Hkv, 16), min(Hkv, 16) if G * Hkv <= 16 else 16, D if S > 2 else 64,
                     ",".join(map(str, n)), causal=rng.random() < 0.4, nb=rng.choice([8, 32, 37]), R=rng.choice([16, 100, 128, 300]))
    S = _log_uniform(rng, 1, 8)
    n = [_log_uniform(rng, 1, 5000 if S <= 3 else 2500) for _ in range(S)]
    if S > 1 and rng.random() < 0.2:  # a sequence of nothing
        n[rng.randrange(S)] = 0
        n[0] = max(n[0], 1)
    if kind == "fwd" and rng.random() < 0.5:  # continued: fewer queries than keys
        return _attn("", "fwd", G * Hkv, Hkv, D, ",".join(str(min(m, rng.randint(1, 600))) for m in n), ",".join(map(str, n)),
                     slack=rng.randint(0, 70))
    if kind == "train":
        G = min(G, max(1, 16 // Hkv))
    return _attn("", "train" if kind == "train" else "fwd", G * Hkv, Hkv, D, ",".join(map(str, n)), causal=rng.random() < 0.8,
                 qkv=rng.random() < 0.5, api="autograd" if kind == "train" and rng.random() < 0.3 else "call")


def _lens(text):
    return [int(t) for t in text.split(",")]


def _ends(lens):
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    return cu


DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _inputs(c, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    new = lambda *shape: torch.randn(shape, generator=gen, device=DEV)  # noqa: E731
    if c["op"] == "norm":
        xd, wd = DT[c["x"]], DT[c["w"]]
        x = {"x": (new(c["rows"], c["cols"]) * 1.5 + 0.3).to(xd), "w": (1 + 0.2 * new(c["cols"])).to(wd),
             "b": (0.1 * new(c["cols"])).to(wd) if c["bias"] else None}
        if c["mode"] == "train":
            x["dy"] = new(c["rows"], c["cols"]).to(xd)
        return x
    lq, lk = _lens(c["lq"]), _lens(c["lk"])
    cu_q, cu_k = _ends(lq), _ends([n + c["slack"] for n in lk])
    H, Hkv, D = c["H"], c["Hkv"], c["D"]
    if c["qkv"]:
        qkv = new(cu_q[-1], H + 2 * Hkv, D).to(torch.bfloat16)
        q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    else:
        q, k, v = (new(n, h, D).to(torch.bfloat16) for n, h in ((cu_q[-1], H), (cu_k[-1], Hkv), (cu_k[-1], Hkv)))
    dev = lambda t: torch.tensor(t, dtype=torch.int32, device=DEV)  # noqa: E731
    x = {"q": q, "k": k, "v": v, "cu_q": dev(cu_q), "cu_k": dev(cu_k), "len_k": dev(lk) if c["slack"] else None,
         "bias": None, "buckets": None}
    if c["nb"]:
        x["bias"] = new(H, c["nb"]).to(torch.bfloat16)
        # near distances have a bucket each, far ones share buckets that widen with the distance
        d = torch.arange(-c["R"], c["R"] + 1, device=DEV)
        half = c["nb"] if c["causal"] else c["nb"] // 2
        exact = max(1, half // 2)
        n = -d.clamp(max=0) if c["causal"] else d.abs()
        far = exact + torch.floor(torch.log(n.clamp(min=1).double() / exact) / math.log(max(c["R"], exact + 1) / exact) * (half - exact) + 1e-9).long()
        b = torch.where(n < exact, n, far.clamp(max=half - 1))
        x["buckets"] = (b if c["causal"] else b + half * (d > 0)).to(torch.int32)
    if c["mode"] == "train":
        x["do"] = new(cu_q[-1], H, D).to(torch.bfloat16)
    return x


def prepare(c, seed):
    s = {"case": c, **_inputs(c, seed)}
    if c["op"] == "attn" and c["mode"] == "train" and c["api"] == "autograd":
        for n in ("q", "k", "v"):
            s[n] = s[n].detach().requires_grad_(True)
    return s


# --- the operators in elementary operations, 32 bits -----------------------------------------

def _plain_norm(s):
    c = s["case"]
    x, w = s["x"].float(), s["w"].float()
    mean = x.mean(-1)
    xc = x - mean[:, None]
    rstd = torch.rsqrt((xc * xc).mean(-1) + 1e-5)
    xh = xc * rstd[:, None]
    y = xh * w
    if s["b"] is not None:
        y = y + s["b"].float()
    out = (y.to(s["x"].dtype), mean, rstd)
    if c["mode"] == "fwd":
        return out
    dy = s["dy"].float()
    g = dy * w
    dx = (g - g.mean(-1, keepdim=True) - xh * (g * xh).mean(-1, keepdim=True)) * rstd[:, None]
    dw = (dy * xh).sum(0).to(s["w"].dtype)
    return out + (dx.to(s["x"].dtype), dw) + ((dy.sum(0).to(s["w"].dtype),) if s["b"] is not None else ())


def _plain_attention(s):
    c = s["case"]
    H, Hkv, D, G = c["H"], c["Hkv"], c["D"], c["H"] // c["Hkv"]
    mq, mk = max(_lens(c["lq"])), max(_lens(c["lk"]))
    cu_q, cu_k = s["cu_q"].long(), s["cu_k"].long()
    S = cu_q.numel() - 1
    nq = cu_q[1:] - cu_q[:-1]
    nk = cu_k[1:] - cu_k[:-1] if s["len_k"] is None else s["len_k"].long()
    i, j = torch.arange(mq, device=DEV), torch.arange(mk, device=DEV)
    at_q = (cu_q[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)
    at_k = (cu_k[:-1, None] + j).clamp(max=s["k"].shape[0] - 1)

    def rows(t, at):  # [S, key heads, query heads of one x rows, D]
        return t.float()[at].view(S, at.shape[1], Hkv, -1, D).permute(0, 2, 3, 1, 4).reshape(S, Hkv, -1, D)

    q, k, v = rows(s["q"].detach(), at_q), rows(s["k"].detach(), at_k), rows(s["v"].detach(), at_k)
    scale = 1 / math.sqrt(D)
    p = torch.matmul(q, k.transpose(2, 3).contiguous()).mul_(scale).view(S, Hkv, G, mq, mk)
    rel = j[None, None, :] - (i[None, :, None] + (nk - nq)[:, None, None])
    ok = (j[None, None, :] < nk[:, None, None]) & (i[None, :, None] < nq[:, None, None])
    if c["causal"]:
        ok = ok & (rel <= 0)
    bucket = None
    if s["bias"] is not None:
        bucket = s["buckets"].long()[rel.clamp(-c["R"], c["R"]) + c["R"]]
        p += s["bias"].float()[:, bucket].view(Hkv, G, S, mq, mk).permute(2, 0, 1, 3, 4)
    p.masked_fill_(~ok[:, None, None], -math.inf)
    m = p.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), torch.zeros_like(m), m)
    p = p.sub_(m).exp_()
    l = p.sum(-1, keepdim=True)
    lse = torch.where(l > 0, torch.log(l) + m, torch.full_like(l, -math.inf))[..., 0]
    p = p.div_(torch.where(l > 0, l, torch.ones_like(l))).view(S, Hkv, G * mq, mk)
    o = torch.matmul(p, v)

    def back(t, cu, total):  # [S, key heads, x rows, D] to [total, heads, D]
        r = torch.arange(total, device=DEV)
        seq = torch.searchsorted(cu[1:].contiguous(), r, right=True).clamp(max=S - 1)
        n = t.shape[3]
        return t[seq, :, :, (r - cu[seq]).clamp(max=n - 1)].reshape(total, -1, *t.shape[4:])

    Tq, Tk = s["q"].shape[0], s["k"].shape[0]
    out = (back(o.view(S, Hkv, G, mq, D), cu_q, Tq).to(torch.bfloat16), back(lse, cu_q, Tq).t().contiguous())
    if c["mode"] == "fwd":
        return out
    do = rows(s["do"], at_q)
    dv = torch.matmul(p.transpose(2, 3).contiguous(), do)
    ds = torch.matmul(do, v.transpose(2, 3).contiguous())
    ds = ds.sub_((ds * p).sum(-1, keepdim=True)).mul_(p)
    del p
    dq = torch.matmul(ds, k).mul_(scale)
    dk = torch.matmul(ds.transpose(2, 3).contiguous(), q).mul_(scale)
    keys = torch.arange(Tk, device=DEV)
    seq = torch.searchsorted(cu_k[1:].contiguous(), keys, right=True).clamp(max=S - 1)
    real = (keys - cu_k[seq] < nk[seq])[:, None, None]
    out += (back(dq.view(S, Hkv, G, mq, D), cu_q, Tq).to(torch.bfloat16),)
    out += tuple((back(t.view(S, Hkv, 1, mk, D), cu_k, Tk) * real).to(torch.bfloat16) for t in (dk, dv))
    if bucket is not None:
        hot = torch.zeros((bucket.numel(), c["nb"]), device=DEV).scatter_(1, bucket.view(-1, 1), 1.0)
        out += (torch.matmul(ds.view(S, H, mq, mk).transpose(0, 1).reshape(H, -1), hot).to(torch.bfloat16),)
    return out[:1] + out[2:] if c["api"] == "autograd" else out


# --- one pass ----------------------------------------------------------------------------------

def _descriptor(s):
    import paper_2501_08453_amd as vc
    c = s["case"]
    lq, lk = _lens(c["lq"]), _lens(c["lk"])
    return vc.make_packed_desc(len(lq), c["H"], c["Hkv"], c["D"], s["q"].shape[0], s["k"].shape[0], max(lq), max(lk) + c["slack"],
                               causal=c["causal"], num_buckets=c["nb"], max_distance=c["R"])


def _own(s):
    import paper_2501_08453_amd as vc
    c = s["case"]
    if c["op"] == "norm":
        out = vc.layer_norm_fwd(s["x"], s["w"], s["b"])
        if c["mode"] == "fwd":
            return out
        dx, dw, db = vc.layer_norm_bwd(s["dy"], s["x"], s["w"], s["b"], out[1], out[2])
        return out + (dx, dw) + ((db,) if db is not None else ())
    desc = _descriptor(s)
    kw = {"len_k": s["len_k"], "bias": s["bias"], "buckets": s["buckets"]}
    if c["mode"] == "train" and c["api"] == "autograd":
        o = vc.packed_attention(s["q"], s["k"], s["v"], desc, s["cu_q"], s["cu_k"], **kw)
        return (o.detach(),) + torch.autograd.grad(o, (s["q"], s["k"], s["v"]), s["do"])
    o, lse = vc.packed_fwd(s["q"], s["k"], s["v"], desc, s["cu_q"], s["cu_k"], **kw)
    if c["mode"] == "fwd":
        return o, lse
    g = vc.packed_bwd(s["q"], s["k"], s["v"], o, lse, s["do"], desc, s["cu_q"], s["cu_k"], **kw)
    return (o, lse) + tuple(t for t in g if t is not None)


def run(s):
    if own:
        return _own(s)
    return _plain_norm(s) if s["case"]["op"] == "norm" else _plain_attention(s)


def work(c):
    train = c["mode"] == "train"
    if c["op"] == "norm":
        n, xb, wb = c["rows"] * c["cols"], (2 if c["x"] == "bf16" else 4), (2 if c["w"] == "bf16" else 4)
        params = c["cols"] * wb * (2 if c["bias"] else 1)
        return {"bytes": n * xb * (4 if train else 2) + 8 * c["rows"] + params * (2 if train else 1), "flops": n * (19 if train else 8)}
    lq, lk = _lens(c["lq"]), _lens(c["lk"])
    H, Hkv, D = c["H"], c["Hkv"], c["D"]
    pairs = 0
    for n, m in zip(lq, lk):
        if c["causal"]:  # row i sees keys 0 .. i + m - n
            full = min(n, m)
            pairs += full * (m - full) + full * (full + 1) // 2
        else:
            pairs += n * m
    tq, tk = sum(lq), sum(lk)
    table = H * c["nb"] * 2
    b = 4 * tq * H * D + 4 * tk * Hkv * D + 4 * tq * H + table
    if train:
        b += 4 * tq * H * D + 4 * tk * Hkv * D + table
    return {"bytes": b, "flops": pairs * H * D * (14 if train else 4)}


# --- the same results in 64 bits, from the definitions -----------------------------------------

def exact(c, seed):
    x = _inputs(c, seed)
    if c["op"] == "norm":
        x = {n: None if t is None else t.double() for n, t in x.items()}
        var, mean = torch.var_mean(x["x"], -1, correction=0, keepdim=True)
        rstd = (var + 1e-5) ** -0.5
        n = (x["x"] - mean) * rstd
        out = [n * x["w"] + (0 if x["b"] is None else x["b"]), mean[:, 0], rstd[:, 0]]
        if c["mode"] == "train":
            g = x["dy"] * x["w"]
            k = c["cols"]
            out += [rstd / k * (k * g - g.sum(-1, keepdim=True) - n * (g * n).sum(-1, keepdim=True)), (x["dy"] * n).sum(0)]
            out += [] if x["b"] is None else [x["dy"].sum(0)]
        return tuple(out)
    train = c["mode"] == "train"
    lq, lk = _lens(c["lq"]), _lens(c["lk"])
    if work(c)["flops"] > 4e13:
        return None
    cu_q, cu_k = _ends(lq), _ends([n + c["slack"] for n in lk])
    H, Hkv, D = c["H"], c["Hkv"], c["D"]
    zero = lambda *shape: torch.zeros(shape, dtype=torch.float64, device=DEV)  # noqa: E731
    o, lse = zero(cu_q[-1], H, D), zero(H, cu_q[-1])
    dq, dk, dv, db = zero(cu_q[-1], H, D), zero(cu_k[-1], Hkv, D), zero(cu_k[-1], Hkv, D), zero(H, max(1, c["nb"]))
    scale = D ** -0.5
    for n, m, a, b in zip(lq, lk, cu_q, cu_k):
        if n == 0:
            continue
        step = max(1, (1 << 26) // max(1, m))
        for r0 in range(0, n, step):
            r1 = min(n, r0 + step)
            gap = torch.arange(m, device=DEV)[None, :] - torch.arange(r0 + m - n, r1 + m - n, device=DEV)[:, None]
            shut = gap > 0 if c["causal"] else torch.zeros_like(gap, dtype=torch.bool)
            which = None if x["bias"] is None else x["buckets"].long()[gap.clamp(-c["R"], c["R"]) + c["R"]]
            for h in range(H):
                kv = h // (H // Hkv)
                qq, kk, vv = x["q"][a + r0:a + r1, h].double(), x["k"][b:b + m, kv].double(), x["v"][b:b + m, kv].double()
                sc = (qq @ kk.t().contiguous()) * scale
                if which is not None:
                    sc += x["bias"][h].double()[which]
                sc = sc.masked_fill_(shut, -math.inf)
                z = torch.logsumexp(sc, -1)
                lse[h, a + r0:a + r1] = z
                pr = torch.exp(sc - z[:, None]).nan_to_num_(0.0)
                o[a + r0:a + r1, h] = pr @ vv
                if train:
                    dd = x["do"][a + r0:a + r1, h].double()
                    dv[b:b + m, kv] += pr.t().contiguous() @ dd
                    dp = dd @ vv.t().contiguous()
                    grad = pr * (dp - (pr * dp).sum(-1, keepdim=True))
                    dq[a + r0:a + r1, h] = grad @ kk * scale
                    dk[b:b + m, kv] += grad.t().contiguous() @ qq * scale
                    if which is not None:
                        db[h] += torch.bincount(which.reshape(-1), grad.reshape(-1), minlength=c["nb"])
    out = (o, lse) + ((dq, dk, dv) if train else ()) + ((db,) if train and c["nb"] else ())
    return out[:1] + out[2:] if train and c["api"] == "autograd" else out
