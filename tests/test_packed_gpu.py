"""Packed attention on the GPU against the fp64 oracle, on every element, and what holds beyond parity: rows that are
left alone, strides, streams, graphs, reproducibility."""
import numpy as np
import pytest

from oracle import ref_tower as T
from parity_util import bf16_values, log

pytestmark = pytest.mark.gpu


def _vc():
    import paper_2501_08453_amd as vc
    return vc


def lse_bound(x, D, n_keys, scale, lse):
    """|LSE - exact| <= ...: the products are exact in fp32 and summed in D / 16 steps of the matrix cores (each a sum of
    16: at most D additions, relative 2^-24 of the sum of magnitudes A = scale * max |q|.|k| + |bias|), the probabilities
    are summed unrounded in fp32 (32 of a lane, one addition per tile, one across lanes), and the exponent's and the
    logarithm's argument and result are rounded (a few 2^-24 of their magnitude; 2^-21 covers the hardware's)."""
    a = scale * np.abs(x["q"]).max() * np.abs(x["k"]).max() * D / 4 + (np.abs(x["bias"][np.abs(x["bias"]) < 65536]).max(initial=0.0) if x.get("bias") is not None else 0.0)
    return a * D * 2.0 ** -24 + (n_keys / 64 + 40) * 2.0 ** -24 + 2.0 ** -21 * max(1.0, np.abs(lse[np.isfinite(lse)]).max(initial=0.0))


def bounds(x, eps, **over):
    """(oracle's results, bound per element of o, dq, dk, dv, dbias). Independent roundings to bf16, each off by a step /
    sqrt(12) with a step at most 2^-7 of the value, add up like a random walk: six standard deviations of it. They are
    P_ij in O = sum_j P_ij v_j and dV_j = sum_i P_ij dO_i; dS_ij in dQ and dK; and O in D_i = <dO_i, O_i>, which moves
    all dS_ij = P_ij (dP_ij - D_i) of its row together, so dQ_i by c P_ij K_j summed over the keys and a bucket's
    dbias by the row's probability of it. To these come half a step of the result (2^-8 relative) and the fp32 part:
    P off by at most eps (relative), dP and D by the rounding of D products."""
    D = x["q"].shape[-1]
    c = 1 / np.sqrt(D) if x["scale"] is None else x["scale"]
    u = 2.0 ** -7 / np.sqrt(12)
    e1 = 2.0 ** -23 * D * np.abs(x["dout"]).max() * np.abs(x["v"]).max() * D / 4
    var = {n: np.zeros(x[m].shape) for n, m in (("o", "q"), ("dq", "q"), ("dk", "k"), ("dv", "k"))}
    fix = {n: np.zeros(t.shape) for n, t in var.items()}
    rows_d, rows_ds = [], []

    def each(rows, keys, h, g, p, ds):
        Q, K, V, dO = x["q"][rows, h], x["k"][keys, g], x["v"][keys, g], x["dout"][rows, h]
        sd = (u * u) * (dO ** 2 * (p @ V) ** 2).sum(1)  # variance of D_i
        ads = p * e1 + eps * np.abs(ds)
        var["o"][rows, h] += u * u * (p ** 2 @ V ** 2)
        fix["o"][rows, h] += 2 * eps * (p @ np.abs(V))
        var["dv"][keys, g] += u * u * (p.T ** 2 @ dO ** 2)
        fix["dv"][keys, g] += eps * (p.T @ np.abs(dO))
        var["dq"][rows, h] += c * c * (sd[:, None] * (p @ K) ** 2 + u * u * (ds ** 2 @ K ** 2))
        fix["dq"][rows, h] += c * (ads @ np.abs(K))
        var["dk"][keys, g] += c * c * ((p ** 2 * sd[:, None]).T @ Q ** 2 + u * u * (ds.T ** 2 @ Q ** 2))
        fix["dk"][keys, g] += c * (ads.T @ np.abs(Q))
        rows_d.append((rows, h, sd))
        rows_ds.append((h, ads.sum()))

    r = oracle(x, each=each, **over)
    tol = {n: 6 * np.sqrt(var[n]) + fix[n] + 2.0 ** -8 * np.abs(r[n]) + 1e-30 for n in var}
    if "dbias" in r:
        vb = np.zeros(r["dbias"].shape)
        fb = np.zeros(r["dbias"].shape[0])
        for rows, h, sd in rows_d:
            vb[h] += (sd[:, None] * r["weight"][rows, h] ** 2).sum(0)
        for h, a in rows_ds:
            fb[h] += a
        tol["dbias"] = 6 * np.sqrt(vb) + fb[:, None] + 2.0 ** -8 * np.abs(r["dbias"]) + 1e-30
    return r, tol


def make(seed, lq, lk, H, Hkv, D, causal=False, nb=0, R=0, scale=None, slack=(0, 0), outside=(0, 0), strided=False, low=None):
    """Inputs on the GPU and their exact values on the host. slack: rows of each query (key) slot behind its length,
    holding NaN; outside: rows before the first and behind the last slot."""
    import torch
    g = torch.Generator().manual_seed(seed)
    f = {}
    x = {"causal": causal, "scale": scale}
    for n, lens, sl in (("q", lq, slack[0]), ("k", lk, slack[1])):
        cu = np.cumsum([outside[0]] + [m + sl for m in lens]).astype(np.int32)
        x["cu_" + n], x["len_" + n] = cu, (np.array(lens, np.int32) if sl else None)
        f["T" + n] = int(cu[-1]) + outside[1]
    bf = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16)  # noqa: E731
    shapes = {"q": (f["Tq"], H, D), "k": (f["Tk"], Hkv, D), "v": (f["Tk"], Hkv, D), "dout": (f["Tq"], H, D)}
    host = {n: bf(*s) for n, s in shapes.items()}
    for n, t in host.items():
        c = "q" if n in ("q", "dout") else "k"
        take = torch.zeros(t.shape[0], dtype=torch.bool)
        for s in range(len(lq)):
            a = int(x["cu_" + c][s])
            take[a:a + (lq if c == "q" else lk)[s]] = True
        t[~take] = float("nan")
    if nb:
        b = bf(H, nb)
        if low is not None:
            b[:, ::2] = low
        host["bias"] = b
        x["buckets"] = torch.randint(0, nb, (2 * R + 1,), generator=g, dtype=torch.int32)
    for n, t in host.items():
        v = t.double().numpy()
        x[n] = np.where(np.isnan(v), 0.0, v) if n != "bias" else v
    dev = {}
    for n, t in host.items():
        if strided and n in ("q", "k", "v"):  # tokens further apart than their heads
            wide = torch.full((t.shape[0], t.shape[1] + 3, D), float("nan"), dtype=torch.bfloat16, device="cuda")
            wide[:, 1:1 + t.shape[1]] = t.cuda()
            dev[n] = wide[:, 1:1 + t.shape[1]]
        else:
            dev[n] = t.cuda()
    for n in ("cu_q", "cu_k", "len_q", "len_k", "buckets"):
        t = x.get(n)
        dev[n] = None if t is None else torch.as_tensor(t).cuda()
    if nb:
        x["buckets"] = x["buckets"].numpy()
    mx = lambda lens, sl: max(max(m + sl for m in lens), 1)  # noqa: E731
    desc = _vc().make_packed_desc(len(lq), H, Hkv, D, f["Tq"], f["Tk"], mx(lq, slack[0]), mx(lk, slack[1]), causal, scale, nb, R)
    return x, dev, desc


def _kw(d):
    return dict(len_q=d["len_q"], len_k=d["len_k"], bias=d.get("bias"), buckets=d["buckets"])


def run(d, desc, **kw):
    vc = _vc()
    o, lse = vc.packed_fwd(d["q"], d["k"], d["v"], desc, d["cu_q"], d["cu_k"], **_kw(d))
    dq, dk, dv, db = vc.packed_bwd(d["q"], d["k"], d["v"], o, lse, d["dout"], desc, d["cu_q"], d["cu_k"], **_kw(d))
    return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv, **({"dbias": db} if db is not None else {})}


def oracle(x, **over):
    y = {n: x[n] for n in ("q", "k", "v", "dout", "cu_q", "cu_k", "len_q", "len_k", "causal", "scale", "bias", "buckets") if n in x}
    return T.packed_attention(**{**y, **over})


def check(x, dev, desc):
    import torch
    out = run(dev, desc)
    torch.cuda.synchronize()
    D = x["q"].shape[-1]
    c = 1 / np.sqrt(D) if x["scale"] is None else x["scale"]
    eps = 2 * lse_bound(x, D, desc.max_k, c, np.zeros(1)) + 2.0 ** -20  # of exp(s - LSE)
    r, tol = bounds(x, eps)
    lse = out["lse"].double().cpu().numpy()
    assert np.array_equal(np.isneginf(lse), np.isneginf(r["lse"]))
    fin = np.isfinite(r["lse"])
    if fin.any():
        off = np.abs(lse[fin] - r["lse"][fin]).max()
        bound = lse_bound(x, D, desc.max_k, c, r["lse"])
        log("   LSE off %.2e, bound %.2e" % (off, bound))
        assert off <= bound
    for n in tol:
        off = np.abs(bf16_values(out[n]) - r[n]) / tol[n]
        log("   %-5s off / bound %.3f" % (n, off.max(initial=0.0)))
        assert off.max(initial=0.0) <= 1, n
    for n in ("o", "dq", "dk", "dv"):
        # Rows that take no part, see no key, or are seen by no query: exactly zero. (Not every zero of the oracle: dq of a
        # row with one key is P (dP - D) K with D a sum of its own, in another order than dP's.)
        zero = np.isneginf(r["lse"].T) if n in ("o", "dq") else np.all(r["dv"] == 0, axis=-1)
        assert (bf16_values(out[n])[zero] == 0).all(), n
    return out


LENS = {
    "ones": ([1], [1]),
    "one-token-long-cache": ([1, 1, 1], [700, 64, 1]),
    "few-tokens": ([5, 2, 3, 17], [1030, 2, 129, 65]),
    "edges": ([31, 32, 33, 63, 64, 65], [31, 32, 33, 63, 64, 65]),
    "blocks": ([255, 257, 300], [255, 257, 300]),
    "empty": ([0, 40, 0, 1, 0], [0, 40, 7, 0, 0]),
    "more-queries": ([100, 70], [30, 69]),
    "continued": ([70, 33], [400, 290]),
}


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("lens", LENS)
def test_lengths(lens, causal, D):
    lq, lk = LENS[lens]
    check(*make(11, lq, lk, 4, 2, D, causal))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("lens", ["ones", "few-tokens", "edges", "blocks", "empty", "more-queries", "continued"])
@pytest.mark.parametrize("nb,R", [(32, 128), (5, 0), (1, 17), (40, 512)])
def test_bias(nb, R, lens, causal, D):
    if R == 512 and lens != "few-tokens" and lens != "continued":
        pytest.skip("short lengths reach a few of its distances only: covered at the smaller ones")
    lq, lk = LENS[lens]
    check(*make(12, lq, lk, 3, 3, D, causal, nb, R))


@pytest.mark.parametrize("H,Hkv", [(1, 1), (8, 1), (6, 2), (5, 5), (16, 8)])
def test_heads(H, Hkv):
    check(*make(13, [130, 1, 47], [130, 1, 47], H, Hkv, 64, True, 8, 20))
    check(*make(14, [1, 3], [300, 77], H, Hkv, 128, True))


@pytest.mark.parametrize("D", [64, 128])
def test_lengths_inside_slots_rows_outside_and_strides(D):
    """Padded slots whose padding holds NaN, rows outside every slot, tokens further apart than their heads."""
    x, d, desc = make(15, [20, 0, 65], [30, 4, 65], 4, 2, D, True, 8, 9, slack=(7, 66), outside=(5, 9), strided=True)
    out = check(x, d, desc)  # outputs made by the helpers: rows outside are 0, -inf (the oracle's)
    import torch
    vc = _vc()
    given = {n: torch.full_like(out[n], 7.0) for n in ("o", "lse", "dq", "dk", "dv")}
    vc.packed_fwd(d["q"], d["k"], d["v"], desc, d["cu_q"], d["cu_k"], out=given["o"], lse=given["lse"], **_kw(d))
    vc.packed_bwd(d["q"], d["k"], d["v"], out["o"], out["lse"], d["dout"], desc, d["cu_q"], d["cu_k"], dq=given["dq"], dk=given["dk"],
                  dv=given["dv"], **_kw(d))
    for n, t in given.items():
        rows = t.t() if n == "lse" else t
        ref = out[n].t() if n == "lse" else out[n]
        a, b = (int(d["cu_k" if n in ("dk", "dv") else "cu_q"][i]) for i in (0, -1))
        assert torch.equal(rows[a:b], ref[a:b]), n
        assert (rows[:a] == 7).all() and (rows[b:] == 7).all(), n


@pytest.mark.parametrize("low", [float("-inf"), float(np.finfo(np.float32).min), -70000.0])
def test_bias_that_shuts_out(low):
    """Every other bucket shut out: some rows keep no key."""
    check(*make(16, [90, 3], [90, 3], 2, 2, 64, True, 4, 40, low=low))
    check(*make(17, [90, 3], [90, 3], 2, 2, 128, False, 1, 40, low=low))  # nothing left at all


def test_bucket_outside_the_table_and_large_bias():
    import torch
    x, d, desc = make(18, [70], [70], 2, 1, 64, False, 4, 12)
    x["buckets"][3:6], x["buckets"][20] = -1, 4
    d["buckets"] = torch.from_numpy(x["buckets"]).cuda()
    check(x, d, desc)


@pytest.mark.parametrize("scale", [1.0, 2.0 ** -24, 3.0])
def test_scales(scale):
    check(*make(19, [100, 5], [100, 50], 2, 1, 64, True, 6, 30, scale=scale))


def test_smallest_and_largest_plain_scale():
    for s in (2.0 ** -60, 8.0):
        check(*make(20, [70, 5], [70, 50], 2, 1, 128, True, scale=s))


def test_many_sequences():
    g = np.random.default_rng(5)
    lens = [int(n) for n in g.integers(0, 80, 150)]
    check(*make(21, lens, lens, 2, 2, 64, False, 12, 33))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("nb", [0, 16])
def test_longer_sequences(nb, causal, D):
    """Slots of more than 2,048 rows (wider blocks), a sequence that ends inside one, and a short one beside it."""
    check(*make(28, [2100, 70, 1], [2100, 300, 1], 2, 1 if nb == 0 else 2, D, causal, nb, 100 if nb else 0))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("nb", [0, 12])
@pytest.mark.parametrize("lq,H,Hkv", [([1, 1, 1, 1, 0], 8, 2), ([4, 4, 4, 4, 4], 16, 2), ([7, 1, 3, 2, 5], 4, 4), ([33, 1, 40, 8, 2], 4, 2)])
def test_few_rows_behind_long_caches(lq, H, Hkv, nb, D):
    """Single and drafted tokens, the rows of a group's heads together (up to 32, and more), keys over several workgroups,
    slots longer than what they hold (NaN behind it), in both directions."""
    x, d, desc = make(29, lq, [9000, 64, 1, 2049, 333], H, Hkv if nb == 0 else H, D, True, nb, 60 if nb else 0, slack=(2, 70), outside=(0, 3))
    check(x, d, desc)


@pytest.mark.parametrize("D,nb", [(64, 0), (64, 9), (128, 0)])
@pytest.mark.parametrize("long", [700, 3000])
def test_one_long_sequence_among_many_short(long, D, nb):
    """Blocks numbered through and looked up; with the longer one its keys shared by several workgroups."""
    g = np.random.default_rng(6)
    lens = [int(n) for n in g.integers(0, 20, 300)]
    lens[137] = long
    x, d, desc = make(30, lens, lens, 2, 2, D, True, nb, 30 if nb else 0, outside=(3, 200))
    check(x, d, desc)
    more = [min(n, 400) for n in lens]  # and keys before the queries', more than 64 x 64 sequences beside
    check(*make(31, more + [1] * 4000, [n + 3 for n in more] + [1] * 4000, 2, 1, D, False))


@pytest.mark.parametrize("D,nb", [(64, 0), (64, 12), (128, 0)])
def test_few_keys_of_unequal_weight(D, nb):
    """Gradients of texts of a few tokens, where dS is much smaller than D = <dO, O>: dQ and dK are off (2-norm) by no more
    than two roundings to bf16 (dS and the result: relative rms at most 2^-8 / sqrt(3) each, where a value stands
    at the bottom of its binade), 2^-8 sqrt(2 / 3) = 0.0032, and 0.0003 for the fp32 part; not by the rounding of O in D."""
    lens = [n for n in range(2, 7)] * 20
    for causal in (False, True):
        x, d, desc = make(33, lens, lens, 2, 2, D, causal, nb, 4 if nb else 0)
        x["bias"] = x["bias"] * 2 if nb else None  # logits of a spread of 2 and more
        if nb:
            d["bias"] = d["bias"] * 2
        out = run(d, desc)
        r = T.packed_attention(**{n: x[n] for n in ("q", "k", "v", "dout", "cu_q", "cu_k", "causal") if n in x},
                               bias=x["bias"], buckets=x.get("buckets"))
        for n in ("dq", "dk"):
            off = np.linalg.norm(bf16_values(out[n]) - r[n]) / np.linalg.norm(r[n])
            log("   %s %.4f" % (n, off))
            assert off <= 0.0035, n


def test_reproducible():
    """Two runs agree bitwise."""
    import torch
    x, d, desc = make(22, [300, 77, 512], [300, 77, 512], 4, 2, 128, True, 8, 50)
    a, b = run(d, desc), run(d, desc)
    for n in a:
        assert torch.equal(a[n], b[n]), n


def test_another_stream_and_two_at_once():
    import torch
    cases = [make(23 + i, [200 + 31 * i, 5], [200 + 31 * i, 5], 4, 2, 64, True, 8, 20) for i in range(2)]
    want = [run(d, desc) for _, d, desc in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [None, None]
    for _ in range(3):
        for i, s in enumerate(streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got[i] = run(cases[i][1], cases[i][2])
        torch.cuda.synchronize()
        for w, h in zip(want, got):
            assert all(torch.equal(w[n], h[n]) for n in w)


def test_graph_replays():
    """Forward and backward captured, replayed with new values in the inputs, eager work between the replays; two graphs
    with workspaces of their own."""
    import torch
    vc = _vc()
    x, d, desc = make(25, [130, 1, 64], [130, 1, 64], 4, 2, 64, True, 8, 20)
    x2, d2, desc2 = make(26, [1, 2], [900, 130], 8, 2, 128, True)
    graphs, outs = [], []
    for dd, de in ((d, desc), (d2, desc2)):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run(dd, de)
        torch.cuda.current_stream().wait_stream(side)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(run(dd, de))
        graphs.append(g)
    for rep in range(4):
        for dd in (d, d2):
            for n in ("q", "k", "v", "dout"):
                dd[n].copy_(torch.randn(dd[n].shape, device="cuda"))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for (dd, de), got in zip(((d, desc), (d2, desc2)), outs):
            want = run(dd, de)
            torch.cuda.synchronize()
            assert all(torch.equal(want[n], got[n]) for n in want), rep


def test_differentiable_form():
    """Gradients of slices of one projection's output, with and without the bias's."""
    import torch
    vc = _vc()
    x, d, desc = make(27, [90, 33], [90, 33], 4, 2, 64, True, 8, 20)
    qkv = torch.cat([d["q"], d["k"], d["v"]], 1).requires_grad_(True)
    bias = d["bias"].clone().requires_grad_(True)
    o = vc.packed_attention(qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], desc, d["cu_q"], d["cu_k"], bias=bias, buckets=d["buckets"])
    o.backward(d["dout"])
    want = run(d, desc)
    assert torch.equal(o, want["o"]) and torch.equal(bias.grad, want["dbias"])
    assert torch.equal(qkv.grad, torch.cat([want["dq"], want["dk"], want["dv"]], 1))
    frozen = vc.packed_attention(qkv[:, :4], qkv[:, 4:6], qkv[:, 6:], desc, d["cu_q"], d["cu_k"], bias=d["bias"], buckets=d["buckets"])
    assert torch.equal(torch.autograd.grad(frozen, qkv, d["dout"])[0], qkv.grad)


def test_offsets_past_32_bits():
    """Slots whose rows start behind 2^31 elements of every tensor: a second sequence of 70 queries and 130 keys there, 3 rows
    of each in the first one's long slot."""
    import torch
    vc = _vc()
    H, D, n = 32, 128, 560_000
    assert (n - 1000) * H * D > 2 ** 31
    g = torch.Generator().manual_seed(40)
    cu = torch.tensor([0, n - 1000, n], dtype=torch.int32).cuda()
    lens = {"q": [3, 70], "k": [3, 130]}
    big = {m: torch.empty((n, H, D), dtype=torch.bfloat16, device="cuda") for m in ("q", "k", "v", "dout")}
    small = {}
    for m, t in big.items():
        a, b = lens["q" if m in ("q", "dout") else "k"]
        small[m] = torch.randn((a + b, H, D), generator=g).to(torch.bfloat16)
        t[:a] = small[m][:a].cuda()
        t[n - 1000:n - 1000 + b] = small[m][a:].cuda()
    desc = vc.make_packed_desc(2, H, H, D, n, n, n - 1000, n - 1000, causal=True)
    kw = {"len_q": torch.tensor(lens["q"], dtype=torch.int32).cuda(), "len_k": torch.tensor(lens["k"], dtype=torch.int32).cuda()}
    o, lse = vc.packed_fwd(big["q"], big["k"], big["v"], desc, cu, cu, **kw)
    dq, dk, dv, _ = vc.packed_bwd(big["q"], big["k"], big["v"], o, lse, big["dout"], desc, cu, cu, **kw)
    x = {m: t.double().numpy() for m, t in small.items()}
    x.update(cu_q=np.array([0, 3, 73]), cu_k=np.array([0, 3, 133]), len_q=None, len_k=None, causal=True, scale=None)
    r, tol = bounds(x, 2 * lse_bound(x, D, 130, 1 / np.sqrt(D), np.zeros(1)) + 2.0 ** -20)
    for m, t in (("o", o), ("dq", dq), ("dk", dk), ("dv", dv)):
        a, b = lens["q" if m in ("o", "dq") else "k"]
        got = bf16_values(torch.cat([t[:a], t[n - 1000:n - 1000 + b]]))
        off = float((np.abs(got - r[m]) / tol[m]).max())
        log("   %-3s off / bound %.3f" % (m, off))
        assert off <= 1, m
        assert not t[a:n - 1000].any() and not t[n - 1000 + b:].any(), m  # rows of the slots behind their lengths
    # one token each at the end of the same caches
    one = vc.make_packed_desc(2, H, H, D, 2, n, 1, n - 1000, causal=True)
    ends = torch.tensor([0, 1, 2], dtype=torch.int32).cuda()
    o1, _ = vc.packed_fwd(torch.cat([big["q"][2:3], big["q"][n - 1000 + 69:n - 1000 + 70]]), big["k"], big["v"], one, ends, cu, len_k=kw["len_k"])
    got, last = bf16_values(o1), [2, 72]
    assert (np.abs(got - r["o"][last]) <= tol["o"][last]).all()


@pytest.mark.parametrize("given", ["out", "lse"])
def test_one_output_given(given):
    """Rows before the first and behind the last slot: left as they were in the output that is given, 0 (lse: -inf) in the one
    that is not, whatever its memory held before."""
    import torch
    vc = _vc()
    x, d, desc = make(41, [20, 0, 65], [30, 4, 65], 4, 2, 64, True, slack=(7, 0), outside=(5, 9))
    want = dict(zip(("out", "lse"), vc.packed_fwd(d["q"], d["k"], d["v"], desc, d["cu_q"], d["cu_k"], **_kw(d))))
    kept = torch.full_like(want[given], 7.0)
    torch.cuda.synchronize()
    used = [torch.full_like(t, 3.0) for t in want.values() for _ in range(4)]  # what the allocator hands out next
    del used
    got = dict(zip(("out", "lse"), vc.packed_fwd(d["q"], d["k"], d["v"], desc, d["cu_q"], d["cu_k"], **{given: kept}, **_kw(d))))
    assert got[given] is kept
    a, b = int(x["cu_q"][0]), int(x["cu_q"][-1])
    for n, t in got.items():
        rows, ref = (t.t(), want[n].t()) if n == "lse" else (t, want[n])
        assert torch.equal(rows[a:b], ref[a:b]), n
        assert all((r == 7).all() if n == given else torch.equal(r, f) for r, f in ((rows[:a], ref[:a]), (rows[b:], ref[b:]))), n


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("R", [129, 300, 512])
def test_distances_of_the_wide_table(R, causal, D):
    """More queries and keys than any distance with a bucket of its own, on both sides, in the kernels for distances past 128; a
    block of queries behind a longer cache, and fewer distances than R."""
    check(*make(42, [1200, 90, 40], [1200, 1500, 40], 2, 2, D, causal, 8, R))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("nb", [256, 257, 1024])
def test_large_tables(nb, D):
    """Tables whose values are loaded along with the bucket numbers (up to 256), and larger ones."""
    check(*make(43, [600, 3], [600, 70], 2, 2, D, False, nb, 512))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
def test_bias_above_the_limit(causal, D):
    """Entries above 65536, +inf among them, count as 65536. Scores exact (whole q . k, scale 1). LSE of about 65536 is held in fp32,
    half a step of which is h = 2^-8: rounded itself, with its base and the sum's logarithm in log2 units (h ln 2 each), and
    by the constants log2 e and ln 2 (h each); P in the backward has the error of LSE, that of LSE in log2 units (h ln 2),
    and far tiles' that of the bias in log2 units (h ln 2): 3 + 4 ln 2 < 6 of h in all."""
    import torch
    x, d, desc = make(44, [70, 9], [70, 200], 2, 1, D, causal, 4, 12, scale=1.0)
    for n in ("q", "k"):
        x[n] = np.clip(np.round(x[n]), -1, 1)
        d[n] = torch.from_numpy(x[n]).to(torch.bfloat16).cuda()
    d["bias"][:, 1], d["bias"][0, 2], d["bias"][1, 2] = 70000.0, float("inf"), 65536.0
    x["bias"] = d["bias"].double().cpu().numpy()
    x["buckets"][12] = 0  # a causal first row sees no large one
    d["buckets"] = torch.from_numpy(x["buckets"]).cuda()
    out = run(d, desc)
    eps = 6 * 2.0 ** -8
    r, tol = bounds(x, eps)
    assert (r["lse"] > 65000).any() and (not causal or (r["lse"] < 100).any())
    assert np.abs(out["lse"].double().cpu().numpy() - r["lse"]).max() <= eps
    for n in tol:
        off = np.abs(bf16_values(out[n]) - r[n]) / tol[n]
        log("   %-5s off / bound %.3f" % (n, off.max()))
        assert off.max() <= 1, n


@pytest.mark.parametrize("given", ["out", "lse"])
@pytest.mark.parametrize("D", [64, 128])
def test_one_output_given_to_a_single_token_step(given, D):
    """The same in the few-row kernel, with keys shared by several workgroups."""
    import torch
    vc = _vc()
    x, d, desc = make(45, [1, 0, 2], [5000, 4, 900], 8, 2, D, True, outside=(3, 40))
    want = dict(zip(("out", "lse"), vc.packed_fwd(d["q"], d["k"], d["v"], desc, d["cu_q"], d["cu_k"], **_kw(d))))
    kept = torch.full_like(want[given], 7.0)
    got = dict(zip(("out", "lse"), vc.packed_fwd(d["q"], d["k"], d["v"], desc, d["cu_q"], d["cu_k"], **{given: kept}, **_kw(d))))
    a, b = int(x["cu_q"][0]), int(x["cu_q"][-1])
    for n, t in got.items():
        ref = want[n].clone()
        if n == given:
            (ref.t() if n == "lse" else ref)[:a] = 7
            (ref.t() if n == "lse" else ref)[b:] = 7
        assert torch.equal(t, ref), n
