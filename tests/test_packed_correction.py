"""The correction of D = <dO, O> by the row sums of dS, in packed attention's backward: over rows of more than 64 keys the
rounding of O in D moves all dS of its row by P, which dK and the bias gradient must not show. Sharp rows
(softmax scale 2), where dS is much smaller than D; errors by their 2-norm. A simulation on the CPU shows that the bounds
hold with the correction and fail without it, with its sign turned, or with the sum over half of the keys."""
import numpy as np
import pytest

from oracle import ref_tower as T
from parity_util import bf16_values, log

SCALE, R, NB = 2.0, 20, 4
U2 = 2.0 ** -16 / 3  # mean square of a rounding to bf16, relative: half a step is at most 2^-8
# P and dS in fp32: scores of up to 110, 160 in log2 units, formed in up to 8 roundings of 2^-24, and as much for LSE
EPS = 2 * 8 * 160 * 2.0 ** -24

# name: (queries, keys), unsplit and with a row block's keys shared by several workgroups in the dQ pass
LENS = {"one": ([300, 130], [300, 130]), "shared": ([64, 20], [4000, 1200])}
H = 4


def bf16(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


def inputs(lens, causal, D, bias, seed=50):
    g = np.random.default_rng(seed)
    lq, lk = LENS[lens]
    x = {n: bf16(g.standard_normal((sum(t), H, D))) for n, t in (("q", lq), ("k", lk), ("v", lk), ("dout", lq))}
    x.update(cu_q=np.cumsum([0] + lq).astype(np.int32), cu_k=np.cumsum([0] + lk).astype(np.int32), causal=causal, scale=SCALE)
    if bias:
        x.update(bias=bf16(g.standard_normal((H, NB))), buckets=g.integers(0, NB, 2 * R + 1).astype(np.int32))
    return x


def reference(x, sim=None):
    """(oracle's results, bound of the error's 2-norm for dq and dk, of every element for dbias). Roundings: dS and the
    result; in dq also O in D, which moves dq_i by c sum_j P_ij K_j for each. dbias sums dS in fp32: the result's
    rounding (at most 2^-8), and P dP as D corrected, whose fp32 sums of D products of unit variance are off by at most about
    2^-24 D for the row. sim(rows, keys, h, g, p): called for every (sequence, head)."""
    var, fix = {"dq": 0.0, "dk": 0.0}, {"dq": 0.0, "dk": 0.0}
    small = np.zeros(H)

    def each(rows, keys, h, g, p, ds):
        Q, K, V, dO = x["q"][rows, h], x["k"][keys, g], x["v"][keys, g], x["dout"][rows, h]
        sd = U2 * (dO ** 2 * (p @ V) ** 2).sum(1)
        var["dq"] += SCALE ** 2 * ((sd[:, None] * (p @ K) ** 2).sum() + U2 * (ds ** 2 @ K ** 2).sum())
        var["dk"] += SCALE ** 2 * U2 * (ds.T ** 2 @ Q ** 2).sum()
        fix["dq"] += (SCALE * EPS) ** 2 * ((np.abs(ds) @ np.abs(K)) ** 2).sum()
        fix["dk"] += (SCALE * EPS) ** 2 * ((np.abs(ds).T @ np.abs(Q)) ** 2).sum()
        small[h] += EPS * np.abs(ds).sum() + 2.0 ** -24 * Q.shape[1] * p.sum()
        if sim is not None:
            sim(rows, keys, h, g, p)

    r = T.packed_attention(**x, each=each)
    tol = {n: np.sqrt(var[n] + U2 * (r[n] ** 2).sum()) + np.sqrt(fix[n]) for n in var}
    if "dbias" in r:
        tol["dbias"] = 2.0 ** -8 * np.abs(r["dbias"]) + small[:, None]
    return r, tol


def off_by(got, r, tol):
    """Error over bound, the largest for dbias."""
    return {n: float((np.abs(got[n] - r[n]) / tol[n]).max()) if n == "dbias" else float(np.linalg.norm(got[n] - r[n]) / tol[n])
            for n in tol if n in got}


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("D", [64, 128])
def test_bounds_tell_the_correction(lens, causal, D):
    x = inputs(lens, causal, D, True)
    kinds = ("right", "none", "turned", "half")
    sums = {k: {"dk": np.zeros(x["k"].shape), "dbias": np.zeros((H, NB))} for k in kinds}

    def sim(rows, keys, h, g, p):
        Q, V, dO = x["q"][rows, h], x["v"][keys, g], x["dout"][rows, h]
        dp = dO @ V.T
        d = (dO * bf16(bf16(p) @ V)).sum(1, keepdims=True)
        raw = p * (dp - d)
        n, m = p.shape
        bucket = T.pair_terms(n, m, causal, x["bias"], x["buckets"])[2]
        for k in kinds:
            fix = {"right": raw.sum(1), "none": 0 * raw[:, 0], "turned": -raw.sum(1), "half": raw[:, m // 2:].sum(1)}[k]
            ds = p * (dp - d - fix[:, None])
            sums[k]["dk"][keys, g] += SCALE * (bf16(ds).T @ Q)
            sums[k]["dbias"][h] += np.array([ds[bucket == u].sum() for u in range(NB)])

    r, tol = reference(x, sim)
    for k in kinds:
        off = off_by({n: bf16(t) for n, t in sums[k].items()}, r, tol)
        log("   %-6s dk %.2f dbias %.2f" % (k, off["dk"], off["dbias"]))
        if k == "right":
            assert off["dk"] <= 1 and off["dbias"] <= 1
        else:
            assert off["dk"] > 1.5 and off["dbias"] > 2


@pytest.mark.gpu
@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bias", [False, True], ids=["plain", "bias"])
def test_sharp_rows_of_many_keys(bias, lens, causal, D):
    import torch

    import paper_2501_08453_amd as vc
    x = inputs(lens, causal, D, bias)
    lq, lk = LENS[lens]
    desc = vc.make_packed_desc(2, H, H, D, sum(lq), sum(lk), max(lq), max(lk), causal, SCALE, NB if bias else 0, R if bias else 0)
    # the dQ pass's fp32 partials are by far the largest part of the workspace where it splits
    assert (vc.vc_packedattn_bwd_workspace_bytes(desc) >= 2 * sum(lq) * H * (D + 1) * 4) == (lens == "shared")
    d = {n: torch.from_numpy(x[n]).to(torch.bfloat16).cuda() for n in ("q", "k", "v", "dout", "bias") if n in x}
    i = {n: torch.from_numpy(x[n]).cuda() for n in ("cu_q", "cu_k", "buckets") if n in x}
    kw = dict(bias=d.get("bias"), buckets=i.get("buckets"))
    o, lse = vc.packed_fwd(d["q"], d["k"], d["v"], desc, i["cu_q"], i["cu_k"], **kw)
    dq, dk, dv, db = vc.packed_bwd(d["q"], d["k"], d["v"], o, lse, d["dout"], desc, i["cu_q"], i["cu_k"], **kw)
    got = {"dq": bf16_values(dq), "dk": bf16_values(dk)}
    if bias:
        got["dbias"] = bf16_values(db)
    r, tol = reference(x)
    off = off_by(got, r, tol)
    log("   error / bound:", " ".join("%s %.2f" % t for t in off.items()))
    assert all(t <= 1 for t in off.values()), off
