"""Refusals of the entry points around a block's attention (CPU: nothing here reaches a launch)."""
import ctypes

import pytest

import paper_2501_08453_amd as vc

P = 1 << 20  # never dereferenced: validation fails first
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return vc._lib()


def no_gpu():
    import torch
    return not torch.cuda.is_available()


def _set(d, kw):
    for n, x in kw.items():
        setattr(d, n, x)
    return d


def res(**kw):
    d = vc.make_residual_desc(40, 100, 4, post_norm="rms")
    d.clear_outside = 0
    return _set(d, kw)


FWD = ("x", "a", "gate", "scale", "shift", "post_weight", "cu", "lens", "h", "y", "mean", "rstd", "post_mean", "post_rstd", "h8",
       "h8_scales", "a8", "a8_scales")
BWD = ("dh", "dy", "h", "a", "h8_scales", "a8_scales", "gate", "scale", "post_weight", "cu", "lens", "mean", "rstd", "post_mean",
       "post_rstd", "dx", "da", "dgate", "dscale", "dshift", "dpost_weight")


def fwd(lib, d, **kw):
    p = {n: None if n in ("cu", "lens") else P for n in FWD} | kw
    return lib.vc_residualnorm_fwd(d and ctypes.byref(d), *[p[n] for n in FWD], None)


def bwd(lib, d, ws=P, n=BIG, **kw):
    p = {n: None if n in ("cu", "lens") else P for n in BWD} | kw
    return lib.vc_residualnorm_bwd(d and ctypes.byref(d), *[p[n] for n in BWD], ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(rows=0), -2), (dict(rows=(1 << 30) + 1), -2), (dict(cols=0), -2), (dict(cols=8193), -2), (dict(samples=0), -2),
    (dict(samples=3), -2), (dict(rows=1 << 30, samples=1 << 22), -2), (dict(x_type=2), -8), (dict(y_type=-1), -8),
    (dict(param_type=2), -8), (dict(y_type=1), -8), (dict(norm=3), -8), (dict(post_norm=-1), -8), (dict(packed=2), -2),
    (dict(plus_one=-1), -2), (dict(checkpoint=2), -2), (dict(clear_outside=3), -2), (dict(residual_scale=float("inf")), -2),
    (dict(residual_scale=float("nan")), -2), (dict(eps=-1.0), -2), (dict(eps=float("inf")), -2), (dict(x_stride=99), -2),
    (dict(a_stride=-1), -2), (dict(dh_stride=99), -2), (dict(dy_stride=(1 << 30) + 1), -2), (dict(gate_stride=99), -2),
    (dict(scale_stride=-2), -2), (dict(shift_stride=1), -2),
])
def test_bad_residual_descriptor(lib, kw, code):
    assert fwd(lib, res(**kw)) == code and bwd(lib, res(**kw)) == code
    assert vc.vc_residualnorm_bwd_workspace_bytes(res(**kw)) == 0


def test_residual_pointers_and_combinations(lib):
    d, k = res(), res(checkpoint=1)
    assert fwd(lib, None) == -1 and bwd(lib, None) == -1
    for n in ("x", "h", "y", "mean", "rstd", "post_mean", "post_rstd"):
        assert fwd(lib, d, **{n: None}) == -1, n
    for n in FWD[:6] + ("h", "y", "mean", "rstd", "post_mean", "post_rstd"):
        assert fwd(lib, d, **{n: P + 1}) == -4, n
    for n in ("h8", "h8_scales", "a8", "a8_scales"):
        assert fwd(lib, k, **{n: None}) == -1, n
    assert fwd(lib, k, h8_scales=P + 2) == -4 and fwd(lib, d, lens=P + 2) == -4 and bwd(lib, d, lens=P + 2) == -4
    assert fwd(lib, res(x_type=1), x=P + 2) == -4 and fwd(lib, res(x_type=1, y_type=1), a=P + 2) == -4
    # offsets go with `packed`, and only with that
    assert fwd(lib, d, cu=P) == -2 and fwd(lib, res(packed=1)) == -1 and bwd(lib, res(packed=1)) == -1
    assert fwd(lib, res(packed=1), cu=P + 2) == -4
    # without a block output there is nothing to gate, norm or scale
    alone = res(post_norm=0)
    none = dict(a=None, gate=None, post_weight=None)
    assert fwd(lib, d, **none) == -2 and fwd(lib, alone, a=None, post_weight=None) == -2 and fwd(lib, alone, a=None, gate=None) == -2
    assert fwd(lib, res(post_norm=0, residual_scale=0.5), **none) == -2 and fwd(lib, res(post_norm=0, norm=0), **none, scale=None, shift=None) == -2
    assert fwd(lib, res(post_norm=0)) == -2  # a weight of a norm that is not there
    assert fwd(lib, res(norm=0)) == -2       # a scale likewise
    for n in ("dh", "dy"):  # one of them may be left out
        assert bwd(lib, d, **{n: None}) == (-6 if no_gpu() else 0) or not no_gpu()
    assert bwd(lib, d, dh=None, dy=None) == -1
    for n in ("h", "mean", "rstd", "post_mean", "post_rstd"):
        assert bwd(lib, d, **{n: None}) == -1, n
    for n in set(BWD) - {"cu", "lens"}:
        assert bwd(lib, d, **{n: P + 1}) == -4, n
    assert bwd(lib, k, h=P + 1, a=P + 3) == -6 or not no_gpu()  # bytes
    assert bwd(lib, k, h8_scales=None) == -1 and bwd(lib, k, a8_scales=None) == -1
    assert bwd(lib, res(norm=0), dy=None) == -2 and bwd(lib, res(norm=0), dh=None, dy=None) == -1
    gone = dict(a=None, gate=None, post_weight=None, da=None, dgate=None, dpost_weight=None)
    for n in ("gate", "post_weight", "da", "dgate", "dpost_weight"):
        assert bwd(lib, alone, **(gone | {n: P})) == -2, n
    nothing = {n: None for n in ("dx", "da", "dgate", "dscale", "dshift", "dpost_weight")}
    assert bwd(lib, d, **nothing) == -1
    need = vc.vc_residualnorm_bwd_workspace_bytes(d)
    assert need > 0 and bwd(lib, d, ws=None) == -5 and bwd(lib, d, n=need - 1) == -5 and bwd(lib, d, ws=P + 16) == -4
    if no_gpu():
        assert fwd(lib, d) == -6 and bwd(lib, d) == -6
        assert bwd(lib, d, ws=None, n=0, **{n: None for n in ("dgate", "dscale", "dshift", "dpost_weight")}) == -6
        assert fwd(lib, alone, **none) == -6 and bwd(lib, alone, **gone) == -6


def test_checkpoint_refusals(lib):
    d = lambda **kw: _set(vc.vc_checkpoint_desc(10, 100, 0, 0), kw)  # noqa: E731
    pack = lambda d, x=P, q=P, s=P: lib.vc_checkpoint_pack(d and ctypes.byref(d), x, q, s, None)  # noqa: E731
    unpack = lambda d, q=P, s=P, y=P: lib.vc_checkpoint_unpack(d and ctypes.byref(d), q, s, y, None)  # noqa: E731
    for kw, code in ((dict(rows=0), -2), (dict(rows=(1 << 32) + 1), -2), (dict(cols=0), -2), (dict(cols=(1 << 24) + 1), -2),
                     (dict(type=2), -8), (dict(stride=99), -2), (dict(stride=(1 << 30) + 1), -2)):
        assert pack(d(**kw)) == code and unpack(d(**kw)) == code, kw
    assert pack(None) == -1 and unpack(None) == -1
    for n in "xqs":
        assert pack(d(), **{n: None}) == -1
    for n in "qsy":
        assert unpack(d(), **{n: None}) == -1
    assert pack(d(), x=P + 1) == -4 and pack(d(type=1), x=P + 2) == -4 and pack(d(), s=P + 2) == -4
    assert unpack(d(), y=P + 1) == -4 and unpack(d(), s=P + 2) == -4 and unpack(d(stride=120)) == -2
    if no_gpu():
        assert pack(d(stride=120), q=P + 1) == -6 and unpack(d(), q=P + 1) == -6


def test_embedding_refusals(lib):
    d = lambda **kw: _set(vc.vc_embedding_desc(10, 50, -1, 0, 64, 1, 0, 0, 1.0, 0), kw)  # noqa: E731
    f = lambda d, ids=P, table=P, out=P: lib.vc_embedding_fwd(d and ctypes.byref(d), ids, table, out, None)  # noqa: E731
    g = lambda d, ids=P, dout=P, dtable=P, ws=P, n=BIG: lib.vc_embedding_bwd(d and ctypes.byref(d), ids, dout, dtable, ws, n, None)  # noqa: E731
    for kw, code in ((dict(tokens=0), -2), (dict(tokens=(1 << 30) + 1), -2), (dict(vocab=0), -2), (dict(vocab=(1 << 27) + 1), -2),
                     (dict(cols=0), -2), (dict(cols=8193), -2), (dict(ids64=2), -2), (dict(table_type=2), -8), (dict(out_type=-1), -8),
                     (dict(scale=float("nan")), -2), (dict(accumulate=2), -2), (dict(row_stride=63), -2)):
        assert f(d(**kw)) == code and g(d(**kw)) == code, kw
        assert vc.vc_embedding_bwd_workspace_bytes(d(**kw)) == 0
    many = d(tokens=(1 << 24) + 1)
    assert g(many) == -2 and vc.vc_embedding_bwd_workspace_bytes(many) == 0
    assert f(None) == -1 and g(None) == -1
    for n in ("ids", "table", "out"):
        assert f(d(), **{n: None}) == -1 and f(d(), **{n: P + 1}) == -4
    for n in ("ids", "dout", "dtable"):
        assert g(d(), **{n: None}) == -1 and g(d(), **{n: P + 1}) == -4
    assert f(d(), ids=P + 4) == -4 and f(d(table_type=1), table=P + 2) == -4
    need = vc.vc_embedding_bwd_workspace_bytes(d())
    assert need > 0 and g(d(), ws=None) == -5 and g(d(), n=need - 1) == -5 and g(d(), ws=P + 16) == -4
    if no_gpu():
        assert f(many) == -6 and f(d(ids64=0), ids=P + 4) == -6 and g(d()) == -6


def test_helpers_check_before_calling():
    torch = pytest.importorskip("torch")
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    x, a, v = bf(40, 100), bf(40, 100), bf(4, 100)
    cu = torch.zeros(5, dtype=torch.int32)
    d = vc.make_residual_desc(40, 100, 4)
    call = lambda *p, **kw: lambda: vc.residual_norm_fwd(*p, d, **kw)  # noqa: E731
    saved = vc.ResidualSaved(d, x, a, None, None, None, None, None, None, torch.zeros(4, 40), torch.bfloat16)
    alone = vc.make_residual_desc(40, 100, 4, norm=None)
    ids, table = torch.zeros(9, dtype=torch.int64), bf(30, 16)
    for match, f in (
            ("must be on a GPU", call(x, a)),
            ("x must be torch", call(x.half(), a)),
            ("a must be torch", call(x, a.int())),
            ("a has shape", call(x, a[:-1])),
            ("gate has shape", call(x, a, gate=v[:-1])),
            ("gate has shape", call(x, a, gate=bf(99))),
            ("scale must be torch.bfloat16", call(x, a, gate=v, scale=v.float())),
            ("shift must be", call(x, a, shift=bf(100, 4).t())),
            ("post_weight has shape", call(x, a, post_weight=v)),
            ("cu must be torch.int32", call(x, a, cu=cu.long())),
            ("cu has shape", call(x, a, cu=cu[:-1])),
            ("lens has shape", call(x, a, lens=cu)),
            ("y has a's type", call(x, a, y_dtype=torch.float32)),
            ("y_dtype must be", call(x, None, y_dtype=torch.half)),
            ("x must be contiguous", call(bf(100, 40).t(), a)),
            ("a norm is", lambda: vc.make_residual_desc(40, 100, norm="batch")),
            ("both None", lambda: vc.residual_norm_bwd(None, None, saved)),
            ("dy must be", lambda: vc.residual_norm_bwd(x, a.float(), saved)),
            ("dh has shape", lambda: vc.residual_norm_bwd(x[:-1], a, saved)),
            ("no y without a norm", lambda: vc.residual_norm_bwd(None, a, saved._replace(desc=alone))),
            ("x must be torch", lambda: vc.checkpoint_pack(x.half())),
            ("x has shape", lambda: vc.checkpoint_pack(x[0, 0])),
            ("must be on a GPU", lambda: vc.checkpoint_pack(x)),
            ("out is of", lambda: vc.checkpoint_pack(x, out=vc.Packed8(x, x, torch.float32))),
            ("out.q must be", lambda: vc.checkpoint_pack(x, out=vc.Packed8(x, x, x.dtype))),
            ("out must be", lambda: vc.checkpoint_unpack(vc.Packed8(x, x, x.dtype), dtype=torch.half)),
            ("ids must be torch", lambda: vc.embedding_fwd(ids.short(), table)),
            ("table has shape", lambda: vc.embedding_fwd(ids, table[0])),
            ("table must be torch", lambda: vc.embedding_fwd(ids, table.half())),
            ("out has shape", lambda: vc.embedding_fwd(ids, table, out=table)),
            ("must be on a GPU", lambda: vc.embedding_fwd(ids, table)),
            ("dout has shape", lambda: vc.embedding_bwd(table, ids, 30)),
            ("into has shape", lambda: vc.embedding_bwd(bf(9, 16), ids, 30, into=bf(29, 16))),
            ("into must be", lambda: vc.embedding_bwd(bf(9, 16), ids, 30, into=table, dtype=torch.float32)),
    ):
        with pytest.raises(ValueError, match=match):
            f()
