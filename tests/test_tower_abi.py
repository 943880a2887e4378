"""Refusals of the packed attention's and the layer norm's entry points (CPU: nothing here reaches a launch)."""
import ctypes

import pytest

import paper_2501_08453_amd as vc

P = 1 << 20  # never dereferenced: validation fails first
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return vc._lib()


def desc(**kw):
    d = vc.make_packed_desc(3, 4, 2, 64, 100, 120, 60, 70)
    for n, x in kw.items():
        setattr(d, n, x)
    return d


def fwd(lib, d, q=P, k=P, v=P, cu_q=P, cu_k=P, len_q=None, len_k=None, bias=None, buckets=None, o=P, lse=P, ws=P, n=BIG):
    return lib.vc_packedattn_fwd(d and ctypes.byref(d), q, k, v, cu_q, cu_k, len_q, len_k, bias, buckets, o, lse, ws, n, None)


def bwd(lib, d, q=P, k=P, v=P, o=P, lse=P, dout=P, cu_q=P, cu_k=P, len_q=None, len_k=None, bias=None, buckets=None, dq=P, dk=P, dv=P,
        dbias=None, ws=P, n=BIG):
    return lib.vc_packedattn_bwd(d and ctypes.byref(d), q, k, v, o, lse, dout, cu_q, cu_k, len_q, len_k, bias, buckets, dq, dk, dv,
                                 dbias, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(head_dim=96), -3), (dict(head_dim=0), -3), (dict(sequences=0), -2), (dict(heads=0), -2), (dict(kv_heads=0), -2),
    (dict(kv_heads=3), -2), (dict(heads=8192, kv_heads=2), -2), (dict(total_q=0), -2), (dict(total_k=0), -2),
    (dict(total_q=1 << 31), -2), (dict(max_q=0), -2), (dict(max_q=101), -2), (dict(max_k=121), -2), (dict(causal=2), -2),
    (dict(clear_outside=-1), -2), (dict(q_stride=255), -2), (dict(q_stride=4 * 64 + 4), -2), (dict(k_stride=120), -2),
    (dict(v_stride=-128), -2), (dict(q_stride=1 << 24), -2), (dict(num_buckets=-1), -2), (dict(num_buckets=1025), -2),
    (dict(num_buckets=4, max_distance=513), -2), (dict(max_distance=-1), -2), (dict(softmax_scale=float("nan")), -2),
    (dict(softmax_scale=float("inf")), -2), (dict(softmax_scale=2.0 ** -61), -2),
    (dict(softmax_scale=2.0 ** -25, num_buckets=4), -2), (dict(softmax_scale=2.0 ** 25, num_buckets=4), -2),
    (dict(sequences=1 << 20, heads=4096, total_q=1 << 29, total_k=1 << 29, max_q=1 << 20, max_k=1), -2),
])
def test_bad_descriptor(lib, kw, code):
    d = desc(**kw)
    assert fwd(lib, d, bias=P, buckets=P) == code
    assert bwd(lib, d, bias=P, buckets=P) == code
    assert vc.vc_packedattn_fwd_workspace_bytes(d) == 0 and vc.vc_packedattn_bwd_workspace_bytes(d) == 0


def test_pointers_and_workspaces(lib):
    d, b = desc(), desc(num_buckets=4, max_distance=3)
    assert fwd(lib, None) == -1 and bwd(lib, None) == -1
    for n in ("q", "k", "v", "cu_q", "cu_k", "o", "lse"):
        assert fwd(lib, d, **{n: None}) == -1, n
        assert fwd(lib, d, **{n: P + 2}) == -4, n
    for n in ("q", "k", "v", "o", "lse", "dout", "cu_q", "cu_k", "dq", "dk", "dv"):
        assert bwd(lib, d, **{n: None}) == -1, n
        assert bwd(lib, d, **{n: P + 2}) == -4, n
    for n in ("len_q", "len_k"):
        assert fwd(lib, d, **{n: P + 2}) == -4 and bwd(lib, d, **{n: P + 2}) == -4
    assert fwd(lib, b, bias=P) == -1 and fwd(lib, b, buckets=P) == -1 and bwd(lib, b, bias=P) == -1
    assert fwd(lib, b, bias=P + 1, buckets=P) == -4 and fwd(lib, b, bias=P, buckets=P + 2) == -4
    assert bwd(lib, d, dbias=P) == -2  # a gradient of a bias that is not there
    for f, need in ((fwd, vc.vc_packedattn_fwd_workspace_bytes(d)), (bwd, vc.vc_packedattn_bwd_workspace_bytes(d))):
        assert need > 0
        assert f(lib, d, ws=None) == -5 and f(lib, d, n=need - 1) == -5 and f(lib, d, ws=P + 16) == -4
    import torch
    if not torch.cuda.is_available():
        assert fwd(lib, d) == -6 and bwd(lib, b, bias=P, buckets=P, dbias=P) == -6


def test_norm_refusals(lib):
    def norm(**kw):
        d = vc.vc_layernorm_desc(10, 100, 0, 1, 1e-5, 0, 0)
        for n, x in kw.items():
            setattr(d, n, x)
        return d

    def f(d, x=P, w=P, b=P, y=P, m=P, r=P):
        return lib.vc_layernorm_fwd(d and ctypes.byref(d), x, w, b, y, m, r, None)

    def g(d, dy=P, x=P, w=P, m=P, r=P, dx=P, dw=P, db=P, ws=P, n=BIG):
        return lib.vc_layernorm_bwd(d and ctypes.byref(d), dy, x, w, m, r, dx, dw, db, ws, n, None)

    for kw, code in ((dict(rows=0), -2), (dict(rows=1 << 31), -2), (dict(cols=0), -2), (dict(cols=65537), -2), (dict(x_type=2), -8),
                     (dict(param_type=-1), -8), (dict(x_stride=99), -2), (dict(dout_stride=-1), -2), (dict(eps=-1.0), -2),
                     (dict(eps=float("nan")), -2)):
        assert f(norm(**kw)) == code and g(norm(**kw)) == code, kw
        assert vc.vc_layernorm_bwd_workspace_bytes(norm(**kw)) == 0
    assert f(None) == -1 and g(None) == -1
    for n in "xymr":
        assert f(norm(), **{n: None}) == -1 and f(norm(), **{n: P + 1}) == -4
    for n in ("dy", "x", "m", "r", "dx"):
        assert g(norm(), **{n: None}) == -1 and g(norm(), **{n: P + 1}) == -4
    assert f(norm(), w=P + 2) == -4 and f(norm(x_type=1), x=P + 2) == -4 and g(norm(), dw=P + 2) == -4
    need = vc.vc_layernorm_bwd_workspace_bytes(norm())
    assert need > 0 and g(norm(), ws=None) == -5 and g(norm(), n=need - 1) == -5 and g(norm(), ws=P + 16) == -4
    import torch
    if not torch.cuda.is_available():
        assert f(norm(), w=None, b=None) == -6 and g(norm(), dw=None, db=None, ws=None, n=0) == -6


def test_helpers_check_before_calling():
    torch = pytest.importorskip("torch")
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    q, k, v = bf(100, 4, 64), bf(120, 2, 64), bf(120, 2, 64)
    cu = torch.zeros(4, dtype=torch.int32)
    d = vc.make_packed_desc(3, 4, 2, 64, 100, 120, 60, 70)
    b = vc.make_packed_desc(3, 4, 2, 64, 100, 120, 60, 70, num_buckets=5, max_distance=2)
    bias, buckets = bf(4, 5), torch.zeros(5, dtype=torch.int32)
    for match, call in (
            ("must be on a GPU", lambda: vc.packed_fwd(q, k, v, d, cu, cu)),
            ("q has shape", lambda: vc.packed_fwd(q[:-1], k, v, d, cu, cu)),
            ("k must be torch.bfloat16", lambda: vc.packed_fwd(q, k.float(), v, d, cu, cu)),
            ("v has shape", lambda: vc.packed_fwd(q, k, bf(120, 4, 64), d, cu, cu)),
            ("cu_q must be torch.int32", lambda: vc.packed_fwd(q, k, v, d, cu.long(), cu)),
            ("cu_k has shape", lambda: vc.packed_fwd(q, k, v, d, cu, cu[:-1])),
            ("len_k has shape", lambda: vc.packed_fwd(q, k, v, d, cu, cu, len_k=cu)),
            ("a bias and its buckets", lambda: vc.packed_fwd(q, k, v, d, cu, cu, bias=bias, buckets=buckets)),
            ("a bias and its buckets", lambda: vc.packed_fwd(q, k, v, b, cu, cu)),
            ("a bias and its buckets", lambda: vc.packed_fwd(q, k, v, b, cu, cu, bias=bias)),
            ("bias must be torch.bfloat16", lambda: vc.packed_fwd(q, k, v, b, cu, cu, bias=bias.float(), buckets=buckets)),
            ("buckets has shape", lambda: vc.packed_fwd(q, k, v, b, cu, cu, bias=bias, buckets=buckets[:-1])),
            ("out has shape", lambda: vc.packed_fwd(q, k, v, d, cu, cu, out=k)),
            ("lse has shape", lambda: vc.packed_fwd(q, k, v, d, cu, cu, lse=torch.zeros(100, 4))),
            ("given together", lambda: vc.packed_bwd(q, k, v, q, torch.zeros(4, 100), q, d, cu, cu, dq=q)),
            ("dout must be", lambda: vc.packed_bwd(q, k, v, q, torch.zeros(4, 100), q.float(), d, cu, cu)),
            ("invalid descriptor", lambda: vc.packed_fwd_workspace(vc.make_packed_desc(3, 4, 3, 64, 9, 9, 9, 9), "cpu")),
            ("relative_buckets", lambda: vc.relative_buckets(2, 8)),
            ("relative_buckets", lambda: vc.relative_buckets(32, 8)),
            ("relative_buckets", lambda: vc.relative_buckets(32, 513)),
            ("x must be torch", lambda: vc.layer_norm_fwd(q.half())),
            ("x must be on a GPU", lambda: vc.layer_norm_fwd(q)),
            ("weight has shape", lambda: vc.layer_norm_fwd(q, bf(63))),
            ("weight and bias", lambda: vc.layer_norm_fwd(q, bf(64), torch.zeros(64))),
            ("rstd has shape", lambda: vc.layer_norm_bwd(q, q, None, None, torch.zeros(100, 4), torch.zeros(100))),
    ):
        with pytest.raises(ValueError, match=match):
            call()


def test_relative_buckets():
    """The borders hold in whole numbers: with 8 buckets a direction, 4 wide ones up to 64 = 4 * 16, distance 8 = 4 * 16^(1/4)
    * ... is the first of its bucket where 8^4 >= 64 * 4^3."""
    b = vc.relative_buckets(16, 64, device="cpu").tolist()
    assert len(b) == 129 and b[64] == 0 and b[63] == 1 and b[65] == 9
    behind = b[64::-1]  # n = 0 .. 64
    assert behind[:4] == [0, 1, 2, 3] and behind[7] == 4 and behind[8] == 5 and behind[15] == 5 and behind[16] == 6
    assert behind[31] == 6 and behind[32] == 7 and behind[64] == 7
    assert b[65:] == [8 + x for x in behind[1:]]
    one = vc.relative_buckets(8, 64, bidirectional=False, device="cpu").tolist()
    assert one[64::-1] == behind and one[65:] == [0] * 64


def test_launches_of_2_32_threads_and_more_are_refused(lib):
    """Workgroups have 256 threads, 32 of them clear the rows outside the slots: a grid of 2^24 - 1 - 32 others is the largest."""
    most = (2 ** 32 - 1) // 256 - 32

    def one(S, H, Hkv, q=1, k=1, **kw):  # S slots of q queries and k keys
        d = vc.make_packed_desc(S, H, Hkv, 64, S * q, S * k, q, k)
        for n, x in kw.items():
            setattr(d, n, x)
        return d

    def sizes(d):
        return vc.vc_packedattn_fwd_workspace_bytes(d), vc.vc_packedattn_bwd_workspace_bytes(d)

    def refused(d, f):
        w = dict(bias=P, buckets=P) if d.num_buckets else {}
        return f(lib, d, **w) == -2

    # single tokens of 17 heads each: sequences x heads workgroups, in both directions
    assert all(sizes(one(most // 17, 17, 17))) and sizes(one(most // 17 + 1, 17, 17)) == (0, 0)
    d = one(most // 17 + 1, 17, 17)
    assert refused(d, fwd) and refused(d, bwd)
    # the heads of a group share a workgroup forward, not in dQ's pass
    d = one(1 << 20, 32, 8)
    assert sizes(d)[0] > 0 and sizes(d)[1] == 0 and refused(d, bwd)
    # two blocks of 128 rows a slot, of the queries or of the keys alone
    d = one(1 << 17, 64, 64, q=200)
    assert sizes(d) == (0, 0) and refused(d, fwd) and refused(d, bwd)
    d = one(1 << 17, 64, 64, k=200)
    assert sizes(d)[0] > 0 and sizes(d)[1] == 0 and refused(d, bwd)
    # with a bias a key block has a workgroup per query head at least
    d = one(1 << 19, 40, 1, num_buckets=4, max_distance=8)
    assert sizes(d) == (0, 0) and refused(d, bwd)
    d = one(1 << 18, 40, 1, num_buckets=4, max_distance=8)
    assert all(sizes(d))
    import torch
    if not torch.cuda.is_available():
        assert fwd(lib, one(1 << 20, 32, 8)) == -6 and fwd(lib, one(1 << 17, 64, 64, k=200)) == -6

    n = vc.vc_layernorm_desc((2 ** 32 - 1) // 256, 8193, 0, 1, 1e-5, 0, 0)  # a workgroup a row
    assert vc.vc_layernorm_bwd_workspace_bytes(n) > 0
    n.rows += 1
    assert vc.vc_layernorm_bwd_workspace_bytes(n) == 0
    assert lib.vc_layernorm_fwd(ctypes.byref(n), P, P, P, P, P, P, None) == -2
    n.cols = 8192
    assert vc.vc_layernorm_bwd_workspace_bytes(n) > 0


def test_chunks_keep_to_the_launch_limit():
    """Whatever the sizes, chunks and grids stay below 2^32 threads: the forward's chunks, as its workspace gives them,
    times its other workgroups, and the waves that join them."""
    import random
    rng = random.Random(7)
    split = 0
    for _ in range(4000):
        S, Hkv, G = 1 << rng.randint(0, 20), 1 << rng.randint(0, 6), 1 << rng.randint(0, 3)
        q = rng.choice([1, 1, 2, 4])
        total_k = min(1 << 30, S * (1 << rng.randint(0, 9)) + (1 << rng.randint(0, 22)))
        d = vc.make_packed_desc(S, Hkv * G, Hkv, 64, S * q, total_k, q, 1 << rng.randint(0, 22), causal=True)
        n = vc.vc_packedattn_fwd_workspace_bytes(d)
        if not n:
            continue
        chunks = 1 if n == 256 else n // (d.total_q * d.heads * (64 + 2) * 4)
        heads = Hkv if q * G <= 32 else Hkv * G  # rows of a group's heads together
        assert S * heads * chunks + 32 < 2 ** 24
        if chunks > 1:
            split += 1
            assert S * q * d.heads * 64 < 2 ** 32
    assert split > 100


@pytest.mark.parametrize("both", [False, True], ids=["one-sided", "bidirectional"])
def test_relative_buckets_up_to_the_largest_table(both):
    """Tables that a call takes, and none beyond."""
    b = vc.relative_buckets(1024 if both else 1022, 512, both, device="cpu")  # one-sided: fewer than 512 exact ones
    assert len(b) == 1025 and int(b.min()) == 0 and int(b.max()) < 1024
    d = vc.make_packed_desc(1, 1, 1, 64, 1, 1, 1, 1, num_buckets=1024, max_distance=512)
    assert vc.vc_packedattn_fwd_workspace_bytes(d) > 0
    d.num_buckets = 1026
    assert vc.vc_packedattn_fwd_workspace_bytes(d) == 0
    with pytest.raises(ValueError, match="relative_buckets"):
        vc.relative_buckets(1026, 512, both, device="cpu")


def test_backward_keeps_the_forwards_descriptor(monkeypatch):
    """A descriptor changed after the forward (reused for the next batch) does not reach the backward."""
    torch = pytest.importorskip("torch")
    from paper_2501_08453_amd import tower
    seen = []

    def forward(q, k, v, desc, *rest):
        return torch.zeros_like(q), torch.zeros(q.shape[1], q.shape[0])

    def backward(q, k, v, o, lse, do, desc, *rest, want_dbias):
        seen.append((desc.causal, desc.softmax_scale, desc.max_k))
        return torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v), None

    monkeypatch.setattr(tower, "packed_fwd", forward)
    monkeypatch.setattr(tower, "packed_bwd", backward)
    q = torch.zeros((8, 2, 64), dtype=torch.bfloat16, requires_grad=True)
    cu = torch.tensor([0, 8], dtype=torch.int32)
    d = vc.make_packed_desc(1, 2, 2, 64, 8, 8, 8, 8, causal=True, scale=0.5)
    o = vc.packed_attention(q, q, q, d, cu, cu)
    d.causal, d.softmax_scale, d.max_k = 0, 0.25, 4
    o.sum().backward()
    assert seen == [(1, 0.5, 8)]


def test_workspace_on_another_device_is_refused(monkeypatch):
    """The kernels write to it: nothing is launched. (Device and layout of the other tensors are left out here.)"""
    torch = pytest.importorskip("torch")
    from paper_2501_08453_amd import tower
    launched = []
    monkeypatch.setattr(tower, "_check_all", lambda every: None)
    monkeypatch.setattr(tower, "_launch", lambda device, f, *args: launched.append(args[-1]))
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)  # noqa: E731
    q, lse, cu = bf(8, 2, 64), torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32)
    x, w, mean = bf(4, 16), torch.ones(16), torch.zeros(4)
    d = vc.make_packed_desc(1, 2, 2, 64, 8, 8, 8, 8)
    calls = (lambda ws: vc.packed_fwd(q, q, q, d, cu, cu, ws=ws), lambda ws: vc.packed_bwd(q, q, q, q, lse, q, d, cu, cu, ws=ws),
             lambda ws: vc.layer_norm_bwd(x, x, w, w, mean, mean, ws=ws))
    for call in calls:
        with pytest.raises(ValueError, match="ws is on meta"):
            call(torch.empty(1 << 20, dtype=torch.uint8, device="meta"))
        with pytest.raises(ValueError, match="ws must be contiguous"):
            call(torch.empty(1, dtype=torch.uint8).expand(1 << 20))
        assert not launched
        call(torch.empty(1 << 10, dtype=torch.float32))
        assert launched.pop() == 1 << 12


def test_clearing_one_output_is_the_forwards(lib):
    """clear_outside 2 and 3 name the forward's outputs."""
    for c, f, b in ((0, True, True), (1, True, True), (2, True, False), (3, True, False), (4, False, False)):
        d = desc(clear_outside=c)
        assert (vc.vc_packedattn_fwd_workspace_bytes(d) > 0) == f and (vc.vc_packedattn_bwd_workspace_bytes(d) > 0) == b
        assert b or bwd(lib, d) == -2
        assert f or fwd(lib, d) == -2
