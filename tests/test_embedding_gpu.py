"""Embedding of tokens on the GPU against the fp64 oracle, on every element.

Bounds, u = 2^-24: a lookup is one product, rounded once to the type (scale in fp32). A row of the gradient is a chain of at most
tokens + 16 additions, off by at most that many u of the sum of magnitudes, one product, and the rounding to its type."""
import numpy as np
import pytest

from oracle import ref_blocks as B
from parity_util import log

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {2: 2.0 ** -8, 4: U}


def _vc():
    import paper_2501_08453_amd as vc
    return vc


def _np(t):
    return t.double().cpu().numpy()


def make(tokens, vocab, cols, t="bf16", ids="i64", how="spread", seed=1):
    import torch
    g = torch.Generator().manual_seed(seed + tokens + vocab + cols)
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[t]
    if how == "spread":
        i = torch.randint(0, vocab, (tokens,), generator=g)
    elif how == "often":  # as words come: the chance of an id falls as its inverse
        i = (torch.exp(torch.rand(tokens, generator=g, dtype=torch.float64) * np.log(vocab + 1.0)) - 1).long().clamp(max=vocab - 1)
    elif how == "one":
        i = torch.full((tokens,), vocab // 2)
    else:  # none: outside the table on both sides
        i = torch.where(torch.rand(tokens, generator=g) < 0.5, torch.randint(-9, 0, (tokens,), generator=g), torch.randint(vocab, vocab + 9, (tokens,), generator=g))
    i = i.to(torch.int64 if ids == "i64" else torch.int32)
    return (i.cuda(), torch.randn((vocab, cols), generator=g).to(dt).cuda(), torch.randn((tokens, cols), generator=g).to(dt).cuda())


def check(ids, table, dout, scale=1.0, padding=None, grad=None):
    import torch
    vc = _vc()
    V, pad, f = table.shape[0], -1 if padding is None else padding, float(np.float32(scale))
    I = ids.cpu().numpy()
    out = vc.embedding_fwd(ids, table, scale, padding)
    want = B.embedding(I, _np(table), f, pad)
    assert out.dtype is table.dtype and (np.abs(_np(out) - want) <= (HALF[table.element_size()] + 2 * U) * np.abs(want)).all()
    g = vc.embedding_bwd(dout, ids, V, scale, padding, dtype=grad)
    assert torch.equal(g, vc.embedding_bwd(dout, ids, V, scale, padding, dtype=grad))
    want, mag, n = B.embedding_grad(I, _np(dout), V, f, pad)
    hg = HALF[g.element_size()]
    tol = (n[:, None] + 18) * U * mag
    tol = tol + hg * (np.abs(want) + tol)
    off = np.abs(_np(g) - want)
    assert (off <= tol).all() and (_np(g)[n == 0] == 0).all()
    if mag.any():
        log("   off / bound %.2f" % float((off[tol > 0] / tol[tol > 0]).max()))
    # added to a gradient that is there: the sum as above (before its rounding), one addition, one rounding
    base = torch.randn(g.shape, generator=torch.Generator().manual_seed(3)).to(g.dtype).cuda()
    got = vc.embedding_bwd(dout, ids, V, scale, padding, into=base.clone())
    total = want + _np(base)
    t2 = (n[:, None] + 20) * U * mag + 2 * U * np.abs(total)
    t2 = t2 + hg * (np.abs(total) + t2)
    assert (np.abs(_np(got) - total) <= t2).all() and torch.equal(got[torch.from_numpy(n == 0).cuda()], base[torch.from_numpy(n == 0).cuda()])
    return out, g


@pytest.mark.parametrize("t,grad,ids", [("bf16", "f32", "i64"), ("f32", None, "i32"), ("bf16", None, "i32")])
@pytest.mark.parametrize("tokens,vocab,cols", [(1, 1, 1), (1, 50, 64), (3, 2, 7), (64, 5, 63), (65, 1000, 129), (7, 513, 8192), (500, 17, 1155),
                                               (1024, 511, 40), (1025, 512, 40), (300, 20000, 256)])
def test_shapes(tokens, vocab, cols, t, grad, ids):
    import torch
    check(*make(tokens, vocab, cols, t, ids), scale=0.37, grad=torch.float32 if grad else None)


@pytest.mark.parametrize("how", ["spread", "often", "one", "none"])
@pytest.mark.parametrize("tokens", [5, 33, 1000, 4096, 4097, 8192, 8193, 20000])
def test_ids(tokens, how):
    check(*make(tokens, 300, 24, how=how), scale=3.0, padding=7)


@pytest.mark.parametrize("vocab", [255, 256, 511, 512, 513, 65535, 65536, 262143, 262144, 300000])
def test_tables_at_the_digits_borders(vocab):
    """One, two and three passes of the sort, by one workgroup and by several."""
    for tokens in (600, 9000):
        ids, table, dout = make(tokens, vocab, 8, t="f32")
        ids[:4] = ids.new_tensor([vocab - 1, 0, vocab - 1, vocab // 2])
        check(ids, table, dout, padding=vocab - 1 if tokens == 600 else None)


def test_many_tokens():
    """More than 131,072: blocks of 16,384 of them; an id that fills hundreds of shares."""
    import torch
    vc = _vc()
    ids, table, dout = make(200003, 1000, 16, t="f32", how="often")
    got = vc.embedding_bwd(dout, ids, 1000, 0.5)
    want, mag = (torch.zeros((1000, 16), dtype=torch.float64).index_add_(0, ids.cpu(), d) * 0.5 for d in (dout.double().cpu(), dout.double().abs().cpu()))
    n = torch.bincount(ids.cpu(), minlength=1000)[:, None]
    assert ((got.double().cpu() - want).abs() <= (n + 20) * U * mag + 1e-30).all()
    again = vc.embedding_bwd(dout, ids, 1000, 0.5)
    assert torch.equal(got, again)


def test_order_of_sums_is_that_of_the_tokens():
    """An id of few tokens, all in one share: the fp32 sum in the order of the tokens, bit by bit."""
    import torch
    vc = _vc()
    ids = torch.tensor([4, 1, 4, 2, 4, 1, 4], device="cuda")
    dout = torch.randn((7, 96), device="cuda") * torch.tensor([1, 1e4, 1e-3, 1, 300, 7, 1.0], device="cuda")[:, None]
    g = vc.embedding_bwd(dout, ids, 6)
    want = torch.zeros(96, device="cuda")
    for t in (0, 2, 4, 6):
        want = want + dout[t]
    assert torch.equal(g[4], want) and torch.equal(g[1], dout[1] + dout[5])


def test_strides_types_and_empty():
    import torch
    vc = _vc()
    ids, table, dout = make(70, 40, 101)
    wt, wd = torch.full((40, 150), float("nan"), device="cuda", dtype=table.dtype), torch.full((70, 150), float("nan"), device="cuda", dtype=table.dtype)
    wt[:, 5:106], wd[:, 5:106] = table, dout
    assert torch.equal(vc.embedding_fwd(ids, wt[:, 5:106]), vc.embedding_fwd(ids, table))
    assert torch.equal(vc.embedding_bwd(wd[:, 5:106], ids, 40), vc.embedding_bwd(dout, ids, 40))
    up = vc.embedding_fwd(ids, table, 0.3, dtype=torch.float32)
    assert up.dtype is torch.float32 and torch.allclose(up, table.float()[ids] * 0.3, rtol=2 * U, atol=0)
    assert torch.equal(vc.embedding_fwd(ids, table.float(), 0.3, dtype=torch.bfloat16), up.to(torch.bfloat16))
    assert torch.equal(vc.embedding_fwd(ids.view(7, 10), table), vc.embedding_fwd(ids, table).view(7, 10, 101))
    assert torch.equal(vc.embedding_bwd(dout.view(7, 10, 101), ids.view(7, 10), 40), vc.embedding_bwd(dout, ids, 40))
    none = ids[:0]
    assert vc.embedding_fwd(none, table).shape == (0, 101)
    assert (vc.embedding_bwd(dout[:0], none, 40) == 0).all()
    base = torch.ones((40, 101), device="cuda")
    assert vc.embedding_bwd(dout[:0], none, 40, into=base) is base and (base == 1).all()


def test_offsets_past_32_bits():
    """A table and a gradient of more than 2^31 elements: ids at both ends."""
    import torch
    vc = _vc()
    V, cols = 300000, 7200
    table = torch.zeros((V, cols), dtype=torch.bfloat16, device="cuda")
    table[-1], table[V // 2], table[0] = 3.0, 2.0, 1.0
    ids = torch.tensor([V - 1, 0, V // 2, V - 1], device="cuda")
    out = vc.embedding_fwd(ids, table)
    assert [float(r.float().mean()) for r in out] == [3.0, 1.0, 2.0, 3.0]
    del table
    g = vc.embedding_bwd(out, ids, V)
    assert float(g[-1].float().min()) == 6.0 and float(g[V // 2].float().max()) == 2.0 and float(g[0].float().min()) == 1.0
    assert int(g.any(1).sum()) == 3


def test_differentiable_graph_and_stream():
    import torch
    vc = _vc()
    ids, table, dout = make(3000, 257, 200, how="often")
    leaf = table.clone().requires_grad_(True)
    out = vc.embedding(ids, leaf, 2.0, 3)
    out.backward(dout)
    want = vc.embedding_bwd(dout, ids, 257, 2.0, 3, dtype=table.dtype)
    assert torch.equal(out, vc.embedding_fwd(ids, table, 2.0, 3)) and torch.equal(leaf.grad, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = vc.embedding_bwd(dout, ids, 257, 2.0, 3, dtype=table.dtype)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    for n in (3000, 9001):
        ids, table, dout = make(n, 257, 200, how="often")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            o = vc.embedding_fwd(ids, table, 2.0, 3)
            d = vc.embedding_bwd(dout, ids, 257, 2.0, 3)
        for _ in range(3):
            ids.copy_(torch.randint(0, 257, ids.shape, device="cuda"))
            dout.copy_(torch.randn(dout.shape, device="cuda"))
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, vc.embedding_fwd(ids, table, 2.0, 3)) and torch.equal(d, vc.embedding_bwd(dout, ids, 257, 2.0, 3))


@pytest.mark.parametrize("how", ["spread", "often", "one", "none"])
@pytest.mark.parametrize("tokens", [1, 2, 8, 9, 63, 64, 65])
def test_few_tokens(tokens, how):
    """Up to 64 tokens there is no sort: rows of one vector, of several waves, with odd ends; more ids than a workgroup clears."""
    for vocab, cols, t in ((3, 5, "f32"), (130, 2056, "bf16"), (700, 1027, "bf16"), (5000, 64, "f32")):
        check(*make(tokens, vocab, cols, t, ids="i32" if tokens % 2 else "i64", how=how), scale=0.75, padding=2)
