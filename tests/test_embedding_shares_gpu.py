"""The embedding's gradient where the plan of its sort and sums takes other forms than small calls have: shares of more tokens than a
wave has lanes, and tables whose ids take four passes."""
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("tokens", [70001, 140000])
@pytest.mark.parametrize("cols,t,grad", [(264, "bf16", "f32"), (264, "f32", "f32"), (1027, "bf16", "bf16"), (1027, "f32", "f32")])
def test_shares_of_more_than_64_tokens(tokens, cols, t, grad):
    """A wave takes such a share 64 tokens a step: ids go on from step to step, and end, begin, or turn into none in a later one. A row of
    n tokens is off by at most (n + 18) u of its magnitudes, u = 2^-24, and by half a step of its type."""
    import torch
    import paper_2501_08453_amd as vc
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}
    g = torch.Generator().manual_seed(tokens + cols)
    for V, none in ((3000, 0.0), (40, 0.4)):
        # the chance of an id falls as its inverse: the first fill hundreds of shares
        ids = (torch.exp(torch.rand(tokens, generator=g, dtype=torch.float64) * torch.log(torch.tensor(V + 1.0))) - 1).long().clamp(max=V - 1)
        ids[torch.rand(tokens, generator=g) < none] = V + 3
        ids[::101] = 2  # the padding
        ids = ids.cuda()
        dout = torch.randn((tokens, cols), generator=g).to(dt[t]).cuda()
        real = (ids < V) & (ids != 2)
        got = vc.embedding_bwd(dout, ids, V, 0.5, 2, dtype=dt[grad])
        n = torch.bincount(ids[real], minlength=V)[:, None]
        where, half = ids[real], 2.0 ** -8 if grad == "bf16" else U
        for c in range(0, cols, 400):
            d = dout[real][:, c:c + 400].double().cpu()
            want, mag = (torch.zeros((V, d.shape[1]), dtype=torch.float64).index_add_(0, where.cpu(), 0.5 * p).cuda() for p in (d, d.abs()))
            tol = (n + 18) * U * mag
            assert ((got[:, c:c + 400].double() - want).abs() <= tol + half * (want.abs() + tol)).all()
        assert not got[n[:, 0] == 0].any() and torch.equal(got, vc.embedding_bwd(dout, ids, V, 0.5, 2, dtype=dt[grad]))


@pytest.mark.parametrize("tokens", [300, 9000, 140000])
def test_the_largest_table(tokens):
    """2^27 ids: keys up to that number itself take 28 bits, four passes of seven. Sums of whole numbers up to 256 are exact."""
    import torch
    import paper_2501_08453_amd as vc
    V = 1 << 27
    g = torch.Generator().manual_seed(tokens)
    ids = torch.randint(0, V, (tokens,), generator=g)
    ids[::3] = V - 1 - ids[::3] % 1000
    ids[1::7], ids[:3] = V + 5, torch.tensor([V - 1, 0, V - 1])
    dout = torch.randint(-2, 3, (tokens, 1), generator=g)
    real = ids < V
    met, where = torch.unique(ids[real], return_inverse=True)
    want = torch.zeros((len(met), 1), dtype=torch.int64).index_add_(0, where, dout[real])
    assert int(want.abs().max()) <= 256
    got = vc.embedding_bwd(dout.to(torch.bfloat16).cuda(), ids.cuda(), V)
    assert torch.equal(got[met.cuda()].cpu().long(), want)
    got[met.cuda()] = 0
    assert not got.any()
