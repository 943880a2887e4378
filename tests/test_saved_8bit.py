"""saved_in_8bit on the CPU, where nothing is packed: what it keeps is what autograd keeps without it."""
import gc
import weakref

import pytest

import paper_2501_08453_amd as vc

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("op", [torch.exp, lambda t: t.softmax(-1), lambda t: t.sigmoid() * t, lambda t: t[:, :3].tanh()])
def test_a_graph_that_is_dropped_is_freed(op):
    """An operation that saves its own result holds it; kept as it is, the result would hold the operation in turn."""
    gone = []
    for context in (torch.enable_grad, vc.saved_in_8bit):
        x = torch.randn((4, 70), requires_grad=True)
        with context():
            y = op(x)
        ref = weakref.ref(y)
        del y
        gc.collect()
        gone.append(ref() is None)
    assert gone == [True, True]


def test_gradients_of_what_is_not_packed():
    """Those without the context, of the first and of the second order."""
    x = torch.randn((5, 70), dtype=torch.float64, requires_grad=True)
    w = torch.randn((70, 66), dtype=torch.float64, requires_grad=True)
    got = []
    for context in (torch.enable_grad, vc.saved_in_8bit):
        with context():
            y = ((x * 2).exp() @ w).softmax(-1)
            g = torch.autograd.grad((y * y).sum(), (x, w), create_graph=True)
            gg = torch.autograd.grad(sum((t * t).sum() for t in g), (x, w))
        got.append(g + gg)
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_changed_in_place_after_it_was_saved():
    """Hooks switch off autograd's own check: without another, the backward would go on with the changed values."""
    x = torch.randn((4, 70), requires_grad=True)
    w = torch.randn((70, 70), requires_grad=True)

    def result(a):
        y = a.exp()
        y.add_(1)
        return y

    def operand(a):
        u = a * 2
        y = u * u
        u[1:].zero_()
        return y

    def weight(a):
        y = a @ w
        with torch.no_grad():
            w.mul_(0.5)
        return y

    for f in (result, operand, weight):
        with vc.saved_in_8bit():
            y = f(x)
        with pytest.raises(RuntimeError, match="in place"):
            torch.autograd.grad(y.sum(), x)
    with vc.saved_in_8bit():  # before it is saved, and what nobody saves, may change
        u = x * 2
        u.add_(1)
        y = u.exp() + 0
        y.mul_(3)
    assert torch.equal(torch.autograd.grad(y.sum(), x)[0], 6 * (2 * x.detach() + 1).exp())


def test_which_tensors_are_of_leaves():
    of = vc.blocks._of_leaves
    w, v, x = (torch.randn((4, 6), requires_grad=True) for _ in range(3))
    plain = torch.randn((4, 6))
    low = w.to(torch.bfloat16)
    for t in (w, plain, w.detach(), w.t(), w[1:], low, low.t().contiguous(), low.clone()[0], torch.cat([w, v]), torch.stack([w, plain]).unbind(0)[0],
              torch.cat([w.t().to(torch.bfloat16), plain.to(torch.bfloat16).t()], 1).view(-1), w.diagonal(), low.unsqueeze(0).expand(2, 4, 6)):
        assert of(t), t.grad_fn
    changed = w.clone()
    changed[0].mul_(2)
    for t in (w * 2, (w * 2).to(torch.bfloat16), (x + 0).t(), torch.cat([w, v * 2]), w.t() @ v, changed, changed.view(-1)):
        assert not of(t), t.grad_fn
    many = w
    for _ in range(40):  # 2^40 ways to the leaf
        many = torch.cat([many[:1], many[:1]])
    assert of(many)
