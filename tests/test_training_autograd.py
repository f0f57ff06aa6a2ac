"""The backward pass and the autograd node of the gated FFN without a device: the two calls are replaced by their formulas, so what is tested
is which gradients the node asks for, what it hands back, and what is refused."""
import pytest
import torch

import training_reference as ref
from paper_2609_31975_b200 import training


@pytest.fixture()
def node(monkeypatch):
    asked = []

    def forward(x, W_g, b_g, W_up, W_down, act="relu", act_up=None, *, save=True):
        f = ref.forward(x, W_g, b_g, W_up, W_down, act, act_up)
        return (f["y"], f["z"], f["u"]) if save else (f["y"], None, None)

    def backward(dy, x, z, u, W_g, W_up, W_down, act="relu", act_up=None, *, need):
        asked.append(sorted(need))
        assert dy.is_contiguous() and dy.shape == x.shape and dy.data_ptr() % 16 == 0   # as the kernels take it
        return {k: v for k, v in ref.backward(dy, x, z, u, W_g, W_up, W_down, act, act_up).items() if k in need}

    monkeypatch.setattr(training, "gated_ffn_forward", forward)
    monkeypatch.setattr(training, "gated_ffn_backward", backward)
    return training.GatedFFNFunction.apply, asked


def leaves(wanted=(True,) * 5):
    g = torch.Generator().manual_seed(7)
    rnd = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    return [t.requires_grad_(w) for t, w in zip((rnd(2, 3, 8), rnd(5, 8), rnd(5), rnd(5, 8), rnd(5, 8)), wanted)]


def plain(x, W_g, b_g, W_up, W_down):
    z = x @ W_g.T + b_g
    return (z * torch.sigmoid(z) * (x @ W_up.T)) @ W_down


def test_second_derivatives_are_refused(node):
    """The backward pass is not a graph of torch's: a gradient taken with create_graph would count as a constant, and what depends on
    it would be lost without a word."""
    apply, _ = node
    t = leaves()
    y = apply(*t, "silu", None)
    loss = y.square().mean()
    g, = torch.autograd.grad(loss, t[1], create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (loss + g.square().sum()).backward()


@pytest.mark.parametrize("wanted", [(True,) * 5, (False, True, True, True, True), (True, False, False, False, False), (False, False, True, False, False),
                                    (True, False, True, False, True)])
def test_frozen_tensors_get_no_gradient(node, wanted):
    apply, asked = node
    t = leaves(wanted)
    apply(*t, "silu", None).sin().sum().backward()
    names = ("dx", "dW_g", "db_g", "dW_up", "dW_down")
    assert asked == [sorted(n for n, w in zip(names, wanted) if w)]
    want = torch.autograd.grad(plain(*t).sin().sum(), [x for x, w in zip(t, wanted) if w])
    got = [x.grad for x in t if x.grad is not None]
    assert len(got) == len(want) and all(torch.allclose(a, b, atol=1e-12) for a, b in zip(got, want))


def test_gradients_that_are_expanded(node):
    apply, _ = node
    t = leaves()
    apply(*t, "silu", None).sum().backward()          # dy is one number, expanded
    want = torch.autograd.grad(plain(*t).sum(), t)
    assert all(torch.allclose(x.grad, w, atol=1e-12) for x, w in zip(t, want))


def test_gradients_that_are_slices(node):
    """dy comes from torch, as whatever it is: here the tail of a longer vector, which does not start on 16 bytes."""
    apply, _ = node
    t = leaves()
    weights = torch.linspace(-1, 1, 1 + 2 * 3 * 8, dtype=torch.float64)
    head = torch.zeros(1, dtype=torch.float64)
    (torch.cat([head, apply(*t, "silu", None).flatten()]) * weights).sum().backward()
    want = torch.autograd.grad((torch.cat([head, plain(*t).flatten()]) * weights).sum(), t)
    assert all(torch.allclose(x.grad, w, atol=1e-12) for x, w in zip(t, want))


def test_outputs_by_a_wrong_name_are_refused():
    """A misspelt output would be made anew, and the caller's tensor stay as it was."""
    w = torch.zeros(8, 8)
    with pytest.raises(ValueError, match="dWg"):
        training.gated_ffn_backward(w, w, w, w, w, w, w, out=dict(dWg=w))
