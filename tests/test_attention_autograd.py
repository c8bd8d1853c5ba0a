"""The autograd function of the attention binding, with the library's two calls replaced by torch on the CPU: first derivatives pass through, and second ones, which
the library does not have, are refused instead of left out."""
import math

import pytest
import torch


@pytest.fixture
def at(monkeypatch):
    from paper_2404_04541_amd import attention

    def forward(handle, plan, q, k, v, scale=None, cap=0.0, slopes=None):
        with torch.enable_grad():
            s = torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(q.shape[2])
            o = torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), v)
        return o, torch.logsumexp(s, -1)

    def backward(handle, plan, q, k, v, o, lse, d_o, scale=None, cap=0.0, slopes=None):
        with torch.enable_grad():
            x = [t.detach().requires_grad_() for t in (q, k, v)]
            return torch.autograd.grad(forward(None, None, *x)[0], x, d_o.detach())

    monkeypatch.setattr(attention, "forward", forward)
    monkeypatch.setattr(attention, "backward", backward)
    return attention


def inputs(seed=0):
    gen = torch.Generator().manual_seed(seed)
    return [torch.randn((7, 2, 4), generator=gen, dtype=torch.float64, requires_grad=True) for _ in range(3)]


def test_first_derivatives(at):
    x = inputs()
    got = torch.autograd.grad(at.attention(None, None, *x).square().sum(), x)
    want = torch.autograd.grad(at.forward(None, None, *x)[0].square().sum(), x)
    assert all(torch.allclose(a, b) for a, b in zip(got, want))


def test_second_derivatives_are_refused(at):
    """A loss with a penalty on its gradients: without a refusal the penalty would add nothing, and nobody would know."""
    x = inputs()
    loss = at.attention(None, None, *x).square().sum()
    grads = torch.autograd.grad(loss, x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (loss + sum(g.square().sum() for g in grads)).backward()
