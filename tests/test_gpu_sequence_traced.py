"""The sequence operators under torch.jit.trace: gradients behave as those of the calls themselves."""
import pytest
import torch

from paper_2501_08455_amd import autograd

gpu = pytest.mark.gpu
SHAPE = (2, 6, 2, 8)


def calls():
    log_decay = torch.full((2,), -0.1, device="cuda")
    f = torch.ones(2, dtype=torch.float64, device="cuda")
    p = torch.arange(6, device="cuda")
    return {"layer_norm": lambda x: autograd.layer_norm(x), "rotary": lambda x: autograd.rotary(x, p, f),
            "linear_attention": lambda x: autograd.linear_attention(x, x, x, log_decay),
            "with a state": lambda x: sum(t.sum() for t in autograd.linear_attention(x, x, x, log_decay, return_state=True))}


def traced(name):
    return torch.jit.trace(calls()[name], (torch.randn(SHAPE, device="cuda"),), check_trace=False)


@gpu
@pytest.mark.parametrize("name", ["layer_norm", "rotary", "linear_attention", "with a state"])
def test_a_graph_can_be_walked_twice(name):
    x = torch.randn(SHAPE, device="cuda", requires_grad=True)
    y = traced(name)(x)
    g = torch.randn_like(y)
    (first,) = torch.autograd.grad(y, x, g, retain_graph=True)
    (second,) = torch.autograd.grad(y, x, g)
    (want,) = torch.autograd.grad(calls()[name](x), x, g)
    assert torch.equal(first, want) and torch.equal(second, want)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(y, x, g)       # and is gone after the second


@gpu
@pytest.mark.parametrize("name", ["layer_norm", "linear_attention"])
def test_a_change_in_place_of_what_is_saved_is_an_error(name):
    x = torch.randn(SHAPE, device="cuda", requires_grad=True)
    between = x * 1.0
    y = traced(name)(between).sum()
    with torch.no_grad():
        between.mul_(2.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        torch.autograd.grad(y, x)


@gpu
@pytest.mark.parametrize("name", ["layer_norm", "rotary", "linear_attention"])
def test_second_derivatives_are_refused_and_not_left_out(name):
    """... also where another part of the loss has one."""
    x = torch.randn(SHAPE, device="cuda", requires_grad=True)
    (gx,) = torch.autograd.grad(traced(name)(x).square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivative"):
        torch.autograd.grad(gx.sum() + x.pow(3).sum(), x)


@gpu
def test_what_has_no_gradient_is_refused_when_it_is_called():
    x = torch.randn(SHAPE, device="cuda")
    log_decay = torch.full((2,), -0.1, device="cuda", requires_grad=True)
    with pytest.raises(ValueError):
        torch.jit.trace(lambda x, d: autograd.linear_attention(x, x, x, d), (x, log_decay), check_trace=False)
