"""The sequence operators with more tokens or heads than one launch's threads can count (2^32), checked where one launch would end and at the
ends, in 64 bits, with the tolerance of tests/test_gpu_sequence_ops.py."""
import pytest
import torch

from paper_2501_08455_amd import autograd, binding
from test_gpu_sequence_ops import assert_near, attention_reference, rotary_reference

gpu = pytest.mark.gpu


def some(n, *edges):
    """places 0 .. n - 1: the first and last few and those around `edges`"""
    at = [torch.arange(max(0, e - 40), min(n, e + 40)) for e in (0, *edges, n)]
    return torch.unique(torch.cat(at))


@gpu
@pytest.mark.parametrize("B,T", [(16411, 16384), (1, (1 << 28) + 77)])
def test_rotary_of_more_tokens_than_a_launch_has_threads(B, T):
    x = torch.randn(B, T, 1, 2, device="cuda", dtype=torch.bfloat16)
    f = torch.tensor([0.01], dtype=torch.float64, device="cuda")
    positions = torch.arange(T, device="cuda")
    y = binding.rotary(x, positions, f)
    assert torch.isfinite(y).all()
    at = some(B * T, 1 << 27, 1 << 28)
    b, t = at // T, at % T
    assert_near(y[b, t][None], rotary_reference(x[b, t][None], t, f, False, 1.0))


@gpu
@pytest.mark.parametrize("B,H,G,T", [((1 << 24) + 41, 1, 1, 1), ((1 << 23) + 3, 2, 1, 1), ((1 << 24) + 41, 1, 1, 5), (5600000, 3, 3, 3)])
def test_linear_attention_of_more_heads_than_a_launch_has_workgroups(B, H, G, T):
    K = V = 2
    gen = torch.Generator(device="cuda").manual_seed(7)
    q, k, v, g = (torch.randn(B, T, n, K, device="cuda", generator=gen) for n in (H, G, G, H))
    state, g_state = (torch.randn(B, H, K, V, device="cuda", generator=gen) for _ in range(2))
    log_decay = torch.log(torch.linspace(0.5, 0.9, H)).cuda()
    lengths = torch.randint(0, T + 1, (B,), device="cuda", generator=gen)
    ins = [t.requires_grad_(True) for t in (q, k, v, state)]
    out = autograd.linear_attention(*ins[:3], log_decay, state=state, lengths=lengths, return_state=True)
    got = list(out) + list(torch.autograd.grad(out, ins, (g, g_state)))
    slices = ((1 << 24) - 1) // H
    at = some(B, slices).cuda()
    want = attention_reference(q[at], k[at], v[at], log_decay, state[at], lengths[at], K ** -0.5, g[at], g_state[at])
    for a, b, name in zip(got, want, ("o", "state", "grad q", "grad k", "grad v", "grad state")):
        assert_near(a[at], b, what=name)


@gpu
def test_shared_heads_gradients_in_slices_of_the_batch():
    """More scratch than a call takes at once: the last slice's gradients as those of a call of their own (which cuts sequences otherwise, so that
    sums differ before they are rounded)."""
    B, T, H, G, K = 9, 65536, 16, 4, 128
    gen = torch.Generator(device="cuda").manual_seed(8)
    q, k, v, g = (torch.randn(B, T, n, K, device="cuda", generator=gen).bfloat16() for n in (H, G, G, H))
    log_decay = torch.log1p(-torch.exp2(-2.0 - 6.0 * torch.arange(H, device="cuda") / H))

    def gradients(*ins):
        ins = [t.detach().requires_grad_(True) for t in ins[:3]] + [ins[3]]
        return torch.autograd.grad(autograd.linear_attention(*ins[:3], log_decay), ins[:3], ins[3])

    got = gradients(q, k, v, g)
    for b in (0, B - 2, B - 1):
        for x, y in zip(got, gradients(*(t[b:b + 1] for t in (q, k, v, g)))):
            assert float((x[b] - y[0]).float().norm()) <= 2.0 ** -8 * float(y.float().norm())
