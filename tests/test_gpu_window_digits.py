"""Digits of small probabilities in window attention: a first token whose score stands `gap` above all others' and whose value is 0, so that the outputs are what the
others' probabilities, e^-gap of the largest, make of their values, which are positive.

Tolerances are those of test_gpu_window_attention.py, and for float16 what its end of range loses: lifted by 2^14 a probability of e^-gap of the largest is a number of
2^14 e^-gap, and off by half a step of 2^-24: 2^-39 e^gap of itself (twice that here, as the scores vary around the gap).  In the gradient each line's terms are
scaled so that steps are 2^-32 of its largest or less: nothing beside the 64 * 2^-24.
"""
import math

import pytest
import torch

from paper_2501_08455_amd import autograd
from test_gpu_window_attention import TYPES, UNIT, noise, reference

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("gap", [6, 12, 17, 19])
@pytest.mark.parametrize("spread", [0.0, 0.5])
@pytest.mark.parametrize("B,T,K,V", [(1, 2500, 16, 32), (3, 300, 64, 64), (2, 400, 16, 130)])      # (the first: its keys cut into pieces)
def test_a_first_token_above_all_others(B, T, K, V, spread, gap, kind):
    k, v, q, g = (noise(B, T, 1, d, seed=i) for i, d in enumerate((K, V, K, V)))
    k, v = k * spread / (K - 1) ** 0.5, v.abs() * 16
    k[..., 0], q[..., 0] = 0.0, 1.0
    k[:, 0], v[:, 0] = 0.0, 0.0
    k[:, 0, :, 0] = gap
    g = g.abs() / 16
    q, k, v, g = (t.to(kind).cuda() for t in (q, k, v, g))
    q, k, v = (t.requires_grad_(True) for t in (q, k, v))
    o = autograd.window_attention(q, k, v, scale=1.0)
    want = reference(q, k, v, None, 0, None, 1.0, g)
    lost = 2.0 ** -38 * math.exp(gap) if kind == torch.float16 else 0.0
    for name, got in zip(("o", "grad q", "grad k", "grad v"), (o, *torch.autograd.grad(o, (q, k, v), g))):
        value, size = want[name]
        err = float((got.detach().cpu().double() - value).norm())
        # (numbers of float16 end at 2^-24: each is off by half of that there)
        floor = 2.0 ** -25 * math.sqrt(value.numel()) if kind == torch.float16 else 0.0
        assert err <= (2 * UNIT[kind] + 64 * 2.0 ** -24 + (lost if name == "o" else 0.0)) * size + floor, (name, err / size, floor / size)


@gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("power", [7, 17, 23, 26])
def test_scores_up_to_many_millions(power, kind):
    """Each token's own score is the largest, by 2^(power - 7).  Scores of 2^power and more are exact, but not times log2 e, which a maximum is kept as: that is rounded by up to
    2^(power - 23)."""
    B, T, K, V = 2, 100, 16, 24
    k = (128.0 + torch.arange(T)).view(1, T, 1, 1).expand(B, T, 1, K).contiguous()
    q = torch.full((B, T, 1, K), 2.0 ** (power - 11))
    v, g = noise(B, T, 1, V, seed=1, kind=kind), noise(B, T, 1, V, seed=2, kind=kind).cuda()
    q, k, v = (t.to(kind).cuda().requires_grad_(True) for t in (q, k, v))
    o = autograd.window_attention(q, k, v, scale=1.0)
    want = reference(q, k, v, None, 0, None, 1.0, g)
    # (what a line's probabilities are kept relative to is the same in both passes, so that its rounding takes nothing from them)
    for name, got in zip(("o", "grad v"), (o, torch.autograd.grad(o, (q, k, v), g)[2])):
        value, size = want[name]
        err = float((got.detach().cpu().double() - value).norm())
        assert err <= (2 * UNIT[kind] + 64 * 2.0 ** -24) * size, (name, err / size)
