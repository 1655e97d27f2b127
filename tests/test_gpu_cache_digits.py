"""Digits of small probabilities in attention over a cache: one place whose score stands `gap` above all others' and whose value is 0, so that the output is what
the others' probabilities, e^-gap of the largest, make of their values.

Tolerances are those of test_gpu_cache.py, and for float16 pages what two float16 numbers of a probability lose at the end of that type's range: lifted by 2^15 they
have steps of 2^-24, so a probability of e^-gap of the largest is off by 2^-25 / (2^15 e^-gap) = 2^-40 e^gap of itself at most (twice that here, as the scores
vary around the gap).  Exponents of up to 18 / ln 2 = 26 are rounded by 2^-20, which is 11 of the 64 * 2^-24.
"""
import math

import pytest
import torch

from paper_2501_08455_amd import binding
from test_gpu_cache import CACHES, Pool, attention_reference
from test_gpu_window_attention import UNIT, noise

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("kind,cache", CACHES)
@pytest.mark.parametrize("gap", [6, 12, 15, 18])
@pytest.mark.parametrize("spread", [0.0, 0.5])
@pytest.mark.parametrize("G,places", [(2, 4000), (512, 300)])      # cut along the places, and whole
def test_one_place_above_all_others(G, places, spread, gap, kind, cache):
    K, V, P = 8, 16, 16
    pool = Pool(1, places, G, P, K, V, cache)
    k, v = noise(1, places, G, K, seed=1, kind=kind).cuda(), noise(1, places, G, V, seed=2, kind=kind).cuda()
    k *= spread / (K - 1) ** 0.5
    k[..., 0] = 0.0
    k[:, 0, :, 0], k[:, 0, :, 1:], v[:, 0] = float(gap), 0.0, 0.0
    q = noise(1, 1, G, K, seed=3, kind=kind).cuda()
    q[..., 0] = 1.0
    binding.cache_append(k, v, pool.keys, pool.values, pool.table, torch.zeros(1, dtype=torch.int64, device="cuda"), **pool.scales())
    lengths = torch.tensor([places], device="cuda")
    got = binding.cache_attention(q, pool.keys, pool.values, pool.table, lengths, scale=1.0, **pool.scales())
    value, size = attention_reference(q, pool, lengths, [1], None, 0, 1.0)
    err = float((got.cpu().double() - value).norm())
    # (outputs of float16 themselves end at 2^-24: each is off by half of that there)
    floor = 2.0 ** -25 * math.sqrt(G * V) if kind == torch.float16 else 0.0
    lost = 2.0 ** -39 * math.exp(gap) if cache == torch.float16 else 0.0
    assert err <= ((1 + 2.0 ** -7) * UNIT[kind] + 64 * 2.0 ** -24 + lost) * size + floor, (err / size, floor / size)


@gpu
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("power", [7, 17, 23, 26])
def test_scores_up_to_many_millions(power, kind):
    """The last place's score is the largest by 2^(power - 7): its value is the output.  Scores of 2^power and more are exact, but not over their maximum times log2 e, which
    is rounded by up to 2^(power - 23)."""
    n, K, V = 100, 16, 24
    k = torch.full((n, 1, 1, K), 2.0) * 64 + torch.arange(n).view(n, 1, 1, 1)
    q = torch.full((n, 1, 1, K), 2.0 ** (power - 11))
    v = noise(n, 1, 1, V, seed=1)
    table = torch.arange(n).int().expand(n, n).cuda()
    got = binding.cache_attention(q.to(kind).cuda(), k.to(kind).cuda(), v.to(kind).cuda(), table, torch.arange(1, n + 1).cuda(), scale=1.0)
    want = v.to(kind).double()[:, 0, 0]
    err = (got.cpu().double()[:, 0, 0] - want).norm()
    # (at 2^7 the place before is e^-1 of the last: that case is the definition's)
    if power == 7:
        p = torch.softmax((torch.arange(n) * 1.0).expand(n, n).masked_fill(torch.arange(n) > torch.arange(n)[:, None], -math.inf).double(), -1)
        want, size = p @ v.to(kind).double()[:, 0, 0], p @ v.to(kind).double().abs()[:, 0, 0]
        err = (got.cpu().double()[:, 0, 0] - want).norm()
    else:
        size = want
    assert err <= ((1 + 2.0 ** -7) * UNIT[kind] + 64 * 2.0 ** -24) * size.norm(), float(err / size.norm())
