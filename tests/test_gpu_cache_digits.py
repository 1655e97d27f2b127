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
