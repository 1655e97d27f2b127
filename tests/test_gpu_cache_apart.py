"""What an append writes lies apart: keys, values and their scales from one another, pages from other pages, and all of them from what is read.  (Calls that would race are
refused before anything is launched.)"""
import itertools
import random

import pytest
import torch

from paper_2501_08455_amd import binding
from test_gpu_cache import E4M3, Pool
from test_gpu_window_attention import noise

gpu = pytest.mark.gpu


def append_nothing(keys, values, **scales):
    """A call without tokens: what it checks, and no launch."""
    n = torch.zeros(1, dtype=torch.int64, device="cuda")
    k, v = (torch.zeros(1, 0, t.shape[1], t.shape[3], device="cuda") for t in (keys, values))
    binding.cache_append(k, v, keys, values, torch.zeros(1, 1, dtype=torch.int32, device="cuda"), n, **scales)


def places_of(t):
    """(numbers of a tensor's values along its storage, whether they are all different)"""
    at = [t.storage_offset() + sum(i * s for i, s in zip(index, t.stride())) for index in itertools.product(*map(range, t.shape))]
    return set(at), len(set(at)) == len(at)


@gpu
def test_layouts_against_the_places_that_they_take():
    rng = random.Random(5)
    buffer = torch.zeros(4000, device="cuda")
    refused = accepted = 0
    for _ in range(1500):
        G, P, pages = (rng.randint(1, 4) for _ in range(3))
        K, V = rng.randint(1, 5), rng.randint(1, 5)
        views = []
        axes = rng.sample(range(3), 3)
        for width in (K, V):
            if rng.random() < 0.3:
                axes = rng.sample(range(3), 3)
            strides, step = [0, 0, 0], width if rng.random() < 0.4 else K + V
            for axis in axes:      # (axes that hold one another, with some room or none, or too little)
                strides[axis] = max(1, step + rng.choice((0, 0, 0, 1, 3, -1)))
                step = strides[axis] * (pages, G, P)[axis]
            views.append(buffer.as_strided((pages, G, P, width), (*strides, 1), rng.choice((0, K, V, K * P, K * P * G, rng.randint(0, 60), 900))))
        (keys, one), (values, other) = map(places_of, views)
        try:
            append_nothing(*views)
            assert one and other and not keys & values, [(v.shape, v.stride(), v.storage_offset()) for v in views]
            accepted += 1
        except ValueError:
            assert not one or not other or keys & values, [(v.shape, v.stride(), v.storage_offset()) for v in views]
            refused += 1
    assert refused > 300 and accepted > 300


@gpu
def test_one_tensor_for_two():
    pool, narrow = Pool(1, 16, 2, 4, 8, 8, torch.float32), Pool(1, 16, 2, 4, 8, 8, E4M3)
    before = [t.clone() for t in (pool.keys, narrow.keys.float(), narrow.key_scales)]
    k = torch.ones(1, 3, 2, 8, device="cuda")
    n, table = torch.zeros(1, dtype=torch.int64, device="cuda"), pool.table
    scales = torch.ones(2 * narrow.key_scales.numel(), device="cuda")
    first, second, between = (scales[i:i + narrow.key_scales.numel()].view_as(narrow.key_scales) for i in (0, narrow.key_scales.numel(), 3))
    for keys, values, more in ((pool.keys, pool.keys, {}), (pool.keys, pool.keys.view_as(pool.keys), {}), (narrow.keys, narrow.values, dict(key_scales=first, value_scales=first)),
                               (narrow.keys, narrow.values, dict(key_scales=first, value_scales=between)), (narrow.keys, narrow.keys, dict(key_scales=first, value_scales=second)),
                               (narrow.keys, narrow.values, dict(key_scales=narrow.values.view(-1)[:40].view(torch.float32).view(5, 2), value_scales=second))):
        with pytest.raises(ValueError, match="must lie apart"):
            binding.cache_append(k, k, keys, values, table, n, **more)
    # a table, lengths and positions that stand in the pages
    inside = pool.keys.view(-1).view(torch.int32)
    f = torch.ones(2, dtype=torch.float64, device="cuda")
    for more in (dict(table=inside[:4].view(1, 4), lengths=n), dict(table=table, lengths=inside[:1]), dict(table=table, lengths=n, positions=inside[:3], frequencies=f)):
        if more["lengths"] is not n:
            more["lengths"] = pool.keys.view(-1).view(torch.int64)[:1]      # (int32 lengths are copied)
        with pytest.raises(ValueError, match="apart from the cache"):
            binding.cache_append(k, k, pool.keys, pool.values, **more)
    for was, t in zip(before, (pool.keys, narrow.keys.float(), narrow.key_scales)):
        assert torch.equal(was, t)
    binding.cache_append(k, k, narrow.keys, narrow.values, table, n, key_scales=first, value_scales=second)
    assert float(first[int(table[0, 0]), 0]) == float(second[int(table[0, 0]), 0]) == 2.0 ** -8
    # attention only reads, and may take keys for values
    q = torch.ones(1, 1, 2, 8, device="cuda")
    assert torch.equal(binding.cache_attention(q, pool.keys, pool.keys, table, n + 3), torch.full((1, 1, 2, 8), 7.0, device="cuda"))


@gpu
@pytest.mark.parametrize("layout", ["pages", "heads", "slots"])
def test_keys_and_values_in_turn(layout):
    """Keys and values of a page, of a head or of a token next to each other, of different widths."""
    B, T, G, P, K, V = 2, 40, 3, 16, 24, 40
    pool = Pool(B, T, G, P, K, V, torch.float32)
    n, zero = pool.keys.shape[0], torch.zeros(B, dtype=torch.int64, device="cuda")
    k, v, q = noise(B, T, G, K, seed=1).cuda(), noise(B, T, G, V, seed=2).cuda(), noise(B, 1, G, K, seed=3).cuda()
    if layout == "pages":
        both = torch.zeros(n, G * P * (K + V), device="cuda")
        keys, values = both[:, :G * P * K].unflatten(1, (G, P, K)), both[:, G * P * K:].unflatten(1, (G, P, V))
    elif layout == "heads":
        both = torch.zeros(n, G, P * (K + V), device="cuda")
        keys, values = both[..., :P * K].unflatten(2, (P, K)), both[..., P * K:].unflatten(2, (P, V))
    else:
        both = torch.zeros(n, P, G * (K + V), device="cuda")
        keys, values = both[..., :G * K].unflatten(2, (G, K)).transpose(1, 2), both[..., G * K:].unflatten(2, (G, V)).transpose(1, 2)
    lengths = torch.tensor([40, 31], device="cuda")
    for a, b in ((pool.keys, pool.values), (keys, values)):
        binding.cache_append(k, v, a, b, pool.table, zero)
    rows = pool.table.long().flatten()
    held = torch.arange(pool.n * P, device="cuda").view(pool.n, P) < T
    for a, b in ((keys, pool.keys), (values, pool.values)):
        assert torch.equal(a[rows].transpose(1, 2)[held.repeat(B, 1)], b[rows].transpose(1, 2)[held.repeat(B, 1)])
    assert torch.equal(binding.cache_attention(q, keys, values, pool.table, lengths), binding.cache_attention(q, pool.keys, pool.values, pool.table, lengths))
