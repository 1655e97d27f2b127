"""What a sequence's output in attention over a cache does not depend on: pages of other sequences."""
import math

import pytest
import torch

from paper_2501_08455_amd import binding
from test_gpu_cache import CACHES, E4M3, Pool
from test_gpu_window_attention import noise

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("kind,cache", CACHES)
@pytest.mark.parametrize("T,window,sinks", [(1, None, 0), (6, 40, 3)])
@pytest.mark.parametrize("D", [64, 40])
def test_pages_of_others_may_hold_anything(D, T, window, sinks, kind, cache):
    """NaN in the first page, which no table names: the same bits, for whole blocks, last blocks and places without a page."""
    B, H, G, P, places = 5, 4, 2, 8, 330
    pool = Pool(B, places, G, P, D, D, cache)
    pool.table = (1 + torch.randperm(B * pool.n, generator=torch.Generator().manual_seed(4))).view(B, pool.n).int().cuda()
    k, v, q = (noise(B, n, h, D, seed=i, kind=kind).cuda() for i, (n, h) in enumerate(((pool.n * P, G), (pool.n * P, G), (T, H))))
    binding.cache_append(k, v, pool.keys, pool.values, pool.table, torch.zeros(B, dtype=torch.int64, device="cuda"), **pool.scales())
    pool.table[1, 3], pool.table[4, :17] = -1, -1      # (the latter: whole blocks)
    lengths = torch.tensor([330, 129, 64, 7, 250], device="cuda")
    attend = lambda: binding.cache_attention(q, pool.keys, pool.values, pool.table, lengths, window=window, sinks=sinks, **pool.scales())      # noqa: E731
    want = attend()
    assert torch.isfinite(want).all()
    for bad in (math.nan, math.inf):
        pool.keys[0], pool.values[0] = (torch.full_like(t[0], bad, dtype=torch.float32).to(cache) for t in (pool.keys, pool.values))
        if cache == E4M3:
            pool.key_scales[0] = pool.value_scales[0] = bad
        assert torch.equal(attend(), want)
