"""A window model's cache that has no room for another point: refused as it is, so that a larger one goes on from it."""
import pytest
import torch

from paper_2501_08455_amd import sequence
from test_gpu_sequence_model import near

gpu = pytest.mark.gpu


def test_a_full_cache_is_refused_before_anything_is_touched():
    model = sequence.SequenceModel(4, 3, 2, 5, heads=2, head_dim=8, device="cpu", mixer="window", window=5)
    cache = model.begin(torch.zeros(2, 4), 3)
    cache["room"] = 0
    before = {name: value.clone() if isinstance(value, torch.Tensor) else value for name, value in cache.items()}
    with pytest.raises(ValueError, match="no room"):
        model.step(torch.ones(2, 4), cache)
    for name, value in before.items():
        assert torch.equal(cache[name].float(), value.float()) if isinstance(value, torch.Tensor) else cache[name] == value, name


@gpu
@pytest.mark.parametrize("kind", [None, torch.float8_e4m3fn])
def test_a_larger_cache_goes_on_from_a_full_one(kind):
    torch.manual_seed(4)
    model = sequence.SequenceModel(4, 3, 3, 5, heads=2, head_dim=24, mixer="window")
    x = torch.randn(3, 30, 4, device="cuda").cumsum(1) * 0.2
    whole, cache, larger = model.begin(x[:, 0], 29, kind=kind), model.begin(x[:, 0], 16, kind=kind), model.begin(x[:, 0], 32, kind=kind)
    for t in range(1, 30):
        want = model.step(x[:, t], whole)
        if t == 17:
            names = [name for name, value in cache.items() if isinstance(value, torch.Tensor)]
            before = {name: cache[name].clone() for name in names}
            with pytest.raises(ValueError, match="no room"):
                model.step(x[:, t], cache)
            for name in names:
                assert torch.equal(cache[name].float(), before[name].float()), name
            for name in ("keys", "values", "key_scales", "value_scales"):
                if cache[name] is not None:
                    larger[name][larger["table"][:, :1].long()] = cache[name][cache["table"].long()]
            cache = dict(larger, point=cache["point"], row=cache["row"], lengths=cache["lengths"], room=16)
        near(model.step(x[:, t], cache), want.cpu(), t)
