"""Float32 window attention and NaN of any bits: one whose upper half alone would read as infinity is NaN all the same, to all tokens that see it and to no other."""
import pytest
import torch

from paper_2501_08455_amd import autograd
from test_gpu_window_attention import noise, visible_reference

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("what", ["q", "k", "v", "grad"])
@pytest.mark.parametrize("bits", [0x7f800001, 0xff800001 - (1 << 32), 0x7f80ffff, 0x7fc00000])
@pytest.mark.parametrize("where", [0, 70, 199])
@pytest.mark.parametrize("K,window,sinks", [(64, 23, 2), (24, 200, 0), (96, 23, 2), (128, 23, 2)])
def test_nan_of_any_bits(K, window, sinks, where, bits, what):
    T = 200
    x = {name: noise(T, K, seed=i) for i, name in enumerate(("q", "k", "v", "grad"))}
    x[what].view(torch.int32)[where, 7] = bits
    assert torch.isnan(x[what]).sum() == 1
    want = visible_reference(x["q"], x["k"], x["v"], window, sinks, x["grad"])
    q, k, v, g = (x[name].cuda()[None, :, None] for name in ("q", "k", "v", "grad"))
    q, k, v = (t.requires_grad_(True) for t in (q, k, v))
    o = autograd.window_attention(q, k, v, window=window, sinks=sinks)
    for name, got, value in zip(("o", "grad q", "grad k", "grad v"), (o, *torch.autograd.grad(o, (q, k, v), g)), want):
        got = got.detach().cpu()[0, :, 0]
        assert torch.equal(torch.isfinite(got), torch.isfinite(value)), name
        if name == "o":
            assert torch.equal(torch.isnan(got), torch.isnan(value))
