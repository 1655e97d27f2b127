"""Softmax attention of few queries that see many keys: cut along the keys, joined by a second launch (the tolerances of test_gpu_window_attention.py)."""
import math

import pytest
import torch

from paper_2501_08455_amd import autograd, binding
from test_gpu_window_attention import TYPES, UNIT, assert_near, noise, reference, seen_by

gpu = pytest.mark.gpu
NAMES = ("o", "grad q", "grad k", "grad v")

# B, T, heads, shared, K, V, window, sinks.  Two pieces or more of each (up to 16)
SHAPES = [(1, 1024, 1, 1, 64, 64, None, 0), (1, 2100, 2, 1, 128, 128, None, 0), (1, 1600, 3, 3, 40, 72, None, 0), (2, 1100, 1, 1, 256, 130, None, 0), (1, 2500, 2, 2, 96, 96, 1100, 5),
          (1, 1800, 2, 2, 33, 33, 600, 500), (1, 1300, 4, 2, 1, 3, None, 0), (1, 512, 1, 1, 128, 128, None, 0), (1, 777, 2, 1, 96, 96, None, 0), (1, 4096, 1, 1, 8, 8, None, 0), (1, 1700, 1, 1, 30, 5, None, 0), (1, 2600, 1, 1, 16, 24, 2599, 1)]


def operands(shape, kind):
    B, T, H, G, K, V = shape[:6]
    return (noise(B, T, H, K, seed=1, kind=kind), noise(B, T, G, K, seed=2, kind=kind), noise(B, T, G, V, seed=3, kind=kind), noise(B, T, H, V, seed=4, kind=kind))


def both(q, k, v, g, **more):
    q, k, v = (t.cuda().requires_grad_(True) for t in (q, k, v))
    o = autograd.window_attention(q, k, v, **more)
    return (o.detach(), *torch.autograd.grad(o, (q, k, v), g.cuda()))


@gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("shape", SHAPES)
def test_outputs_and_gradients(shape, kind):
    q, k, v, g = operands(shape, kind)
    window, sinks = shape[6:]
    got = both(q, k, v, g, window=window, sinks=sinks)
    want = reference(q, k, v, window, sinks, None, None, g)
    for name, x in zip(NAMES, got):
        assert_near(x, want[name], (name, shape))
    # (without a gradient, and again: the same bits)
    assert torch.equal(binding.window_attention(q.cuda(), k.cuda(), v.cuda(), window=window, sinks=sinks), got[0])
    for x, y in zip(got, both(q, k, v, g, window=window, sinks=sinks)):
        assert torch.equal(x, y)


@gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("window,sinks", [(None, 0), (1000, 30), (7, 1200)])
def test_ragged_sequences(window, sinks, kind):
    """Lengths that leave whole pieces and whole sequences without a token; what stands behind them is NaN."""
    B, T, H, G, K, V = 5, 1500, 2, 1, 40, 24
    lengths = torch.tensor([0, 1, 1499, 700, 5000])
    q, k, v, g = operands((B, T, H, G, K, V), kind)
    want = reference(q, k, v, window, sinks, lengths, None, g)
    behind = torch.arange(T) >= lengths[:, None]
    q, k, v, g = (t.masked_fill(behind[:, :, None, None], math.nan) for t in (q, k, v, g))
    got = both(q, k, v, g, window=window, sinks=sinks, lengths=lengths.cuda())
    for name, x in zip(NAMES, got):
        assert_near(x, want[name], name)
        assert not x.cpu()[behind].any(), name


@gpu
@pytest.mark.parametrize("kind", TYPES)
def test_scores_that_lie_far_apart(kind):
    """Pieces whose maxima differ by hundreds: the smaller ones count for nothing, and nothing overflows."""
    T, K = 1200, 64
    q, k, v, g = operands((1, T, 1, 1, K, K), kind)
    k = k.clone()
    k[:, 500:700] *= 20
    want = reference(q, k, v, None, 0, None, None)["o"]
    got = binding.window_attention(q.cuda(), k.cuda(), v.cuda())
    # (scores of up to some 300, each off by 64 * 2^-24 of that)
    value, size = want
    assert float((got.cpu().double() - value).norm()) <= (2 * UNIT[kind] + (64 + 64 * 300) * 2.0 ** -24) * size


@gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("what,bad", [("k", math.nan), ("v", math.inf), ("v", -math.inf), ("q", math.nan), ("grad", math.inf)])
@pytest.mark.parametrize("where", [3, 640, 1199])
def test_what_is_not_finite_reaches_only_what_sees_it(where, what, bad, kind):
    T, window, K = 1200, 1100, 32
    ops = dict(zip(("q", "k", "v", "grad"), operands((1, T, 1, 1, K, K), kind)))
    clean = both(*ops.values(), window=window)
    ops[what] = ops[what].clone()
    ops[what][0, where, 0, 7] = bad
    got = both(*ops.values(), window=window)
    seen = seen_by(T, window, 0)
    rows = seen[:, where] if what in "kv" else torch.arange(T) == where      # tokens whose output or gradient it spoils
    keys = seen[rows].any(0)
    o, gq, gk, gv = (torch.isfinite(x[0, :, 0].cpu()) for x in got)
    if what == "grad":
        assert bool(o.all())
    else:
        assert bool(o[~rows].all()) and not bool((o[rows].all(1) if what in "qk" else o[rows, 7]).any())
    assert bool(gq[~rows].all()) and not bool(gq[rows].all(1).any())
    for x in (gk, gv):
        assert bool(x[~keys].all())
    for x, y, spoilt in zip(got, clean, (rows, rows, keys, keys)):
        x, y = (t[0, :, 0].cpu()[~spoilt].double() for t in (x, y))
        assert float((x - y).norm()) <= 8 * (2 * UNIT[kind] + 64 * 2.0 ** -24) * float(y.norm())


@gpu
def test_captured_calls_replay():
    q, k, v, g = (t.cuda() for t in operands((1, 2000, 2, 1, 64, 64), torch.bfloat16))
    want = binding.window_attention(q, k, v)
    graph, stream = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        binding.window_attention(q, k, v)
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            o = binding.window_attention(q, k, v)
    torch.cuda.current_stream().wait_stream(stream)
    for _ in range(4):
        o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want)
        assert torch.equal(binding.window_attention(q, k, v), want)
        q.mul_(1.25)
        want = binding.window_attention(q, k, v)
