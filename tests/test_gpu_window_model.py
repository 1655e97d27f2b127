"""The sequence model with softmax attention over a window (paper_2501_08455_amd/sequence.py): against the same chain in 64 bits, trained, and served from a
paged cache.

Tolerance: 1e-4, relative Frobenius, for float32, as for the model with linear attention.
"""
import math

import pytest
import torch

from paper_2501_08455_amd import autograd, sequence
from test_gpu_sequence_model import near, norm64, turn64

gpu = pytest.mark.gpu


def model64(model, rows, lengths, grad):
    """Outputs, and gradients of the signature rows and of all parameters behind them, in float64 on the CPU."""
    P = {n: p.detach().cpu().double().requires_grad_(True) for n, p in model.named_parameters() if not n.startswith("path.")}
    rows = rows.detach().cpu().double().requires_grad_(True)
    H, K = model.heads, model.head_dim
    B, T, _ = rows.shape
    mixed = (norm64(rows, P["norm_weight"], P["norm_bias"]) @ P["mix.weight"].t() + P["mix.bias"]).view(B, T, 3 * H, K)
    turned, v = turn64(mixed[:, :, :2 * H], model.frequencies.cpu(), model.scale), mixed[:, :, 2 * H:].transpose(1, 2)
    q, k = turned[:, :, :H].transpose(1, 2), turned[:, :, H:].transpose(1, 2)
    at = torch.arange(T)
    gap = at[:, None] - at
    seen = (gap >= 0) & ((gap < (model.window or T)) | (at < model.sinks))
    p = torch.softmax((K ** -0.5 * q @ k.transpose(2, 3)).masked_fill(~seen, -math.inf), -1)
    o = (p @ v).transpose(1, 2) * (at < lengths.cpu()[:, None])[..., None, None]
    y = norm64(o, P["head_weight"]).flatten(2) @ P["out.weight"].t() + P["out.bias"]
    names = list(P)
    return y.detach(), dict(zip(["rows"] + names, torch.autograd.grad(y, [rows] + [P[n] for n in names], grad.cpu().double())))


@gpu
@pytest.mark.parametrize("L,heads,head_dim,window,sinks", [(41, 2, 24, 7, 2), (90, 3, 64, None, 0), (150, 1, 40, 32, 5)])
def test_model_and_its_gradients(L, heads, head_dim, window, sinks):
    torch.manual_seed(1)
    torch.backends.cuda.matmul.allow_tf32 = False
    B = 3
    model = sequence.SequenceModel(7, 3, 3, 6, heads=heads, head_dim=head_dim, mixer="window", window=window, sinks=sinks)
    x = torch.randn(B, L, 7, device="cuda").cumsum(1) / L ** 0.5
    lengths = torch.tensor([L - 1, (L - 1) // 2, 1], device="cuda")
    y = model(x, lengths=lengths)
    grad = torch.randn_like(y) * (torch.arange(L - 1, device="cuda") < lengths[:, None])[..., None]
    grads = dict(zip([n for n, _ in model.named_parameters()], torch.autograd.grad(y, list(model.parameters()), grad)))
    rows = autograd.signature(model._points(x), model.depth, stream=True)
    want, want_grads = model64(model, rows, lengths, grad)
    near(y, want, "outputs")
    # through the signature and the points by the kernels that the other model's test holds to the oracle
    path = [p for n, p in model.named_parameters() if n.startswith("path.")]
    for p, g in zip(path, torch.autograd.grad(rows, path, want_grads.pop("rows").float().cuda())):
        name = next(n for n, other in model.named_parameters() if other is p)
        near(grads[name], g.cpu(), name)
    for name, g in want_grads.items():
        near(grads[name], g, name)


@gpu
@pytest.mark.parametrize("window,sinks,page", [(None, 0, 16), (9, 2, 4), (1, 0, 16), (16, 5, 16), (5, 33, 8)])
def test_points_one_at_a_time_give_the_rows_of_the_whole_path(window, sinks, page):
    """... also where the window's pages are used again."""
    torch.manual_seed(2)
    model = sequence.SequenceModel(4, 3, 3, 5, heads=3, head_dim=40, turned=16, mixer="window", window=window, sinks=sinks)
    x = torch.randn(6, 70, 4, device="cuda").cumsum(1) * 0.2
    with torch.no_grad():
        want = model(x)
    cache = model.begin(x[:, 0], 69, page_tokens=page)
    if window is not None:
        assert len(cache["keys"]) <= 6 * (-(-sinks // page) + -(-window // page) + 1)
    for t in range(1, 70):
        near(model.step(x[:, t], cache), want[:, t - 1].cpu(), t)
    with pytest.raises(ValueError):
        model.step(x[:, 69], cache)


@gpu
@pytest.mark.parametrize("convert", ["float", "bfloat16", "half"])
@pytest.mark.parametrize("narrow", [False, True])
def test_converted_models_and_narrow_caches(convert, narrow):
    """Roundings of some eight results of 2^-8 or 2^-11 each, as in the model with linear attention; keys and values of 8 bits are off by 2^-4 at most, 2^-5 on average,
    and the norm behind the attention at most doubles that."""
    torch.manual_seed(5)
    model = sequence.SequenceModel(4, 3, 3, 5, heads=2, head_dim=32, mixer="window", window=12, sinks=2)
    x = torch.randn(3, 40, 4, device="cuda").cumsum(1) * 0.2
    kind = {"bfloat16": torch.bfloat16, "half": torch.float16}.get(convert, torch.float32)
    with torch.no_grad():
        for p in model.parameters():
            p.copy_(p.to(kind))
        want = model(x)
        model = getattr(model, convert)()
        assert model.frequencies.dtype == torch.float64 and "log_decay" not in model.state_dict()
        got = model(x)
    tolerance = {torch.float32: 64 * 2.0 ** -24, torch.bfloat16: 16 * 2.0 ** -8, torch.float16: 16 * 2.0 ** -11}[kind]
    assert got.dtype == kind and float((got.float() - want).norm()) <= tolerance * float(want.norm())
    cache = model.begin(x[:, 0], 39, kind=torch.float8_e4m3fn if narrow else None)
    tolerance = max(tolerance, 1e-4) + (2.0 ** -3 if narrow else 0.0)
    for t in range(1, 40):
        row = model.step(x[:, t], cache)
        assert row.dtype == kind and float((row.float() - want[:, t - 1]).norm()) <= tolerance * float(want[:, t - 1].norm()), t
    grads = torch.autograd.grad(model(x).float().square().sum(), list(model.parameters()))
    assert all(torch.isfinite(g).all() and g.dtype == kind for g in grads)


@gpu
def test_a_captured_training_step_repeats_the_eager_one():
    torch.manual_seed(3)
    model = sequence.SequenceModel(4, 3, 3, 1, heads=2, head_dim=32, mixer="window", window=20, sinks=1)
    x = torch.randn(16, 300, 4, device="cuda").cumsum(1) * 0.2
    # (not the bias of the Dense layer in front of the attention: its gradient is torch's sum over many rows, which clears memory in a way that graphs do not
    # repeat; the other mixer's model has the same)
    parameters = [p for n, p in model.named_parameters() if n != "mix.bias"]

    def step():
        return torch.autograd.grad(model(x).square().mean(), parameters)

    graph, grads = autograd.capture(step)
    for _ in range(3):
        x.copy_(torch.randn_like(x).cumsum(1) * 0.2)
        want = [g.clone() for g in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(grads, want))


def test_arguments():
    make = lambda **more: sequence.SequenceModel(4, 3, 2, 5, heads=2, head_dim=8, device="cpu", **more)      # noqa: E731
    for bad in (dict(mixer="other"), dict(window=5), dict(sinks=1), dict(mixer="window", window=0), dict(mixer="window", sinks=-1)):
        with pytest.raises(ValueError):
            make(**bad)
    model = make(mixer="window", window=5)
    for bad in (dict(), dict(room=0), dict(room=4, page_tokens=0), dict(room=4, kind=torch.float16)):
        with pytest.raises(ValueError):
            model.begin(torch.zeros(2, 4), **bad)
    for bad in (dict(room=4), dict(kind=torch.float32)):
        with pytest.raises(ValueError):
            make().begin(torch.zeros(2, 4), **bad)
    assert "log_decay" in make().state_dict() and "log_decay" not in model.state_dict()
    # pages behind the first prefixes' come round when the window has left them
    cache = model.begin(torch.zeros(2, 4), 100, page_tokens=4)
    table = cache["table"]
    assert table.shape == (2, 25) and len(cache["keys"]) == 6 and not set(table[0].tolist()) & set(table[1].tolist())
    for place in range(100):
        seen = [p // 4 for p in range(max(0, place - 4), place + 1)]
        assert len({int(table[0, i]) for i in seen}) == len(set(seen))
