"""The sequence model that runs the signature of every prefix, layer norm, rotary positions and linear attention together
(paper_2501_08455_amd/sequence.py): against the same chain in 64 bits around the oracle, trained, and one point at a time.

Tolerance: 1e-4, relative Frobenius, as for the training step of the paper's model; the chain is in float32 on the GPU.
"""
import numpy as np
import pytest
import torch

from paper_2501_08455_amd import autograd, sequence

TOL = 1e-4
gpu = pytest.mark.gpu


def near(got, want, what):
    got, want = got.detach().cpu().double(), torch.as_tensor(want).double()
    assert got.shape == want.shape, what
    err = float((got - want).norm() / want.norm())
    assert err <= TOL, (what, err)


def norm64(x, w, b=0.0):
    c = x - x.mean(-1, keepdim=True)
    return c / torch.sqrt((c * c).mean(-1, keepdim=True) + 1e-5) * w + b


def turn64(x, f, scale):
    half = f.numel()
    a = torch.arange(x.shape[1], dtype=torch.float64)[:, None] * f
    c, s = torch.cos(a)[:, None], torch.sin(a)[:, None]
    p, q = x[..., :half], x[..., half:2 * half]
    return scale * torch.cat((p * c - q * s, p * s + q * c, x[..., 2 * half:] / scale), -1)


def model64(oracle, model, x, lengths, grad):
    """Outputs, and gradients of every parameter, in float64 on the CPU."""
    P = {n: p.detach().cpu().double().requires_grad_(True) for n, p in model.named_parameters()}
    H, K = model.heads, model.head_dim
    f = model.frequencies.cpu()
    x = x.cpu().double()
    hidden = torch.tanh(x @ P["path.weight"].t() + P["path.bias"])
    z32 = hidden.detach().numpy().astype(np.float32)
    rows = torch.tensor(oracle.signature(z32, model.depth, stream=True), requires_grad=True)
    B, T, _ = rows.shape
    mixed = (norm64(rows, P["norm_weight"], P["norm_bias"]) @ P["mix.weight"].t() + P["mix.bias"]).view(B, T, 3 * H, K)
    qk, v = turn64(mixed[:, :, :2 * H], f, model.scale), mixed[:, :, 2 * H:]
    l = torch.exp(model.log_decay.cpu().double())[:, None, None]
    live = (torch.arange(T) < lengths.cpu()[:, None]).double()[..., None, None]
    s, outs = torch.zeros(B, H, K, K, dtype=torch.float64), []
    for t in range(T):
        s = l * s + qk[:, t, H:, :, None] * v[:, t, :, None, :]
        outs.append(K ** -0.5 * (qk[:, t, :H, None, :] @ s)[:, :, 0])
    o = torch.stack(outs, 1) * live
    y = norm64(o, P["head_weight"]).flatten(2) @ P["out.weight"].t() + P["out.bias"]
    after = [n for n in P if not n.startswith("path.")]
    grads = dict(zip(after + ["rows"], torch.autograd.grad(y, [P[n] for n in after] + [rows], grad.cpu().double())))
    dz = torch.tensor(oracle.signature_backward(z32, model.depth, grads.pop("rows").numpy().astype(np.float32), stream=True))
    grads["path.weight"], grads["path.bias"] = torch.autograd.grad(hidden, [P["path.weight"], P["path.bias"]], dz)
    return y.detach(), grads


@gpu
@pytest.mark.parametrize("B,L,channels,depth,heads,head_dim,positions", [
    (5, 41, 3, 3, 2, 24, {}), (3, 100, 5, 2, 3, 64, {"turned": 32, "scaling": "parts", "factor": 4.0, "trained_length": 50}),
    (2, 130, 4, 4, 4, 32, {"scaling": "base", "factor": 2.0})])
def test_model_and_its_gradients(oracle, B, L, channels, depth, heads, head_dim, positions):
    torch.manual_seed(1)
    torch.backends.cuda.matmul.allow_tf32 = False
    model = sequence.SequenceModel(7, channels, depth, 6, heads=heads, head_dim=head_dim, **positions)
    x = torch.randn(B, L, 7, device="cuda").cumsum(1) / L ** 0.5
    lengths = torch.tensor([L - 1] + [(L - 1) // (b + 1) for b in range(1, B)], device="cuda")
    y = model(x, lengths=lengths)
    grad = torch.randn_like(y) * (torch.arange(L - 1, device="cuda") < lengths[:, None])[..., None]
    grads = torch.autograd.grad(y, list(model.parameters()), grad)
    want, want_grads = model64(oracle, model, x, lengths, grad)
    near(y, want, "outputs")
    for (name, _), g in zip(model.named_parameters(), grads):
        near(g, want_grads[name], name)


@gpu
def test_points_one_at_a_time_give_the_rows_of_the_whole_path():
    torch.manual_seed(2)
    model = sequence.SequenceModel(4, 3, 4, 5, heads=3, head_dim=40, turned=16)
    x = torch.randn(6, 30, 4, device="cuda").cumsum(1) * 0.2
    with torch.no_grad():
        want = model(x)
    cache = model.begin(x[:, 0])
    for t in range(1, 30):
        near(model.step(x[:, t], cache), want[:, t - 1].cpu(), t)


@gpu
def test_training_as_a_graph_lowers_the_loss():
    torch.manual_seed(3)
    model = sequence.SequenceModel(4, 3, 3, 1, heads=2, head_dim=32)
    x = torch.randn(16, 60, 4, device="cuda").cumsum(1) * 0.2
    target = x[:, 1:].square().sum(-1, keepdim=True).cumsum(1) * 0.05
    parameters = list(model.parameters())

    def step():
        loss = (model(x) - target).square().mean()
        grads = torch.autograd.grad(loss, parameters)
        with torch.no_grad():
            for p, g in zip(parameters, grads):
                p -= 0.02 * g
        return loss.detach()

    first = float(step())
    graph, loss = autograd.capture(step)
    for _ in range(60):
        graph.replay()
    torch.cuda.synchronize()
    assert float(loss) < 0.5 * first, (first, float(loss))


@gpu
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_a_captured_attention_that_is_cut_along_time_replays_like_the_eager_call(kind):
    """Context scratch inside a graph, with the program's own calls on the same context between the replays."""
    from paper_2501_08455_amd import binding
    q, k, v = (torch.randn(1, 3001, 2, 64, device="cuda").to(kind) for _ in range(3))
    log_decay = torch.log(torch.tensor([0.9, 0.99], device="cuda"))
    call = lambda: binding.linear_attention(q, k, v, log_decay, return_state=True)   # noqa: E731
    graph, out = autograd.capture(call)
    for _ in range(3):
        for t in (q, k, v):
            t.normal_()
        want = [t.clone() for t in call()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_rotary_frequencies():
    plain, one = sequence.rotary_frequencies(8, device="cpu")
    assert one == 1.0 and torch.allclose(plain, torch.tensor([1.0, 0.1, 0.01, 0.001], dtype=torch.float64), rtol=1e-15)
    linear, one = sequence.rotary_frequencies(8, scaling="linear", factor=4.0, device="cpu")
    assert one == 1.0 and torch.equal(linear, plain / 4.0)
    other, _ = sequence.rotary_frequencies(8, scaling="base", factor=4.0, device="cpu")
    assert other[0] == 1.0 and abs(float(other[-1] / plain[-1]) - 0.25) < 1e-14
    parts, scale = sequence.rotary_frequencies(64, scaling="parts", factor=8.0, trained_length=1000, device="cpu")
    plain, _ = sequence.rotary_frequencies(64, device="cpu")
    turns = 1000 * plain / (2 * np.pi)
    assert torch.equal(parts[turns >= 32], plain[turns >= 32]) and torch.allclose(parts[turns < 1], plain[turns < 1] / 8, rtol=1e-15)
    between = (turns >= 1) & (turns < 32)
    assert ((parts < plain) & (parts > plain / 8))[between].all() and abs(scale - 1 - 0.1 * np.log(8.0)) < 1e-15
    assert sequence.rotary_frequencies(0, device="cpu")[0].numel() == 0
    for bad in (dict(turned=7), dict(turned=-2), dict(turned=8, factor=0.5), dict(turned=8, scaling="parts"), dict(turned=8, scaling="other"),
                dict(turned=8, factor=float("nan"))):
        with pytest.raises(ValueError):
            sequence.rotary_frequencies(device="cpu", **bad)
