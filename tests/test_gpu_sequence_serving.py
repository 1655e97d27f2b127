"""The sequence model where it runs for long, and where its parameters are converted (paper_2501_08455_amd/sequence.py)."""
import pytest
import torch

from paper_2501_08455_amd import sequence

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("reached", [2 ** 24 - 2, 2 ** 31 - 2, 2 ** 40])
def test_points_are_counted_beyond_what_float32_counts(reached):
    """Far into a stream the cache still counts every point, so that two points' angles differ by one position's: the same as from zero on, but for
    the common turn, which leaves queries times keys alone."""
    torch.manual_seed(4)
    model = sequence.SequenceModel(4, 3, 3, 5, heads=2, head_dim=32)
    x = torch.randn(3, 8, 4, device="cuda").cumsum(1) * 0.2
    near, far = model.begin(x[:, 0]), model.begin(x[:, 0])
    far["position"] += reached
    for t in range(1, 8):
        a, b = model.step(x[:, t], near), model.step(x[:, t], far)
        assert int(far["position"]) == reached + t
        # angles are reduced in 64 bits: at 2^40 turns of one radian 2^-53 * 2^40 / 2 pi are left, far below float32
        assert float((a - b).norm() / a.norm()) <= 1e-4, t


@gpu
@pytest.mark.parametrize("convert", ["float", "bfloat16", "half", "double and back", "to"])
def test_a_converted_model_still_computes(convert):
    """Types of parameters change, those that the operators ask for do not.  In a 16-bit model about eight roundings lie behind the float32
    signature (norm, mix, rotation, attention, norm of heads, products' operands), 2^-8 each in bfloat16; the heads' norm at most doubles them.
    In float32 nothing changes but, at most, the order of a library product's sums."""
    torch.manual_seed(5)
    model = sequence.SequenceModel(4, 3, 3, 5, heads=2, head_dim=32)
    frequencies, log_decay = model.frequencies.clone(), model.log_decay.clone()
    x = torch.randn(3, 20, 4, device="cuda").cumsum(1) * 0.2
    kind = {"bfloat16": torch.bfloat16, "half": torch.float16}.get(convert, torch.float32)
    with torch.no_grad():
        if kind != torch.float32:
            for p in model.parameters():
                p.copy_(p.to(kind))
        want = model(x)
        model = {"double and back": lambda: model.double().float(), "to": lambda: model.to("cuda", torch.float32)}.get(convert, lambda: getattr(model, convert)())()
        assert torch.equal(model.frequencies, frequencies) and model.frequencies.dtype == torch.float64
        assert torch.equal(model.log_decay, log_decay) and model.log_decay.dtype == torch.float32
        assert set(model.state_dict()) >= {"frequencies", "log_decay"}
        got = model(x)
    assert got.dtype == kind and all(p.dtype == kind for p in model.parameters())
    tolerance = {torch.float32: 64 * 2.0 ** -24, torch.bfloat16: 16 * 2.0 ** -8, torch.float16: 16 * 2.0 ** -11}[kind]
    assert float((got.float() - want).norm()) <= tolerance * float(want.norm())
    cache = model.begin(x[:, 0])
    for t in range(1, 20):
        row = model.step(x[:, t], cache)
        assert row.dtype == kind
        assert float((row.float() - want[:, t - 1]).norm()) <= max(tolerance, 1e-4) * float(want[:, t - 1].norm()), t
    grads = torch.autograd.grad(model(x).float().square().sum(), list(model.parameters()))
    assert all(torch.isfinite(g).all() and g.dtype == kind for g in grads)
