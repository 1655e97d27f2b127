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
