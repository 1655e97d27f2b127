"""Linear attention where the number of heads is about that of the compute units: sequences that are cut along time there, against the 64-bit
references and with the tolerances of tests/test_gpu_sequence_ops.py."""
import pytest
import torch

from paper_2501_08455_amd import autograd
from test_gpu_sequence_ops import assert_near, attention_inputs, attention_reference, noise

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,T,H,G,K,V", [(50, 2100, 4, 4, 24, 33), (61, 2600, 5, 5, 16, 64), (75, 3200, 4, 2, 40, 24), (64, 3300, 2, 2, 128, 100), (24, 3200, 2, 1, 100, 130),
                                         (128, 3100, 2, 2, 72, 16), (4, 200, 8, 8, 128, 128), (1, 700, 8, 8, 64, 100), (2, 1500, 12, 12, 96, 72)])
def test_some_sequences_of_a_batch(B, T, H, G, K, V, kind):
    """Ragged, with states, both directions.  The reference takes three of the batch's sequences: a batch element is no other's concern."""
    q, k, v, log_decay, state, lengths = attention_inputs(B, T, H, G, K, V, kind, ragged=B > 2, seed=150)
    g, gs = noise(B, T, H, V, seed=155, kind=kind).cuda(), noise(B, H, K, V, seed=156).float().cuda()
    ins = [t.requires_grad_(True) for t in (q, k, v, state)]
    out = autograd.linear_attention(*ins[:3], log_decay, state=state, lengths=lengths, return_state=True)
    got = list(out) + list(torch.autograd.grad(out, ins, (g, gs)))
    for b in sorted({0, B // 3, B - 1}):
        n = T if lengths is None else int(lengths[b])
        for t in (got[0], got[2], got[3], got[4]):
            assert not t[b, n:].any()
        few = torch.arange(H, device="cuda")[:2 * (H // G)]      # heads of the first two shared heads, or of one
        few = few[few < H]
        shared = torch.arange(max(1, len(few) * G // H), device="cuda")
        part = lambda t, heads: t[b:b + 1, :n][:, :, heads]   # noqa: E731
        want = attention_reference(part(q, few), part(k, shared), part(v, shared), log_decay[few], state[b:b + 1, few], None, K ** -0.5, part(g, few), gs[b:b + 1, few])
        assert_near(part(got[0], few), want[0], what=("o", b))
        assert_near(got[1][b:b + 1, few], want[1], what=("state", b))
        for name, a, heads, w in zip(("grad q", "grad k", "grad v"), got[2:5], (few, shared, shared), want[2:5]):
            assert_near(part(a, heads), w, what=(name, b))
        assert_near(got[5][b:b + 1, few], want[5], what=("grad state", b))
