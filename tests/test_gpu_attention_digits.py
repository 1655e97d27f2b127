"""Bfloat16 attention: the running state keeps float32's digits in every pass, so that no result depends on which others are asked for."""
import pytest
import torch

from paper_2501_08455_amd import autograd
from test_gpu_sequence_ops import attention_inputs, noise

gpu = pytest.mark.gpu


@gpu
@pytest.mark.parametrize("B,T,H,G,K,V", [(2, 130, 2, 2, 64, 64), (1, 700, 2, 2, 128, 128), (3, 300, 4, 2, 40, 72), (1, 90, 2, 1, 256, 33)])
def test_gradients_have_the_same_bits_with_and_without_the_states(B, T, H, G, K, V):
    q, k, v, log_decay, state, _ = attention_inputs(B, T, H, G, K, V, torch.bfloat16, seed=140)
    grad = noise(B, T, H, V, seed=145, kind=torch.bfloat16).cuda()
    ins = [t.requires_grad_(True) for t in (q, k, v)]
    alone = torch.autograd.grad(autograd.linear_attention(*ins, log_decay, state=state), ins, grad)
    state = state.clone().requires_grad_(True)
    both = torch.autograd.grad(autograd.linear_attention(*ins, log_decay, state=state), ins + [state], grad)
    for a, b in zip(alone, both):
        assert torch.equal(a, b)
