"""Linear attention of values that are not finite: NaN and infinities reach what they reach in the recurrence, and nothing else.

The reference is the recurrence and its gradient written out in 64 bits, token by token, so that 0 x infinity, infinity - infinity and
what decay does to them are IEEE's.  Outputs have to be NaN and infinite, with their signs, in the same places; the finite ones
are held to the tolerance of tests/test_gpu_sequence_ops.py.
"""
import math

import pytest
import torch

from paper_2501_08455_amd import autograd, binding
from test_gpu_sequence_ops import TYPES, attention_inputs, noise, tolerance, wide

gpu = pytest.mark.gpu


def reference(q, k, v, log_decay, state, scale, grad, grad_state):
    q, k, v, grad = (wide(t) for t in (q, k, v, grad))
    B, T, H, K = q.shape
    share = torch.arange(H) // (H // k.shape[2])
    keys, values = k[:, :, share], v[:, :, share]
    l = torch.exp(wide(log_decay))[:, None, None]
    s, outs, gq, gk, gv = wide(state), [], [], [], []
    for t in range(T):
        s = l * s + keys[:, t, :, :, None] * values[:, t, :, None, :]
        outs.append(scale * (q[:, t, :, :, None] * s).sum(2))
        gq.append(scale * (s * grad[:, t, :, None, :]).sum(3))
    r = wide(grad_state)
    for t in reversed(range(T)):
        r = r + scale * q[:, t, :, :, None] * grad[:, t, :, None, :]
        gk.append((r * values[:, t, :, None, :]).sum(3))
        gv.append((r * keys[:, t, :, :, None]).sum(2))
        r = l * r
    o, gq, gk, gv = (torch.stack(x, 1) for x in (outs, gq, gk[::-1], gv[::-1]))
    gk, gv = (t.unflatten(2, (k.shape[2], -1)).sum(3) for t in (gk, gv))
    return o, s, gq, gk, gv, r


def assert_same(got, want, what):
    kind, got = got.dtype, got.detach().cpu().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), (what, int(torch.isnan(got).sum()), int(torch.isnan(want).sum()))
    infinite = torch.isinf(want)
    assert torch.equal(torch.isinf(got), infinite) and torch.equal(got[infinite], want[infinite]), what
    fine = torch.isfinite(want)
    err, size = float((got[fine] - want[fine]).norm()), float(want[fine].norm())
    assert err <= tolerance(kind) * size or err == 0.0, (what, err, size)


def check(q, k, v, log_decay, state, grad, grad_state):
    scale = q.shape[-1] ** -0.5
    want = reference(q, k, v, log_decay, state, scale, grad, grad_state)
    for a, b, name in zip(binding.linear_attention(q, k, v, log_decay, state=state, return_state=True), want, ("o", "state")):
        assert_same(a, b, name)
    ins = [t.detach().requires_grad_(True) for t in (q, k, v, state)]
    out = autograd.linear_attention(*ins[:3], log_decay, state=ins[3], return_state=True)
    for a, b, name in zip(torch.autograd.grad(out, ins, (grad, grad_state)), want[2:], ("grad q", "grad k", "grad v", "grad state")):
        assert_same(a, b, name)


def inputs(B, T, H, G, K, V, kind, decay="spread", seed=100):
    q, k, v, log_decay, state, _ = attention_inputs(B, T, H, G, K, V, kind, decay=decay, seed=seed)
    return [q, k, v, log_decay, state, noise(B, T, H, V, seed=seed + 5, kind=kind).cuda(), noise(B, H, K, V, seed=seed + 6).float().cuda()]


PLACES = {"q": 0, "k": 1, "v": 2, "state": 4, "grad": 5, "grad_state": 6}


@gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("where", PLACES)
@pytest.mark.parametrize("T", [1, 3, 200])
def test_one_value(T, where, value, kind):
    for token in sorted({0, T // 2, T - 1}):
        x = inputs(2, T, 2, 1, 40, 72, kind)
        t = x[PLACES[where]]
        if t.shape[1] == T and where not in ("state", "grad_state"):
            t[1, token, -1, 7] = value
        else:
            t[1, 1, 7, 11] = value
        check(*x)


@gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("where", PLACES)
@pytest.mark.parametrize("K,V", [(40, 96), (130, 33), (256, 64), (64, 128)])
def test_sequences_that_are_cut_along_time(K, V, where, value, kind):
    """Few heads' 700 tokens: segments of different workgroups, their own states first."""
    for token in (0, 300, 699) if where not in ("state", "grad_state") else (0,):
        x = inputs(1, 700, 2, 2, K, V, kind, seed=110)
        t = x[PLACES[where]]
        if where in ("state", "grad_state"):
            t[0, 1, K - 1, 3] = value
        else:
            t[0, token, 1, -1] = value
        check(*x)


@gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("decay", ["none", "all", "strong"])
@pytest.mark.parametrize("T", [2, 90, 700])
def test_infinities_of_both_signs_under_extreme_decays(T, decay, kind):
    """l = 1 keeps them, l = exp(-90) does too, and 0 x infinity is not a number."""
    x = inputs(1, T, 3, 3, 32, 48, kind, decay=decay, seed=120)
    x[1][0, T // 2, 0, 3], x[1][0, T // 2, 1, 3], x[1][0, T // 2, 2, 3] = math.inf, -math.inf, math.inf
    x[2][0, T - 1, 1, 3], x[2][0, 0, 2, 5] = math.inf, -math.inf
    x[4][0, :, 2, 2], x[6][0, :, 4, 4] = math.inf, -math.inf
    check(*x)


@gpu
@pytest.mark.parametrize("kind", TYPES)
def test_one_token_after_the_other_keeps_infinite_states(kind):
    q, k, v, log_decay, state, grad, grad_state = inputs(2, 6, 2, 2, 24, 40, kind, seed=130)
    k[0, 2, 0, 5], state[1, 1, 3, 8], v[1, 4, 0, 2] = math.inf, -math.inf, math.nan
    want = reference(q, k, v, log_decay, state, 24 ** -0.5, grad, grad_state)
    for t in range(6):
        assert_same(binding.linear_attention_step(q[:, t], k[:, t], v[:, t], log_decay, state), want[0][:, t], t)
    assert_same(state, want[1], "state")


def microseconds(call):
    """the fastest of a few calls"""
    call()
    best = math.inf
    for _ in range(5):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        call()
        b.record()
        b.synchronize()
        best = min(best, 1000.0 * a.elapsed_time(b))
    return best


@gpu
@pytest.mark.parametrize("kind", TYPES)
def test_a_passing_infinity_costs_its_own_chunk_only(kind):
    """An infinite query reaches its own output and no state, an infinite upstream gradient the gradient of its own query: the chunks behind are
    worked on as chunks again.  (One of 32 or 64 chunks token by token: 1.1 to 1.6 times as long; all of them 16 to 36 times.)"""
    B, T, H, K = 8, 2048, 64, 64
    q, k, v = (torch.randn(B, T, H, K, device="cuda").to(kind) for _ in range(3))
    log_decay = torch.full((H,), -0.05, device="cuda")
    call = lambda: binding.linear_attention(q, k, v, log_decay)   # noqa: E731
    clean, want = microseconds(call), call()
    q[:, 5, :, 3] = math.inf
    assert microseconds(call) <= 3.0 * clean
    got = call()
    assert not torch.isfinite(got[:, 5]).any()
    # (the rest of the spoilt chunk is worked out in another order)
    others = [t for t in range(T) if t != 5]
    assert float((got[:, others] - want[:, others]).float().norm()) <= tolerance(kind) * float(want[:, others].float().norm())


@gpu
@pytest.mark.parametrize("kind", TYPES)
def test_chunks_after_several_spoilt_ones(kind):
    """Spoilt chunks one behind another, apart, the first and the last, ragged, forward and both reversed passes; and a state that stays infinite
    behind chunks that were only passed through."""
    x = inputs(3, 500, 2, 1, 40, 72, kind, seed=160)
    for t in (0, 40, 70, 100, 101, 300, 499):
        x[0][1, t, 0, 2], x[5][1, 499 - t, 1, 4] = math.inf, -math.inf
    check(*x)
    x = inputs(1, 400, 3, 3, 128, 64, kind, seed=170)
    x[0][0, 20, 1, 5], x[5][0, 390, 1, 7] = math.nan, math.nan
    x[1][0, 200, 1, 5] = math.inf
    check(*x)
