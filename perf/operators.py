"""The sequence-model operators behind the every-prefix signature: layer norm, rotary positions, linear attention with decay.

Listed cases, and draws from the ranges they stand for.  Every case is one call, or one forward/backward pair, through the
Python entry points a program uses: `binding` without a gradient, `autograd` with one.  Where `own` is false the same
outputs come from elementary torch operations in 32 bits, rounded once at the end.

Formulas (c a scale, l the decay of a head):
  layer norm   h = (x - mean x) / sqrt(mean (x - mean x)^2 + eps), y = h w + b over the last axis
  rotary       a pair (x1, x2) of a head's first components becomes (x1 cos a - x2 sin a, x1 sin a + x2 cos a), a = position * frequency
  attention    S_t = l S_{t-1} + k_t (x) v_t, o_t = c q_t S_t; tokens from a path's length on give zeros and leave the state alone
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
_EPS = 1e-5


# ---------------------------------------------------------------- the cases
def _norm(rows, width, kind, train, name=None):
    return _named({"op": "norm", "rows": rows, "width": width, "type": kind, "train": train}, name)


def _rotary(B, T, heads, dim, turned, kind, interleaved, train, first, name=None):
    return _named({"op": "rotary", "B": B, "T": T, "heads": heads, "dim": dim, "turned": turned, "type": kind,
                   "interleaved": interleaved, "train": train, "first": first}, name)


def _token(B, heads, shared, K, V, kind, name=None):
    return _named({"op": "token", "B": B, "heads": heads, "shared": shared, "K": K, "V": V, "type": kind}, name)


def _attention(B, T, heads, shared, K, V, kind, train, state, ragged, name=None):
    return _named({"op": "attention", "B": B, "T": T, "heads": heads, "shared": shared, "K": K, "V": V, "type": kind,
                   "train": train, "state": state, "ragged": ragged}, name)


def _named(case, name):
    return case if name is None else dict(case, name=name)


def listed():
    return [
        # rows of one mini-batch's signatures in front of a Dense layer: an interactive call, all latency
        _norm(128, 780, "f32", False, name="norm_batch"),
        # every prefix of a mini-batch (64 paths, 255 prefixes, 340 coefficients), a training step
        _norm(64 * 255, 340, "f32", True, name="norm_stream_train"),
        # few paths with 1.1 million coefficients each (ten channels at depth six)
        _norm(16, 1111110, "f32", True, name="norm_large_train"),
        # a whole data set's rows in a training step of a model that runs in bfloat16
        _norm(65536, 780, "bf16", True, name="norm_bulk_train"),
        # queries and keys of one new token of 128 sequences, far into a long context
        _rotary(128, 1, 16, 64, 64, "bf16", False, False, 130000, name="rotary_token"),
        # queries and keys of a training batch, half of each head turned, neighbouring pairs
        _rotary(4, 8192, 24, 128, 64, "bf16", True, True, 0, name="rotary_train"),
        # one token of a mini-batch through a small model
        _token(128, 4, 4, 64, 64, "f32", name="attention_token"),
        # one token of many sequences through wide heads: the states are 268 MB
        _token(256, 16, 16, 128, 128, "bf16", name="attention_token_wide"),
        # a mixer over every prefix of a mini-batch, as large as the signature layer's own stream case
        _attention(64, 255, 4, 4, 64, 64, "f32", False, False, False, name="attention_stream"),
        # one long prompt, split over its length, with the state that its tokens go on from
        _attention(1, 65536, 8, 8, 128, 128, "bf16", False, True, False, name="attention_prompt"),
        # a training batch of long sequences
        _attention(8, 4096, 16, 16, 128, 128, "bf16", True, False, False, name="attention_train"),
        # the ragged last batch of an epoch: odd sizes, heads that share keys and values, a state carried on
        _attention(93, 499, 8, 4, 40, 72, "f32", True, True, True, name="attention_train_ragged"),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


# a drawn case moves and computes no more than the largest listed ones of its kind, and keeps no more states
_MOST_VALUES = {"norm": 65536 * 780, "rotary": 4 * 8192 * 24 * 128, "token": 256 * 16 * 128 * 128}
_MOST_HEAD_TOKENS = 8 * 4096 * 16
_MOST_PRODUCTS = 8 * 4096 * 16 * 128 * 128


def draw(rng):
    op = rng.choice(("norm", "norm", "rotary", "token", "attention", "attention", "attention"))
    kind = rng.choice(("f32", "f32", "bf16", "bf16", "f16"))
    if op == "norm":
        rows = _log_uniform(rng, 1, 65536)
        width = 1111110 if rng.random() < 0.08 else _log_uniform(rng, 2, 12000)
        rows = max(1, min(rows, _MOST_VALUES[op] // width))
        return _norm(rows, width, kind, rng.random() < 0.6)
    if op == "rotary":
        B, T, heads = _log_uniform(rng, 1, 256), _log_uniform(rng, 1, 16384), _log_uniform(rng, 1, 48)
        dim = rng.choice((32, 40, 64, 80, 96, 128, 192, 256, 57))
        turned = rng.choice((dim - dim % 2, dim // 2 - dim // 2 % 2, dim // 4 - dim // 4 % 2))
        B = max(1, min(B, _MOST_VALUES[op] // (T * heads * dim)))
        return _rotary(B, T, heads, dim, turned, kind, rng.random() < 0.5, rng.random() < 0.5, rng.choice((0, 0, 1000, 130000, 1000000)))
    shared = _log_uniform(rng, 1, 16)
    heads = shared * rng.choice((1, 1, 1, 2, 4))
    sizes = (16, 24, 32, 40, 64, 64, 72, 96, 128, 128, 130, 192, 256, 33)
    K, V = rng.choice(sizes), rng.choice(sizes)
    if op == "token":
        B = _log_uniform(rng, 1, 256)
        B = max(1, min(B, _MOST_VALUES[op] // (heads * K * V)))
        return _token(B, heads, shared, K, V, kind)
    B, T = _log_uniform(rng, 1, 256), _log_uniform(rng, 1, 65536)
    train = rng.random() < 0.5
    most = min(_MOST_HEAD_TOKENS, _MOST_PRODUCTS // (K * V))
    B = max(1, min(B, most // (heads * T)))
    T = max(1, min(T, most // (heads * B)))
    return _attention(B, T, heads, shared, K, V, kind, train, rng.random() < 0.5, rng.random() < 0.3)


def work(case):
    size = _BYTES[case["type"]]
    if case["op"] == "norm":
        values, extra = case["rows"] * case["width"], 2 * 4 * case["width"]
        # forward: in and out; backward: the input and the upstream gradient in, the gradient out; weights and their gradients
        passes = 5 if case["train"] else 2
        return {"bytes": float(passes * values * size + (3 if case["train"] else 1) * extra), "flops": float((22 if case["train"] else 8) * values)}
    if case["op"] == "rotary":
        heads = case["B"] * case["T"] * case["heads"]
        passes = 4 if case["train"] else 2
        return {"bytes": float(passes * heads * case["dim"] * size), "flops": float(passes / 2 * 3 * heads * case["turned"])}
    B, H, G, K, V = case["B"], case["heads"], case["shared"], case["K"], case["V"]
    if case["op"] == "token":
        # the state in and out
        return {"bytes": float(8 * B * H * K * V + size * B * (H * (K + V) + G * (K + V))), "flops": float(5 * B * H * K * V)}
    tokens = B * case["T"]
    ins, outs = tokens * (H * K + G * (K + V)), tokens * H * V
    values = ins + outs
    if case["train"]:
        values += 2 * ins + outs           # q, k, v and the upstream gradient in, three gradients out
    states = (2 if case["state"] else 0) * (2 if case["train"] else 1) * B * H * K * V
    # the recurrence's products: the state from k and v, the output from q; their five in the gradient
    return {"bytes": float(size * values + 4 * states), "flops": float((14 if case["train"] else 4) * tokens * H * K * V)}


# ---------------------------------------------------------------- inputs
def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    kind = _TYPES[case["type"]]
    state = dict(case)

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=gen)

    if case["op"] == "norm":
        R, D = case["rows"], case["width"]
        # rows whose stretches differ in size, as the levels of a signature do (a coefficient of level n has variance about 1/n!)
        level = torch.exp2(-4.0 * torch.arange(D, device="cuda") / D)
        state["x"] = (normal(R, D) * level + 0.1 * normal(R, 1)).to(kind)
        state["weight"], state["bias"] = 1.0 + 0.2 * normal(D), 0.2 * normal(D)
        if case["train"]:
            state["grad"] = normal(R, D).to(kind)
            for name in ("x", "weight", "bias"):
                state[name].requires_grad_(True)
        return state
    if case["op"] == "rotary":
        B, T, H, D = case["B"], case["T"], case["heads"], case["dim"]
        # queries and keys side by side in front of the values, as one projection leaves them
        fused = normal(B, T, H + max(1, H // 3), D).to(kind)
        state["x"] = fused[:, :, :H]
        start = torch.randint(0, 1000, (B, 1), device="cuda", generator=gen)
        state["positions"] = case["first"] + start + torch.arange(T, device="cuda")
        half = case["turned"] // 2
        state["frequencies"] = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / max(half, 1))
        if case["train"]:
            state["grad"] = normal(B, T, H, D).to(kind)
            state["x"].requires_grad_(True)
        return state
    B, H, G, K, V = case["B"], case["heads"], case["shared"], case["K"], case["V"]
    # decays from one eighth to one five-hundredth a token lost, over the heads
    state["log_decay"] = torch.log1p(-torch.exp2(-3.0 - 6.0 * torch.arange(H, device="cuda", dtype=torch.float32) / H))
    if case["op"] == "token":
        state["q"], state["k"], state["v"] = normal(B, H, K).to(kind), normal(B, G, K).to(kind), normal(B, G, V).to(kind)
        state["state"] = 4.0 * normal(B, H, K, V)
        state["next"] = torch.empty_like(state["state"])
        return state
    T = case["T"]
    state["q"], state["k"], state["v"] = normal(B, T, H, K).to(kind), normal(B, T, G, K).to(kind), normal(B, T, G, V).to(kind)
    state["initial"] = 4.0 * normal(B, H, K, V) if case["state"] else None
    state["lengths"] = torch.randint(0, T + 1, (B,), device="cuda", generator=gen) if case["ragged"] else None
    if case["train"]:
        state["grad"] = normal(B, T, H, V).to(kind)
        state["grad_state"] = normal(B, H, K, V) if case["state"] else None
        for name in ("q", "k", "v", "initial"):
            if state[name] is not None:
                state[name].requires_grad_(True)
    return state


# ---------------------------------------------------------------- one pass
def run(state):
    if not own:
        with torch.no_grad():
            return _PLAIN[state["op"]](state)
    from paper_2501_08455_amd import autograd, binding
    if state["op"] == "norm":
        if not state["train"]:
            return binding.layer_norm(state["x"], state["weight"], state["bias"], eps=_EPS)
        y = autograd.layer_norm(state["x"], state["weight"], state["bias"], eps=_EPS)
        return (y,) + torch.autograd.grad(y, (state["x"], state["weight"], state["bias"]), state["grad"])
    if state["op"] == "rotary":
        if not state["train"]:
            return binding.rotary(state["x"], state["positions"], state["frequencies"], interleaved=state["interleaved"])
        y = autograd.rotary(state["x"], state["positions"], state["frequencies"], interleaved=state["interleaved"])
        return (y,) + torch.autograd.grad(y, state["x"], state["grad"])
    if state["op"] == "token":
        o = binding.linear_attention_step(state["q"], state["k"], state["v"], state["log_decay"], state["state"], out_state=state["next"])
        return o, state["next"]
    args = (state["q"], state["k"], state["v"], state["log_decay"])
    more = {"state": state["initial"], "lengths": state["lengths"], "return_state": state["initial"] is not None}
    if not state["train"]:
        return binding.linear_attention(*args, **more)
    out = autograd.linear_attention(*args, **more)
    if state["initial"] is None:
        return (out,) + torch.autograd.grad(out, (state["q"], state["k"], state["v"]), state["grad"])
    return out + torch.autograd.grad(out, (state["q"], state["k"], state["v"], state["initial"]), (state["grad"], state["grad_state"]))


def _plain_norm(state):
    x, w = state["x"].float(), state["weight"]
    centred = x - x.mean(1, keepdim=True)
    r = torch.rsqrt((centred * centred).mean(1, keepdim=True) + _EPS)
    h = centred * r
    y = (h * w + state["bias"]).to(state["x"].dtype)
    if not state["train"]:
        return y
    g = state["grad"].float()
    gw = g * w
    gx = r * (gw - gw.mean(1, keepdim=True) - h * (gw * h).mean(1, keepdim=True))
    return y, gx.to(state["x"].dtype), (g * h).sum(0), g.sum(0)


def _plain_rotary(state):
    # (the angle of a far position has to be reduced in 64 bits: it has no correct digit left in 32)
    angle = state["positions"].double().unsqueeze(-1) * state["frequencies"]
    turn = (torch.cos(angle).float().unsqueeze(2), torch.sin(angle).float().unsqueeze(2))
    y = _plain_turn(state["x"], turn, state["turned"], state["interleaved"], 1.0)
    if not state["train"]:
        return y
    return y, _plain_turn(state["grad"], turn, state["turned"], state["interleaved"], -1.0)


def _plain_turn(x, turn, turned, interleaved, sign):
    cos, sin = turn[0], sign * turn[1]
    z = x[..., :turned].float()
    a, b = (z[..., 0::2], z[..., 1::2]) if interleaved else (z[..., :turned // 2], z[..., turned // 2:])
    a, b = a * cos - b * sin, a * sin + b * cos
    z = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((z.to(x.dtype), x[..., turned:]), -1)


def _plain_token(state):
    H, G = state["heads"], state["shared"]
    q, k, v = (state[n].float() for n in ("q", "k", "v"))
    k, v = k.repeat_interleave(H // G, 1), v.repeat_interleave(H // G, 1)
    s = torch.exp(state["log_decay"])[:, None, None] * state["state"] + k.unsqueeze(-1) * v.unsqueeze(-2)
    o = (q.unsqueeze(-2) @ s).squeeze(-2) * state["K"] ** -0.5
    return o.to(state["q"].dtype), s


def _chunked(x, y, z, log_decay, initial):
    """o_t = sum_{s <= t} l^(t-s) (x_t . y_s) z_s + l^(t+1) x_t initial, all [B, H, T, .] in 32 bits: pairs of tokens inside chunks of
    128, and what lies before a chunk as the state that the chunks' own states add up to."""
    B, H, T, K = x.shape
    C, N = 128, -(-T // 128)
    pad = N * C - T
    x, y, z = (torch.nn.functional.pad(t, (0, 0, 0, pad)).view(B, H, N, C, -1) for t in (x, y, z))
    g = log_decay.view(H, 1, 1)
    at = torch.arange(C, device=x.device)
    gap = at[:, None] - at
    inside = torch.where(gap >= 0, torch.exp(g * gap.clamp(min=0)), torch.zeros((), device=x.device)).view(H, 1, C, C)
    o = ((x @ y.transpose(-1, -2)) * inside) @ z
    if N == 1 and initial is None:
        return o.view(B, H, N * C, -1)[:, :, :T]
    own_state = (y * torch.exp(g * (C - 1 - at).view(1, 1, C)).view(H, 1, C, 1)).transpose(-1, -2) @ z
    chunk = torch.arange(N, device=x.device)
    apart = chunk[:, None] - chunk - 1
    across = torch.where(apart >= 0, torch.exp(g * C * apart.clamp(min=0)), torch.zeros((), device=x.device))
    before = (across @ own_state.view(B, H, N, -1)).view(B, H, N, K, -1)
    if initial is not None:
        before = before + torch.exp(g * C * chunk.view(1, 1, N)).view(H, N, 1, 1) * initial.unsqueeze(2)
    o = o + (x * torch.exp(g * (at + 1)).view(H, 1, C, 1)) @ before
    return o.view(B, H, N * C, -1)[:, :, :T]


def _plain_attention(state):
    B, T, H, G, K = (state[n] for n in ("B", "T", "heads", "shared", "K"))
    kind, c, g = state["q"].dtype, state["K"] ** -0.5, state["log_decay"]
    q, k, v = (state[n].float().transpose(1, 2) for n in ("q", "k", "v"))
    k, v = k.repeat_interleave(H // G, 1), v.repeat_interleave(H // G, 1)
    length = torch.full((B,), T, device=q.device) if state["lengths"] is None else state["lengths"]
    at = torch.arange(T, device=q.device)
    live = (at < length[:, None]).float().view(B, 1, T, 1)
    q, k, v = q * live, k * live, v * live
    o = (c * _chunked(q, k, v, g, state["initial"])).transpose(1, 2).to(kind)
    outs = [o]
    if state["initial"] is not None:
        left = (length[:, None] - 1 - at).clamp(min=0).view(B, 1, T)
        ahead = torch.exp(g.view(1, H, 1) * left).unsqueeze(-1) * live            # l^(length - 1 - t)
        whole = torch.exp(g * length[:, None]).view(B, H, 1, 1)                   # l^length
        outs.append((k * ahead).transpose(-1, -2) @ v + whole * state["initial"])
    if not state["train"]:
        return outs[0] if len(outs) == 1 else tuple(outs)
    go = state["grad"].float().transpose(1, 2) * live
    initial = None if state["initial"] is None else state["initial"].transpose(-1, -2)
    gq = c * _chunked(go, v, k, g, initial)
    gk = c * _chunked(v.flip(2), go.flip(2), q.flip(2), g, None).flip(2)
    gv = c * _chunked(k.flip(2), q.flip(2), go.flip(2), g, None).flip(2)
    if state["initial"] is not None:
        last = state["grad_state"]
        gk = gk + (v * ahead) @ last.transpose(-1, -2)
        gv = gv + (k * ahead) @ last
        behind = torch.exp(g.view(H, 1, 1) * (at + 1).view(1, T, 1)) * live
        first = c * (q * behind).transpose(-1, -2) @ go + whole * last
    gk, gv = (t.view(B, G, H // G, T, -1).sum(2) for t in (gk, gv))
    outs += [t.transpose(1, 2).to(kind) for t in (gq, gk, gv)]
    if state["initial"] is not None:
        outs.append(first)
    return tuple(outs)


_PLAIN = {"norm": _plain_norm, "rotary": _plain_rotary, "token": _plain_token, "attention": _plain_attention}


# ---------------------------------------------------------------- the definitions in 64 bits
@torch.no_grad()
def exact(case, seed):
    state = prepare(case, seed)
    d = {name: t.detach().double() for name, t in state.items() if isinstance(t, torch.Tensor) and t.is_floating_point()}
    if case["op"] == "norm":
        var, mean = torch.var_mean(d["x"], 1, keepdim=True, correction=0)
        deviation = torch.sqrt(var + _EPS)
        unit = (d["x"] - mean) / deviation
        y = d["weight"] * unit + d["bias"]
        if not case["train"]:
            return y
        up = d["grad"] * d["weight"]
        D = case["width"]
        gx = (D * up - up.sum(1, keepdim=True) - unit * (up * unit).sum(1, keepdim=True)) / (D * deviation)
        return y, gx, torch.linalg.vecdot(d["grad"], unit, dim=0), d["grad"].sum(0)
    if case["op"] == "rotary":
        turn = torch.exp(1j * d["frequencies"] * state["positions"][:, :, None, None])
        y = _exact_turn(d["x"], turn, case["turned"], case["interleaved"])
        return (y, _exact_turn(d["grad"], turn.conj(), case["turned"], case["interleaved"])) if case["train"] else y
    B, H, G, K, V = case["B"], case["heads"], case["shared"], case["K"], case["V"]
    l, c = torch.exp(d["log_decay"])[:, None, None], 1.0 / math.sqrt(K)
    if case["op"] == "token":
        share = torch.arange(H, device="cuda") // (H // G)
        s = l * d["state"] + d["k"][:, share, :, None] * d["v"][:, share, None, :]
        return c * (d["q"][..., None] * s).sum(2), s
    T = case["T"]
    length = state["lengths"] if case["ragged"] else torch.full((B,), T, device="cuda")
    share = torch.arange(H, device="cuda") // (H // G)
    s = d["initial"] if case["state"] else torch.zeros((B, H, K, V), dtype=torch.float64, device="cuda")
    keys, values = d["k"][:, :, share], d["v"][:, :, share]
    o = torch.zeros((B, T, H, V), dtype=torch.float64, device="cuda")
    gq = torch.zeros_like(d["q"])
    live = (torch.arange(T, device="cuda")[:, None] < length).view(T, B, 1, 1, 1)
    for t in range(T):
        k, v = keys[:, t], values[:, t]
        s = torch.where(live[t], torch.addcmul(l * s, k[..., :, None], v[..., None, :]), s)
        o[:, t] = c * (d["q"][:, t, :, None, :] @ s).squeeze(2) * live[t, :, :, 0]
        if case["train"]:
            gq[:, t] = c * (s @ d["grad"][:, t, :, :, None]).squeeze(3) * live[t, :, :, 0]
    outs = (o, s) if case["state"] else (o,)
    if not case["train"]:
        return outs if case["state"] else o
    gk, gv = (torch.zeros((B, T, H, n), dtype=torch.float64, device="cuda") for n in (K, V))
    r = d["grad_state"] if case["state"] else torch.zeros((B, H, K, V), dtype=torch.float64, device="cuda")
    for t in reversed(range(T)):           # r: the gradient of the state behind token t
        k, v = keys[:, t], values[:, t]
        own_part = torch.addcmul(r, d["q"][:, t, :, :, None], d["grad"][:, t, :, None, :], value=c)
        gk[:, t] = (own_part @ v[..., None]).squeeze(3) * live[t, :, :, 0]
        gv[:, t] = (k[:, :, None, :] @ own_part).squeeze(2) * live[t, :, :, 0]
        r = torch.where(live[t], l * own_part, r)
    gk, gv = (t.unflatten(2, (G, H // G)).sum(3) for t in (gk, gv))
    return outs + (gq, gk, gv) + ((r,) if case["state"] else ())


def _exact_turn(x, turn, turned, interleaved):
    half = turned // 2
    first = torch.arange(half, device=x.device) * (2 if interleaved else 1)
    second = first + (1 if interleaved else half)
    z = torch.complex(x[..., first], x[..., second]) * turn
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y
