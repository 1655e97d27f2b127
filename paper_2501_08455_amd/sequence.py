"""A sequence model on every prefix of a path: signature -> layer norm -> rotary positions -> linear attention with decay.

The model of the paper (Section 4.2, Eq. 11) reads one signature of a whole path.  This one reads the signature of every prefix
(Eq. 10) and mixes them along time, with one output for each prefix: sequence-to-sequence training on whole paths, and serving
one point after the other, where the signature grows by Chen's identity and the attention by its recurrence.  The
operators run in libsig's kernels (include/sig.h, include/sig_sequence.h), the Dense layers in torch.
"""
import math

import torch

from . import autograd, binding


def rotary_frequencies(turned, base=10000.0, scaling=None, factor=1.0, trained_length=None, device="cuda"):
    """Frequencies (float64 [turned / 2], radians a position) and the scale of rotary positions over `turned` components.

    f_i = base^(-2 i / turned).  For sequences `factor` times as long as the model was trained on, `scaling` is
      None      f as it is
      "linear"  f / factor: positions interpolated (Chen et al. 2023, arXiv 2306.15595)
      "base"    base * factor^(turned / (turned - 2)): the lowest frequency is divided by factor, the highest kept
      "parts"   f where a pair turns 32 times or more within `trained_length`, f / factor where it turns less than once, and in
                proportion between; the scale is 1 + 0.1 ln factor, for queries and keys each (Peng et al. 2023, arXiv 2309.00071)
    """
    if turned < 0 or turned % 2:
        raise ValueError("turned must be even and not negative")
    if not factor >= 1.0:
        raise ValueError("factor must be at least 1")
    if scaling == "base" and turned > 2:
        base = base * factor ** (turned / (turned - 2))
    f = base ** (-2.0 * torch.arange(turned // 2, dtype=torch.float64) / max(turned, 1))
    scale = 1.0
    if scaling == "linear":
        f = f / factor
    elif scaling == "parts":
        if not trained_length or trained_length <= 0:
            raise ValueError("scaling by parts needs the length that the model was trained on")
        turns = trained_length * f / (2.0 * math.pi)
        kept = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
        f = f / factor * (1.0 - kept) + f * kept
        scale = 1.0 + 0.1 * math.log(factor)
    elif scaling not in (None, "base"):
        raise ValueError("scaling is None, 'linear', 'base' or 'parts'")
    return f.to(device), scale


class SequenceModel(torch.nn.Module):
    """Dense(inputs -> channels, tanh) -> signature of every prefix -> layer norm -> Dense -> rotary positions -> linear attention
    with a decay for each head -> layer norm of each head -> Dense(outputs).

    `model(x)` with x [B, L, inputs] gives [B, L - 1, outputs], one row for each prefix; `lengths` [B] counts the prefixes that are there.
    `model.begin(x0)` and `model.step(x, cache)` give the same rows one point at a time.

    A model whose parameters are converted (`model.bfloat16()`, `.half()`) mixes and attends in that type; paths, signatures and states are float32."""

    def __init__(self, inputs, channels, depth, outputs, heads=4, head_dim=64, turned=None, decays=(0.125, 0.002), device="cuda", **positions):
        super().__init__()
        self.depth, self.heads, self.head_dim = depth, heads, head_dim
        width = binding.sig_size(channels, depth)
        self.path = torch.nn.Linear(inputs, channels, device=device)
        self.norm_weight = torch.nn.Parameter(torch.ones(width, device=device))
        self.norm_bias = torch.nn.Parameter(torch.zeros(width, device=device))
        self.mix = torch.nn.Linear(width, 3 * heads * head_dim, device=device)
        self.head_weight = torch.nn.Parameter(torch.ones(head_dim, device=device))
        self.out = torch.nn.Linear(heads * head_dim, outputs, device=device)
        frequencies, self.scale = rotary_frequencies(head_dim // 2 * 2 if turned is None else turned, device=device, **positions)
        self.register_buffer("frequencies", frequencies)
        # a fraction of the state that a token costs, from the first head to the last in equal ratios
        lost = decays[0] * (decays[1] / decays[0]) ** (torch.arange(heads, dtype=torch.float64) / max(heads - 1, 1))
        self.register_buffer("log_decay", torch.log1p(-lost).float().to(device))

    def _apply(self, fn, *args, **kwargs):
        # the operators take these two in their own types, whatever the parameters are converted to: they only move
        own = {name: self._buffers[name] for name in ("frequencies", "log_decay")}
        super()._apply(fn, *args, **kwargs)
        for name, buffer in own.items():
            if self._buffers[name].dtype != buffer.dtype:
                self._buffers[name] = buffer.to(self._buffers[name].device)
        return self

    def _points(self, x):
        """The path's points, float32 (differences of rounded points would lose the steps between them)."""
        if self.path.weight.dtype == torch.float32:
            return torch.tanh(self.path(x.float()))
        return torch.tanh(torch.nn.functional.linear(x.float(), self.path.weight.float(), self.path.bias.float()))

    def _normed(self, layer_norm, rows):
        """Signature rows, float32, through the layer norm and into the parameters' type (their range may be beyond float16's before)."""
        return layer_norm(rows, self.norm_weight.float(), self.norm_bias.float()).to(self.mix.weight.dtype)

    def forward(self, x, lengths=None):
        rows = autograd.signature(self._points(x), self.depth, stream=True)
        B, T, _ = rows.shape
        mixed = self.mix(self._normed(autograd.layer_norm, rows)).view(B, T, 3 * self.heads, self.head_dim)
        positions = torch.arange(T, device=x.device)
        # queries and keys are turned together
        turned = autograd.rotary(mixed[:, :, :2 * self.heads], positions, self.frequencies, scale=self.scale)
        o = autograd.linear_attention(turned[:, :, :self.heads], turned[:, :, self.heads:], mixed[:, :, 2 * self.heads:], self.log_decay, lengths=lengths)
        return self.out(autograd.layer_norm(o, self.head_weight).flatten(2))

    @torch.no_grad()
    def begin(self, x0):
        """The cache behind the first point, x0 [B, inputs]."""
        B = x0.shape[0]
        state = torch.zeros(B, self.heads, self.head_dim, self.head_dim, dtype=torch.float32, device=x0.device)
        # (counted in whole numbers, as forward() does: float32 stops at 2^24)
        return {"point": self._points(x0), "row": None, "state": state, "position": torch.zeros(1, dtype=torch.int64, device=x0.device)}

    @torch.no_grad()
    def step(self, x, cache):
        """The next point, x [B, inputs]: the outputs [B, outputs] of the prefix that ends there.  Updates `cache` in place."""
        point = self._points(x)
        segment = binding.signature(torch.stack((cache["point"], point), 1), self.depth)
        if cache["row"] is None:
            cache["row"] = segment
        else:
            row = torch.empty_like(segment)
            rc = binding.sig_combine(binding.default_ctx(), cache["row"], segment, point.shape[1], self.depth, row)
            if rc != binding.SIG_OK:
                raise binding.SigError(rc, "sig_combine")
            cache["row"] = row
        cache["point"] = point
        mixed = self.mix(self._normed(binding.layer_norm, cache["row"])).view(-1, 1, 3 * self.heads, self.head_dim)
        turned = mixed[:, :, :2 * self.heads]
        binding.rotary(turned, cache["position"], self.frequencies, scale=self.scale, out=turned)
        cache["position"] += 1
        q, k, v = mixed[:, 0].split(self.heads, 1)
        o = binding.linear_attention_step(q, k, v, self.log_decay, cache["state"])
        return self.out(binding.layer_norm(o, self.head_weight).flatten(1))
