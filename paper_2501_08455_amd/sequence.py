"""A sequence model on every prefix of a path: signature -> layer norm -> rotary positions -> linear attention with decay, or softmax
attention with a sliding window.

The model of the paper (Section 4.2, Eq. 11) reads one signature of a whole path.  This one reads the signature of every prefix
(Eq. 10) and mixes them along time, with one output for each prefix: sequence-to-sequence training on whole paths, and serving
one point after the other, where the signature grows by Chen's identity, linear attention by its recurrence, and softmax
attention reads the window's keys and values from a paged cache.  The operators run in libsig's kernels (include/sig.h, include/sig_sequence.h), the Dense layers in torch.
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
    """Dense(inputs -> channels, tanh) -> signature of every prefix -> layer norm -> Dense -> rotary positions -> attention -> layer norm
    of each head -> Dense(outputs).

    `mixer` is "linear", linear attention with a decay for each head (`decays`), or "window", softmax attention over the last `window` prefixes
    (None: all) and the first `sinks`.

    `model(x)` with x [B, L, inputs] gives [B, L - 1, outputs], one row for each prefix; `lengths` [B] counts the prefixes that are there.
    `model.begin(x0)` and `model.step(x, cache)` give the same rows one point at a time; a "window" model needs to know how many points may follow,
    `model.begin(x0, room)`, and keeps pages for its window and first prefixes alone.

    A model whose parameters are converted (`model.bfloat16()`, `.half()`) mixes and attends in that type; paths, signatures and states are float32."""

    mixer, window, sinks = "linear", None, 0      # (of models that were pickled without)

    def __init__(self, inputs, channels, depth, outputs, heads=4, head_dim=64, turned=None, decays=(0.125, 0.002), device="cuda",
                 mixer="linear", window=None, sinks=0, **positions):
        super().__init__()
        if mixer not in ("linear", "window"):
            raise ValueError("mixer is 'linear' or 'window'")
        if (window is not None and window < 1) or sinks < 0 or (mixer == "linear" and (window is not None or sinks)):
            raise ValueError("a 'window' mixer has a window of 1 or more, or None, and no fewer than 0 sinks; a 'linear' one has neither")
        self.mixer, self.window, self.sinks = mixer, window, sinks
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
        if mixer == "window":
            return
        # a fraction of the state that a token costs, from the first head to the last in equal ratios
        lost = decays[0] * (decays[1] / decays[0]) ** (torch.arange(heads, dtype=torch.float64) / max(heads - 1, 1))
        self.register_buffer("log_decay", torch.log1p(-lost).float().to(device))

    def _apply(self, fn, *args, **kwargs):
        # the operators take these two in their own types, whatever the parameters are converted to: they only move
        own = {name: self._buffers[name] for name in ("frequencies", "log_decay") if name in self._buffers}
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
        q, k, v = turned[:, :, :self.heads], turned[:, :, self.heads:], mixed[:, :, 2 * self.heads:]
        if self.mixer == "window":
            o = autograd.window_attention(q, k, v, window=self.window, sinks=self.sinks, lengths=lengths)
        else:
            o = autograd.linear_attention(q, k, v, self.log_decay, lengths=lengths)
        return self.out(autograd.layer_norm(o, self.head_weight).flatten(2))

    def _pages(self, B, room, page_tokens, kind, device):
        """An empty paged cache for `room` prefixes of each of B sequences.  Behind the first prefixes' pages, pages that the window has left are used again:
        the table names them anew."""
        pages = -(-room // page_tokens)
        number = torch.arange(pages, device=device)
        if self.window is not None:
            front, ring = -(-self.sinks // page_tokens), -(-self.window // page_tokens) + 1
            number = torch.where(number < front, number, front + (number - front) % ring)
            pages = min(pages, front + ring)
        table = (torch.arange(B, device=device)[:, None] * pages + number).int()
        cache = {name: torch.zeros(B * pages, self.heads, page_tokens, self.head_dim, device=device).to(kind) for name in ("keys", "values")}
        for name in ("key_scales", "value_scales"):
            cache[name] = torch.ones(B * pages, self.heads, device=device) if kind == torch.float8_e4m3fn else None
        return dict(cache, table=table, lengths=torch.zeros(B, dtype=torch.int64, device=device), room=room)

    @torch.no_grad()
    def begin(self, x0, room=None, page_tokens=16, kind=None):
        """The cache behind the first point, x0 [B, inputs].  Of a "window" model: for `room` more points, in pages of `page_tokens`, their type the parameters',
        or `kind`, torch.float8_e4m3fn for 8 bits."""
        B = x0.shape[0]
        cache = {"point": self._points(x0), "row": None}
        if self.mixer == "window":
            if room is None or room < 1 or page_tokens < 1:
                raise ValueError("a 'window' model's cache has room for 1 point or more, in pages of 1 or more")
            if kind not in (None, self.mix.weight.dtype, torch.float8_e4m3fn):
                raise ValueError("the cache has the parameters' type or float8_e4m3fn")
            return dict(cache, **self._pages(B, room, page_tokens, kind or self.mix.weight.dtype, x0.device))
        if room is not None or kind is not None:
            raise ValueError("room and kind are for 'window' models")
        state = torch.zeros(B, self.heads, self.head_dim, self.head_dim, dtype=torch.float32, device=x0.device)
        # (counted in whole numbers, as forward() does: float32 stops at 2^24)
        return dict(cache, state=state, position=torch.zeros(1, dtype=torch.int64, device=x0.device))

    def _attend(self, mixed, cache):
        """Attention of one prefix, mixed [B, 1, 3 heads, head_dim]: [B, heads, head_dim]."""
        q, k, v = mixed.split(self.heads, 2)
        if self.mixer == "window":
            cache["room"] -= 1
            pages = [cache[name] for name in ("keys", "values", "table", "lengths")]
            scales = {name: cache[name] for name in ("key_scales", "value_scales")}
            q = binding.cache_append(k, v, *pages, q=q, frequencies=self.frequencies, scale=self.scale, **scales)
            cache["lengths"] += 1
            return binding.cache_attention(q, *pages, window=self.window, sinks=self.sinks, **scales)[:, 0]
        turned = mixed[:, :, :2 * self.heads]
        binding.rotary(turned, cache["position"], self.frequencies, scale=self.scale, out=turned)
        cache["position"] += 1
        return binding.linear_attention_step(q[:, 0], k[:, 0], v[:, 0], self.log_decay, cache["state"])

    @torch.no_grad()
    def step(self, x, cache):
        """The next point, x [B, inputs]: the outputs [B, outputs] of the prefix that ends there.  Updates `cache` in place; a full one is refused as it is."""
        if self.mixer == "window" and cache["room"] == 0:
            raise ValueError("the cache has no room for another point")
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
        o = self._attend(mixed, cache)
        return self.out(binding.layer_norm(o, self.head_weight).flatten(1))
