"""The signature, and the sequence-model operators behind it, as differentiable torch operations.

Marshalling only: both directions run in libsig's kernels (include/sig.h, include/sig_sequence.h), and the autograd nodes are
native (csrc/sig_torch.cpp, csrc/sig_torch_sequence.cpp), so that the engine's thread never waits for the interpreter.  This is
what lets the layer sit between trainable layers as in the paper's model (Section 4.2, Eq. 11).
"""
import torch

from . import binding


class _Traced(torch.autograd.Function):
    """The layer while torch.jit.trace is recording: the tracer keeps a Function as one operation of the graph, but sees nothing
    of a native call except the allocation of its result."""

    @staticmethod
    def forward(ctx, path, depth, stream):
        path = path.contiguous()
        out = binding.signature(path, depth, stream=stream)
        ctx.save_for_backward(path, out)
        ctx.depth, ctx.stream = int(depth), bool(stream)
        return out

    @staticmethod
    def backward(ctx, grad_out):
        path, out = ctx.saved_tensors
        grad_path = torch.empty_like(path)
        rc = binding.sig_backward(binding.default_ctx(), path, ctx.depth, int(ctx.stream), out, grad_out.contiguous(), grad_path)
        if rc != binding.SIG_OK:
            raise binding.SigError(rc, "sig_backward")
        return grad_path, None, None


def signature(path, depth, stream=False):
    """Depth-`depth` signatures of `path` (float32 CUDA tensor [B, L, d]) with gradient support:
    [B, D], or [B, L-1, D] with stream=True."""
    if torch.jit.is_tracing():
        return _Traced.apply(path, depth, stream)
    return (binding._torch_lib or binding.torch_lib()).autograd_signature(path, depth, stream)


class _FirstOrderOnly(torch.autograd.Function):
    """The first `count` of `tensors`, the gradients; a derivative of those with respect to any of them is an error, not a zero."""

    @staticmethod
    def forward(ctx, count, *tensors):
        return tuple(t.view_as(t) for t in tensors[:count])

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("libsig's operators have no second derivative")


class _TracedCall(torch.autograd.Function):
    """A native differentiable call while torch.jit.trace is recording (see _Traced): `call` takes the tensors.  The backward pass makes
    it again from the saved inputs and goes through its own node, which is gone behind each call: what a graph may do with a saved
    tensor (be walked twice, notice a change in place, be freed) stays with this Function's."""

    @staticmethod
    def _recorded(call, tensors, needed):
        inputs = [t.detach().requires_grad_(n) if torch.is_tensor(t) else t for t, n in zip(tensors, needed)]
        with torch.enable_grad():
            out = call(*inputs)
        return inputs, (out,) if torch.is_tensor(out) else out

    @staticmethod
    def forward(ctx, call, *tensors):
        ctx.call = call
        ctx.save_for_backward(*tensors)
        # (recorded, so that it refuses here what it has no gradient for)
        out = [t.detach() for t in _TracedCall._recorded(call, tensors, ctx.needs_input_grad[1:])[1]]
        return out[0] if len(out) == 1 else tuple(out)

    @staticmethod
    def backward(ctx, *grads):
        needed = ctx.needs_input_grad[1:]
        inputs, out = _TracedCall._recorded(ctx.call, ctx.saved_tensors, needed)
        got = torch.autograd.grad(out, [t for t, n in zip(inputs, needed) if n], [g.detach() for g in grads])
        if torch.is_grad_enabled():
            got = _FirstOrderOnly.apply(len(got), *got, *(t for t in ctx.saved_tensors + grads if t is not None))
        got = iter(got)
        return (None,) + tuple(next(got) if n else None for n in needed)


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """binding.layer_norm with a gradient with respect to `x`, `weight` and `bias`."""
    call = (binding._torch_lib or binding.torch_lib()).autograd_layer_norm
    if torch.jit.is_tracing():
        return _TracedCall.apply(lambda x, weight, bias: call(x, weight, bias, eps), x, weight, bias)
    return call(x, weight, bias, eps)


def rotary(x, positions, frequencies, interleaved=False, scale=1.0):
    """binding.rotary with a gradient with respect to `x`."""
    call = (binding._torch_lib or binding.torch_lib()).autograd_rotary
    if torch.jit.is_tracing():
        return _TracedCall.apply(lambda x, p, f: call(x, p, f, interleaved, scale), x, positions, frequencies)
    return call(x, positions, frequencies, interleaved, scale)


def linear_attention(q, k, v, log_decay, state=None, lengths=None, scale=None, return_state=False):
    """binding.linear_attention with a gradient with respect to `q`, `k`, `v` and `state` (log_decay is a constant of the model)."""
    call = (binding._torch_lib or binding.torch_lib()).autograd_linear_attention
    if torch.jit.is_tracing():
        return _TracedCall.apply(lambda *t: call(*t, scale, return_state), q, k, v, log_decay, state, lengths)
    return call(q, k, v, log_decay, state, lengths, scale, return_state)


def window_attention(q, k, v, window=None, sinks=0, lengths=None, scale=None):
    """binding.window_attention with a gradient with respect to `q`, `k` and `v`."""
    call = (binding._torch_lib or binding.torch_lib()).autograd_window_attention
    if torch.jit.is_tracing():
        return _TracedCall.apply(lambda q, k, v, n: call(q, k, v, window, sinks, n, scale), q, k, v, lengths)
    return call(q, k, v, window, sinks, lengths, scale)


def capture(step_fn, warmup=3):
    """One call of `step_fn()` as a HIP graph: (graph, what the captured call returned).

    A training step of the paper's model at batch 128 is a few dozen short kernels, and launching them one by one costs
    several times what they take to run; replayed as a graph the step is one launch.  `step_fn` must read its inputs from
    tensors that stay where they are (copy each batch into them before `graph.replay()`) and may update its parameters
    in place.  It is first run `warmup` times outside the graph, on a side stream of default priority, so that libsig has
    sized its context scratch and torch its workspaces: neither may allocate while the capture is on.
    """
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(warmup):
            step_fn()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step_fn()
    return graph, out
