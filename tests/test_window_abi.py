"""The C entry points of window attention and the paged cache (include/sig_sequence.h): what they refuse, before anything is read or launched."""
import ctypes

import pytest

from paper_2501_08455_amd import binding

INVALID, LARGE, UNSUPPORTED, OK = binding.SIG_ERR_INVALID, binding.SIG_ERR_TOO_LARGE, binding.SIG_ERR_UNSUPPORTED, binding.SIG_OK


def test_the_structures_are_laid_out_as_in_c():
    assert ctypes.sizeof(binding.sig_window_t) == 2 * 8 + 6 * 4 + 2 * 8 + 9 * 8
    assert ctypes.sizeof(binding.sig_cache_t) == 2 * 8 + 4 * 4 + 4 * 8 + 6 * 8 + 3 * 8
    assert ctypes.sizeof(binding.sig_append_t) == 2 * 8 + 2 * 4 + 9 * 8 + 8 + 2 * 4 + 2 * 8 + 3 * 8
    assert ctypes.sizeof(binding.sig_queries_t) == 2 * 8 + 3 * 4 + 4 + 2 * 8 + 3 * 8


def window(**change):
    shape = binding.sig_window_t(1, 1, 2, 1, 4, 4, 0, 1.0, 0, 0)
    for name, value in change.items():
        setattr(shape, name, value)
    return shape


def cache(p, **change):
    shape = binding.sig_cache_t(1, 4, 1, 4, 4, 0, p, p, None, None)
    shape.table, shape.table_pages, shape.table_stride = p, 1, 1
    for name, value in change.items():
        setattr(shape, name, value)
    return shape


def test_calls_without_a_context_are_refused():
    lib, none = binding.load(), None
    assert lib.sig_window_attention(none, ctypes.byref(window()), *[none] * 8) == INVALID
    assert lib.sig_window_attention_backward(none, ctypes.byref(window()), *[none] * 12) == INVALID
    c = cache(none)
    assert lib.sig_cache_append(none, ctypes.byref(c), ctypes.byref(binding.sig_append_t(1, 1, 1, 0)), *[none] * 7) == INVALID
    assert lib.sig_cache_attention(none, ctypes.byref(c), ctypes.byref(binding.sig_queries_t(1, 1, 1, 0, 1.0)), *[none] * 5) == INVALID


@pytest.mark.gpu
def test_bad_arguments_are_refused():
    import torch
    lib, ctx = binding.load(), binding.default_ctx()
    room = torch.zeros(4096, device="cuda")
    p = ctypes.c_void_p(room.data_ptr())

    def attention(q=p, k=p, v=p, out=p, **change):
        shape = window(**change)
        both = (lib.sig_window_attention(ctx, ctypes.byref(shape), q, k, v, None, out, None, None, None),
                lib.sig_window_attention_backward(ctx, ctypes.byref(shape), q, k, v, None, out, p, None, p, out, p, p, None))
        assert both[0] == both[1]
        return both[0]

    assert attention(q=None) == attention(k=None) == attention(v=None) == attention(out=None) == INVALID
    assert (attention(B=-1) == attention(T=-1) == attention(heads=0) == attention(shared_heads=0) == attention(heads=3, shared_heads=2) == attention(key_dim=0)
            == attention(value_dim=0) == attention(type=3) == attention(window=-1) == attention(sinks=-1) == attention(scale=float("nan"))
            == attention(scale=float("inf")) == INVALID)
    assert attention(key_dim=257) == attention(value_dim=1000) == UNSUPPORTED
    assert attention(B=1 << 31) == attention(T=(1 << 31) - 1024) == attention(B=1 << 20, T=1 << 28) == LARGE
    assert attention(B=0, q=None) == attention(T=0, q=None) == OK
    assert lib.sig_window_attention(ctx, None, p, p, p, None, p, None, None, None) == INVALID
    assert lib.sig_window_attention_backward(ctx, ctypes.byref(window()), p, p, p, None, p, None, None, p, p, p, p, None) == INVALID      # (no stats)
    for kind in (binding.SIG_BF16, binding.SIG_F16):      # (no rest)
        assert lib.sig_window_attention(ctx, ctypes.byref(window(type=kind)), p, p, p, None, p, p, None, None) == INVALID
        assert lib.sig_window_attention_backward(ctx, ctypes.byref(window(type=kind)), p, p, p, None, p, p, None, p, p, p, p, None) == INVALID

    def append(q=p, k=p, v=p, lengths=p, q_out=p, of=(), B=1, T=1, heads=1, kind=0, **change):
        shape, c = binding.sig_append_t(B, T, heads, kind), cache(p, **dict(of))
        shape.scale = 1.0
        for name, value in change.items():
            setattr(shape, name, value)
        return lib.sig_cache_append(ctx, ctypes.byref(c), ctypes.byref(shape), q, k, v, lengths, None, q_out, None)

    assert append(q=None) == append(k=None) == append(v=None) == append(lengths=None) == append(q_out=None) == append(turned=2) == INVALID
    assert (append(B=-1) == append(T=-1) == append(heads=-1) == append(kind=3) == append(turned=3, frequencies=p) == append(turned=6, frequencies=p)
            == append(positions=p, position_type=4) == INVALID)
    narrow = dict(type=binding.SIG_E4M3)
    for of in (dict(pages=-1), dict(page_tokens=0), dict(heads=0), dict(key_dim=0), dict(value_dim=0), dict(table_pages=-1), dict(type=1), dict(keys=None), dict(values=None),
               dict(table=None), narrow, dict(narrow, key_scales=p)):
        assert append(of=of) == INVALID, of
    assert append(B=1 << 20, T=1 << 20) == append(heads=(1 << 31) - 1) == append(of=dict(page_tokens=1 << 40)) == LARGE
    assert append(of=dict(key_dim=8192), turned=8192, frequencies=p) == UNSUPPORTED
    assert append(B=0, k=None) == append(T=0, k=None) == OK

    def attend(q=p, lengths=p, out=p, of=(), B=1, T=1, heads=1, kind=0, scale=1.0, window=0, sinks=0):
        shape, c = binding.sig_queries_t(B, T, heads, kind, scale, window, sinks), cache(p, **dict(of))
        return lib.sig_cache_attention(ctx, ctypes.byref(c), ctypes.byref(shape), q, lengths, None, out, None)

    assert attend(q=None) == attend(lengths=None) == attend(out=None) == INVALID
    assert (attend(B=-1) == attend(T=-1) == attend(heads=0) == attend(kind=3) == attend(window=-1) == attend(sinks=-1) == attend(scale=float("nan"))
            == attend(heads=3, of=dict(heads=2)) == attend(of=dict(type=1)) == attend(of=narrow) == INVALID)
    assert attend(of=dict(key_dim=257)) == attend(of=dict(value_dim=257)) == UNSUPPORTED
    assert attend(T=(1 << 31) - 1024) == attend(B=1 << 31) == attend(B=1 << 20, T=1 << 20) == attend(of=dict(page_tokens=1 << 40)) == LARGE
    assert attend(B=0, q=None) == attend(T=0, q=None) == OK
    torch.cuda.synchronize()
    assert not room.any()                                                    # nothing was launched
