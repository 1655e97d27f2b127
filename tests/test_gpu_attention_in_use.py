"""Window attention and the paged cache as programs use them: graphs walked twice, traced calls, other streams, captured calls that share scratch, pages that
sequences share, long caches, and one call's results against another's that has to give the same numbers."""
import copy

import pytest
import torch

from paper_2501_08455_amd import autograd, binding, sequence
from test_gpu_cache import CACHES, E4M3, Pool, filled
from test_gpu_window_attention import TYPES, assert_near, noise, reference

gpu = pytest.mark.gpu


def heads_of(B, T, H, G, D, kind=torch.float32, seed=0):
    return [noise(B, T, h, D, seed=seed + i, kind=kind).cuda() for i, h in enumerate((H, G, G))]


# ---------------------------------------------------------------- gradients
@gpu
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("shape", [(1, 1500, 4, 2, 64, 10, 700), (2, 900, 2, 1, 128, 33, 129), (1, 800, 2, 2, 16, 1, 1)])
def test_many_first_tokens(shape, kind):
    B, T, H, G, D, window, sinks = shape
    q, k, v = (t.requires_grad_(True) for t in heads_of(B, T, H, G, D, kind))
    g = noise(B, T, H, D, seed=5, kind=kind).cuda()
    o = autograd.window_attention(q, k, v, window=window, sinks=sinks)
    want = reference(q, k, v, window, sinks, None, None, g)
    assert_near(o, want["o"], "o")
    for name, got in zip(("grad q", "grad k", "grad v"), torch.autograd.grad(o, (q, k, v), g)):
        assert_near(got, want[name], name)


@gpu
@pytest.mark.parametrize("kind", TYPES)
def test_many_sequences_with_many_first_tokens(kind):
    """Enough keys and queries to be left whole; the sequences that are compared, by themselves, have theirs cut (so their sums are in another order)."""
    B, T, H, G, D, window, sinks = 300, 520, 4, 4, 8, 5, 400
    q, k, v = (t.requires_grad_(True) for t in heads_of(B, T, H, G, D, kind))
    g = noise(B, T, H, D, seed=5, kind=kind).cuda()
    o = autograd.window_attention(q, k, v, window=window, sinks=sinks)
    grads = torch.autograd.grad(o, (q, k, v), g)
    some = slice(7, 300, 150)
    few = [t[some].detach().clone().requires_grad_(True) for t in (q, k, v)]
    o_few = autograd.window_attention(*few, window=window, sinks=sinks)
    want = reference(*few, window, sinks, None, None, g[some])
    assert_near(o[some], want["o"], "o")
    assert_near(o_few, want["o"], "o")
    for name, got, alone in zip(("grad q", "grad k", "grad v"), grads, torch.autograd.grad(o_few, few, g[some].contiguous())):
        assert_near(got[some], want[name], name)
        assert_near(alone, want[name], name)


@gpu
def test_a_graph_walked_twice_and_gradients_of_some_inputs():
    q, k, v = (t.requires_grad_(True) for t in heads_of(2, 90, 4, 2, 24))
    o = autograd.window_attention(q, k, v, window=30, sinks=2)
    g = torch.randn_like(o)
    first = torch.autograd.grad(o, (q, k, v), g, retain_graph=True)
    for a, b in zip(first, torch.autograd.grad(o, (q, k, v), g, retain_graph=True)):
        assert torch.equal(a, b)
    (only,) = torch.autograd.grad(o, v, g, retain_graph=True)
    assert torch.equal(only, first[2])
    # an upstream gradient that is a broadcast number, and one whose rows are not next to each other
    (total,) = torch.autograd.grad(o.sum(), q, retain_graph=True)
    assert torch.equal(total, torch.autograd.grad(o, q, torch.ones_like(o), retain_graph=True)[0])
    turned = g.transpose(1, 2).contiguous().transpose(1, 2)
    assert torch.equal(torch.autograd.grad(o, q, turned)[0], first[0])
    k.requires_grad_(False)
    q.requires_grad_(False)
    (alone,) = torch.autograd.grad(autograd.window_attention(q, k, v, window=30, sinks=2), v, g)
    assert torch.equal(alone, first[2])


@gpu
def test_one_tensor_for_all_three():
    x = noise(2, 70, 2, 16, seed=1).cuda().requires_grad_(True)
    (got,) = torch.autograd.grad(autograd.window_attention(x, x, x, window=9).square().sum(), x)
    q, k, v = (x.detach().clone().requires_grad_(True) for _ in range(3))
    grads = torch.autograd.grad(autograd.window_attention(q, k, v, window=9).square().sum(), (q, k, v))
    assert float((got - sum(grads)).abs().max()) <= 4 * 2.0 ** -24 * float(sum(t.abs() for t in grads).max())      # (three sums, in any order)


@gpu
def test_what_changes_between_the_passes_is_noticed():
    q, k, v = (t.requires_grad_(True) for t in heads_of(1, 20, 1, 1, 8))
    o = autograd.window_attention(q, k, v)
    with torch.no_grad():
        k.add_(1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        o.sum().backward()


@gpu
def test_forward_mode_and_transforms_are_refused():
    x = torch.randn(1, 5, 2, 8, device="cuda", requires_grad=True)
    call = lambda t: autograd.window_attention(t, t, t)      # noqa: E731
    with torch.autograd.forward_ad.dual_level(), pytest.raises(NotImplementedError):
        call(torch.autograd.forward_ad.make_dual(x, x))
    for bad in (lambda: torch.vmap(call)(x[None]), lambda: torch.func.grad(lambda t: call(t).sum())(x.detach())):
        with pytest.raises(RuntimeError):
            bad()


@gpu
def test_traced_calls_compute_with_their_own_input():
    lengths = torch.tensor([6, 4], device="cuda")
    model = lambda x: autograd.window_attention(x, x, x, window=3, sinks=1, lengths=lengths) * 2.0      # noqa: E731
    first, other = torch.randn(2, 6, 2, 8, device="cuda"), torch.randn(2, 6, 2, 8, device="cuda")
    traced = torch.jit.trace(model, (first,), check_trace=False)
    for base in (first, other):
        a, b = base.clone().requires_grad_(True), base.clone().requires_grad_(True)
        got, want = traced(a), model(b)
        assert torch.equal(got, want)
        got.square().sum().backward()
        want.square().sum().backward()
        assert torch.equal(a.grad, b.grad)


# ---------------------------------------------------------------- streams and graphs
@gpu
def test_a_stream_of_ones_own():
    q, k, v = (t.requires_grad_(True) for t in heads_of(2, 700, 4, 2, 64, torch.bfloat16))
    g = noise(2, 700, 4, 64, seed=4, kind=torch.bfloat16).cuda()
    pool = filled(2, 700, 2, 16, 64, 64, torch.bfloat16, torch.bfloat16)
    lengths = torch.tensor([700, 555], device="cuda")

    def work():
        o = autograd.window_attention(q, k, v, window=100, sinks=3)
        return [o, *torch.autograd.grad(o, (q, k, v), g), binding.cache_attention(q[:, :1], pool.keys, pool.values, pool.table, lengths)]

    want = work()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = work()
    again = work()      # (beside it: each stream has scratch of its own)
    torch.cuda.synchronize()
    for a, b, c in zip(want, got, again):
        assert torch.equal(a, b) and torch.equal(a, c)


@gpu
def test_captured_calls_that_share_scratch():
    """Two graphs, a gradient and an attention that is cut along its places, replayed in turn with eager calls of other sizes between."""
    B, T, H, G, D = 2, 600, 4, 2, 32
    base = heads_of(B, T, H, G, D)
    g = noise(B, T, H, D, seed=4).cuda()
    pool = filled(B, 3000, G, 16, D, D, torch.float32, torch.float32)
    query, lengths = noise(B, 1, H, D, seed=6).cuda(), torch.tensor([3000, 2500], device="cuda")

    def gradient():
        leaves = [t.detach().requires_grad_(True) for t in base]
        return torch.autograd.grad(autograd.window_attention(*leaves, window=70, sinks=2), leaves, g)

    def attention():
        return binding.cache_attention(query, pool.keys, pool.values, pool.table, lengths)

    (first, grads), (second, out) = autograd.capture(gradient), autograd.capture(attention)
    large = heads_of(3, 1100, 6, 3, 64, seed=9)
    for turn in range(3):
        for t in (*base, query):
            t.copy_(torch.randn_like(t))
        lengths.sub_(turn * 100)
        want, want_out = [t.clone() for t in gradient()], attention().clone()
        binding.window_attention(*large, window=500)
        first.replay()
        second.replay()
        first.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want_out) and all(torch.equal(a, b) for a, b in zip(grads, want)), turn
        gradient()
        torch.cuda.synchronize()


# ---------------------------------------------------------------- caches
@gpu
@pytest.mark.parametrize("kind,cache", CACHES)
def test_sequences_that_share_pages(kind, cache):
    """A common beginning is kept once; what stands behind it differs."""
    B, G, P, D, common, T = 3, 2, 8, 32, 4, 5
    pool = filled(B, 64, G, P, D, D, kind, cache)
    shared = pool.table.clone()
    shared[:, :common] = pool.table[:1, :common]
    apart = Pool(B, 64, G, P, D, D, cache, seed=3)
    for name in ("keys", "values", "key_scales", "value_scales"):
        pages = getattr(pool, name)
        if pages is not None:
            getattr(apart, name)[apart.table.long()] = pages[shared.long()]
    q, lengths = noise(B, T, 4, D, seed=8, kind=kind).cuda(), torch.tensor([60, 41, 64], device="cuda")
    for window in (None, 37):
        assert torch.equal(binding.cache_attention(q, pool.keys, pool.values, shared, lengths, window=window, **pool.scales()),
                           binding.cache_attention(q, apart.keys, apart.values, apart.table, lengths, window=window, **apart.scales()))


@gpu
@pytest.mark.parametrize("kind,cache,pages", [(torch.bfloat16, torch.bfloat16, 17000), (torch.bfloat16, E4M3, 34000)])
def test_pages_behind_32_bits(kind, cache, pages):
    """The last pages of a pool whose values, or bytes, are more than 2^32 of each, against the same pages in a small one."""
    G, P, D, places, B = 8, 64, 256, 640, 2
    width = 2 if cache == kind else 1
    assert pages * G * P * D * width > 1 << 32
    keys, values = (torch.empty(pages, G, P, D, device="cuda", dtype=cache) for _ in range(2))
    scales = {name: torch.ones(pages, G, device="cuda") for name in ("key_scales", "value_scales")} if cache == E4M3 else {}
    n = places // P
    table = (pages - 1 - torch.randperm(B * n, generator=torch.Generator().manual_seed(1))).view(B, n).int().cuda()
    small = Pool(B, places, G, P, D, D, cache)
    k, v, q = (noise(B, places, h, D, seed=h + i, kind=kind).cuda() for i, h in enumerate((G, G, 2 * G)))
    zero, lengths = torch.zeros(B, dtype=torch.int64, device="cuda"), torch.tensor([places, places - 77], device="cuda")
    f, _ = sequence.rotary_frequencies(D)
    turned = [binding.cache_append(k, v, a, b, t, zero, q=q, frequencies=f, **s) for a, b, t, s in ((keys, values, table, scales), (small.keys, small.values, small.table, small.scales()))]
    assert torch.equal(*turned)
    q = turned[0][:, :3].contiguous()
    for window in (None, 100):
        assert torch.equal(binding.cache_attention(q, keys, values, table, lengths, window=window, sinks=2, **scales),
                           binding.cache_attention(q, small.keys, small.values, small.table, lengths, window=window, sinks=2, **small.scales()))


@gpu
@pytest.mark.parametrize("kind,cache", CACHES)
def test_caches_with_nothing_in_them(kind, cache):
    B, T, G, D = 2, 3, 2, 16
    k, v, q = (noise(B, T, h, D, seed=i, kind=kind).cuda() for i, h in enumerate((G, G, 4)))
    zero = torch.zeros(B, dtype=torch.int64, device="cuda")
    f, _ = sequence.rotary_frequencies(D)
    pool = Pool(B, 32, G, 16, D, D, cache)
    none = {name: None if t is None else t[:0] for name, t in (("keys", pool.keys), ("values", pool.values), *pool.scales().items())}
    for table, pages in ((pool.table, none), (pool.table[:, :0], dict(keys=pool.keys, values=pool.values, **pool.scales())), (pool.table[:, :0], none)):
        turned = binding.cache_append(k, v, table=table, lengths=zero, q=q, frequencies=f, **pages)
        assert torch.equal(turned, binding.rotary(q, torch.arange(T, device="cuda"), f))
        assert not binding.cache_attention(q, table=table, lengths=zero + 3, **pages).any()
    assert (pool.keys.float() == 7.0).all()
    # more queries than tokens: those in front of the first one see nothing
    full = filled(B, 32, G, 16, D, D, kind, cache)
    got = binding.cache_attention(q, full.keys, full.values, full.table, zero + 1, **full.scales())
    assert not got[:, :2].any() and got[:, 2].any()
    many = noise(B, 300, 4, D, seed=5, kind=kind).cuda()
    got = binding.cache_attention(many, full.keys, full.values, full.table, zero + 1, window=4, sinks=2, **full.scales())
    assert not got[:, :299].any() and got[:, 299].any()


@gpu
def test_zeros_behind_scales_of_zero():
    """Pages whose scales are still 0, as they were allocated: zeros behind their first slot are zeros, and what follows counts."""
    keys, values = (torch.zeros(1, 1, 8, 4, device="cuda").to(E4M3) for _ in range(2))
    scales = {name: torch.zeros(1, 1, device="cuda") for name in ("key_scales", "value_scales")}
    table, zeros = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.zeros(1, 1, 1, 4, device="cuda")
    at = torch.full((1,), 3, dtype=torch.int64, device="cuda")
    binding.cache_append(zeros, zeros, keys, values, table, at, **scales)
    assert not keys.float().any() and not values.float().any()
    binding.cache_append(zeros + 3.0, zeros - 448.0, keys, values, table, at + 1, **scales)
    assert float(scales["value_scales"]) == 1.0 and (values[0, 0, 4].float() == -448.0).all() and (keys[0, 0, 4].float() * scales["key_scales"] == 3.0).all()
    assert not values[0, 0, :4].float().any()


@gpu
def test_operands_inside_the_cache_are_refused():
    pool = Pool(1, 16, 2, 16, 8, 8, torch.float32)
    n = torch.zeros(1, dtype=torch.int64, device="cuda")
    inside, other = pool.keys[:1].transpose(1, 2)[:, :3], torch.zeros(1, 3, 2, 8, device="cuda")
    for k, v, q in ((inside, other, None), (other, inside, None), (other, other, inside)):
        with pytest.raises(ValueError, match="apart from the cache"):
            binding.cache_append(k, v, pool.keys, pool.values, pool.table, n, q=q)
    binding.cache_append(other, other, pool.keys, pool.values, pool.table, n.int(), q=other)


@gpu
def test_pages_of_one_buffer():
    """Keys and values next to each other, page by page."""
    B, T, G, P, D = 2, 40, 2, 16, 24
    k, v = noise(B, T, G, D, seed=1).cuda(), noise(B, T, G, D, seed=2).cuda()
    pool, both = Pool(B, T, G, P, D, D, torch.float32), torch.zeros(7, 2, P, G, D, device="cuda")
    keys, values = both[:, 0].transpose(1, 2), both[:, 1].transpose(1, 2)
    zero, lengths, q = torch.zeros(B, dtype=torch.int64, device="cuda"), torch.tensor([40, 31], device="cuda"), noise(B, 1, 4, D, seed=3).cuda()
    out = []
    for a, b in ((pool.keys, pool.values), (keys, values)):
        binding.cache_append(k, v, a, b, pool.table, zero)
        out.append(binding.cache_attention(q, a, b, pool.table, lengths, window=20, sinks=1))
    assert torch.equal(*out)


# ---------------------------------------------------------------- the model
@gpu
def test_models_from_before_their_mixer():
    """A linear model's attributes are those that it had without a choice of mixers."""
    torch.manual_seed(1)
    model = sequence.SequenceModel(3, 3, 2, 2, heads=2, head_dim=8)
    old = copy.deepcopy(model)
    for name in ("mixer", "window", "sinks"):
        del old.__dict__[name]
    x = torch.randn(2, 9, 3, device="cuda")
    assert torch.equal(old(x), model(x))
    cache = old.begin(x[:, 0])
    assert old.step(x[:, 1], cache).shape == (2, 2)
