"""GPU tests of the decoder that runs norm, rotary positions, causal attention, the cache in pages and the KAT MLP together.

The plain decoder below computes the same from float32 copies of the parameters, with the formulas written out (and the KAT MLP in float32,
which has tests of its own).  Bound, as a relative norm, as for the cross decoder: a block rounds about 14 tensors one behind the other, each by
u at most (2^-11 or 2^-8) and by no more than the norms' rows scale back up; the backward pass rounds each of them and its gradient: blocks x 14 u
forward, three times that for gradients.  Tokens over what a cache holds differ from a whole sequence's by both sides' roundings: twice that."""
import copy

import pytest

pytestmark = pytest.mark.gpu

UNIT = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def _plain_norm(h, m):
    return h * (h.square().mean(-1, keepdim=True) + m.eps).rsqrt() * m.weight


def _plain_rotary(torch, x, positions, m):
    f, axis = m.frequency_bits.view(torch.float64), m.axis.long()
    angle = (positions.double()[..., axis] * f).float()
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    n = f.numel()
    a, b = x[..., :n], x[..., n:2 * n]
    return torch.cat([a * c - b * s, a * s + b * c, x[..., 2 * n:]], -1)


def _plain(torch, m, x, offsets, positions=None):
    """x [tokens, dim], every token in a sequence"""
    for block in m.blocks:
        qkv = block.to_qkv(_plain_norm(x, block.norm1)).unflatten(-1, (-1, block.head_dim))
        q, k, v = qkv.split((block.heads, block.kv_heads, block.kv_heads), -2)
        if block.rotary is not None:
            q, k = _plain_rotary(torch, q, positions, block.rotary), _plain_rotary(torch, k, positions, block.rotary)
        group, parts = block.heads // block.kv_heads, []
        for first, end in zip(offsets, offsets[1:]):
            Q, K, V = (t[first:end].transpose(0, 1) for t in (q, k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)))
            s = Q @ K.transpose(-1, -2).contiguous() * block.head_dim ** -0.5
            p = s.masked_fill(torch.ones_like(s, dtype=torch.bool).triu(1), -1e30).softmax(-1)
            parts.append((p @ V.contiguous()).transpose(0, 1).flatten(-2))
        x = x + block.proj(torch.cat(parts))
        x = x + block.mlp(_plain_norm(x, block.norm2))
    return _plain_norm(x, m.norm)


def _decoder(torch, dtype, depth=2, seed=0, **block):
    from paper_2505_13813_amd.transformer import KATDecoder

    torch.manual_seed(seed)
    m = KATDecoder(depth, 192, 3, **block).cuda()
    with torch.no_grad():
        for name, p in m.named_parameters():
            if "norm" in name:
                p.uniform_(0.5, 1.5)
    return m if dtype == "f32" else m.to({"f16": torch.float16, "bf16": torch.bfloat16}[dtype])


def _near(got, want, bound, label):
    got, want = got.detach().float(), want.detach().float()
    off = float((got - want).norm() / want.norm())
    assert off <= bound, (label, off, bound)


def _places(torch, lengths):
    return torch.cat([torch.arange(n, dtype=torch.int32, device="cuda:0") for n in lengths])[:, None]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rotary", [(), (32,), (20,)])
@pytest.mark.parametrize("kv_heads", [3, 1])
def test_training_step(kv_heads, rotary, dtype):
    import torch

    print(kv_heads, rotary, dtype, flush=True)
    m = _decoder(torch, dtype, rotary_pairs=rotary, kv_heads=kv_heads)
    reference = copy.deepcopy(m).float()
    lengths = [70, 1, 0, 129]
    offsets = [0, 70, 71, 71, 200]
    at = _places(torch, lengths) if rotary else None
    torch.manual_seed(1)
    io = next(m.parameters()).dtype
    x = torch.randn(200, 192, device="cuda:0").to(io)
    leaf, plain = x.clone().requires_grad_(), x.float().requires_grad_()
    out = m(leaf, torch.tensor(offsets, device="cuda:0"), at)
    want = _plain(torch, reference, plain, offsets, at)
    assert out.dtype == io
    bound = 2 * 14 * UNIT[dtype]
    _near(out, want, bound, "out")
    dout = torch.randn_like(want).to(io)
    out.backward(dout)
    want.backward(dout.float())
    _near(leaf.grad, plain.grad, 3 * bound, "x")
    for (name, p), (_, w) in zip(m.named_parameters(), reference.named_parameters()):
        assert p.grad is not None and bool(p.grad.isfinite().all()), name
        if "norm" in name or "proj.weight" in name or "to_" in name and name.endswith("weight"):
            _near(p.grad, w.grad, 3 * bound, name)


def test_float32_parameters_under_autocast():
    import torch

    m = _decoder(torch, "f32", rotary_pairs=(32,))
    at = _places(torch, [40, 24])
    torch.manual_seed(2)
    x = torch.randn(64, 192, device="cuda:0", requires_grad=True)
    with torch.autocast("cuda", dtype=torch.bfloat16):
        out = m(x, torch.tensor([0, 40, 64], device="cuda:0"), at)
    assert out.dtype == torch.float32
    other, reference = x.detach().clone().requires_grad_(), copy.deepcopy(m)
    want = _plain(torch, reference, other, [0, 40, 64], at)
    bound = 2 * 14 * UNIT["bf16"]
    _near(out, want, bound, "out")
    dout = torch.randn_like(out)
    out.backward(dout)
    want.backward(dout)
    _near(x.grad, other.grad, 3 * bound, "x")


def test_a_batch_is_sequences_of_one_length():
    import torch

    m = _decoder(torch, "bf16", rotary_pairs=(32,), kv_heads=1)
    torch.manual_seed(3)
    x = torch.randn(3, 50, 192, device="cuda:0", dtype=torch.bfloat16)
    with torch.no_grad():
        whole = m(x, positions=_places(torch, [50]))
        packed = m(x.flatten(0, 1), torch.arange(4, device="cuda:0") * 50, _places(torch, [50] * 3))
    assert torch.equal(whole.flatten(0, 1), packed)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("page", [16, 64])
def test_prompts_and_then_tokens(page, dtype):
    """Prompts of different lengths into a cache, then a token at a time, and a few at once: near what the whole sequences get in one call; the
    same bits from a captured step that is replayed as the cache grows; a released row that another sequence takes."""
    import torch

    m = _decoder(torch, dtype, rotary_pairs=(32,), kv_heads=1)
    io = next(m.parameters()).dtype
    lengths, steps = [33, 1, 150, 64], 9
    torch.manual_seed(4)
    whole = [torch.randn(n + steps, 192, device="cuda:0", dtype=io) for n in lengths]
    every = torch.cat(whole)
    offsets = torch.tensor([0, *torch.tensor([n + steps for n in lengths]).cumsum(0).tolist()], device="cuda:0")
    bound = 2 * 14 * UNIT[dtype]
    with torch.no_grad():
        want = m(every, offsets, _places(torch, [n + steps for n in lengths]))
        want = [want[a:b] for a, b in zip(offsets.tolist(), offsets[1:].tolist())]

        def prompts():
            cache = m.cache(40, page, 4, 200)
            cache.grow(lengths)
            at = torch.tensor([0, *torch.tensor(lengths).cumsum(0).tolist()], device="cuda:0")
            out = m(torch.cat([t[:n] for t, n in zip(whole, lengths)]), at, _places(torch, lengths), cache)
            for i, n in enumerate(lengths):
                _near(out[at[i]:at[i + 1]], want[i][:n], bound, ("prompt", i))
            return cache

        def tokens(first, count):
            x = torch.stack([t[n + first:n + first + count] for t, n in zip(whole, lengths)])
            place = torch.tensor([[[n + first + j] for j in range(count)] for n in lengths], dtype=torch.int32, device="cuda:0")
            return x, place

        cache, found = prompts(), []
        for i in range(steps):
            cache.grow([1] * 4)
            x, place = tokens(i, 1)
            found.append(m.step(x, cache, place))
            for s, n in enumerate(lengths):
                _near(found[-1][s], want[s][n + i:n + i + 1], 2 * bound, (i, s))
        assert cache.counts == [n + steps for n in lengths] and cache.lengths.tolist() == cache.counts
        other = prompts()
        other.grow([steps] * 4)
        at_once = m.step(*((lambda t: (t[0], other, t[1]))(tokens(0, steps))))
        for s, n in enumerate(lengths):
            _near(at_once[s], want[s][n:], 2 * bound, ("at once", s))
        # captured: the cache's table and lengths stay where they are
        third = prompts()
        x, place = tokens(0, 1)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            m.step(x, m.cache(40, page, 4, 200), place)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = m.step(x, third, place)
        for i in range(steps):
            third.grow([1] * 4)
            for to, t in zip((x, place), tokens(i, 1)):
                to.copy_(t)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(held, found[i])
        # a row for another sequence
        free = cache.free_pages
        cache.release(2)
        assert cache.free_pages == free + -(-(150 + steps) // page)
        cache.grow([0, 0, 20, 0])
        x = torch.randn(20, 192, device="cuda:0", dtype=io)
        got = m(x, torch.tensor([0, 0, 0, 20, 20], device="cuda:0"), _places(torch, [20]), cache)
        _near(got, m(x, torch.tensor([0, 20], device="cuda:0"), _places(torch, [20])), 0.0, "same bits")
        assert cache.lengths.tolist() == cache.counts == [33 + steps, 1 + steps, 20, 64 + steps]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_a_cache_under_autocast(dtype):
    """Float32 parameters and streams, the cache of autocast's type: prompts and then tokens as the whole sequences in float32.  A cache of float32 is refused."""
    import torch

    io = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    m = _decoder(torch, "f32", rotary_pairs=(32,), kv_heads=1)
    lengths, steps = [40, 1, 23], 5
    torch.manual_seed(6)
    whole = [torch.randn(n + steps, 192, device="cuda:0") for n in lengths]
    ends = lambda counts: [sum(counts[:i]) for i in range(len(counts) + 1)]  # noqa: E731
    bound = 2 * 14 * UNIT[dtype]
    with torch.no_grad():
        every = [n + steps for n in lengths]
        want = _plain(torch, m, torch.cat(whole), ends(every), _places(torch, every)).split(every)
        with torch.autocast("cuda", dtype=io):
            cache = m.cache(20, 16, 3, 64, dtype=io)
            cache.grow(lengths)
            out = m(torch.cat([t[:n] for t, n in zip(whole, lengths)]), torch.tensor(ends(lengths), device="cuda:0"), _places(torch, lengths), cache)
            assert out.dtype == torch.float32 and cache.k_pages[0].dtype == io
            for got, w, n in zip(out.split(lengths), want, lengths):
                _near(got, w[:n], bound, ("prompt", n))
            for i in range(steps):
                cache.grow([1] * 3)
                place = torch.tensor([[[n + i]] for n in lengths], dtype=torch.int32, device="cuda:0")
                out = m.step(torch.stack([t[n + i:n + i + 1] for t, n in zip(whole, lengths)]), cache, place)
                assert out.dtype == torch.float32
                for got, w, n in zip(out, want, lengths):
                    _near(got, w[n + i:n + i + 1], 2 * bound, (n, i))
            wide = m.cache(20, 16, 3, 64)
            wide.grow([1] * 3)
            with pytest.raises(TypeError, match="k_pages"):
                m.step(torch.stack([t[:1] for t in whole]), wide, torch.zeros(3, 1, 1, dtype=torch.int32, device="cuda:0"))


def test_growing_is_no_part_of_a_captured_step():
    import torch

    m = _decoder(torch, "bf16", kv_heads=1)
    cache = m.cache(10, 16, 2, 64)
    x = torch.randn(2, 1, 192, device="cuda:0", dtype=torch.bfloat16)
    with torch.no_grad():
        cache.grow([1, 1])
        want = m.step(x, cache)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for call in (lambda: cache.grow([1, 1]), lambda: cache.grow([16, 0]), lambda: cache.release(0)):
                with pytest.raises(RuntimeError, match="captur"):
                    call()
            got = m.step(x, cache)
        graph.replay()
        torch.cuda.synchronize()
    assert cache.counts == cache.lengths.tolist() == [1, 1] and cache.free_pages == 8 and torch.equal(got, want)


def test_saved_tensor_hooks():
    """Operands that come back from hooks in another layout, and of the wrong shape or type."""
    import torch

    from paper_2505_13813_amd import transformer as T

    q, k, v = (torch.randn(50, h, 64, device="cuda:0", dtype=torch.bfloat16, requires_grad=True) for h in (4, 2, 2))
    offsets = torch.tensor([0, 20, 50], device="cuda:0")

    def loss():
        return T.causal_attention(q, k, v, offsets).square().mean()

    want = torch.autograd.grad(loss(), (q, k, v))
    turned = lambda t: t.transpose(0, 1).contiguous().transpose(0, 1) if t.dim() == 3 and t.shape[1] == 2 else t  # noqa: E731
    with torch.autograd.graph.saved_tensors_hooks(turned, lambda t: t):
        out = loss()
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(out, (q, k, v)), want))
    for cut in (lambda t: t[:-1] if t.dim() == 3 else t, lambda t: t.float(), lambda t: t.cpu(), lambda t: t[:, :-1] if t.dim() == 3 else t):
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, cut):
            out = loss()
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            torch.autograd.grad(out, (q, k, v))


def test_under_compile():
    """torch.compile leaves the calls as they are, between its graphs."""
    import torch

    from paper_2505_13813_amd import transformer as T

    pool = torch.zeros(2, 4, 16, 3, 32, device="cuda:0", dtype=torch.bfloat16)
    table, lengths = torch.arange(4, dtype=torch.int32, device="cuda:0").view(2, 2), torch.tensor([20, 20], device="cuda:0")

    def f(x):
        q = (x * 2).view(2, 20, 3, 32)
        T.paged_write(q, q + 1, pool[0], pool[1], table, lengths)
        return T.causal_attention(q, q + 1, q) * 2, T.paged_attention(q[:, -1:], pool[0], pool[1], table, lengths) + 1

    x = torch.randn(40, 96, device="cuda:0", dtype=torch.bfloat16)
    with torch.no_grad():
        assert all(torch.equal(a, b) for a, b in zip(torch.compile(f, backend="eager")(x), f(x)))


def test_transforms_modes_and_forward_differentiation_are_refused():
    import torch
    from torch.autograd import forward_ad
    from torch.utils._python_dispatch import TorchDispatchMode

    from paper_2505_13813_amd import transformer as T

    class Mode(TorchDispatchMode):
        def __torch_dispatch__(self, function, types, args=(), kwargs=None):
            return function(*args, **(kwargs or {}))

    pool = torch.zeros(2, 4, 16, 2, 32, device="cuda:0", dtype=torch.bfloat16)
    table, lengths = torch.arange(4, dtype=torch.int32, device="cuda:0").view(2, 2), torch.tensor([20, 20], device="cuda:0")
    x = torch.randn(2, 3, 2, 32, device="cuda:0", dtype=torch.bfloat16)

    def write(t):
        T.paged_write(t, t, pool[0], pool[1], table, lengths)
        return t

    with torch.no_grad():
        for call in (lambda t: T.causal_attention(t, t, t), write, lambda t: T.paged_attention(t, pool[0], pool[1], table, lengths)):
            with pytest.raises(NotImplementedError):
                torch.func.vmap(call)(x[None])
            with pytest.raises(NotImplementedError):
                torch.func.jvp(call, (x,), (x,))
            with pytest.raises(NotImplementedError):
                torch.func.grad(lambda t: call(t).float().sum())(x)
            with forward_ad.dual_level(), pytest.raises(NotImplementedError):
                call(forward_ad.make_dual(x, x))
            with Mode(), pytest.raises(NotImplementedError):
                call(x)
            assert call(x).shape == x.shape
    torch.cuda.synchronize()
    assert int(pool.count_nonzero()) == 2 * x.count_nonzero()  # the one write that was not refused
