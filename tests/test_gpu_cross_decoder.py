"""GPU tests of the decoder that runs norm, rotary positions, cross attention and the KAT MLP together.

The plain decoder below computes the same from float32 copies of the parameters, with the formulas written out (and the KAT MLP in
float32, which has tests of its own).  Bound, as a relative norm: a block in float16 rounds about 14 tensors one behind the other (two norms and
their streams, q, k and v, their rotations, P, the attention's output, the projection, four in the MLP), each by 2^-11 at most and by no more than
the norms' rows scale back up; the backward pass rounds each of them and its gradient.  blocks x 14 x 2^-11 forward, three times that for gradients;
bfloat16: 2^-8 in its place."""
import copy

import pytest

pytestmark = pytest.mark.gpu

UNIT = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def _plain_norm(h, m):
    return h * (h.square().mean(-1, keepdim=True) + m.eps).rsqrt() * m.weight


def _plain_rotary(torch, x, positions, m):
    f, axis = m.frequency_bits.view(torch.float64), m.axis.long()
    angle = (positions.double()[..., axis] * f).float()
    if angle.dim() == 2:
        angle = angle[None]
    c, s = angle.cos()[:, :, None], angle.sin()[:, :, None]
    n = f.numel()
    a, b = x[..., :n], x[..., n:2 * n]
    return torch.cat([a * c - b * s, a * s + b * c, x[..., 2 * n:]], -1)


def _plain_block(torch, m, x, context, positions, context_positions, valid):
    y = _plain_norm(x, m.norm1)
    q = m.to_q(y).unflatten(-1, (m.heads, m.head_dim))
    k, v = m.keys_values(context)
    if m.rotary is not None:
        q, k = _plain_rotary(torch, q, positions, m.rotary), _plain_rotary(torch, k, context_positions, m.rotary)
    group = m.heads // m.kv_heads
    k, v = (t.repeat_interleave(group, 2).transpose(1, 2) for t in (k, v))
    s = q.transpose(1, 2) @ k.transpose(-1, -2).contiguous() * m.head_dim ** -0.5
    p = s.masked_fill(~valid[:, None, None], -1e30).softmax(-1) * valid[:, None, None]
    x = x + m.proj((p @ v.contiguous()).transpose(1, 2).flatten(-2))
    return x + m.mlp(_plain_norm(x, m.norm2))


def _plain(torch, m, x, context, positions=None, context_positions=None, valid=None):
    if valid is None:
        valid = torch.ones(context.shape[:2], dtype=torch.bool, device=x.device)
    for block in m.blocks:
        x = _plain_block(torch, block, x, context, positions, context_positions, valid)
    return _plain_norm(x, m.norm)


def _decoder(torch, dtype, depth=2, seed=0, **block):
    from paper_2505_13813_amd.transformer import KATCrossDecoder

    torch.manual_seed(seed)
    m = KATCrossDecoder(depth, 192, 3, **block).cuda()
    with torch.no_grad():
        for name, p in m.named_parameters():
            if "norm" in name:
                p.uniform_(0.5, 1.5)
    return m if dtype == "f32" else m.to({"f16": torch.float16, "bf16": torch.bfloat16}[dtype])


def _near(got, want, bound, label):
    got, want = got.detach().float(), want.detach().float()
    off = float((got - want).norm() / want.norm())
    assert off <= bound, (label, off, bound)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("kind", ["image", "video", "no positions"])
def test_training_step(kind, dtype):
    import torch

    from paper_2505_13813_amd.transformer import grid_positions

    print(kind, dtype, flush=True)
    io = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
    torch.manual_seed(1)
    if kind == "image":
        m, queries, keys = _decoder(torch, dtype, rotary_pairs=(16, 16)), grid_positions(7, 9, device="cuda:0"), grid_positions(12, 11, device="cuda:0")
    elif kind == "video":
        m, queries, keys = _decoder(torch, dtype, rotary_pairs=(8, 12, 12), kv_heads=1), grid_positions(2, 5, 6, device="cuda:0"), grid_positions(4, 6, 5, device="cuda:0")
    else:
        m, queries, keys = _decoder(torch, dtype, context_dim=128), torch.zeros(50, 1), torch.zeros(90, 1)
    with_positions = kind != "no positions"
    reference = copy.deepcopy(m).float()
    x = torch.randn(3, len(queries), 192, device="cuda:0").to(io)
    context = torch.randn(3, len(keys), 128 if kind == "no positions" else 192, device="cuda:0").to(io)
    lengths = torch.tensor([len(keys), 17, 1], device="cuda:0")
    valid = torch.arange(len(keys), device="cuda:0") < lengths[:, None]
    places = dict(positions=queries, context_positions=keys) if with_positions else {}
    leaves = [t.clone().requires_grad_() for t in (x, context)]
    plain = [t.float().requires_grad_() for t in (x, context)]
    out = m(*leaves, key_lengths=lengths, **places)
    want = _plain(torch, reference, *plain, valid=valid, **places)
    assert out.dtype == io
    bound = 2 * 14 * UNIT[dtype]
    _near(out, want, bound, "out")
    dout = torch.randn_like(want).to(io)
    out.backward(dout)
    want.backward(dout.float())
    for got, w, label in zip(leaves, plain, ("x", "context")):
        _near(got.grad, w.grad, 3 * bound, label)
    assert (leaves[1].grad[1, 17:] == 0).all()
    # every parameter has its gradient; the weights' as near as the tensors' (the rational's coefficients are sums that cancel)
    for (name, p), (_, w) in zip(m.named_parameters(), reference.named_parameters()):
        assert p.grad is not None and bool(p.grad.isfinite().all()), name
        if "norm" in name or "proj.weight" in name or "to_" in name and name.endswith("weight"):
            _near(p.grad, w.grad, 3 * bound, name)


def test_float32_parameters_under_autocast():
    import torch

    m = _decoder(torch, "f32", rotary_pairs=(16, 16))
    from paper_2505_13813_amd.transformer import grid_positions

    torch.manual_seed(2)
    at, of = grid_positions(6, 6, device="cuda:0"), grid_positions(8, 9, device="cuda:0")
    x, context = torch.randn(2, 36, 192, device="cuda:0", requires_grad=True), torch.randn(2, 72, 192, device="cuda:0")
    with torch.autocast("cuda", dtype=torch.bfloat16):
        out = m(x, context, at, of)
    assert out.dtype == torch.float32
    bound = 2 * 14 * UNIT["bf16"]
    other = x.detach().clone().requires_grad_()
    reference = copy.deepcopy(m)
    want = _plain(torch, reference, other, context, at, of)
    _near(out, want, bound, "out")
    dout = torch.randn_like(out)
    out.backward(dout)
    want.backward(dout)
    _near(x.grad, other.grad, 3 * bound, "x")


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_single_tokens_on_cached_states(dtype):
    """A token at a time on states laid out once: the same bits as with the states anew, near what all tokens get in one call, and the same
    bits from a captured step, replayed with eager work between."""
    import torch

    from paper_2505_13813_amd.transformer import grid_positions

    m = _decoder(torch, dtype, rotary_pairs=(16, 16), kv_heads=1)
    io = next(m.parameters()).dtype
    torch.manual_seed(3)
    of = grid_positions(30, 40, device="cuda:0")
    x, context = torch.randn(4, 5, 192, device="cuda:0", dtype=io), torch.randn(4, 1200, 192, device="cuda:0", dtype=io)
    lengths = torch.tensor([1200, 1, 600, 0], device="cuda:0")
    at = torch.stack([torch.arange(5, dtype=torch.int32), torch.arange(5, dtype=torch.int32) % 3], -1).cuda()
    with torch.no_grad():
        every = m(x, context, at, of, key_lengths=lengths)
        cache = m.cached(context, of)
        token, place = torch.empty_like(x[:, :1]), torch.empty_like(at[:1])
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            m(token.zero_(), positions=place.zero_(), key_lengths=lengths, cache=cache)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = m(token, positions=place, key_lengths=lengths, cache=cache)
        for i in range(5):
            one = m(x[:, i:i + 1], positions=at[i:i + 1], key_lengths=lengths, cache=cache)
            assert torch.equal(one, m(x[:, i:i + 1], context, at[i:i + 1], of, key_lengths=lengths))
            _near(one, every[:, i:i + 1], 2 * 14 * UNIT[dtype], i)
            token.copy_(x[:, i:i + 1])
            place.copy_(at[i:i + 1])
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(held, one)


def test_under_compile():
    """torch.compile leaves the calls as they are, between its graphs."""
    import torch

    from paper_2505_13813_amd import transformer as T

    x = torch.randn(40, 96, device="cuda:0", dtype=torch.bfloat16)
    w = torch.rand(96, device="cuda:0", dtype=torch.bfloat16)

    def f(x, w):
        y, h = T.rms_norm(x * 2, w, x)
        q = y.view(2, 20, 3, 32)
        return T.cross_attention(q, q + 1, q) * 2, h

    assert all(torch.equal(a, b) for a, b in zip(torch.compile(f, backend="eager")(x, w), f(x, w)))


def test_saved_tensor_hooks():
    """Operands that come back from hooks in another layout, and of the wrong shape."""
    import torch

    from paper_2505_13813_amd import transformer as T

    x = torch.randn(30, 64, device="cuda:0", dtype=torch.bfloat16, requires_grad=True)
    w = torch.rand(64, device="cuda:0", dtype=torch.bfloat16, requires_grad=True)
    q, k, v = (torch.randn(2, 20, 2, 64, device="cuda:0", dtype=torch.bfloat16, requires_grad=True) for _ in range(3))
    leaves = [x, w, q, k, v]

    def both():
        return (T.rms_norm(x, w).square().mean() + T.cross_attention(q, k, v).square().mean())

    want = torch.autograd.grad(both(), leaves)
    strided = lambda t: t.t().contiguous().t() if t.dim() == 2 and t.is_floating_point() else t  # noqa: E731
    with torch.autograd.graph.saved_tensors_hooks(strided, lambda t: t):
        out = both()
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(out, leaves), want))
    for cut in (lambda t: t[:-1] if t.dim() == 2 else t, lambda t: t[:, :-1] if t.dim() == 4 else t, lambda t: t.float(), lambda t: t.cpu()):
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, cut):
            out = both()
        with pytest.raises((ValueError, TypeError, RuntimeError)):
            torch.autograd.grad(out, leaves)
