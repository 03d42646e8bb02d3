"""GPU tests of causal attention over packed sequences, forward and backward, against the formulas in 64 bits (bounds: attention_bounds.py)."""
import math

import pytest
from attention_bounds import assert_within, formulas

pytestmark = pytest.mark.gpu

# lengths of the sequences, tokens in front and behind, heads, key heads, dim
CASES = [([1], 0, 0, 1, 1, 8), ([16], 0, 0, 3, 3, 64), ([5, 0, 1, 30], 0, 3, 2, 1, 64), ([33, 31, 32], 2, 0, 2, 2, 32), ([129], 0, 1, 6, 2, 128),
         ([64, 65, 63, 1, 0, 0, 127], 0, 40, 3, 1, 96), ([197, 100], 1, 1, 12, 3, 72), ([700], 0, 0, 1, 1, 40), ([300, 2, 513], 5, 0, 8, 8, 64),
         ([1100, 90], 0, 0, 8, 2, 128), ([3] * 70, 0, 2, 4, 2, 64), ([0, 0], 3, 4, 2, 2, 64), ([], 0, 9, 2, 1, 64), ([250, 60], 0, 0, 5, 1, 104),
         ([17] * 200, 7, 0, 6, 6, 24), ([1500, 640], 0, 0, 16, 8, 80), ([600], 0, 0, 40, 1, 64), ([2000, 900], 0, 100, 10, 10, 64),
         ([300, 65, 1], 1, 0, 200, 100, 128), ([129, 0, 40], 2, 3, 1100, 550, 96), ([400, 200], 0, 1, 128, 64, 104),
         ([300], 0, 0, 294, 21, 128), ([1100], 2, 0, 80, 20, 128), ([1500, 0, 730], 0, 40, 42, 7, 128), ([64], 0, 0, 512, 8, 128),
         ([700, 600], 0, 0, 110, 110, 64), ([400], 0, 1, 256, 256, 32), ([300, 200], 0, 0, 130, 130, 80), ([600, 300], 3, 0, 160, 40, 64), ([900], 0, 0, 12, 12, 96)]


def _type(torch, dtype):
    return {"bf16": torch.bfloat16, "f16": torch.float16}[dtype]


def _rand(torch, gen, dtype, *shape, std=1.0):
    return (torch.randn(*shape, device="cuda:0", generator=gen) * std).to(_type(torch, dtype))


def _operands(torch, case, dtype, seed=0, poison=True):
    """q, k, v of one projection, dout, offsets.  With `poison` NaN and infinities in the tokens of no sequence."""
    lengths, front, behind, heads, kv, dim = case
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(100 * seed + len(lengths) + dim)
    tokens = front + sum(lengths) + behind
    every = _rand(torch, gen, dtype, tokens, heads + 2 * kv, dim, std=1.3)
    dout = _rand(torch, gen, dtype, tokens, heads, dim)
    offsets = [front]
    for n in lengths:
        offsets.append(offsets[-1] + n)
    if poison:
        bad = torch.tensor([math.nan, math.inf, -math.inf], device="cuda:0").to(every.dtype)
        for t in (every, dout):
            for part in (t[:front], t[offsets[-1]:]):
                part.copy_(bad[torch.randint(0, 3, part.shape, generator=gen, device="cuda:0")])
    return every[:, :heads], every[:, heads:heads + kv], every[:, heads + kv:], dout, offsets


def _sequences(torch, q, k, v, offsets, scale, dtype, dout=None):
    """(slice, [(exact, bound)]) of each sequence"""
    for first, end in zip(offsets, offsets[1:]):
        at = slice(first, end)
        if end > first:
            ok = torch.ones(end - first, end - first, dtype=torch.bool, device="cuda:0").tril()
            yield at, formulas(torch, q[at], k[at], v[at], ok, scale, dtype, None if dout is None else dout[at])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "%s+%s+%s %sx%s %s" % (len(c[0]), sum(c[0]), c[2], c[3], c[4], c[5]))
def test_forward_and_gradients(case, dtype):
    import torch

    from paper_2505_13813_amd.transformer import causal_attention

    print(case, dtype, flush=True)
    q, k, v, dout, offsets = _operands(torch, case, dtype)
    given = torch.tensor(offsets, device="cuda:0", dtype=torch.int32 if len(offsets) % 2 else torch.int64)
    leaves = [t.detach().requires_grad_() for t in (q, k, v)]
    out = causal_attention(*leaves, given)
    got = (out.detach(),) + torch.autograd.grad(out, leaves, dout)
    assert all(t.is_contiguous() and t.dtype == q.dtype for t in got)
    with torch.no_grad():
        assert torch.equal(causal_attention(q, k, v, given), out)
    for at, wanted in _sequences(torch, q, k, v, offsets, case[-1] ** -0.5, dtype, dout):
        assert_within([t[at] for t in got], wanted, (case, at))
    for t in got:
        assert (t[:offsets[0]] == 0).all() and (t[offsets[-1]:] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", [(1, 50, 2, 2, 64), (3, 130, 6, 3, 96), (2, 1000, 12, 12, 64), (70, 1, 2, 1, 128), (2, 0, 2, 2, 64)])
def test_a_batch_of_one_length(shape, dtype):
    """[batch, tokens, heads, dim] without offsets: the bits of the packed call; and one sequence without offsets."""
    import torch

    from paper_2505_13813_amd.transformer import causal_attention

    batch, tokens, heads, kv, dim = shape
    q, k, v, dout, offsets = _operands(torch, ([tokens] * batch, 0, 0, heads, kv, dim), dtype, 1)
    found = []
    for packed in (True, False):
        leaves = [(t if packed else t.unflatten(0, (batch, tokens))).detach().requires_grad_() for t in (q, k, v)]
        up = dout if packed else dout.unflatten(0, (batch, tokens))
        out = causal_attention(*leaves, torch.tensor(offsets, device="cuda:0")) if packed else causal_attention(*leaves)
        found.append([t.reshape(-1, *t.shape[-2:]) for t in (out.detach(), *torch.autograd.grad(out, leaves, up))])
    assert all(torch.equal(a, b) for a, b in zip(*found))
    if batch == 1:
        assert torch.equal(causal_attention(q, k, v), found[0][0])


@pytest.mark.parametrize("scale", [0.02, 0.5, 3.0])
def test_scales(scale):
    import torch

    from paper_2505_13813_amd.transformer import causal_attention

    q, k, v, dout, offsets = _operands(torch, ([90, 200], 0, 0, 4, 2, 64), "bf16", 2)
    leaves = [t.detach().requires_grad_() for t in (q, k, v)]
    out = causal_attention(*leaves, torch.tensor(offsets, device="cuda:0"), scale=scale)
    got = (out.detach(),) + torch.autograd.grad(out, leaves, dout)
    for at, wanted in _sequences(torch, q, k, v, offsets, scale, "bf16", dout):
        assert_within([t[at] for t in got], wanted, scale)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", [([40], 2, 2, 64), ([300, 80], 4, 1, 128), ([1000, 60], 60, 20, 64), ([700, 300], 64, 16, 72), ([1000], 64, 64, 32),
                                   ([900], 64, 64, 96), ([900], 64, 64, 128), ([200, 30], 420, 420, 88), ([1100], 80, 20, 128),
                                   ([700, 300], 72, 8, 128)])
def test_later_tokens_have_no_influence(shape, dtype):
    """NaN and infinities in the keys and values of later tokens: the bits of the earlier ones' outputs as with ordinary numbers there, also where they share
    a tile; the tokens behind see them."""
    import torch

    from paper_2505_13813_amd.transformer import causal_attention

    lengths, heads, kv, dim = shape
    q, k, v, _, offsets = _operands(torch, (lengths, 0, 0, heads, kv, dim), dtype, 3)
    given = torch.tensor(offsets, device="cuda:0")
    want = causal_attention(q, k, v, given)
    for at in {0, 1, 17, 31, 32, 37, lengths[0] // 2, lengths[0] - 1}:
        for value in (math.nan, math.inf):
            k2, v2 = k.clone(), v.clone()
            k2[at], v2[at] = value, -value
            got = causal_attention(q, k2, v2, given)
            assert torch.equal(got[:at], want[:at]), (at, value)
            assert torch.equal(got[offsets[1]:], want[offsets[1]:]), (at, value)
            assert bool((~got[at].isfinite()).all()), (at, value)
            v2 = v.clone()
            v2[at, :, 3] = value
            got = causal_attention(q, k, v2, given)
            assert torch.equal(got[:at], want[:at]) and torch.equal(got[offsets[1]:], want[offsets[1]:]), (at, value)
            other = [c for c in range(dim) if c != 3]
            assert torch.equal(got[..., other], want[..., other]), (at, value)
            assert bool((got[at, :, 3] == value).all() if value == math.inf else got[at, :, 3].isnan().all())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_sequences_have_no_influence_on_one_another(dtype):
    """A sequence of NaN and infinities, gradients too: the others' outputs and gradients are the same bits."""
    import torch

    from paper_2505_13813_amd.transformer import causal_attention

    for lengths, heads, kv, dim in (([70, 45, 100], 4, 2, 64), ([300, 129, 1000, 5], 12, 4, 128), ([130, 60, 20], 3, 3, 40)):
        q, k, v, dout, offsets = _operands(torch, (lengths, 0, 0, heads, kv, dim), dtype, 4)
        given, found = torch.tensor(offsets, device="cuda:0"), []
        at = slice(offsets[1], offsets[2])
        for bad in (False, True):
            leaves, up = [t.clone() for t in (q, k, v)], dout.clone()
            if bad:
                for t, value in zip((*leaves, up), (math.nan, math.inf, math.nan, -math.inf)):
                    t[at] = value
            for t in leaves:
                t.requires_grad_()
            out = causal_attention(*leaves, given)
            found.append((out.detach(), *torch.autograd.grad(out, leaves, up)))
        for a, b in zip(*found):
            assert torch.equal(a[:at.start], b[:at.start]) and torch.equal(a[at.stop:], b[at.stop:])


def test_gradients_against_differences():
    """The gradient along a direction, against the outputs' difference over a step of 64 bits' formulas (float16, small tensors)."""
    import torch

    from paper_2505_13813_amd.transformer import causal_attention

    q, k, v, dout, offsets = _operands(torch, ([20, 11], 0, 0, 2, 1, 16), "f16", 5)
    leaves = [t.detach().requires_grad_() for t in (q, k, v)]
    got = torch.autograd.grad(causal_attention(*leaves, torch.tensor(offsets, device="cuda:0")), leaves, dout)

    def value(*operands):
        total = 0.0
        for first, end in zip(offsets, offsets[1:]):
            Q, K, V = (t[first:end].transpose(0, 1) for t in operands)
            K, V = K.expand(2, -1, -1), V.expand(2, -1, -1)
            S = Q @ K.transpose(-1, -2) / 4
            S = S.masked_fill(torch.ones_like(S, dtype=torch.bool).triu(1), -math.inf)
            total = total + ((S.softmax(-1) @ V).transpose(0, 1) * dout[first:end].double()).sum()
        return float(total)

    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(6)
    exact = [t.detach().double() for t in (q, k, v)]
    for i, g in enumerate(got):
        for _ in range(4):
            way = torch.randn(g.shape, generator=gen, device="cuda:0", dtype=torch.float64)
            step = 1e-5
            ends = [value(*(t + s * step * way if j == i else t for j, t in enumerate(exact))) for s in (1, -1)]
            slope = (ends[0] - ends[1]) / (2 * step)
            # each element is off by some 2^-10 of the gradients' size at most (P, S' and the result rounded); the directions' signs are random
            bound = 8 * 2.0 ** -10 * float((g.double().abs() * way.abs()).square().sum().sqrt() + g.double().abs().mean() * way.norm())
            assert abs(float((g.double() * way).sum()) - slope) <= bound, (i, slope)


def test_layouts():
    """Strided, transposed, misaligned and broadcast operands, and upstream gradients of such layouts: the bits of dense ones."""
    import torch

    from paper_2505_13813_amd.transformer import causal_attention

    for heads, kv, dim, lengths in ((4, 2, 64, [50, 70]), (6, 2, 40, [33, 100])):
        q, k, v, dout, offsets = _operands(torch, (lengths, 0, 0, heads, kv, dim), "bf16", 7)
        given = torch.tensor(offsets, device="cuda:0")
        dense = [t.contiguous() for t in (q, k, v, dout)]

        def run(q, k, v, dout):
            leaves = [t.detach().requires_grad_() for t in (q, k, v)]
            out = causal_attention(*leaves, given)
            return out.detach(), *torch.autograd.grad(out, leaves, dout)

        want = run(*dense)
        heads_first = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in dense]
        channels_first = [t.permute(2, 0, 1).contiguous().permute(1, 2, 0) for t in dense]
        off = [torch.empty(t.numel() + 4, dtype=t.dtype, device="cuda:0")[4:].view(t.shape).copy_(t) for t in dense]
        wide = [torch.zeros(t.shape[0], t.shape[1], dim + 24, dtype=t.dtype, device="cuda:0")[..., 8:8 + dim].copy_(t) for t in dense]
        for other in (heads_first, channels_first, off, wide, [q, k, v, dout]):
            assert all(torch.equal(a, b) for a, b in zip(want, run(*other)))
        one = dout[:1, :1].expand_as(dout)
        assert all(torch.equal(a, b) for a, b in zip(run(*dense[:3], one.contiguous()), run(*dense[:3], one)))
        g = torch.autograd.grad(causal_attention(*(leaves := [t.detach().requires_grad_() for t in dense[:3]]), given).sum(), leaves)
        assert all(torch.equal(a, b) for a, b in zip(g, run(*dense[:3], torch.ones_like(dense[0]))[1:]))


def test_offsets_outside_the_buffer_are_clamped():
    """Offsets past the end and below the beginning end there; falling ones leave the tokens that rising ones name as they would be."""
    import torch

    from paper_2505_13813_amd.transformer import causal_attention

    q, k, v, _, _ = _operands(torch, ([100], 0, 0, 2, 1, 64), "bf16", 8)
    for kind in (torch.int32, torch.int64):
        want = causal_attention(q, k, v, torch.tensor([0, 40, 100], device="cuda:0", dtype=kind))
        got = causal_attention(q, k, v, torch.tensor([-7, 40, 1000000007 if kind == torch.int32 else 2 ** 40 + 3, 2 ** 31 - 1], device="cuda:0", dtype=kind))
        assert torch.equal(got, want)
    falling = torch.tensor([0, 60, 20, 100], device="cuda:0")
    leaves = [t.detach().requires_grad_() for t in (q, k, v)]
    out = causal_attention(*leaves, falling)
    grads = torch.autograd.grad(out, leaves, torch.ones_like(out))
    assert out.shape == q.shape and all(g.shape == t.shape for g, t in zip(grads, leaves))


def test_far_tokens():
    """Keys and values that lie past 2^32 bytes from the first."""
    import torch

    from paper_2505_13813_amd.transformer import causal_attention

    tokens, heads, dim = 700, 2, 64
    q, k, v, dout, offsets = _operands(torch, ([300, 400], 0, 0, heads, heads, dim), "bf16", 9)
    far = torch.empty(tokens, 4 << 20, dtype=torch.bfloat16, device="cuda:0")  # 8 MiB a token
    held = [far[:, i * 1024:i * 1024 + heads * dim].unflatten(1, (heads, dim)) for i in range(4)]
    for to, t in zip(held, (q, k, v, dout)):
        to.copy_(t)
    given = torch.tensor(offsets, device="cuda:0")
    found = []
    for operands in ((q, k, v, dout), held):
        leaves = [t.detach().requires_grad_() for t in operands[:3]]
        out = causal_attention(*leaves, given)
        found.append((out.detach(), *torch.autograd.grad(out, leaves, operands[3])))
    assert all(torch.equal(a, b) for a, b in zip(*found))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_long_sequence_of_a_few_heads(dtype):
    """Long walks, cut into slabs and split over wavefronts; rows in places of the sequence against the formulas, gradients of keys too."""
    import torch

    from paper_2505_13813_amd.transformer import causal_attention

    n, heads, kv, dim = 9000, 2, 1, 64
    q, k, v, dout, _ = _operands(torch, ([n], 0, 0, heads, kv, dim), dtype, 10)
    leaves = [t.detach().requires_grad_() for t in (q, k, v)]
    out = causal_attention(*leaves)
    got = (out.detach(),) + torch.autograd.grad(out, leaves, dout)
    ok = torch.ones(n, n, dtype=torch.bool, device="cuda:0").tril()
    assert_within(got, formulas(torch, q, k, v, ok, dim ** -0.5, dtype, dout), (n, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_upstream_gradients_of_a_small_sequence(dtype):
    """A sequence whose gradients are 2^-12 of its neighbour's is as exact as alone: its scales are its own."""
    import torch

    from paper_2505_13813_amd.transformer import causal_attention

    q, k, v, dout, offsets = _operands(torch, ([130, 400], 0, 0, 4, 2, 64), dtype, 11)
    dout = torch.cat([dout[:130], (dout[130:].double() * 2.0 ** -12).to(dout.dtype)])
    leaves = [t.detach().requires_grad_() for t in (q, k, v)]
    out = causal_attention(*leaves, torch.tensor(offsets, device="cuda:0"))
    got = (out.detach(),) + torch.autograd.grad(out, leaves, dout)
    for at, wanted in _sequences(torch, q, k, v, offsets, 0.125, dtype, dout):
        assert_within([t[at] for t in got], wanted, at)


def test_refusals():
    import torch

    import paper_2505_13813_amd as grkan
    from paper_2505_13813_amd.transformer import causal_attention

    def t(*shape, dtype=torch.bfloat16):
        return torch.zeros(*shape, dtype=dtype, device="cuda:0")

    q, k = t(10, 4, 64), t(10, 2, 64)
    offsets = torch.tensor([0, 10], device="cuda:0")
    for bad in ((q, t(9, 2, 64), t(9, 2, 64)), (q, k, t(10, 1, 64)), (t(10, 3, 64), k, k), (q, t(10, 2, 32), t(10, 2, 32)), (t(10, 4, 60), t(10, 2, 60), t(10, 2, 60)),
                (t(10, 4, 136), t(10, 2, 136), t(10, 2, 136)), (t(10, 4), t(10, 4), t(10, 4)), (q[None], k[None], k[None], offsets), (q, k, k, offsets[None]),
                (q, k, k, offsets[:0]), (q, k, k, offsets.cpu()), (q, k.cpu(), k), (t(1, 10, 4, 64), t(2, 10, 4, 64), t(2, 10, 4, 64))):
        with pytest.raises(ValueError):
            causal_attention(*bad)
    for bad in ((q.float(), k.float(), k.float()), (q, k.half(), k), (q, k, k, offsets.float()), (q, k, None), (q, k, k, [0, 10])):
        with pytest.raises(TypeError):
            causal_attention(*bad)
    for scale in (0.0, -1.0, math.inf, math.nan, 1e39):
        with pytest.raises(ValueError):
            causal_attention(q, k, k, scale=scale)
    g, = torch.autograd.grad(causal_attention(w := q.clone().requires_grad_(), k, k).sum(), w, create_graph=True)
    with pytest.raises(RuntimeError, match="not differentiable twice"):
        torch.autograd.grad(g.sum(), w)
    assert isinstance(grkan.GrkanError(8, "x"), RuntimeError)
    assert causal_attention(q[:0], k[:0], k[:0]).shape == (0, 4, 64)
    assert causal_attention(q[:0], k[:0], k[:0], offsets).shape == (0, 4, 64)


def test_some_gradients_and_no_grad():
    import torch

    from paper_2505_13813_amd.transformer import causal_attention

    q, k, v, dout, offsets = _operands(torch, ([60, 200], 0, 0, 4, 2, 64), "bf16", 12)
    given = torch.tensor(offsets, device="cuda:0")
    leaves = [t.detach().requires_grad_() for t in (q, k, v)]
    want = torch.autograd.grad(causal_attention(*leaves, given), leaves, dout)
    for i in range(3):
        some = [t.detach().requires_grad_(j == i) for j, t in enumerate((q, k, v))]
        g, = torch.autograd.grad(causal_attention(*some, given), some[i], dout)
        assert torch.equal(g, want[i])
    # the same leaf in all three places
    one = q.detach().contiguous().requires_grad_()
    g, = torch.autograd.grad(causal_attention(one, one, one, given), one, dout)
    three = [q.detach().contiguous().requires_grad_() for _ in range(3)]
    each = torch.autograd.grad(causal_attention(*three, given), three, dout)
    assert torch.equal(g, (each[0] + each[1] + each[2])) or float((g.double() - sum(e.double() for e in each)).norm() / g.double().norm()) < 2.0 ** -7


def test_on_another_stream_and_in_a_graph():
    """On a stream of its own behind work there; forward and backward kernels captured and replayed with other operands, eager calls between."""
    import torch

    from paper_2505_13813_amd.transformer import causal_attention

    case = ([200, 0, 61, 333], 0, 6, 8, 2, 64)
    sets = [_operands(torch, case, "bf16", seed) for seed in (20, 21, 22)]
    given = torch.tensor(sets[0][4], device="cuda:0")

    def step(q, k, v, dout):
        leaves = [t.detach().requires_grad_() for t in (q, k, v)]
        out = causal_attention(*leaves, given)
        return (out.detach(), *torch.autograd.grad(out, leaves, dout))

    want = [step(*s[:4]) for s in sets]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        held = [torch.empty_like(t, memory_format=torch.contiguous_format) for t in sets[0][:4]]
        for to, t in zip(held, sets[1]):
            to.copy_(t)
        got = step(*held)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want[1]))
    with torch.cuda.stream(side):
        step(*held)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        result = step(*held)
    for i in (0, 2, 1, 0):
        for to, t in zip(held, sets[i]):
            to.copy_(t)
        graph.replay()
        eager = step(*sets[(i + 1) % 3][:4])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(result, want[i]))
        assert all(torch.equal(a, b) for a, b in zip(eager, want[(i + 1) % 3]))


def test_the_same_bits_every_time():
    import torch

    from paper_2505_13813_amd.transformer import causal_attention

    for case in (([1000, 500, 77], 0, 0, 12, 3, 128), ([900, 1000], 0, 0, 12, 12, 64), ([1100], 0, 0, 80, 20, 128)):
        q, k, v, dout, offsets = _operands(torch, case, "f16", 30)
        given, first = torch.tensor(offsets, device="cuda:0"), None
        for _ in range(4):
            leaves = [t.detach().requires_grad_() for t in (q, k, v)]
            out = causal_attention(*leaves, given)
            got = (out.detach(), *torch.autograd.grad(out, leaves, dout))
            first = first or got
            assert all(torch.equal(a, b) for a, b in zip(first, got))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", [([40, 3, 1, 17], 0, 0, 3, 3, 64), ([17], 0, 0, 8, 2, 96), ([38, 100, 12], 0, 2, 6, 3, 128), ([50] * 30, 0, 0, 16, 16, 64),
                                  ([50] * 30, 0, 0, 12, 12, 32), ([120] * 8, 0, 0, 64, 64, 128)])
def test_gradients_of_short_sequences_are_rounded_once(case, dtype):
    """dQ and dK as relative norms: their own rounding alone takes every element by at most u = eps / 2 of itself.  What else there is, the second
    parts' roundings (u squared) and float32 sums, is below a twentieth of that."""
    import torch

    from paper_2505_13813_amd.transformer import causal_attention

    print(case, dtype, flush=True)
    q, k, v, dout, offsets = _operands(torch, case, dtype, 7, poison=False)
    leaves = [t.detach().requires_grad_() for t in (q, k, v)]
    got = torch.autograd.grad(causal_attention(*leaves, torch.tensor(offsets, device="cuda:0")), leaves, dout)
    off, whole = [0.0, 0.0], [0.0, 0.0]
    for at, wanted in _sequences(torch, q, k, v, offsets, case[-1] ** -0.5, dtype, dout):
        for i in range(2):
            exact = wanted[1 + i][0]
            off[i] += float((got[i][at].double() - exact).square().sum())
            whole[i] += float(exact.square().sum())
    u = torch.finfo(q.dtype).eps / 2
    assert all(math.sqrt(a / b) <= 1.05 * u for a, b in zip(off, whole)), [math.sqrt(a / b) / u for a, b in zip(off, whole)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", [([200, 77], 0, 3, 6, 2, 64), ([30, 5], 0, 0, 4, 4, 128), ([300], 0, 0, 294, 21, 128)])
def test_from_c_with_and_without_the_rest(case, dtype):
    """Without what the output's rounding left the gradients are within the formulas' bounds too, and the outputs, which do not need it, have the same bits."""
    import ctypes

    import torch

    from paper_2505_13813_amd import binding

    print(case, dtype, flush=True)
    lib = binding.load_library()
    q, k, v, dout, offsets = _operands(torch, case, dtype, 8)
    heads, kv, dim = case[3:]
    given = torch.tensor(offsets, device="cuda:0", dtype=torch.int32)
    a = binding.CausalAttention(q=q.data_ptr(), k=k.data_ptr(), v=v.data_ptr(), offsets=given.data_ptr(), tokens=q.shape[0], sequences=len(case[0]), heads=heads,
                                kv_heads=kv, dim=dim, q_token_stride=q.stride(0), q_head_stride=q.stride(1), k_token_stride=k.stride(0), k_head_stride=k.stride(1),
                                v_token_stride=v.stride(0), v_head_stride=v.stride(1), scale=dim ** -0.5)
    io, stream = {"bf16": 1, "f16": 2}[dtype], torch.cuda.current_stream().cuda_stream
    need = lib.grkan_causal_attention_bwd_workspace_bytes(ctypes.byref(a))
    results = []
    for with_rest in (True, False):
        out, rest, dq = (torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda:0") for _ in range(3))
        dk, dv = (torch.full(k.shape, 7.0, dtype=q.dtype, device="cuda:0") for _ in range(2))
        lse = torch.full((lib.grkan_causal_attention_lse_count(ctypes.byref(a)),), 7.0, device="cuda:0")
        work = torch.full((need,), 255, dtype=torch.uint8, device="cuda:0")
        left = rest.data_ptr() if with_rest else None
        assert lib.grkan_causal_attention_fwd(ctypes.byref(a), out.data_ptr(), left, lse.data_ptr(), io, stream) == 0
        assert lib.grkan_causal_attention_bwd(ctypes.byref(a), out.data_ptr(), left, lse.data_ptr(), dout.data_ptr(), dout.stride(0), dout.stride(1), dq.data_ptr(),
                                              dk.data_ptr(), dv.data_ptr(), work.data_ptr(), need, io, stream) == 0
        torch.cuda.synchronize()
        for at, wanted in _sequences(torch, q, k, v, offsets, dim ** -0.5, dtype, dout):
            assert_within([t[at] for t in (out, dq, dk, dv)], wanted, (case, at, with_rest))
        assert with_rest or bool((rest == 7.0).all())
        results.append((out, lse, dv))
    assert all(torch.equal(x, y) for x, y in zip(*results))


FALLING = [[0, 60, 20, 100], [100, 0], [50, 40, 30, 700], [0] + [1000, 0] * 6 + [1000, 1100], [-5, 900, 3, 3, 1200, 0, 650, 2 ** 31 - 1], [700] * 70 + [10] * 70]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", [(2, 1, 64), (12, 12, 64), (32, 8, 128), (6, 2, 72)])
def test_falling_offsets_stay_in_the_buffers(shape, dtype):
    """What comes out is unspecified, but nothing around the outputs and the workspace is written (that nothing outside is reached: test_packed_host.py)."""
    import ctypes

    import torch

    from paper_2505_13813_amd import binding

    heads, kv, dim = shape
    lib, io, stream = binding.load_library(), {"bf16": 1, "f16": 2}[dtype], torch.cuda.current_stream().cuda_stream
    guard = 4096
    for offsets in FALLING:
        print(shape, dtype, offsets[:8], flush=True)
        tokens = min(1200, max(offsets))
        q, k, v, dout, _ = _operands(torch, ([tokens], 0, 0, heads, kv, dim), dtype, 9)
        given = torch.tensor(offsets, device="cuda:0", dtype=torch.int32)
        a = binding.CausalAttention(q=q.data_ptr(), k=k.data_ptr(), v=v.data_ptr(), offsets=given.data_ptr(), tokens=tokens, sequences=len(offsets) - 1, heads=heads,
                                    kv_heads=kv, dim=dim, q_token_stride=q.stride(0), q_head_stride=q.stride(1), k_token_stride=k.stride(0), k_head_stride=k.stride(1),
                                    v_token_stride=v.stride(0), v_head_stride=v.stride(1), scale=dim ** -0.5)
        need = lib.grkan_causal_attention_bwd_workspace_bytes(ctypes.byref(a))
        sizes = [2 * q.numel(), 2 * q.numel(), 4 * lib.grkan_causal_attention_lse_count(ctypes.byref(a)), 2 * q.numel(), 2 * k.numel(), 2 * v.numel(), need]
        held = [torch.full((guard + -(-n // 16) * 16 + guard,), 77, dtype=torch.uint8, device="cuda:0") for n in sizes]
        out, rest, lse, dq, dk, dv, work = (t.data_ptr() + guard for t in held)
        assert lib.grkan_causal_attention_fwd(ctypes.byref(a), out, rest, lse, io, stream) == 0
        assert lib.grkan_causal_attention_bwd(ctypes.byref(a), out, rest, lse, dout.data_ptr(), dout.stride(0), dout.stride(1), dq, dk, dv, work, need, io, stream) == 0
        torch.cuda.synchronize()
        for t, n in zip(held, sizes):
            assert bool((t[:guard] == 77).all()) and bool((t[guard + n:] == 77).all()), offsets
