"""GPU tests of rotary positions with several axes, against the formula in 64 bits."""
import math

import pytest

pytestmark = pytest.mark.gpu

UNIT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
FLOOR = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}
# sine and cosine of an angle reduced in 64 bits and rounded to 24: pi 2^-25 of the angle, 2^-22 of the function, and the
# products' roundings
TURN = 2.0 ** -20

# batch, tokens, heads, key heads, dim, pairs of each axis: every vector width, one token and many, parts of the channels, no pair
CASES = [(1, 1, 1, 1, 2, (1,)), (2, 5, 3, 1, 64, (16, 16)), (1, 196, 12, 12, 64, (8, 24)), (2, 33, 4, 2, 128, (16, 24, 24)),
         (3, 17, 2, 2, 80, (10, 10, 20)), (2, 9, 5, 5, 72, (12, 13)), (1, 700, 6, 3, 96, (16, 8)), (2, 40, 1, 1, 30, (7, 8)),
         (4, 3, 8, 8, 64, (0, 4)), (2, 6, 3, 3, 16, (0,)), (1, 3000, 32, 8, 128, (32, 16, 16)), (0, 4, 2, 2, 64, (16, 16)),
         (2, 0, 2, 2, 64, (16, 16)), (1, 7, 2, 1, 4096, (1024, 1024))]


def _types(torch):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _rand(torch, seed, dtype, *shape):
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(seed)
    return torch.randn(*shape, device="cuda:0", generator=gen).to(dtype)


def _exact(torch, x, positions, frequencies, axis, interleaved, sign=1.0):
    """The turned x and the magnitudes |a| + |b| of each channel's pair."""
    n = axis.numel()
    x = x.double()
    out, size = x.clone(), torch.zeros_like(x)
    p = positions if positions.dim() == 3 else positions[None]
    angle = sign * p.double()[..., axis.long()] * frequencies
    cos, sin = angle.cos()[:, :, None], angle.sin()[:, :, None]
    j = torch.arange(n, device=x.device)
    ia, ib = (2 * j, 2 * j + 1) if interleaved else (j, n + j)
    a, b = x[..., ia], x[..., ib]
    out[..., ia], out[..., ib] = a * cos - b * sin, a * sin + b * cos
    size[..., ia] = size[..., ib] = a.abs() + b.abs()
    return out, size


def _near(got, want, size, dtype):
    return ((got.double() - want).abs() <= UNIT[dtype] * want.abs() + TURN * size + FLOOR[dtype]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("case", CASES)
def test_forward_and_backward(case, interleaved, dtype):
    """Queries and keys of one projection, positions for each batch entry; both directions, the same bits again."""
    import torch

    from paper_2505_13813_amd.transformer import rotary, rotary_frequencies

    batch, tokens, heads, kv, dim, pairs = case
    t = _types(torch)[dtype]
    frequencies, axis = rotary_frequencies(pairs, device="cuda:0")
    joint = _rand(torch, 1, t, batch, tokens, heads + kv, dim)
    q, k = joint[:, :, :heads], joint[:, :, heads:]
    positions = torch.randint(-40, 300, (batch, tokens, len(pairs)), device="cuda:0")
    leaves = [v.detach().requires_grad_() for v in (q, k)]
    got = rotary(leaves[0], positions, frequencies, axis, k=leaves[1], interleaved=interleaved)
    again = rotary(q, positions, frequencies, axis, k=k, interleaved=interleaved)
    ups = [_rand(torch, 2 + i, t, *v.shape) for i, v in enumerate((q, k))]
    grads = torch.autograd.grad(got, leaves, ups)
    for i, x in enumerate((q, k)):
        assert torch.equal(got[i], again[i]) and got[i].is_contiguous()
        assert _near(got[i].detach(), *_exact(torch, x, positions, frequencies, axis, interleaved), dtype)
        assert _near(grads[i], *_exact(torch, ups[i], positions, frequencies, axis, interleaved, -1.0), dtype)
        rest = 2 * sum(pairs)
        assert torch.equal(got[i][..., rest:], x[..., rest:])


@pytest.mark.parametrize("kind", ["int32", "int64", "float32"])
def test_positions(kind):
    """Every type of position, a view of them, one set for all batch entries; positions of millions as exact as small ones."""
    import torch

    from paper_2505_13813_amd.transformer import rotary, rotary_frequencies

    frequencies, axis = rotary_frequencies((5, 3, 8), theta=500.0, shared=True, device="cuda:0")
    x = _rand(torch, 3, torch.float32, 3, 50, 4, 32)
    far = torch.randint(0, 16_000_000, (3, 50, 6), device="cuda:0").to(getattr(torch, kind))
    if kind == "float32":
        far = far / 8 + 0.125
    for positions in (far[:, :, 1:4], far[:, :, ::2], far[0, :, :3], far[:1, :, :3]):
        got = rotary(x, positions, frequencies, axis)
        assert _near(got, *_exact(torch, x, positions, frequencies, axis, False), "f32")


def test_layouts():
    """Strides of batch, token and head of their own, and a copied layout: the same bits; keys with positions and a length of their
    own."""
    import torch

    from paper_2505_13813_amd.transformer import grid_positions, rotary, rotary_frequencies

    frequencies, axis = rotary_frequencies((8, 8), device="cuda:0")
    positions = grid_positions(3, 7, device="cuda:0")
    assert positions.shape == (21, 2) and positions[8].tolist() == [1, 1]
    base = _rand(torch, 4, torch.bfloat16, 2, 4, 21, 3, 40)
    for x in (base[:, :, :, 1, :32].transpose(1, 2), base[:, :, :, 2, 1:33].transpose(1, 2), base[..., 4].permute(0, 2, 3, 1).repeat(1, 1, 1, 8)[..., ::1],
              base[:, :, :, 0, :32].permute(0, 2, 1, 3).flip(0)):
        assert torch.equal(rotary(x, positions, frequencies, axis), rotary(x.contiguous(), positions, frequencies, axis))
    odd = base[:, :, :, 1, :32].transpose(1, 2).transpose(2, 3).contiguous().transpose(2, 3)  # channels apart: copied
    assert odd.stride(-1) != 1
    assert torch.equal(rotary(odd, positions, frequencies, axis), rotary(odd.contiguous(), positions, frequencies, axis))
    q, k = base[:, 0, :, :, :32], base[:, 1, :13, :2, :32]
    where = torch.randint(0, 99, (2, 13, 2), device="cuda:0", dtype=torch.int32)
    got = rotary(q, positions, frequencies, axis, k, where)
    assert torch.equal(got[0], rotary(q, positions, frequencies, axis)) and torch.equal(got[1], rotary(k, where, frequencies, axis))


def test_rotation_keeps_what_it_should():
    """A query and a key meet by their positions' difference alone; turning back gives what was there (float32)."""
    import torch

    from paper_2505_13813_amd.transformer import RotaryAxes

    turn = RotaryAxes((16, 16)).to("cuda:0").to(torch.bfloat16)
    assert turn.frequency_bits.dtype == torch.int64
    q, k = _rand(torch, 5, torch.float32, 1, 60, 2, 64), _rand(torch, 6, torch.float32, 1, 60, 2, 64)
    p = torch.randint(0, 50, (60, 2), device="cuda:0")
    shift = torch.tensor([1000, -77], device="cuda:0")
    a, b = turn(q, p, k, p.flip(0)), turn(q, p + shift, k, p.flip(0) + shift)
    dots = [(u.double() * v.double()).sum(-1) for u, v in (a, b)]
    size = (q.norm(dim=-1) * k.norm(dim=-1)).double()
    assert ((dots[0] - dots[1]).abs() <= 4 * TURN * math.sqrt(2) * size).all()


def test_refusals():
    import torch

    import paper_2505_13813_amd as grkan
    from paper_2505_13813_amd.transformer import rotary, rotary_frequencies

    f, axis = rotary_frequencies((4, 4), device="cuda:0")
    x = _rand(torch, 7, torch.bfloat16, 2, 6, 3, 32)
    p = torch.zeros(6, 2, dtype=torch.int32, device="cuda:0")
    bad = [((x.cpu(), p, f, axis), ValueError), ((x.double(), p, f, axis), TypeError), ((x[0], p, f, axis), ValueError),
           ((x, p[:5], f, axis), ValueError), ((x, p.double(), f, axis), TypeError), ((x, p.cpu(), f, axis), ValueError),
           ((x, p, f.float(), axis), TypeError), ((x, p, f, axis.long()), TypeError), ((x, p, f[:-1], axis), ValueError),
           ((x[..., :14], p, f, axis), ValueError), ((x, p.expand(3, 6, 2), f, axis), ValueError),
           ((x, p, f, axis, x.half()), TypeError), ((x, p, f, axis, x[..., :30]), ValueError), ((x, p, f, axis, None, p), ValueError),
           ((x, p, f, axis, x[:, :5]), ValueError)]
    for args, error in bad:
        with pytest.raises(error):
            rotary(*args)
    with pytest.raises(grkan.GrkanError):
        rotary(x[..., :31], p, f, axis)
    with pytest.raises(ValueError):
        rotary_frequencies(())
    y = rotary(x.requires_grad_(), p, f, axis)
    g, = torch.autograd.grad(y, x, torch.ones_like(y).requires_grad_(), create_graph=True)
    with pytest.raises(RuntimeError, match="not differentiable twice"):
        g.sum().backward()


def test_axis_out_of_range_reads_the_last_one():
    """Entries of `axis` past the positions' axes read the last axis, never what lies behind."""
    import torch

    from paper_2505_13813_amd.transformer import rotary, rotary_frequencies

    f, _ = rotary_frequencies((8,), device="cuda:0")
    x = _rand(torch, 8, torch.float32, 1, 5, 1, 16)
    p = torch.randint(0, 9, (5, 2), device="cuda:0")
    far = torch.tensor([0, 1, 2, 7, -1, 1, 100000, 0], dtype=torch.int32, device="cuda:0")
    assert torch.equal(rotary(x, p, f, far), rotary(x, p, f, far.clamp(0, 1)))


def test_tokens_past_32_bits():
    """Tokens 0.5 GB apart, and a contiguous tensor of 4.6 GB: as the same tokens dense, or alone."""
    import torch

    from paper_2505_13813_amd.transformer import rotary, rotary_frequencies

    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(13)
    f, axis = rotary_frequencies((32,), device="cuda:0")
    far = torch.empty(10 * 2 ** 28 + 128, dtype=torch.bfloat16, device="cuda:0").as_strided((1, 10, 2, 64), (0, 2 ** 28, 64, 1))
    far.copy_(torch.randn(1, 10, 2, 64, device="cuda:0", generator=gen))
    at = torch.arange(10, device="cuda:0")[:, None] * 100003
    assert torch.equal(rotary(far, at, f, axis), rotary(far.contiguous(), at, f, axis))
    del far
    tokens = 280000
    x = torch.empty(1, tokens, 128, 64, dtype=torch.bfloat16, device="cuda:0").normal_(generator=gen)
    assert x.numel() * 2 > 2 ** 32
    at = torch.arange(tokens, device="cuda:0", dtype=torch.int32)[:, None]
    assert torch.equal(rotary(x, at, f, axis)[:, -5:], rotary(x[:, -5:], at[-5:], f, axis))
