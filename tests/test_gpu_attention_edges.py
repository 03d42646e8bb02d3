"""GPU tests of cross attention at the edges of what it takes."""
import math

import pytest
from test_gpu_attention import _assert_within, _formulas, _operands, _rand, _type

pytestmark = pytest.mark.gpu


def _off(t, elements):
    """A contiguous copy of t that starts `elements` elements behind a multiple of 256 bytes."""
    import torch

    flat = torch.empty(t.numel() + elements, dtype=t.dtype, device=t.device)
    view = flat[elements:].view(t.shape)
    view.copy_(t)
    assert view.is_contiguous() and view.data_ptr() % 16 == elements * t.element_size() % 16
    return view


@pytest.mark.parametrize("elements", [1, 4])
@pytest.mark.parametrize("which", ["q", "k", "v", "dout", "all"])
def test_contiguous_operands_off_16_bytes(which, elements):
    """Tensors that are contiguous and start 2 or 8 bytes off: the same bits, forward and backward."""
    import torch

    from paper_2505_13813_amd.transformer import cross_attention

    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(21)
    dense = {n: _rand(torch, gen, "bf16", 2, t, h, 64) for n, t, h in (("q", 37, 4), ("k", 70, 2), ("v", 70, 2), ("dout", 37, 4))}
    moved = {n: _off(t, elements) if which in (n, "all") else t for n, t in dense.items()}
    found = []
    for given in (dense, moved):
        leaves = [given[n].detach().requires_grad_() for n in "qkv"]
        out = cross_attention(*leaves)
        found.append((out.detach(), *torch.autograd.grad(out, leaves, given["dout"])))
    assert all(torch.equal(a, b) for a, b in zip(*found))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", [(3, 1, 3000, 4, 2, 64), (4, 40, 700, 2, 2, 128), (2, 900, 300, 4, 2, 128), (3, 20, 100, 2, 2, 64),
                                   (2, 300, 5000, 2, 2, 64)])
def test_no_key_in_an_entry_whatever_its_queries_hold(shape, dtype):
    """NaN and infinities in the queries and upstream gradients of an entry whose mask leaves nothing (padding): zeros there, and the
    other entries' bits as with zeros in their place."""
    import torch

    from paper_2505_13813_amd.transformer import cross_attention

    q, k, v, *_ = _operands(torch, shape, dtype, "none")
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(22)
    dout = _rand(torch, gen, dtype, *q.shape)
    mask = torch.rand(shape[0], shape[2], generator=gen, device="cuda:0") < 0.7
    mask[1] = False
    bad = torch.tensor([math.nan, math.inf, -math.inf, 1.0], device="cuda:0").to(_type(torch, dtype))
    found = []
    for poison in (False, True):
        leaves = [t.detach().clone() for t in (q, k, v)]
        up = dout.clone()
        for t in (leaves[0], up):
            t[1] = bad[torch.randint(0, 4, t[1].shape, generator=gen, device="cuda:0")] if poison else 0.0
        if poison:
            leaves[1][1], leaves[2][1] = math.nan, math.inf
        for t in leaves:
            t.requires_grad_()
        out = cross_attention(*leaves, key_mask=mask)
        found.append((out.detach(), *torch.autograd.grad(out, leaves, up)))
        assert torch.equal(out, cross_attention(*(t.detach() for t in leaves), key_mask=mask))
    for name, a, b in zip(("out", "dq", "dk", "dv"), *found):
        assert (b[1] == 0).all(), name
        assert torch.equal(a, b), name


def test_as_many_workgroups_as_a_launch_takes():
    """14,000,000 entries of one query and one key give their values; 2^24 are refused, and nothing is left behind for the next call."""
    import torch

    import paper_2505_13813_amd as grkan
    from paper_2505_13813_amd.transformer import cross_attention

    for entries, taken in ((14000000, True), (2 ** 24, False)):
        v = torch.arange(entries, device="cuda:0").remainder(251).to(torch.bfloat16)[:, None, None, None].repeat(1, 1, 1, 8)
        leaves = [t.requires_grad_() for t in (torch.ones_like(v), torch.ones_like(v), v)]
        if taken:
            out = cross_attention(*leaves)
            dq, dk, dv = torch.autograd.grad(out, leaves, v.detach())
            assert torch.equal(out, v) and torch.equal(dv, v) and (dq == 0).all() and (dk == 0).all()
        else:
            with pytest.raises(grkan.GrkanError):
                cross_attention(*leaves)
            assert float(v.detach()[:3].float().sum()) == 24.0


@pytest.mark.parametrize("shape", [(1, 60, 1500, 2, 2, 64), (2, 45, 4001, 6, 2, 128), (1, 300, 700, 1, 1, 32), (1, 33, 2000, 3, 1, 96)])
def test_float16_gradients_of_rows_of_different_sizes(shape):
    """Upstream gradients of 2^6 to 2^-8 of the same size otherwise, row by row: a query's gradient is as exact as if all were of its size
    (its own bound times its factor, and half a step of float16 below 2^-14 for the result); the keys' within their bounds."""
    import torch

    from paper_2505_13813_amd.transformer import cross_attention

    q, k, v, _, _, valid = _operands(torch, shape, "f16", "none")
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(23)
    each = _rand(torch, gen, "f16", *q.shape).clamp(-4.0, 4.0)
    by = torch.exp2((6 - torch.arange(shape[1], device="cuda:0") % 15).double())[None, :, None, None]
    dout = (each.double() * by).half()
    leaves = [t.detach().requires_grad_() for t in (q, k, v)]
    out = cross_attention(*leaves)
    dq, dk, dv = torch.autograd.grad(out, leaves, dout)
    scale = shape[-1] ** -0.5
    # (a row's largest is 1 at least, where the bound allows for 4 everywhere)
    assert each.abs().amax(-1).min() >= 1 and each.abs().max() <= 4
    exact, bound = _formulas(torch, q, k, v, valid, scale, "f16", each)[1]
    off = ((dq.double() - by * exact).abs() - by * bound - 2.0 ** -25) / by
    assert bool((off <= 0).all()), (shape, float(off.max()), off.amax((0, 2, 3))[:15].tolist())
    wanted = _formulas(torch, q, k, v, valid, scale, "f16", dout)
    _assert_within([out.detach()], wanted[:1], shape)
    _assert_within([dk, dv], wanted[2:], shape)


@pytest.mark.parametrize("shape", [(2, 40, 3, 2, 1, 128), (1, 40, 200, 1, 1, 128), (2, 200, 130, 2, 2, 64), (1, 33, 40, 3, 3, 24)])
@pytest.mark.parametrize("size", [300.0, 3000.0, 20000.0])
@pytest.mark.parametrize("masked", [False, True])
def test_float16_gradients_with_large_values(masked, size, shape):
    """Values of thousands whose channels agree in sign, and a small loss: its gradients are in float16's range, and what they are summed
    of stays in it as well.  Beside the bound: the terms' steps of 2^-24 are those of at most
    4 max |dO| max(1, 2 sqrt(dim) max |v_j| / 32768) times a number below 1."""
    import torch

    from paper_2505_13813_amd.transformer import cross_attention

    batch, queries, keys, heads, kv, dim = shape
    q, k, _, _, _, valid = _operands(torch, shape, "f16", "none")
    q = q / 4
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(24)

    def spread(*shape):
        return 0.5 + torch.rand(*shape, generator=gen, device="cuda:0")

    sign = torch.where(torch.arange(keys, device="cuda:0") % 2 == 0, 1.0, -1.0)[None, :, None, None]
    v = (size * sign * spread(batch, keys, kv, dim)).half()
    dout = (0.02 / size * spread(*q.shape)).half()
    mask = None
    if masked:  # every third key, NaN and infinities there
        mask = torch.arange(keys, device="cuda:0").remainder(3)[None].repeat(batch, 1) != 2
        valid, k, v = mask, k.clone(), v.clone()
        k[:, 2::3], v[:, 2::3] = math.nan, math.inf
    leaves = [t.detach().requires_grad_() for t in (q, k, v)]
    out = cross_attention(*leaves, key_mask=mask)
    got = (out.detach(),) + torch.autograd.grad(out, leaves, dout)
    assert all(bool(t.isfinite().all()) for t in got), [int((~t.isfinite()).sum()) for t in got]
    scale = dim ** -0.5
    wanted = _formulas(torch, q, k, v, valid, scale, "f16", dout)
    step = 2.0 ** -25 * 4 * float(dout.max()) * max(1.0, 2 * dim ** 0.5 * float(v[valid].double().norm(dim=-1).max()) / 32768) * scale
    group = heads // kv
    more = [0.0, step * torch.where(valid[..., None, None], k, 0).double().abs().sum(1, keepdim=True).repeat_interleave(group, 2),
            step * q.double().abs().sum(1, keepdim=True).unflatten(2, (kv, group)).sum(3), 0.0]
    _assert_within(got, [(exact, bound + m) for (exact, bound), m in zip(wanted, more)], (shape, size))
