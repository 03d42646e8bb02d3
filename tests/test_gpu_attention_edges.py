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
