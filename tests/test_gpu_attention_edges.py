"""GPU tests of cross attention at the edges of what it takes."""
import pytest
from test_gpu_attention import _rand

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
