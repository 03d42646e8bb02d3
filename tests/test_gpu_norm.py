"""GPU tests of the root-mean-square norm with the residual's addition: forward, to 8 bits, backward, against the formulas in
64 bits."""
import pytest

pytestmark = pytest.mark.gpu

UNIT = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}  # one rounding, relative
FLOOR = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}              # of the smallest numbers
# float32 sums of a row: at most 32 elements a lane one after the other, six levels over a wavefront, sixteen wavefronts; a few
# operations an element around them
SUM = 64 * 2.0 ** -24
EPS = 1e-6

# rows, D: less than a vector, one vector, odd lengths, both sides of every number of wavefronts, more rows than workgroups
SIZES = [(1, 1), (3, 5), (7, 8), (1, 13), (5, 64), (9, 197), (4, 512), (4, 516), (6, 768), (5, 1023), (3, 1111), (3, 2048), (2, 2056),
         (2, 4095), (3, 4096), (2, 5000), (2, 8192), (2, 8197), (1, 16384), (2, 16383), (9001, 192), (4500, 1111), (600, 9000), (0, 64)]


def _types(torch):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _rand(torch, rows, D, dtype, seed, std=1.0):
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(seed)
    return (torch.randn(rows, D, device="cuda:0", generator=gen) * std).to(_types(torch)[dtype])


def _operands(torch, rows, D, dtype, weight32=False, residual=True):
    x, r = _rand(torch, rows, D, dtype, 1), _rand(torch, rows, D, dtype, 2, 2.0)
    w = (1 + 0.3 * _rand(torch, 1, D, "f32", 3)[0]).to(torch.float32 if weight32 else x.dtype)
    return x, r if residual else None, w


def _exact(h, w):
    h, w = h.double(), w.double()
    s = 1 / (h.square().mean(-1, keepdim=True) + EPS).sqrt()
    return h, w, s


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,D", SIZES)
def test_forward_and_backward(rows, D, dtype):
    """h to the bit; y, dx, dweight element by element within the roundings of their sums; the same bits again."""
    import torch

    from paper_2505_13813_amd.transformer import rms_norm

    for residual, weight32 in ((True, False), (False, dtype != "f32")):
        x, r, w = _operands(torch, rows, D, dtype, weight32, residual)
        dy, dh = _rand(torch, rows, D, dtype, 4, 0.5), _rand(torch, rows, D, dtype, 5)
        leaves = [t.requires_grad_() for t in (x, r, w) if t is not None]

        def both():
            out = rms_norm(x, w, r, EPS)
            grads = torch.autograd.grad(out, leaves, (dy, dh) if residual else dy)
            return (out if residual else (out,)) + grads

        got = both()
        assert all(torch.equal(a, b) for a, b in zip(got, both()))
        with torch.no_grad():
            h = (x.float() + r.float()).to(x.dtype) if residual else x
            if residual:
                assert torch.equal(got[1], h)
                assert torch.equal(got[2], got[3])
            f, wd, s = _exact(h, w)
            y = f * s * wd
            u, floor = UNIT[dtype], FLOOR[dtype]
            assert ((got[0].double() - y).abs() <= (u + SUM) * y.abs() + floor).all()
            n, g = f * s, dy.double() * wd
            along = (g * n).mean(-1, keepdim=True)
            dx = s * (g - n * along) + (dh.double() if residual else 0)
            terms = s * (g.abs() + n.abs() * (g * n).abs().mean(-1, keepdim=True))
            assert ((got[-2].double() - dx).abs() <= u * dx.abs() + 2 * SUM * terms + floor).all()
            # rows / 4096 in a lane at most, four wavefronts, 16 rows of sums a lane, 64 slices
            dw = (dy.double() * n).sum(0)
            assert got[-1].dtype == w.dtype
            uw = 2.0 ** -24 if weight32 else u
            assert ((got[-1].double() - dw).abs() <= uw * dw.abs() + 2 * SUM * (dy.double() * n).abs().sum(0) * 2 + floor).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,D", SIZES)
def test_to_8_bits(rows, D, dtype):
    """scale is the largest magnitude / 448; what each byte stands for is within half a step of y."""
    import torch

    from paper_2505_13813_amd.transformer import rms_norm_8bit

    for residual in (True, False):
        x, r, w = _operands(torch, rows, D, dtype, False, residual)
        out = rms_norm_8bit(x, w, r, EPS)
        q, scale = out[:2]
        assert q.dtype == torch.float8_e4m3fn and q.shape == x.shape and scale.shape == x.shape[:-1] and scale.dtype == torch.float32
        h = (x.float() + r.float()).to(x.dtype) if residual else x
        if residual:
            assert torch.equal(out[2], h)
        f, wd, s = _exact(h, w)
        y = f * s * wd
        if not rows:
            continue
        most = y.abs().amax(-1)
        assert ((scale.double() - most / 448).abs() <= (SUM + 2.0 ** -22) * most / 448).all()
        # three bits behind the leading one: half a step is 2^-4 relative, and 2^-10 of the scale for the smallest
        off = (q.double() * scale.double()[:, None] - y).abs()
        assert (off <= (2.0 ** -4 + 2 * SUM) * y.abs() + 2.0 ** -10 * scale.double()[:, None] * (1 + 2 * SUM)).all()


def test_8_bits_of_special_rows():
    """A row of zeros has scale 0 and zeros; NaN and infinities give the row NaN as its scale and leave the others alone;
    the smallest rows keep their values."""
    import torch

    from paper_2505_13813_amd.transformer import rms_norm, rms_norm_8bit

    x = _rand(torch, 6, 300, "f32", 7)
    x[1] = 0
    x[2, 17] = float("nan")
    x[3, 299] = float("inf")
    x[4] *= 1e-30
    w = torch.full((300,), 1e-12, device="cuda:0")
    q, scale = rms_norm_8bit(x, w, eps=1e-6)
    assert scale[1] == 0 and (q[1].float() == 0).all()
    assert torch.isnan(scale[2]) and torch.isnan(scale[3])
    for row in (0, 4, 5):
        y = rms_norm(x, w, eps=1e-6)[row].double()
        found = q[row].double() * scale[row].double()
        assert scale[row] > 0 and ((found - y).abs() <= 2.0 ** -4 * y.abs() + 2.0 ** -9 * scale[row].double()).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D", [5, 768, 5000])
def test_8_bits_of_zeros_without_eps(D, dtype):
    """With eps 0, too, a row of zeros has scale 0 and zeros; the others as with an eps that does not matter (float32 sums of a row, and one
    rounding)."""
    import torch

    from paper_2505_13813_amd.transformer import rms_norm_8bit

    x, _, w = _operands(torch, 6, D, dtype)
    x[::2] = 0.0
    q, scale = rms_norm_8bit(x, w, eps=0.0)
    assert (scale[::2] == 0).all() and (q[::2].float() == 0).all()
    h, w64 = x[1::2].double(), w.double()
    y = h / h.square().mean(-1, keepdim=True).sqrt() * w64
    exact = y.abs().amax(-1) / 448
    assert ((scale[1::2].double() - exact).abs() <= (SUM + 2.0 ** -22) * exact).all()
    assert torch.equal(q[1::2].float(), rms_norm_8bit(x, w, eps=1e-30)[0][1::2].float())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_alignment(dtype):
    """Rows apart, rows off 16-byte boundaries, and layouts that are copied: the same bits as from contiguous tensors."""
    import torch

    from paper_2505_13813_amd.transformer import rms_norm

    D = 200
    base = _rand(torch, 2 * 11, 3 * D + 1, dtype, 8).reshape(2, 11, 3 * D + 1)
    res = _rand(torch, 2 * 12, D + 3, dtype, 9).reshape(2, 12, D + 3)
    w = 1 + 0.1 * _rand(torch, 1, D, "f32", 10)[0]
    views = [(base[:, :, 1:D + 1], res[:, 1:, 2:D + 2]), (base[:, :, D:2 * D], res[:, :11, :D]), (base[:, 2:5, :D], res[:, 3:6, 1:D + 1]),
             (base[:1, :, :D].expand(2, 11, D), res[:, :11, 3:D + 3])]
    views.append((base[0, :, :D].t().contiguous().t(), res[0, :11, :D]))
    for x, r in views:
        dy = _rand(torch, x.numel() // D, D, dtype, 11).reshape(x.shape)
        leaves = [t.detach().requires_grad_() for t in (x, r, w)]
        dense = [t.detach().contiguous().requires_grad_() for t in (x, r, w)]
        out, want = rms_norm(leaves[0], leaves[2], leaves[1]), rms_norm(dense[0], dense[2], dense[1])
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        strided = torch.stack((dy, dy), -2)[..., 1, :]  # an upstream gradient with rows apart
        a = torch.autograd.grad(out[0], leaves, strided)
        b = torch.autograd.grad(want[0], dense, dy)
        assert all(torch.equal(s, t) for s, t in zip(a, b))


def test_gradient_against_differences():
    """The gradients along a direction, against a central difference of the formula in 64 bits (truncation of the difference and
    the float32 sums: 1e-4 of the terms)."""
    import torch

    from paper_2505_13813_amd.transformer import rms_norm

    x, r, w = _operands(torch, 6, 300, "f32")
    dy, dh = _rand(torch, 6, 300, "f32", 12), _rand(torch, 6, 300, "f32", 13)
    to = [_rand(torch, *(t.shape if t.dim() == 2 else (1, 300)), "f32", 14 + i).reshape(t.shape) for i, t in enumerate((x, r, w))]
    leaves = [t.requires_grad_() for t in (x, r, w)]
    grads = torch.autograd.grad(rms_norm(x, w, r, EPS), leaves, (dy, dh))
    got = sum((g.double() * t.double()).sum() for g, t in zip(grads, to))
    size = sum((g.double() * t.double()).abs().sum() for g, t in zip(grads, to))

    def loss(step):
        a, b, c = (t.detach().double() + step * d.double() for t, d in zip((x, r, w), to))
        h = a + b
        y = h / (h.square().mean(-1, keepdim=True) + EPS).sqrt() * c
        return (y * dy.double()).sum() + (h * dh.double()).sum()

    want = (loss(1e-5) - loss(-1e-5)) / 2e-5
    assert (got - want).abs() <= 1e-4 * size


def test_parts_of_the_gradient():
    """Only y used, only h used, and only some operands recorded."""
    import torch

    from paper_2505_13813_amd.transformer import rms_norm

    x, r, w = _operands(torch, 5, 96, "f32")
    dy = _rand(torch, 5, 96, "f32", 20)
    for t in (x, r, w):
        t.requires_grad_()
    y, h = rms_norm(x, w, r)
    both = torch.autograd.grad((y, h), (x, w), (dy, torch.zeros_like(dy)), retain_graph=True)
    only_y = torch.autograd.grad(y, (x, w), dy, retain_graph=True)
    assert torch.equal(both[1], only_y[1]) and torch.allclose(both[0], only_y[0], rtol=0, atol=0)
    only_h = torch.autograd.grad(h, (x, r), dy, retain_graph=True)
    assert torch.equal(only_h[0], dy) and torch.equal(only_h[1], dy)
    assert torch.autograd.grad(h, w, dy, allow_unused=True)[0] is None
    y2 = rms_norm(x.detach(), w, None)
    assert torch.autograd.grad(y2, w, dy)[0].shape == w.shape
    with torch.no_grad():
        assert not rms_norm(x, w, r)[0].requires_grad
    y, h = rms_norm(x, w, r)
    gx, = torch.autograd.grad(y, x, dy, create_graph=True)
    with pytest.raises(RuntimeError, match="not differentiable twice"):
        gx.sum().backward()


def test_refusals():
    import torch

    import paper_2505_13813_amd as grkan
    from paper_2505_13813_amd.transformer import rms_norm, rms_norm_8bit

    x, r, w = _operands(torch, 5, 96, "bf16")
    bad = [((x.cpu(), w), ValueError), ((x, w.cpu()), ValueError), ((x, w[:-1]), ValueError), ((x, w.half()), TypeError),
           ((x.double(), w.double()), TypeError), ((x, w, r[:-1]), ValueError), ((x, w, r.float()), TypeError),
           ((x, w, None, -1.0), ValueError), ((x, w, None, float("nan")), ValueError), ((x[:, :0], w[:0]), ValueError)]
    for args, error in bad:
        with pytest.raises(error):
            rms_norm(*args)
        with pytest.raises(error):
            rms_norm_8bit(*args)
    wide = torch.zeros(1, 16385, device="cuda:0")
    with pytest.raises(grkan.GrkanError):
        rms_norm(wide, wide[0])
    with pytest.raises(RuntimeError, match="no gradient"):
        rms_norm_8bit(x, w.requires_grad_())
    with pytest.raises(NotImplementedError):
        torch.func.vmap(lambda t: rms_norm(t, w.detach()))(x)


def test_on_another_stream_and_in_a_graph():
    """On a stream of its own behind work there; captured, and replayed three times with eager calls between."""
    import torch

    from paper_2505_13813_amd.transformer import rms_norm

    x, r, w = _operands(torch, 3000, 768, "bf16")
    want = rms_norm(x, w, r)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        late = x * 1.0
        got = rms_norm(late, w, r)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    held = x.clone()
    with torch.cuda.graph(graph):
        out = rms_norm(held, w, r)
    for k in range(3):
        held.copy_(x * (k + 1))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, rms_norm(x * (k + 1), w, r)))


def test_rows_past_32_bits():
    """Rows 0.5 GB apart, 5 GB in all, and a contiguous tensor of 4.6 GB: as the same rows dense, or alone."""
    import torch

    from paper_2505_13813_amd.transformer import rms_norm

    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(12)
    w = torch.rand(1000, device="cuda:0", generator=gen).bfloat16()
    far = torch.empty(10 * (2 ** 28 + 3), dtype=torch.bfloat16, device="cuda:0").as_strided((10, 1000), (2 ** 28 + 3, 1))
    far.copy_(torch.randn(10, 1000, device="cuda:0", generator=gen))
    near = far.contiguous()
    dy = torch.randn(10, 1000, device="cuda:0", generator=gen).bfloat16()
    found = []
    for x in (far, near):
        x = x.detach().requires_grad_()
        y = rms_norm(x, w)
        found.append((y, *torch.autograd.grad(y, x, dy)))
    assert all(torch.equal(a, b) for a, b in zip(*found))
    del far
    rows, dim = 1150000, 2000
    assert rows * dim * 2 > 2 ** 32
    x = torch.empty(rows, dim, dtype=torch.bfloat16, device="cuda:0").normal_(generator=gen)
    w = torch.rand(dim, device="cuda:0", generator=gen)
    x.requires_grad_()
    y = rms_norm(x, w)
    dx, = torch.autograd.grad(y, x, x.detach())
    end = x.detach()[-9:].clone().requires_grad_()
    alone = rms_norm(end, w)
    assert torch.equal(y[-9:], alone) and torch.equal(dx[-9:], torch.autograd.grad(alone, end, end.detach())[0])
