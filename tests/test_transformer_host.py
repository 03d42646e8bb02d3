"""Norm, rotary positions and cross attention without a GPU: the C interface's structures, sizes and refusals (each before anything is
launched), the helpers that make frequencies and positions, and the refusal of tensors on the CPU."""
import ctypes
import math
import re
from pathlib import Path

import pytest

from paper_2505_13813_amd import binding

ROOT = Path(__file__).resolve().parent.parent
OK, NULL, SHAPE, ALIGN, WORKSPACE, DTYPE, UNSUPPORTED = 0, 1, 2, 4, 5, 6, 8
F32, BF16, F16 = binding.GRKAN_F32, binding.GRKAN_BF16, binding.GRKAN_F16


@pytest.fixture(scope="module")
def lib():
    return binding.load_library()


@pytest.mark.parametrize("name,struct", [("grkan_rotary_t", binding.RotaryOperand), ("grkan_attention_t", binding.Attention)])
def test_structures_match_the_header(name, struct):
    text = re.sub(r"/\*.*?\*/", "", (ROOT / "include" / "grkan_transformer.h").read_text(), flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\} %s;" % name, text).group(1)
    kinds = {"void": ctypes.c_void_p, "int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float,
             "grkan_positions_t": ctypes.c_int}
    fields = []
    for line in body.split(";"):
        if line.strip():
            kind, names = re.match(r"\s*(?:const )?(\w+)\s+(.*)", line, flags=re.S).groups()
            fields += [(n.strip(" *\n"), kinds[kind]) for n in names.split(",")]
    assert fields == list(struct._fields_)


def test_header_is_plain_c(tmp_path):
    import shutil
    import subprocess

    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    src = tmp_path / "use.c"
    src.write_text(
        '#include "grkan_transformer.h"\n'
        "int use(void *p, float *f, const double *d, const int32_t *i, void *s) {\n"
        "  grkan_rotary_t r = {0}; grkan_attention_t a = {0};\n"
        "  grkan_status_t st = grkan_rms_norm_fwd(p, p, p, p, p, f, 1, 8, 8, 8, 1e-6f, GRKAN_BF16, GRKAN_F32, s);\n"
        "  st = grkan_rms_norm_bwd(p, p, p, p, p, p, p, grkan_rms_norm_bwd_workspace_bytes(1, 8, GRKAN_BF16), 1, 8, 8, 8, 8, 1e-6f, GRKAN_BF16,\n"
        "                          GRKAN_F32, s);\n"
        "  r.positions_dtype = GRKAN_POSITIONS_F32;\n"
        "  st = grkan_rotary(&r, 1, d, i, 4, 1, 8, 0, 0, GRKAN_F16, s);\n"
        "  st = grkan_attention_fwd(&a, p, f, p, grkan_attention_workspace_bytes(&a, 0), GRKAN_BF16, s);\n"
        "  st = grkan_attention_bwd(&a, p, f, p, 8, 8, 8, p, p, p, p, grkan_attention_workspace_bytes(&a, 1), GRKAN_BF16, s);\n"
        "  return (int)st + (int)grkan_attention_lse_count(&a);\n"
        "}\n")
    res = subprocess.run([gcc, "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-fsyntax-only", "-I", str(ROOT / "include"), str(src)],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr


def test_norm_refusals(lib):
    def fwd(x=16, r=None, w=16, h=None, y=16, scale=None, rows=4, D=64, eps=1e-6, io=BF16, wt=BF16):
        return lib.grkan_rms_norm_fwd(x, r, w, h, y, scale, rows, D, D, D, eps, io, wt, None)

    assert fwd(x=None) == NULL and fwd(y=None) == NULL and fwd(w=None) == NULL and fwd(r=16) == NULL
    assert fwd(x=17) == ALIGN and fwd(y=17) == ALIGN and fwd(w=17) == ALIGN and fwd(r=16, h=17) == ALIGN and fwd(scale=18) == ALIGN
    assert fwd(io=F32, wt=F32, x=18) == ALIGN and fwd(wt=F32, w=18) == ALIGN
    assert fwd(rows=-1) == SHAPE and fwd(D=0) == SHAPE
    assert fwd(D=16385) == UNSUPPORTED
    assert fwd(io=9) == DTYPE and fwd(wt=F16) == DTYPE and fwd(io=F32, wt=BF16) == DTYPE
    assert fwd(rows=0, x=None, y=None) == OK

    def bwd(h=16, dy=16, dh=None, w=16, dx=16, dw=16, ws=16, size=1 << 30, rows=4, D=64, io=BF16, wt=BF16):
        return lib.grkan_rms_norm_bwd(h, dy, dh, w, dx, dw, ws, size, rows, D, D, D, D, 1e-6, io, wt, None)

    assert bwd(h=None) == NULL and bwd(dy=None) == NULL and bwd(dx=None) == NULL and bwd(dw=None) == NULL and bwd(w=None) == NULL
    assert bwd(h=17) == ALIGN and bwd(dh=17) == ALIGN and bwd(dw=17) == ALIGN
    need = lib.grkan_rms_norm_bwd_workspace_bytes(4, 64, BF16)
    assert need > 0 and bwd(size=need - 1) == WORKSPACE and bwd(ws=None) == WORKSPACE and bwd(ws=24) == WORKSPACE
    assert bwd(D=16385) == UNSUPPORTED and bwd(io=7) == DTYPE and bwd(rows=-1) == SHAPE
    assert lib.grkan_rms_norm_bwd_workspace_bytes(4, 16385, BF16) == 0 and lib.grkan_rms_norm_bwd_workspace_bytes(-1, 64, BF16) == 0


def test_rotary_refusals(lib):
    def call(count=1, frequencies=16, axis=16, pairs=16, axes=2, dim=64, io=BF16, none=False, **fields):
        given = dict(x=16, out=16, positions=16, batch=2, tokens=3, heads=2, batch_stride=384, token_stride=128, head_stride=64,
                     position_batch_stride=6, position_token_stride=2, positions_dtype=0)
        given.update(fields)
        operands = (binding.RotaryOperand * 2)(binding.RotaryOperand(**given), binding.RotaryOperand(**given))
        return lib.grkan_rotary(None if none else operands, count, frequencies, axis, pairs, axes, dim, 0, 0, io, None)

    assert call(none=True) == NULL and call(x=None) == NULL and call(out=None) == NULL and call(positions=None) == NULL
    assert call(frequencies=None) == NULL and call(axis=None) == NULL
    assert call(count=0) == SHAPE and call(count=3) == SHAPE and call(pairs=33) == SHAPE and call(pairs=-1) == SHAPE and call(axes=0) == SHAPE
    assert call(batch=-1) == SHAPE and call(tokens=-1) == SHAPE and call(heads=0) == SHAPE and call(dim=0, pairs=0) == SHAPE
    assert call(io=5) == DTYPE and call(positions_dtype=3) == DTYPE
    assert call(dim=65) == UNSUPPORTED and call(dim=4098) == UNSUPPORTED and call(heads=65537) == UNSUPPORTED
    assert call(batch=1 << 31) == UNSUPPORTED and call(batch=1 << 30, tokens=1 << 10, heads=8) == UNSUPPORTED
    assert call(x=17) == ALIGN and call(out=17) == ALIGN and call(frequencies=20) == ALIGN and call(axis=18) == ALIGN
    assert call(positions=20, positions_dtype=1) == ALIGN and call(positions=18) == ALIGN and call(x=18, io=F32) == ALIGN
    assert call(batch=0) == OK and call(tokens=0, x=None, out=None, positions=None) == OK


def _attention(**fields):
    given = dict(q=16, k=16, v=16, batch=2, queries=5, keys=7, heads=4, kv_heads=2, dim=64, q_batch_stride=1280, q_token_stride=256,
                 q_head_stride=64, k_batch_stride=896, k_token_stride=128, k_head_stride=64, v_batch_stride=896, v_token_stride=128,
                 v_head_stride=64, scale=0.125)
    given.update(fields)
    return binding.Attention(**given)


BAD_ATTENTION = [({"q": None}, NULL), ({"k": None}, NULL), ({"v": None}, NULL), ({"batch": -1}, SHAPE), ({"queries": -1}, SHAPE),
                 ({"keys": -1}, SHAPE), ({"heads": 0}, SHAPE), ({"kv_heads": 0}, SHAPE), ({"heads": 5}, SHAPE), ({"dim": 0}, SHAPE),
                 ({"dim": 60}, UNSUPPORTED), ({"dim": 136}, UNSUPPORTED), ({"scale": 0.0}, UNSUPPORTED), ({"scale": -1.0}, UNSUPPORTED),
                 ({"scale": math.inf}, UNSUPPORTED), ({"scale": math.nan}, UNSUPPORTED), ({"keys": 1 << 31}, UNSUPPORTED),
                 ({"queries": 1 << 31}, UNSUPPORTED), ({"queries": 1 << 30, "heads": 8}, UNSUPPORTED), ({"k_token_stride": -128}, UNSUPPORTED),
                 ({"v_token_stride": 1 << 25}, UNSUPPORTED), ({"q": 24}, ALIGN), ({"k": 24}, ALIGN), ({"v": 24}, ALIGN),
                 ({"q_token_stride": 257}, ALIGN), ({"k_head_stride": 60}, ALIGN), ({"v_batch_stride": 4}, ALIGN),
                 ({"key_lengths": 18}, ALIGN), ({"key_lengths": 20, "key_lengths_64": 1}, ALIGN)]


@pytest.mark.parametrize("fields,status", BAD_ATTENTION)
def test_attention_refusals(lib, fields, status):
    a = _attention(**fields)
    assert lib.grkan_attention_fwd(ctypes.byref(a), 16, None, 16, 1 << 40, BF16, None) == status
    assert lib.grkan_attention_bwd(ctypes.byref(a), 16, 16, 16, 1280, 256, 64, 16, 16, 16, 16, 1 << 40, BF16, None) == status
    assert lib.grkan_attention_workspace_bytes(ctypes.byref(a), 0) == 0 and lib.grkan_attention_workspace_bytes(ctypes.byref(a), 1) == 0


def test_attention_refusals_of_outputs(lib):
    a = _attention()
    assert lib.grkan_attention_fwd(None, 16, None, 16, 0, BF16, None) == NULL
    assert lib.grkan_attention_fwd(ctypes.byref(a), None, None, 16, 0, BF16, None) == NULL
    assert lib.grkan_attention_fwd(ctypes.byref(a), 24, None, 16, 0, BF16, None) == ALIGN
    assert lib.grkan_attention_fwd(ctypes.byref(a), 16, 18, 16, 0, BF16, None) == ALIGN
    for io in (F32, 9):
        assert lib.grkan_attention_fwd(ctypes.byref(a), 16, None, 16, 0, io, None) == DTYPE
    need = lib.grkan_attention_workspace_bytes(ctypes.byref(a), 1)

    def bwd(out=16, lse=16, dout=16, strides=(1280, 256, 64), dq=16, dk=16, dv=16, ws=16, size=need):
        return lib.grkan_attention_bwd(ctypes.byref(a), out, lse, dout, *strides, dq, dk, dv, ws, size, BF16, None)

    for name in ("out", "lse", "dout", "dq", "dk", "dv"):
        assert bwd(**{name: None}) == NULL, name
        assert bwd(**{name: 18}) == ALIGN, name
    assert bwd(strides=(1280, 257, 64)) == ALIGN
    assert need > 0 and bwd(size=need - 1) == WORKSPACE and bwd(ws=None) == WORKSPACE and bwd(ws=24) == WORKSPACE
    long = _attention(queries=1, keys=8000, k_batch_stride=8000 * 128, v_batch_stride=8000 * 128)
    need = lib.grkan_attention_workspace_bytes(ctypes.byref(long), 0)
    assert need > 0 and lib.grkan_attention_fwd(ctypes.byref(long), 16, None, 16, need - 1, BF16, None) == WORKSPACE
    assert lib.grkan_attention_fwd(ctypes.byref(_attention(queries=0, q=None)), None, None, None, 0, BF16, None) == OK
    assert lib.grkan_attention_lse_count(ctypes.byref(a)) == 2 * 5 * 4


def test_frequencies():
    import torch

    from paper_2505_13813_amd.transformer import rotary_frequencies

    f, axis = rotary_frequencies((3, 0, 2), theta=100.0)
    assert f.dtype == torch.float64 and axis.dtype == torch.int32 and axis.tolist() == [0, 0, 0, 2, 2]
    assert f.tolist() == pytest.approx([1.0, 100.0 ** (-1 / 3), 100.0 ** (-2 / 3), 1.0, 0.1], rel=1e-15)
    f, axis = rotary_frequencies((3, 2), theta=32.0, shared=True)
    assert f.tolist() == pytest.approx([32.0 ** (-j / 5) for j in range(5)], rel=1e-15) and axis.tolist() == [0, 0, 0, 1, 1]
    assert rotary_frequencies((0,))[0].numel() == 0
    for bad in ((), (-1, 3)):
        with pytest.raises(ValueError):
            rotary_frequencies(bad)
    with pytest.raises(ValueError):
        rotary_frequencies((4,), theta=0.0)


def test_grids():
    import torch

    from paper_2505_13813_amd.transformer import grid_positions

    assert grid_positions(4).tolist() == [[0], [1], [2], [3]]
    assert grid_positions(2, 3).tolist() == [[i, j] for i in range(2) for j in range(3)]
    g = grid_positions(3, 2, 5)
    assert g.shape == (30, 3) and g.dtype == torch.int32 and g[-1].tolist() == [2, 1, 4]


def test_tensors_on_the_cpu_are_refused():
    import torch

    from paper_2505_13813_amd import transformer as T

    x, w = torch.zeros(4, 64), torch.ones(64)
    with pytest.raises(ValueError, match="GPU"):
        T.rms_norm(x, w)
    with pytest.raises(ValueError, match="GPU"):
        T.rms_norm_8bit(x, w)
    q = torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="GPU"):
        T.rotary(q, T.grid_positions(4), *T.rotary_frequencies((8,)))
    with pytest.raises(ValueError, match="GPU"):
        T.cross_attention(q, q, q)


def test_the_modules_keep_their_frequencies():
    """float64 through conversions of the module, out of the state's dictionary."""
    import torch

    from paper_2505_13813_amd.transformer import KATCrossBlock, RotaryAxes, rotary_frequencies

    m = RotaryAxes((8, 8))
    for to in (m.half(), m.bfloat16(), m.double(), m.float()):
        assert torch.equal(to.frequency_bits.view(torch.float64), rotary_frequencies((8, 8))[0])
    assert not m.state_dict()
    for bad in (dict(heads=5), dict(heads=6, kv_heads=4)):
        with pytest.raises(ValueError):
            KATCrossBlock(192, **bad)


def test_attention_workspaces_of_every_small_size(lib):
    """The plan is made for every combination of few and many queries, keys, heads and channels; what is asked for can be had."""
    for queries in (0, 1, 5, 32, 33, 129, 4096):
        for keys in (0, 1, 64, 129, 300, 700, 1000, 9000, 100000):
            for batch, kv_heads in ((1, 1), (1, 12), (30, 10), (300, 8)):
                for dim in (8, 64, 128):
                    for lengths in (None, 16):
                        a = _attention(batch=batch, queries=queries, keys=keys, heads=kv_heads, kv_heads=kv_heads, dim=dim, key_lengths=lengths)
                        assert lib.grkan_attention_workspace_bytes(ctypes.byref(a), 0) < 1 << 30
                        need = lib.grkan_attention_workspace_bytes(ctypes.byref(a), 1)
                        assert need < (1 << 30) + 16 * batch * queries * kv_heads


def test_more_workgroups_than_a_launch_takes(lib):
    """A launch has less than 2^32 threads: sizes that need more are refused as unsupported, not left to the launch."""
    many = 1 << 24
    for queries in (1, 200):
        a = _attention(batch=many, queries=queries, heads=1, kv_heads=1)
        assert lib.grkan_attention_fwd(ctypes.byref(a), 16, None, 16, 1 << 60, BF16, None) == UNSUPPORTED
        for io in (BF16, F16):
            assert lib.grkan_attention_bwd(ctypes.byref(a), 16, 16, 16, 64, 64, 64, 16, 16, 16, 16, 1 << 60, io, None) == UNSUPPORTED
    # 12 x 40 items of two channels to a token, a token to a workgroup
    t = binding.RotaryOperand(x=16, out=16, positions=16, batch=1, tokens=many, heads=12, batch_stride=0, token_stride=960, head_stride=80,
                              position_batch_stride=0, position_token_stride=1, positions_dtype=0)
    assert lib.grkan_rotary(ctypes.byref(t), 1, 16, 16, 13, 1, 80, 0, 0, BF16, None) == UNSUPPORTED


def test_positions_and_frequencies_have_no_gradient():
    """What has none is refused where it would be wanted, and taken where it is not (and then refused for lying on the CPU)."""
    import torch

    from paper_2505_13813_amd import transformer as T

    q = torch.zeros(1, 4, 2, 64)
    p, (f, axis) = T.grid_positions(4).float(), T.rotary_frequencies((8,))
    for x in (q, q.clone().requires_grad_()):
        for bad in ((x, p, f.clone().requires_grad_(), axis), (x, p.clone().requires_grad_(), f, axis),
                    (x, p, f, axis, q, p.clone().requires_grad_())):
            with pytest.raises(RuntimeError, match="no gradient"):
                T.rotary(*bad)
            with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
                T.rotary(*bad)


def test_the_decoder_has_one_eps():
    from paper_2505_13813_amd.transformer import KATCrossDecoder

    for given, eps in (({}, 1e-6), ({"eps": 1e-3}, 1e-3)):
        m = KATCrossDecoder(2, 64, 2, groups=4, **given)
        assert [n.eps for b in m.blocks for n in (b.norm1, b.norm2)] + [m.norm.eps] == [eps] * 5


def test_a_block_with_rotation_wants_all_positions():
    """An encoder's states are never turned by the queries' positions."""
    import torch

    from paper_2505_13813_amd import transformer as T

    m = T.KATCrossDecoder(1, 64, 2, groups=4, rotary_pairs=(8,))
    x, at = torch.zeros(1, 4, 64), T.grid_positions(4)
    for call in (lambda: m(x, x, at), lambda: m.blocks[0](x, x, None, at)):
        with pytest.raises(ValueError, match="context_positions"):
            call()
    cache = [(x, x)]
    for call in (lambda: m(x, x, None, at), lambda: m(x, cache=cache), lambda: m.cached(x), lambda: m.blocks[0].cached(x)):
        with pytest.raises(ValueError, match=r"\bpositions\b"):
            call()


def test_missing_operands_are_named():
    import torch

    from paper_2505_13813_amd import transformer as T

    x, w, q = torch.zeros(4, 64), torch.ones(64), torch.zeros(1, 4, 2, 64)
    p, (f, axis) = T.grid_positions(4), T.rotary_frequencies((8,))
    for call, name in ((lambda: T.rms_norm(None, w), "x"), (lambda: T.rms_norm(x, None), "weight"), (lambda: T.rms_norm(x, w, 1.0), "residual"),
                       (lambda: T.rms_norm_8bit(x, w.tolist()), "weight"), (lambda: T.rotary(None, p, f, axis), "q"),
                       (lambda: T.rotary(q, None, f, axis), "positions"), (lambda: T.rotary(q, p, None, axis), "frequencies"),
                       (lambda: T.rotary(q, p, f, [0] * 8), "axis"), (lambda: T.rotary(q, p, f, axis, q, [[0]]), "k_positions"),
                       (lambda: T.cross_attention(q, None, q), "k"), (lambda: T.cross_attention(q, q, None), "v"),
                       (lambda: T.cross_attention(q, q, q, [4]), "key_lengths"), (lambda: T.cross_attention(q, q, q, None, [True]), "key_mask")):
        with pytest.raises(TypeError, match=r"^%s must be a tensor" % name):
            call()
