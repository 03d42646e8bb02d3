"""Causal attention and the cache in pages without a GPU: the C interface's structures and refusals (each before anything is launched), workspaces, and the refusal
of tensors on the CPU."""
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


@pytest.mark.parametrize("name,struct", [("grkan_causal_attention_t", binding.CausalAttention), ("grkan_paged_cache_t", binding.PagedCacheOperand),
                                         ("grkan_paged_queries_t", binding.PagedQueries)])
def test_structures_match_the_header(name, struct):
    text = re.sub(r"/\*.*?\*/", "", (ROOT / "include" / "grkan_transformer.h").read_text(), flags=re.S)
    body = re.search(r"typedef struct \{([^}]*)\} %s;" % name, text).group(1)
    kinds = {"void": ctypes.c_void_p, "int32_t": ctypes.c_int32, "int64_t": ctypes.c_int64, "float": ctypes.c_float}
    fields = []
    for line in body.split(";"):
        if line.strip():
            kind, names = re.match(r"\s*(?:const )?(\w+)\s+(.*)", line, flags=re.S).groups()
            fields += [(n.strip(" *\n"), ctypes.c_void_p if "*" in n else kinds[kind]) for n in names.split(",")]
    assert fields == list(struct._fields_)


def _causal(**fields):
    given = dict(q=16, k=16, v=16, offsets=16, tokens=40, sequences=3, heads=4, kv_heads=2, dim=64, q_token_stride=256, q_head_stride=64, k_token_stride=128,
                 k_head_stride=64, v_token_stride=128, v_head_stride=64, scale=0.125)
    given.update(fields)
    return binding.CausalAttention(**given)


BAD_CAUSAL = [({"q": None}, NULL), ({"k": None}, NULL), ({"v": None}, NULL), ({"tokens": -1}, SHAPE), ({"sequences": -1}, SHAPE), ({"heads": 0}, SHAPE),
              ({"heads": 5}, SHAPE), ({"kv_heads": 0}, SHAPE), ({"dim": 0}, SHAPE), ({"offsets": None}, SHAPE), ({"offsets": None, "sequences": 0}, SHAPE),
              ({"dim": 60}, UNSUPPORTED), ({"dim": 136}, UNSUPPORTED), ({"scale": 0.0}, UNSUPPORTED), ({"scale": -1.0}, UNSUPPORTED),
              ({"scale": math.inf}, UNSUPPORTED), ({"scale": math.nan}, UNSUPPORTED), ({"scale": 3e38}, UNSUPPORTED), ({"tokens": 1 << 30}, UNSUPPORTED),
              ({"tokens": 1 << 29, "heads": 8}, UNSUPPORTED), ({"heads": 2 << 20, "tokens": 1}, UNSUPPORTED), ({"k_token_stride": -128}, UNSUPPORTED),
              ({"q_token_stride": 1 << 25}, UNSUPPORTED), ({"v_token_stride": 1 << 25}, UNSUPPORTED), ({"q_head_stride": -64}, UNSUPPORTED),
              ({"q_head_stride": 1 << 30}, UNSUPPORTED), ({"sequences": 1 << 30}, UNSUPPORTED), ({"q": 24}, ALIGN), ({"k": 24}, ALIGN), ({"v": 24}, ALIGN),
              ({"q_token_stride": 257}, ALIGN), ({"k_head_stride": 60}, ALIGN), ({"offsets": 18}, ALIGN), ({"offsets": 20, "offsets_64": 1}, ALIGN)]


@pytest.mark.parametrize("fields,status", BAD_CAUSAL)
def test_causal_refusals(lib, fields, status):
    a = _causal(**fields)
    assert lib.grkan_causal_attention_fwd(ctypes.byref(a), 16, 16, None, BF16, None) == status
    assert lib.grkan_causal_attention_bwd(ctypes.byref(a), 16, 16, 16, 16, 256, 64, 16, 16, 16, 16, 1 << 40, BF16, None) == status
    assert lib.grkan_causal_attention_bwd_workspace_bytes(ctypes.byref(a)) == 0


def test_causal_refusals_of_outputs(lib):
    a = _causal()
    assert lib.grkan_causal_attention_fwd(None, 16, None, None, BF16, None) == NULL
    assert lib.grkan_causal_attention_fwd(ctypes.byref(a), None, None, None, BF16, None) == NULL
    assert lib.grkan_causal_attention_fwd(ctypes.byref(a), 24, None, None, BF16, None) == ALIGN
    assert lib.grkan_causal_attention_fwd(ctypes.byref(a), 16, 24, None, BF16, None) == ALIGN
    assert lib.grkan_causal_attention_fwd(ctypes.byref(a), 16, None, 18, BF16, None) == ALIGN
    for io in (F32, 9):
        assert lib.grkan_causal_attention_fwd(ctypes.byref(a), 16, None, None, io, None) == DTYPE
    need = lib.grkan_causal_attention_bwd_workspace_bytes(ctypes.byref(a))

    def bwd(out=16, rest=16, lse=16, dout=16, strides=(256, 64), dq=16, dk=16, dv=16, ws=16, size=need):
        return lib.grkan_causal_attention_bwd(ctypes.byref(a), out, rest, lse, dout, *strides, dq, dk, dv, ws, size, BF16, None)

    for name in ("out", "lse", "dout", "dq", "dk", "dv"):
        assert bwd(**{name: None}) == NULL, name
        assert bwd(**{name: 18}) == ALIGN, name
    assert bwd(rest=24) == ALIGN
    assert bwd(strides=(257, 64)) == ALIGN and bwd(strides=(1 << 25, 64)) == UNSUPPORTED and bwd(strides=(-256, 64)) == UNSUPPORTED
    assert need > 0 and bwd(size=need - 1) == WORKSPACE and bwd(ws=None) == WORKSPACE and bwd(ws=24) == WORKSPACE
    none = _causal(tokens=0, q=None, k=None, v=None)
    assert lib.grkan_causal_attention_fwd(ctypes.byref(none), None, None, None, BF16, None) == OK
    assert lib.grkan_causal_attention_bwd(ctypes.byref(none), None, None, None, None, 0, 0, None, None, None, None, 0, BF16, None) == OK
    assert lib.grkan_causal_attention_lse_count(ctypes.byref(a)) == 40 * 4


def test_causal_workspaces(lib):
    """The plan is made for every combination of few and many tokens, sequences and heads; what is asked for can be had."""
    for tokens in (1, 127, 5000, 70000, 1 << 20):
        for sequences in (1, 3, 200, 40000):
            for heads, kv in ((1, 1), (12, 12), (32, 4), (40, 1)):
                for dim in (8, 64, 128):
                    a = _causal(tokens=tokens, sequences=sequences, heads=heads, kv_heads=kv, dim=dim)
                    need = lib.grkan_causal_attention_bwd_workspace_bytes(ctypes.byref(a))
                    assert 0 < need < (1 << 30) + 64 * (tokens + sequences) * heads


def test_more_workgroups_than_a_launch_takes(lib):
    for fields in (dict(tokens=1 << 24, heads=64, kv_heads=64, sequences=1 << 24), dict(tokens=1000, heads=1 << 20, kv_heads=1 << 20),
                   dict(tokens=(1 << 30) - 1, heads=2147483647, kv_heads=2147483647), dict(tokens=1 << 29, heads=4, kv_heads=2)):
        a = _causal(**fields)
        assert lib.grkan_causal_attention_fwd(ctypes.byref(a), 16, None, None, BF16, None) == UNSUPPORTED
        assert lib.grkan_causal_attention_bwd(ctypes.byref(a), 16, 16, 16, 16, 256, 64, 16, 16, 16, 16, 1 << 60, BF16, None) == UNSUPPORTED
        assert lib.grkan_causal_attention_bwd_workspace_bytes(ctypes.byref(a)) == 0


def _cache(**fields):
    given = dict(k_pages=16, v_pages=16, table=16, lengths=16, pages=100, page_size=16, sequences=3, table_entries=20, kv_heads=2, dim=64, lengths_64=0, table_stride=20,
                 k_page_stride=2048, k_token_stride=128, k_head_stride=64, v_page_stride=2048, v_token_stride=128, v_head_stride=64)
    given.update(fields)
    return binding.PagedCacheOperand(**given)


def _queries(**fields):
    given = dict(q=16, tokens=1, heads=4, sequence_stride=256, token_stride=256, head_stride=64, scale=0.125)
    given.update(fields)
    return binding.PagedQueries(**given)


BAD_CACHE = [({"k_pages": None}, NULL), ({"v_pages": None}, NULL), ({"table": None}, NULL), ({"lengths": None}, NULL), ({"pages": -1}, SHAPE), ({"page_size": 0}, SHAPE),
             ({"sequences": -1}, SHAPE), ({"table_entries": -1}, SHAPE), ({"kv_heads": 0}, SHAPE), ({"dim": 0}, SHAPE), ({"dim": 60}, UNSUPPORTED), ({"dim": 136}, UNSUPPORTED),
             ({"pages": 1 << 31}, UNSUPPORTED), ({"page_size": 1 << 20, "table_entries": 1 << 10}, UNSUPPORTED), ({"k_token_stride": -128}, UNSUPPORTED),
             ({"v_token_stride": 1 << 25}, UNSUPPORTED), ({"k_pages": 24}, ALIGN), ({"v_pages": 24}, ALIGN), ({"table": 18}, ALIGN), ({"lengths": 18}, ALIGN),
             ({"lengths": 20, "lengths_64": 1}, ALIGN), ({"k_page_stride": 2047}, ALIGN), ({"v_head_stride": 60}, ALIGN)]


@pytest.mark.parametrize("fields,status", BAD_CACHE)
def test_cache_refusals(lib, fields, status):
    c, q = _cache(**fields), _queries()
    assert lib.grkan_paged_attention(ctypes.byref(c), ctypes.byref(q), 16, 16, 1 << 40, BF16, None) == status
    assert lib.grkan_paged_write(ctypes.byref(c), 16, 16, 16, 0, 5, 128, 64, 128, 64, BF16, None) == status
    assert lib.grkan_paged_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(q)) == 0


@pytest.mark.parametrize("fields,status", [({"q": None}, NULL), ({"tokens": -1}, SHAPE), ({"heads": 0}, SHAPE), ({"heads": 3}, SHAPE), ({"tokens": 1 << 30}, UNSUPPORTED),
                                           ({"tokens": 1 << 29, "heads": 8}, UNSUPPORTED), ({"scale": 0.0}, UNSUPPORTED), ({"scale": math.nan}, UNSUPPORTED),
                                           ({"q": 24}, ALIGN), ({"token_stride": 60}, ALIGN)])
def test_queries_refusals(lib, fields, status):
    c, q = _cache(), _queries(**fields)
    assert lib.grkan_paged_attention(ctypes.byref(c), ctypes.byref(q), 16, 16, 1 << 40, BF16, None) == status
    assert lib.grkan_paged_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(q)) == 0


def test_other_refusals_of_pages(lib):
    c, q = _cache(), _queries()

    def attend(cache=c, queries=q, out=16, ws=16, size=1 << 40, io=BF16):
        return lib.grkan_paged_attention(ctypes.byref(cache) if cache else None, ctypes.byref(queries) if queries else None, out, ws, size, io, None)

    assert attend(cache=None) == NULL and attend(queries=None) == NULL and attend(out=None) == NULL and attend(out=24) == ALIGN
    for io in (F32, 9):
        assert attend(io=io) == DTYPE
        assert lib.grkan_paged_write(ctypes.byref(c), 16, 16, 16, 0, 5, 128, 64, 128, 64, io, None) == DTYPE
    long = _cache(table_entries=1000)
    need = lib.grkan_paged_attention_workspace_bytes(ctypes.byref(long), ctypes.byref(q))
    assert need > 0 and attend(long, size=need - 1) == WORKSPACE and attend(long, ws=None, size=need) == WORKSPACE and attend(long, ws=24, size=need) == WORKSPACE
    assert attend(_cache(sequences=0), out=None) == OK and attend(queries=_queries(tokens=0, q=None), out=None) == OK
    for many in (1 << 24, 1 << 23):  # 512 threads each
        assert attend(_cache(sequences=many)) == UNSUPPORTED

    def write(cache=c, k=16, v=16, offsets=16, wide=0, tokens=5, strides=(128, 64, 128, 64)):
        return lib.grkan_paged_write(ctypes.byref(cache) if cache else None, k, v, offsets, wide, tokens, *strides, BF16, None)

    assert write(cache=None) == NULL and write(k=None) == NULL and write(v=None) == NULL
    assert write(tokens=-1) == SHAPE and write(offsets=None, tokens=5) == SHAPE and write(cache=_cache(sequences=0), offsets=None) == SHAPE
    assert write(k=24) == ALIGN and write(v=24) == ALIGN and write(offsets=18) == ALIGN and write(offsets=20, wide=1) == ALIGN and write(strides=(60, 64, 128, 64)) == ALIGN
    assert write(tokens=1 << 30) == UNSUPPORTED and write(cache=_cache(kv_heads=1 << 21)) == UNSUPPORTED
    assert write(tokens=0, k=None, v=None) == OK and write(cache=_cache(pages=0, k_pages=None, v_pages=None)) == OK


def test_writes_of_more_tokens_than_a_launch_takes(lib):
    """64 tokens of a workgroup of 256: from 2^24 workgroups on there are 2^32 threads."""
    most = 64 * ((1 << 24) - 1)
    for tokens in (most + 1, (1 << 30) - 1):
        assert lib.grkan_paged_write(ctypes.byref(_cache()), 16, 16, 16, 0, tokens, 128, 64, 128, 64, BF16, None) == UNSUPPORTED


def test_paged_workspaces(lib):
    for sequences in (1, 7, 300, 5000):
        for entries in (1, 30, 10000):
            for kv, heads in ((1, 1), (8, 32), (12, 12)):
                for tokens in (1, 5, 100):
                    for dim in (8, 64, 128):
                        c = _cache(sequences=sequences, table_entries=entries, kv_heads=kv, dim=dim)
                        need = lib.grkan_paged_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(_queries(heads=heads, tokens=tokens)))
                        assert need <= 4 * 32 * 129 * (1024 + 4096 + 8)


def test_no_tokens_or_no_sequences_over_long_tables():
    """Nothing to do, whatever the table has place for: no workspace, no error.  (In a process of its own, which a division by zero would end.)"""
    import subprocess
    import sys

    text = """
import ctypes, itertools, sys
sys.path[:0] = [%r, %r]
import test_decoder_host as t
lib = t.binding.load_library()
for sequences, tokens, entries, dim, page in itertools.product((0, 3), (0, 1), (1, 20, 200, 100000), (64, 128), (16, 32)):
    if sequences and tokens:
        continue
    c, q = t._cache(sequences=sequences, table_entries=entries, dim=dim, page_size=page), t._queries(tokens=tokens)
    print(sequences, tokens, entries, dim, page, flush=True)
    assert lib.grkan_paged_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(q)) == 0
    assert lib.grkan_paged_attention(ctypes.byref(c), ctypes.byref(q), None, None, 0, t.BF16, None) == t.OK
""" % (str(ROOT), str(ROOT / "tests"))
    found = subprocess.run([sys.executable, "-c", text], capture_output=True, text=True, timeout=300)
    assert found.returncode == 0, (found.returncode, found.stdout[-200:], found.stderr[-2000:])


def test_tensors_on_the_cpu_and_missing_ones_are_refused():
    import torch

    from paper_2505_13813_amd import transformer as T

    q, pool = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16)
    table, lengths, offsets = torch.zeros(4, 1, dtype=torch.int32), torch.zeros(4, dtype=torch.int32), torch.zeros(5, dtype=torch.int32)
    for call in (lambda: T.causal_attention(q, q, q), lambda: T.causal_attention(q, q, q, offsets), lambda: T.paged_attention(q[:, None], pool, pool, table, lengths),
                 lambda: T.paged_write(q, q, pool, pool, table, lengths, offsets)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    for call, name in ((lambda: T.causal_attention(None, q, q), "q"), (lambda: T.causal_attention(q, q, q, [0, 4]), "offsets"),
                       (lambda: T.paged_attention(q, pool, None, table, lengths), "v_pages"), (lambda: T.paged_attention(q, pool, pool, None, lengths), "table"),
                       (lambda: T.paged_attention(q, pool, pool, table, 4), "lengths"), (lambda: T.paged_write(q, None, pool, pool, table, lengths), "v"),
                       (lambda: T.paged_write(q, q, None, pool, table, lengths), "k_pages")):
        with pytest.raises(TypeError, match=r"^%s must be a tensor" % name):
            call()


def _host_cache(**given):
    import torch

    from paper_2505_13813_amd.transformer import PagedCache

    return PagedCache(**{**dict(depth=2, pages=6, page_size=4, kv_heads=2, dim=8, sequences=3, longest=14, dtype=torch.bfloat16, device="cpu"), **given})


def test_pages_are_given_out_and_taken_back():
    c = _host_cache()
    assert [t.shape for t in (*c.k_pages, *c.v_pages)] == [(6, 4, 2, 8)] * 4 and c.table.shape == (3, 4) and c.free_pages == 6
    at = c.table.data_ptr(), c.lengths.data_ptr()
    c.grow([5, 0, 4])
    assert c.counts == c.lengths.tolist() == [5, 0, 4] and c.free_pages == 3
    c.grow([3, 1, 0])
    assert c.counts == c.lengths.tolist() == [8, 1, 4] and c.free_pages == 2
    held = [[p for p in row if p >= 0] for row in c.table.tolist()]
    assert [len(h) for h in held] == [2, 1, 1] and len(set(sum(held, []))) == 4
    before = c.table.clone()
    with pytest.raises(RuntimeError, match="pages"):
        c.grow([1, 4, 8])
    with pytest.raises(ValueError, match="most"):
        c.grow([7, 0, 0])
    for bad in ([1, 1], [1, 1, -1]):
        with pytest.raises(ValueError):
            c.grow(bad)
    assert c.counts == [8, 1, 4] and c.free_pages == 2 and (c.table == before).all()
    c.release(0)
    assert c.free_pages == 4 and c.lengths.tolist() == [0, 1, 4] and (c.table[0] == -1).all() and (c.table[1:] == before[1:]).all()
    c.grow([14, 0, 0])
    assert c.free_pages == 0 and sorted(sum(([p for p in row if p >= 0] for row in c.table.tolist()), [])) == list(range(6))
    assert (c.table.data_ptr(), c.lengths.data_ptr()) == at
    for bad in (dict(pages=0), dict(page_size=0), dict(sequences=0), dict(longest=0), dict(depth=0)):
        with pytest.raises(ValueError):
            _host_cache(**bad)


def test_pages_are_not_given_out_in_a_capture(monkeypatch):
    """The host's part would be done once and the device's at every replay."""
    c = _host_cache()
    c.grow([3, 0, 4])
    state = lambda: (list(c.counts), c.free_pages, c.table.tolist(), c.lengths.tolist())  # noqa: E731
    before = state()
    monkeypatch.setattr(type(c), "_capturing", lambda self: True, raising=False)
    for call in (lambda: c.grow([1, 1, 1]), lambda: c.grow([1, 0, 0]), lambda: c.grow([0, 0, 4]), lambda: c.release(0)):
        with pytest.raises(RuntimeError, match="captur"):
            call()
        assert state() == before
    monkeypatch.undo()
    c.grow([1, 1, 1])
    assert c.counts == c.lengths.tolist() == [4, 1, 5]


def test_a_decoder_wants_positions_and_heads_that_divide():
    import torch

    from paper_2505_13813_amd import transformer as T

    m = T.KATDecoder(1, 64, 2, groups=4, rotary_pairs=(8,))
    x = torch.zeros(4, 64)
    for call in (lambda: m(x), lambda: m.step(x[None], _host_cache())):
        with pytest.raises(ValueError, match="positions"):
            call()
    for bad in (dict(heads=5), dict(heads=6, kv_heads=4)):
        with pytest.raises(ValueError):
            T.KATDecoderBlock(192, **bad)
    for given, eps in (({}, 1e-6), ({"eps": 1e-3}, 1e-3)):
        m = T.KATDecoder(2, 64, 2, groups=4, **given)
        assert [n.eps for b in m.blocks for n in (b.norm1, b.norm2)] + [m.norm.eps] == [eps] * 5
    c = T.KATDecoder(3, 64, 4, kv_heads=2, groups=4).bfloat16().cache(5, 16, 2, 40)
    assert len(c.k_pages) == 3 and c.k_pages[0].shape == (5, 16, 2, 16) and c.k_pages[0].dtype == torch.bfloat16 and c.table.shape == (2, 3)


def _decoder_without_kernels():
    """Its blocks return what they are given."""
    import torch

    from paper_2505_13813_amd import transformer as T

    class Block(torch.nn.Module):
        def forward(self, x, stream=None, **given):
            return x, x

    class Norm(torch.nn.Module):
        def forward(self, x, stream):
            return x, stream

    m = T.KATDecoder(2, 16, 2, groups=4)
    m.blocks, m.norm = torch.nn.ModuleList([Block(), Block()]), Norm()
    return m


def test_a_step_of_rows_that_have_not_grown_is_refused():
    """A row that holds something and has no new position would have its last one's keys and values overwritten."""
    import torch

    m, c = _decoder_without_kernels(), _host_cache(pages=20, longest=40)
    one, two = torch.zeros(3, 1, 16), torch.zeros(3, 2, 16)
    m.step(one, c)  # (nothing is held)
    c.grow([5, 0, 4])
    m(torch.zeros(9, 16), torch.tensor([0, 5, 5, 9]), cache=c)
    with pytest.raises(ValueError, match=r"rows? 0, 2"):  # the prompts have taken what they grew by
        m.step(one, c)
    c.grow([1, 0, 0])
    with pytest.raises(ValueError, match=r"row 2"):
        m.step(one, c)
    c.grow([0, 0, 1])
    m.step(one, c)  # (grown one after the other, and row 1 is free)
    m.step(one, c)  # the same places once more, as before a capture
    c.grow([1, 0, 0])
    with pytest.raises(ValueError, match=r"row 2"):
        m.step(one, c)
    c.release(2)
    m.step(one, c)
    c.grow([1, 3, 0])
    m(torch.zeros(3, 16), torch.tensor([0, 0, 3, 3]), cache=c)  # a prompt into a free row, while row 0 has grown for a step
    c.grow([0, 1, 0])
    m.step(one, c)
    with pytest.raises(ValueError, match=r"rows? 0, 1"):
        m.step(two, c)
    c.grow([1, 1, 0])
    c.grow([1, 1, 0])
    m.step(two, c)
    c.grow([2, 2, 0])
    m.step(one, c)  # (what else the rows grew by is the caller's)


def test_a_batch_into_rows_that_hold_something_else_is_refused():
    """[batch, tokens, dim] into a cache are whole sequences: behind what a row holds already they would not see it, and of a row with fewer positions the
    first ones would be lost."""
    import torch

    m, c = _decoder_without_kernels(), _host_cache(pages=20, longest=40)
    x = torch.zeros(3, 4, 16)
    m(x, cache=c)  # (rows of nothing take nothing)
    c.grow([4, 0, 4])
    m(x, cache=c)
    m(x, cache=c)
    c.grow([4, 4, 0])
    with pytest.raises(ValueError, match=r"row 0$"):
        m(x, cache=c)
    c.release(0)
    c.grow([3, 0, 0])
    with pytest.raises(ValueError, match=r"row 0$"):
        m(x, cache=c)
    m(x.flatten(0, 1), torch.tensor([0, 3, 3, 3]), cache=c)  # (where the sequences end is on the device)


def test_steps_under_compile_are_compiled_once():
    """What the host keeps of the cache is no part of a graph: it changes from step to step, and each would be compiled anew."""
    import torch

    m, c = _decoder_without_kernels(), _host_cache(pages=20, longest=40)
    graphs = []

    def count(graph, example):
        graphs.append(graph)
        return graph.forward

    calls = (lambda run: run(torch.zeros(3, 1, 16), c)), (lambda run: run(torch.zeros(5, 16), torch.tensor([0, 1, 1, 5]), cache=c))
    for form, call in zip((m.step, m.forward), calls):
        torch._dynamo.reset()
        run, first = torch.compile(form, backend=count), None
        for i in range(1, 6):
            for row in range(3):
                c.release(row)
            c.grow([i, 0, 2])
            call(run)
            first = len(graphs) if first is None else first
        assert len(graphs) == first, form
    run = torch.compile(m.step, backend=count)
    c.grow([1, 0, 1])
    calls[0](run)
    c.grow([1, 0, 0])
    with pytest.raises(ValueError, match="row 2"):
        calls[0](run)
