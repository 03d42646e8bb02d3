"""What stands around the KAT MLP in a transformer block: root-mean-square norm with the residual's addition (forward, backward,
and in inference to 8 bits), rotary positions with several axes for tokens of images and video, cross attention to an
encoder's states of another length (forward, backward, and split over the keys where there are few queries, single tokens
among them), causal attention over packed sequences (forward, backward), and a cache of keys and values in pages with the attention
of the newest tokens over it.

The functions run hand-written kernels (C ABI: include/grkan_transformer.h) through native autograd functions; there is no other
route, and nothing falls back.  They take plain tensors on the GPU, outside of function transforms, tracing and
forward-mode differentiation; under torch.compile they are calls that break the graph.  Work is enqueued on the current stream;
results are the same bits from run to run.

KATCrossBlock and KATCrossDecoder run them together with KATMlp, as a decoder of image or video tokens does; KATDecoderBlock and
KATDecoder as one that answers token by token, with a PagedCache.
"""
from __future__ import annotations

from functools import wraps
from typing import Optional, Sequence, Tuple

import torch
from torch import nn

from . import binding
from .nn import KATMlp


def _taken(out, name: str):
    if out is None:
        raise NotImplementedError(
            "%s takes plain tensors, outside of tracing, function transforms, dispatch modes and forward-mode "
            "differentiation" % name)
    return out


def _outside_graphs(function):
    """A call that torch.compile leaves as it is, between two graphs."""
    broken = torch.compiler.disable(function)

    @wraps(function)
    def call(*args, **kwargs):
        return (broken if torch.compiler.is_compiling() else function)(*args, **kwargs)

    return call


@_outside_graphs
def rms_norm(x, weight, residual=None, eps: float = 1e-6):
    """y = h / sqrt(mean(h^2) + eps) * weight over the last dimension, h = x + residual.

    x [..., D] float32, bfloat16 or float16, D up to 16384; weight [D] float32 or of x's type; residual as x.  Returns y, or with a
    residual (y, h): the new residual stream, rounded to x's type, and y made of that.  Differentiable (once) with respect to x,
    weight and residual.  Rows a constant number of elements apart are read as they lie, other layouts are copied."""
    out = _taken(binding.load_native().rms_norm(x, weight, residual, eps), "rms_norm")
    return out[0] if residual is None else (out[0], out[1])


@_outside_graphs
def rms_norm_8bit(x, weight, residual=None, eps: float = 1e-6):
    """rms_norm with y in 8 bits: (q, scale) or, with a residual, (q, scale, h).  q [..., D] float8_e4m3fn, scale [...] float32, one for
    each row: its largest magnitude / 448 (0 for a row of zeros, NaN for one with a NaN or an infinity); y = q * scale.  For inference: no
    gradient."""
    return tuple(_taken(binding.load_native().rms_norm_8bit(x, weight, residual, eps), "rms_norm_8bit"))


def rotary_frequencies(pairs: Sequence[int], theta: float = 10000.0, shared: bool = False,
                       device=None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(frequencies, axis) for `rotary`: pairs[a] pairs of channels turn with axis a.  Each axis has a ladder of its own,
    theta^(-i / pairs[a]) radians per step; with `shared` there is one over all pairs, theta^(-j / sum(pairs)), cut into the axes."""
    counts = [int(n) for n in pairs]
    if not counts or min(counts) < 0 or theta <= 0:
        raise ValueError("pairs must be counts of channel pairs, one for each axis, and theta positive")
    total = sum(counts)
    if shared:
        steps = torch.arange(total, dtype=torch.float64) / max(total, 1)
    else:
        steps = torch.cat([torch.arange(n, dtype=torch.float64) / max(n, 1) for n in counts])
    axis = torch.cat([torch.full((n,), a, dtype=torch.int32) for a, n in enumerate(counts)])
    return (float(theta) ** -steps).to(device), axis.to(device)


def grid_positions(*extents: int, device=None) -> torch.Tensor:
    """int32 [tokens, axes]: the points of a grid (time, height, width, ...) in row order, the tokens' usual one."""
    points = torch.cartesian_prod(*(torch.arange(n, dtype=torch.int32) for n in extents))
    return points.reshape(-1, len(extents)).to(device)


@_outside_graphs
def rotary(q, positions, frequencies, axis, k=None, k_positions=None, interleaved: bool = False):
    """Turns pair j of each head's channels by the angle positions[token, axis[j]] * frequencies[j].

    q (and k) [batch, tokens, heads, dim], any strides with dense channels; positions (of q, and of k where no k_positions
    are given) [tokens, axes] or [batch, tokens, axes], int32, int64 or float32.  A pair is channels (j, pairs + j) or, interleaved,
    (2 j, 2 j + 1); channels behind the pairs are copied.  Entries of `axis` are below `axes`.  Returns q, or (q, k) from one
    launch, contiguous.  Differentiable (once) with respect to q and k; positions or frequencies that want a gradient are refused."""
    if k is not None and k_positions is None:
        k_positions = positions
    out = _taken(binding.load_native().rotary(q, positions, frequencies, axis, k, k_positions, bool(interleaved)), "rotary")
    return out[0] if k is None else (out[0], out[1])


@_outside_graphs
def cross_attention(q, k, v, key_lengths=None, key_mask=None, scale: Optional[float] = None):
    """softmax(scale q k^T) v: q [batch, queries, heads, dim] attends to k, v [batch, keys, kv_heads, dim], head h to key head
    h // (heads / kv_heads).  bfloat16 or float16, dim a multiple of 8 up to 128, any strides with dense channels; scale: dim ** -0.5.

    key_lengths: int [batch], the keys below it are valid; key_mask: bool [batch, keys], True where a key is; both may be given.  What
    lies in other keys and values (NaN, infinities) has no influence; a query without a valid key gets zeros.  Differentiable (once) with
    respect to q, k and v."""
    return _taken(binding.load_native().cross_attention(q, k, v, key_lengths, key_mask, scale), "cross_attention")


@_outside_graphs
def causal_attention(q, k, v, offsets=None, scale: Optional[float] = None):
    """softmax(scale q k^T) v over the tokens of the same sequence up to the token itself, head h reading key head h // (heads / kv_heads).

    q [tokens, heads, dim], k, v [tokens, kv_heads, dim]: sequences packed one behind the other, sequence s being tokens offsets[s] up to, not with,
    offsets[s + 1] (int [sequences + 1]; one sequence where there are none; where they fall, all that comes out is unspecified).  Tokens in front of the first and behind the last belong to no sequence:
    zeros, and zeros as their gradients.  Or q [batch, tokens, heads, dim], k and v alike, without offsets: a sequence each.
    bfloat16 or float16, dim a multiple of 8 up to 128, any strides with dense channels; scale: dim ** -0.5.
    No sequence has any influence on another, and no later token on an earlier one's output, NaN and infinities included.  Differentiable (once) with
    respect to q, k and v."""
    return _taken(binding.load_native().causal_attention(q, k, v, offsets, scale), "causal_attention")


@_outside_graphs
def paged_write(k, v, k_pages, v_pages, table, lengths, offsets=None) -> None:
    """Keys and values of new tokens into a cache in pages, in place.  Position p of sequence s lies in row p % page_size of page table[s, p // page_size].

    k_pages, v_pages [pages, page_size, kv_heads, dim] bfloat16 or float16, whose strides and address are whole 16 bytes, channels dense (they may be a view
    of [pages, kv_heads, page_size, dim]); table int32 [sequences, entries]; lengths int [sequences]: with the new tokens.  k, v [tokens, kv_heads, dim] packed, with
    offsets as in causal_attention, or [sequences, tokens, kv_heads, dim].  A sequence's last new token goes to position lengths[s] - 1, the
    others in front of it.  Tokens of no sequence go nowhere, and neither do those whose entry is no page (below 0, or too large), whose position would be below 0, or
    whose sequence is longer than its row of the table has place for.  Where two tokens have one place (a page in two rows), which of them it holds is
    unspecified.  k and v share no memory with the pages.  No gradient."""
    _taken(binding.load_native().paged_write(k, v, k_pages, v_pages, table, lengths, offsets), "paged_write")


@_outside_graphs
def paged_attention(q, k_pages, v_pages, table, lengths, scale: Optional[float] = None):
    """Attention of the newest tokens over a cache in pages (paged_write): q [sequences, tokens, heads, dim], token i of sequence s being that of position
    lengths[s] - tokens + i, sees the positions up to its own, its keys and values having been written.  One token, or a few.

    A token that sees nothing (an empty sequence, an entry that is no page) gets zeros.  What the pages hold elsewhere, NaN and infinities included, has no
    influence.  Split over the cache's length where that pays, and joined.  scale: dim ** -0.5.  No gradient."""
    return _taken(binding.load_native().paged_attention(q, k_pages, v_pages, table, lengths, scale), "paged_attention")


class RMSNorm(nn.Module):
    """rms_norm with its weight: forward(x) gives y, forward(x, residual) gives (y, x + residual)."""

    def __init__(self, dim: int, eps: float = 1e-6):
        super().__init__()
        self.eps = float(eps)
        self.weight = nn.Parameter(torch.ones(dim))

    def forward(self, x, residual=None):
        return rms_norm(x, self.weight, residual, self.eps)

    def quantized(self, x, residual=None):
        """As rms_norm_8bit."""
        return rms_norm_8bit(x, self.weight, residual, self.eps)


class RotaryAxes(nn.Module):
    """rotary with its frequencies: forward(q, positions, k=None, k_positions=None).  The frequencies stay float64 whatever the
    module is converted to."""

    def __init__(self, pairs: Sequence[int], theta: float = 10000.0, shared: bool = False, interleaved: bool = False):
        super().__init__()
        self.interleaved = bool(interleaved)
        frequencies, axis = rotary_frequencies(pairs, theta, shared)
        # (a conversion of the module leaves whole numbers alone)
        self.register_buffer("frequency_bits", frequencies.view(torch.int64), persistent=False)
        self.register_buffer("axis", axis, persistent=False)

    def forward(self, q, positions, k=None, k_positions=None):
        return rotary(q, positions, self.frequency_bits.view(torch.float64), self.axis, k, k_positions, self.interleaved)


class KATCrossBlock(nn.Module):
    """A decoder block with a KAT MLP: x + attention(norm(x), context), then x + KATMlp(norm(x)).

    The last addition is left to the norm behind it, which has the sum in registers anyway: a block takes (branch, stream) and
    returns (branch, stream), the value being their sum; stream None means that branch is the value.

    Parameters and inputs are bfloat16 or float16, or float32 under autocast to one of the two, which keeps the stream in float32.
    `rotary_pairs`: rotated channel pairs of each head for each axis of the positions; none: no rotation.  With rotation the tokens'
    positions are given and, with a context, the context's own.  `context_dim`: channels of
    the encoder's states (default: dim)."""

    def __init__(self, dim: int, heads: int, kv_heads: Optional[int] = None, context_dim: Optional[int] = None,
                 rotary_pairs: Sequence[int] = (), groups: int = 8, hidden: Optional[int] = None, eps: float = 1e-6):
        super().__init__()
        kv_heads = heads if kv_heads is None else kv_heads
        if dim % heads or heads % kv_heads:
            raise ValueError("dim must be a multiple of heads, and heads of kv_heads")
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, dim // heads
        self.norm1 = RMSNorm(dim, eps)
        self.to_q = nn.Linear(dim, dim)
        self.to_kv = nn.Linear(dim if context_dim is None else context_dim, 2 * kv_heads * self.head_dim)
        self.rotary = RotaryAxes(rotary_pairs) if len(rotary_pairs) else None
        self.proj = nn.Linear(dim, dim)
        self.norm2 = RMSNorm(dim, eps)
        self.mlp = KATMlp(dim, hidden, groups)

    def _positions(self, **given):
        for name, positions in given.items():
            if self.rotary is not None and positions is None:
                raise ValueError("a block with rotation needs %s" % name)

    def keys_values(self, context):
        """(k, v) [batch, keys, kv_heads, head_dim] of the encoder's states, not rotated yet."""
        kv = self.to_kv(context).unflatten(-1, (2, self.kv_heads, self.head_dim))
        return kv[..., 0, :, :], kv[..., 1, :, :]

    def cached(self, context, positions=None):
        """(k, v) as forward(keys_values=...) takes them: made once where single tokens attend to the same states again and
        again."""
        self._positions(positions=positions)
        k, v = self.keys_values(context)
        if self.rotary is not None:
            k = self.rotary(k, positions)
        return k, v

    def forward(self, branch, context=None, stream=None, positions=None, context_positions=None, key_lengths=None,
                key_mask=None, keys_values=None):
        if keys_values is None:
            self._positions(positions=positions, context_positions=context_positions)
        else:
            self._positions(positions=positions)
        y, x = (self.norm1(branch), branch) if stream is None else self.norm1(branch.to(stream.dtype), stream)
        q = self.to_q(y).unflatten(-1, (self.heads, self.head_dim))
        if keys_values is not None:
            k, v = keys_values
            if self.rotary is not None:
                q = self.rotary(q, positions)
        else:
            k, v = self.keys_values(context)
            if self.rotary is not None:
                q, k = self.rotary(q, positions, k, context_positions)
        out = cross_attention(q, k, v, key_lengths, key_mask)
        y, x = self.norm2(self.proj(out.flatten(-2)).to(x.dtype), x)
        return self.mlp(y), x


class KATCrossDecoder(nn.Module):
    """KATCrossBlocks one behind the other, and a norm: queries [batch, tokens, dim] to an encoder's states
    [batch, keys, context_dim].  `eps` is that of every norm."""

    def __init__(self, depth: int, dim: int, heads: int, *, eps: float = 1e-6, **block):
        super().__init__()
        self.blocks = nn.ModuleList(KATCrossBlock(dim, heads, eps=eps, **block) for _ in range(depth))
        self.norm = RMSNorm(dim, eps)

    def cached(self, context, positions=None):
        """What forward(cache=...) takes: the keys and values of every block."""
        return [block.cached(context, positions) for block in self.blocks]

    def forward(self, x, context=None, positions=None, context_positions=None, key_lengths=None, key_mask=None, cache=None):
        stream = None
        for i, block in enumerate(self.blocks):
            x, stream = block(x, context, stream, positions, context_positions, key_lengths, key_mask,
                              None if cache is None else cache[i])
        return self.norm(x) if stream is None else self.norm(x.to(stream.dtype), stream)[0]


class PagedCache:
    """Pages of keys and values for a KATDecoder, or another caller of paged_write and paged_attention: `depth` blocks' k_pages[i] and
    v_pages[i] [pages, page_size, kv_heads, dim], and for `sequences` rows a table and lengths, int32 on the device, which the blocks share and
    whose addresses stay (a captured step reads what grow() wrote).  Which pages are free is kept on the host.

    `longest`: positions that a sequence may have at most."""

    def __init__(self, depth: int, pages: int, page_size: int, kv_heads: int, dim: int, sequences: int, longest: int,
                 dtype=torch.bfloat16, device="cuda"):
        if min(depth, pages, page_size, kv_heads, dim, sequences, longest) < 1:
            raise ValueError("a cache needs a block, a page, a position, a head, a channel and a sequence at least")
        pools = torch.zeros(2, depth, pages, page_size, kv_heads, dim, dtype=dtype, device=device)
        self.k_pages, self.v_pages = list(pools[0].unbind(0)), list(pools[1].unbind(0))
        self.page_size, self.longest = page_size, longest
        self.table = torch.full((sequences, -(-longest // page_size)), -1, dtype=torch.int32, device=device)
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device=device)
        self.counts = [0] * sequences
        self._grown, self._stepped = [0] * sequences, False  # new positions that no step or prompt has had; since when they are counted anew
        self._held = torch.full(self.table.shape, -1, dtype=torch.int32)  # the table on the host
        self._free = list(range(pages - 1, -1, -1))

    @property
    def free_pages(self) -> int:
        return len(self._free)

    def _pages(self, count: int) -> int:
        return -(-count // self.page_size)

    def grow(self, counts: Sequence[int]) -> None:
        """Makes room for counts[s] new positions of each sequence and adds them to the lengths, before the step that writes them, on the
        stream that it runs on.  Refused as a whole where the pages do not suffice, and in a capture."""
        self._outside_captures()
        counts = [int(n) for n in counts]
        if len(counts) != len(self.counts) or min(counts) < 0:
            raise ValueError("counts must be a number of new positions, not negative, for each of the cache's sequences")
        after = [a + b for a, b in zip(self.counts, counts)]
        if max(after) > self.longest:
            raise ValueError("a sequence would have %d positions, and %d is the most" % (max(after), self.longest))
        wanted = [self._pages(b) - self._pages(a) for a, b in zip(self.counts, after)]
        if sum(wanted) > len(self._free):
            raise RuntimeError("%d more pages are needed, and %d are free" % (sum(wanted), len(self._free)))
        for i, n in enumerate(wanted):
            if n:
                first = self._pages(self.counts[i])
                self._held[i, first:first + n] = torch.tensor([self._free.pop() for _ in range(n)], dtype=torch.int32)
        self.counts = after
        if self._stepped:
            self._grown, self._stepped = [0] * len(counts), False
        self._grown = [a + b for a, b in zip(self._grown, counts)]
        if any(wanted):
            self.table.copy_(self._held)
        if min(counts) == max(counts):
            self.lengths.add_(counts[0])  # (nothing from the host, which would wait for the device)
        else:
            self.lengths.copy_(torch.tensor(after, dtype=torch.int32))

    def release(self, sequence: int) -> None:
        """Takes a sequence's pages back: its row, of length 0, is free for another one.  Not in a capture."""
        self._outside_captures()
        row = self._held[sequence]
        self._free += row[:self._pages(self.counts[sequence])].tolist()[::-1]
        row.fill_(-1)
        self.counts[sequence] = self._grown[sequence] = 0
        self.table[sequence].fill_(-1)
        self.lengths[sequence].zero_()

    def _capturing(self) -> bool:
        """Whether a call is recorded and not run: then the counts are not those of its replays."""
        return self.table.is_cuda and torch.cuda.is_current_stream_capturing()

    def _outside_captures(self) -> None:
        if self._capturing():
            raise RuntimeError("a cache grows and releases outside of captured graphs: which pages are free is kept on the host, which has no part in a replay")

    @_outside_graphs
    def _prompts(self, tokens: Optional[int]) -> None:
        """Whole sequences go into the rows that held nothing before they grew; tokens: of each, where all have as many."""
        if self._capturing():
            return
        other = [s for s, held in enumerate(self.counts) if tokens is not None and held not in (0, tokens)]
        if other:
            raise ValueError("whole sequences of %d go into rows that hold nothing else, and have grown by as many: not so row %s" % (tokens, ", ".join(map(str, other))))
        self._grown = [0 if grown == held else grown for grown, held in zip(self._grown, self.counts)]

    @_outside_graphs
    def _newest(self, tokens: int) -> None:
        """So many tokens go into each row that holds something; once more into the same places, until it grows again."""
        if self._capturing():
            return
        short = [s for s, (grown, held) in enumerate(zip(self._grown, self.counts)) if held and grown < tokens]
        if short:
            raise ValueError("a step of %d would overwrite older positions in rows that have not grown by as many since the step or prompt before: row %s"
                             % (tokens, ", ".join(map(str, short))))
        self._stepped = True


class KATDecoderBlock(nn.Module):
    """A decoder block with a KAT MLP: x + attention(norm(x)) within the token's sequence, then x + KATMlp(norm(x)).

    As KATCrossBlock it takes and returns (branch, stream).  Parameters and inputs are bfloat16 or float16, or float32 under autocast to one
    of the two, which keeps the stream in float32.  `rotary_pairs`: rotated channel pairs of each head for each axis of the positions, which are
    then needed; none: no rotation."""

    def __init__(self, dim: int, heads: int, kv_heads: Optional[int] = None, rotary_pairs: Sequence[int] = (), groups: int = 8,
                 hidden: Optional[int] = None, eps: float = 1e-6):
        super().__init__()
        kv_heads = heads if kv_heads is None else kv_heads
        if dim % heads or heads % kv_heads:
            raise ValueError("dim must be a multiple of heads, and heads of kv_heads")
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, dim // heads
        self.norm1 = RMSNorm(dim, eps)
        self.to_qkv = nn.Linear(dim, (heads + 2 * kv_heads) * self.head_dim)
        self.rotary = RotaryAxes(rotary_pairs) if len(rotary_pairs) else None
        self.proj = nn.Linear(dim, dim)
        self.norm2 = RMSNorm(dim, eps)
        self.mlp = KATMlp(dim, hidden, groups)

    def forward(self, branch, stream=None, offsets=None, positions=None, cache: Optional[PagedCache] = None, index: int = 0,
                newest: bool = False):
        """branch [tokens, dim] with offsets, or [batch, tokens, dim].  cache: keys and values go to its pages number `index`, too.  `newest`: the
        tokens are the last of the cache's sequences, [sequences, tokens, dim], and see all that those hold."""
        if self.rotary is not None and positions is None:
            raise ValueError("a block with rotation needs positions")
        y, x = (self.norm1(branch), branch) if stream is None else self.norm1(branch.to(stream.dtype), stream)
        qkv = self.to_qkv(y).unflatten(-1, (-1, self.head_dim))
        q, k, v = qkv.split((self.heads, self.kv_heads, self.kv_heads), -2)
        if self.rotary is not None:
            packed = branch.dim() == 2  # one batch entry
            q, k = self.rotary(q[None] if packed else q, positions, k[None] if packed else k)
            q, k = (q[0], k[0]) if packed else (q, k)
        if cache is not None:
            k_pages, v_pages = cache.k_pages[index], cache.v_pages[index]
            paged_write(k, v, k_pages, v_pages, cache.table, cache.lengths, offsets)
        if newest:
            out = paged_attention(q, k_pages, v_pages, cache.table, cache.lengths)
        else:
            out = causal_attention(q, k, v, offsets)
        y, x = self.norm2(self.proj(out.flatten(-2)).to(x.dtype), x)
        return self.mlp(y), x


class KATDecoder(nn.Module):
    """KATDecoderBlocks one behind the other, and a norm.  `eps` is that of every norm."""

    def __init__(self, depth: int, dim: int, heads: int, *, eps: float = 1e-6, **block):
        super().__init__()
        self.blocks = nn.ModuleList(KATDecoderBlock(dim, heads, eps=eps, **block) for _ in range(depth))
        self.norm = RMSNorm(dim, eps)

    def cache(self, pages: int, page_size: int, sequences: int, longest: int, dtype=None) -> PagedCache:
        """An empty PagedCache on the parameters' device, of their type or (under autocast) `dtype`."""
        block, weight = self.blocks[0], self.norm.weight
        return PagedCache(len(self.blocks), pages, page_size, block.kv_heads, block.head_dim, sequences, longest, dtype or weight.dtype,
                          weight.device)

    def _run(self, x, **given):
        stream = None
        for i, block in enumerate(self.blocks):
            x, stream = block(x, stream, index=i, **given)
        return self.norm(x) if stream is None else self.norm(x.to(stream.dtype), stream)[0]

    def forward(self, x, offsets=None, positions=None, cache: Optional[PagedCache] = None):
        """Whole sequences: x [tokens, dim] packed, offsets as in causal_attention, positions [tokens, axes]; or [batch, tokens, dim].  With a
        cache, whose rows held nothing before they grew by these sequences (a batch is refused where they did), their keys and values are left there;
        without gradients."""
        if cache is not None:
            cache._prompts(x.shape[1] if x.dim() == 3 else None)
        return self._run(x, offsets=offsets, positions=positions, cache=cache)

    def step(self, x, cache: PagedCache, positions=None):
        """The newest tokens [sequences, tokens, dim] of the cache's sequences, by which each has grown, or has been released; positions
        [sequences, tokens, axes].  Refused where a row that holds something has not grown since the step or the prompt before; what a captured
        step is replayed for is not looked at."""
        cache._newest(x.shape[-2])
        return self._run(x, positions=positions, cache=cache, newest=True)
