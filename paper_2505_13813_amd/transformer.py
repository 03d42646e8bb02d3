"""What stands around the KAT MLP in a transformer block: root-mean-square norm with the residual's addition (forward, backward,
and in inference to 8 bits), rotary positions with several axes for tokens of images and video, and cross attention to an
encoder's states of another length (forward, backward, and split over the keys where there are few queries, single tokens
among them).

The functions run hand-written kernels (C ABI: include/grkan_transformer.h) through native autograd functions; there is no other
route, and nothing falls back.  They take plain tensors on the GPU, outside of function transforms, tracing and
forward-mode differentiation; under torch.compile they are calls that break the graph.  Work is enqueued on the current stream;
results are the same bits from run to run.

KATCrossBlock and KATCrossDecoder run them together with KATMlp, as a decoder of image or video tokens does.
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
