"""A softmax attention layer between the mixer layers of a hybrid model, served
end to end on one MI355X: prompts and single tokens over a paged cache of keys
and values in 4 bits, with the norm and 8-bit projections around it.

    u        = norm(x + residual)                     8 bits
    q, k, v  = u qkv_proj                             8-bit product
    k, v     -> the cache, q and k rotated on the way
    y        = attention(q, cache)                    8 bits
    out      = y out_proj                             8-bit product

torch supplies device memory and the stream; every computation of `prefill` and
`step` is a call into libsketchssm.so.
"""
from __future__ import annotations

import math

import torch
from torch import Tensor

from . import ops
from .mixer import quantize_weight


def rotary_angles(places: int, dim: int, base: float = 10000.0, *, factor: float = 1.0, original: int | None = None, low: float = 1.0,
                  high: float = 32.0, magnitude: float | None = None, device="cuda") -> Tensor:
    """The table that ops.rotary and ops.cache_append turn by: [places][dim]
    float32, row p the cosines and then the sines of p base^(-2 i / dim), i <
    dim / 2, from angles in 64 bits.  Made once, for the longest context.

    Scaled for longer contexts than a model was trained on, `factor` > 1:
    `original` None: every angle over factor (interpolated positions).
    `original` the trained length: by parts (YaRN, arXiv 2309.00071) -- an angle
    that turns at least `high` times over it stays, one that turns at most
    `low` times is divided by factor, those between are mixed linearly, and
    cosines and sines are multiplied by 1 + 0.1 ln factor unless `magnitude`
    is given."""
    if places < 1 or dim < 2 or dim % 2 or not base > 0.0 or not factor >= 1.0:
        raise ValueError(f"{places} places, {dim} channels, base {base}, factor {factor}: at least one place, an even number of channels, a "
                         f"positive base and a factor from 1 are needed")
    if original is not None and (original < 1 or not 0.0 <= low < high):
        raise ValueError(f"original {original}, low {low}, high {high}: a length and 0 <= low < high are needed")
    f = base ** (-torch.arange(0, dim, 2, dtype=torch.float64, device=device) / dim)
    scaled = f / factor
    if original is not None:
        turns = f * (original / (2.0 * math.pi))
        keep = ((turns - low) / (high - low)).clamp(0.0, 1.0)
        f = keep * f + (1.0 - keep) * scaled
        m = 1.0 + 0.1 * math.log(factor) if magnitude is None else magnitude
    else:
        f, m = scaled, 1.0 if magnitude is None else magnitude
    a = torch.arange(places, dtype=torch.float64, device=device)[:, None] * f
    return torch.cat([torch.cos(a) * m, torch.sin(a) * m], 1).float()


class Attention:
    """Weights (`weights`, a dict): norm [hidden], qkv_proj [(heads + 2
    kv_heads) dim][hidden] with the rows of the queries, keys and values in this
    order, out_proj [hidden][heads dim].  The projections are quantised here.
    The cache has `pages` pages of `page` tokens; rotation is a table of
    rotary_angles (None: no positions).  A head is 64 channels (with an even
    number of heads a key head), 128 or 256, hidden a multiple of 16.  Shapes
    that do not fit raise ValueError here.

    The sequences' pages and lengths belong to the caller, who keeps them once
    for all layers of a model: table [batch][columns], the pages of each
    sequence in order, and lengths [batch], its tokens with the new ones of this
    call (int32, as ops.cache_append takes them)."""

    def __init__(self, weights: dict, heads: int, kv_heads: int, dim: int, pages: int, page: int, rotation: Tensor | None = None,
                 interleaved: bool = False, scale: float | None = None, io: str = "bf16", eps: float = 1e-5, device="cuda"):
        dev = torch.device(device)
        self._check(weights, heads, kv_heads, dim, rotation)
        self.heads, self.kv_heads, self.dim, self.scale, self.eps = heads, kv_heads, dim, scale, eps
        self.interleaved = interleaved
        self.rotation = None if rotation is None else rotation.to(dev, torch.float32).contiguous()
        self.dtype = torch.bfloat16 if io == "bf16" else torch.float32
        self.norm = weights["norm"].to(dev, torch.float32).contiguous()
        self.qkv_proj, self.qkv_scale = quantize_weight(weights["qkv_proj"].to(dev))
        self.out_proj, self.out_scale = quantize_weight(weights["out_proj"].to(dev))
        self.cache = ops.new_cache(pages, kv_heads, page, dim, dev)

    @staticmethod
    def _check(weights: dict, heads: int, kv_heads: int, dim: int, rotation: Tensor | None) -> None:
        if kv_heads < 1 or heads < 1 or heads % kv_heads:
            raise ValueError(f"{kv_heads} key heads do not divide {heads} heads")
        if dim not in (64, 128, 256) or dim == 64 and heads // kv_heads % 2:
            raise ValueError(f"{heads // kv_heads} heads of {dim} channels a key head: 64 channels with an even number, 128 or 256 end in 8 bits")
        hidden = weights["qkv_proj"].shape[1]
        if hidden % 16:
            raise ValueError(f"hidden size {hidden}: a multiple of 16 is projected in 8 bits")
        for name, shape in (("qkv_proj", ((heads + 2 * kv_heads) * dim, hidden)), ("out_proj", (weights["out_proj"].shape[0], heads * dim)),
                            ("norm", (hidden,))):
            if weights[name].shape != shape:
                raise ValueError(f"{name}: {list(weights[name].shape)}, not {list(shape)}")
        if rotation is not None and (rotation.dim() != 2 or not 2 <= rotation.shape[1] <= dim or rotation.shape[1] % 2):
            raise ValueError(f"rotation: {list(rotation.shape)}, not [places][rotated] of an even number up to {dim}")

    def prefill(self, x: Tensor, residual: Tensor, table: Tensor, lengths: Tensor, offsets: Tensor | None = None) -> tuple[Tensor, Tensor]:
        """Packed new tokens x [T][hidden] of every sequence (rows offsets[b] ..
        offsets[b+1]-1; None: T / batch each) behind what the cache holds of it,
        with the residual stream: (out [T][hidden], the residual stream with x
        added).  Single tokens over long contexts are faster in a `step` of
        their own than in a call with prompts."""
        H, G, D = self.heads, self.kv_heads, self.dim
        u, s, residual = ops.norm(x, self.norm, self.eps, residual=residual, out_dtype=ops.F8)
        qkv = ops.matmul_fp8(u, s, self.qkv_proj, self.qkv_scale, out_dtype=self.dtype).view(-1, H + 2 * G, D)
        q = qkv[:, :H]
        turned = ops.cache_append(self.cache, table, lengths, qkv[:, H:H + G], qkv[:, H + G:], offsets=offsets, rotation=self.rotation,
                                  interleaved=self.interleaved, q=None if self.rotation is None else q,
                                  q_out=None if self.rotation is None else q)
        y, s = ops.attention(self.cache, table, lengths, q if turned is None else turned, offsets=offsets, scale=self.scale, out_dtype=ops.F8)
        return ops.matmul_fp8(y.view(-1, H * D), s, self.out_proj, self.out_scale, out_dtype=self.dtype), residual

    def step(self, x: Tensor, residual: Tensor, table: Tensor, lengths: Tensor) -> tuple[Tensor, Tensor]:
        """One token of every sequence, x and residual [batch][hidden]; lengths count it."""
        if x.shape[0] != lengths.numel():
            raise ValueError(f"{x.shape[0]} tokens of {lengths.numel()} sequences: one of each is a step")
        return self.prefill(x, residual, table, lengths)
