"""A Mamba-2 mixer layer served end to end on one MI355X: prompts through the
convolution and the scan, single tokens through the sketch's decode path
(`SketchSSMLayer`), with the norms and 8-bit projections around both.

    u        = norm(x + residual)                        8 bits
    z, xBC, dt = u in_proj                               8-bit product
    x, B, C  = silu(conv(xBC))
    y        = scan(x, B, C, dt)  (prompts)   or   token -> replay buffer -> read
    out      = norm((y + D x) silu(z)) out_proj          8 bits, 8-bit product

torch supplies device memory and the stream; every computation of `prefill` and
`step` is a call into libsketchssm.so.
"""
from __future__ import annotations

import torch
from torch import Tensor

from . import ops
from .layer import SketchSSMLayer


def quantize_weight(w: Tensor) -> tuple[Tensor, Tensor]:
    """A weight matrix [N][K] as matmul_fp8 reads it: e4m3 values over the scale
    of their 128 x 128 block, scales [ceil(N / 128)][ceil(K / 128)].  Done once,
    when the weights are loaded."""
    N, K = w.shape
    nb, kb = -(-N // 128), -(-K // 128)
    p = torch.nn.functional.pad(w.float(), (0, kb * 128 - K, 0, nb * 128 - N)).reshape(nb, 128, kb, 128)
    s = (p.abs().amax((1, 3)) / 448.0).clamp_min(2.0 ** -64)
    q = (p / s[:, None, :, None]).reshape(nb * 128, kb * 128)[:N, :K]
    return q.to(ops.F8).contiguous(), s.contiguous()


class Mamba2Mixer:
    """Weights (`weights`, a dict): norm [hidden], in_proj [H V + C + H][hidden]
    with the rows of z, of the C = H V + 2 G K convolution channels and of dt in
    this order, taps [C][w], conv_bias [C] (or None), dt_bias, A and D [H]
    (A < 0), out_norm [H V], out_proj [hidden][H V].  The projections are
    quantised here.  omega and coef are the sketch's, and the other sketch
    arguments those of SketchSSMLayer.  The gated norm's groups (H V / G columns
    each, where G > 1) are whole blocks of 128, hidden and H V multiples of 16.
    Shapes that do not fit raise ValueError here, before a prompt moves any state."""

    def __init__(self, weights: dict, batch: int, heads: int, groups: int, dk: int, dv: int, rank: int, window: int,
                 omega: Tensor, coef: Tensor, io: str = "bf16", eps: float = 1e-5, device="cuda", **sketch):
        dev = torch.device(device)
        self._check(weights, heads, groups, dk, dv)
        f32 = lambda n: None if weights.get(n) is None else weights[n].to(dev, torch.float32).contiguous()  # noqa: E731
        self.batch, self.heads, self.groups, self.dk, self.dv, self.eps = batch, heads, groups, dk, dv, eps
        self.dtype = torch.bfloat16 if io == "bf16" else torch.float32
        self.norm, self.taps, self.conv_bias, self.out_norm = f32("norm"), f32("taps"), f32("conv_bias"), f32("out_norm")
        self.dt_bias, self.A, self.D = f32("dt_bias"), f32("A"), f32("D")
        self.in_proj, self.in_scale = quantize_weight(weights["in_proj"].to(dev))
        self.out_proj, self.out_scale = quantize_weight(weights["out_proj"].to(dev))
        self.hidden = self.in_proj.shape[1]
        self.inner, self.channels = heads * dv, heads * dv + 2 * groups * dk
        self.layer = SketchSSMLayer("mamba2", batch, heads, dk, dv, rank, window, io, device, omega=omega, coef=coef, **sketch)
        self.conv_state = torch.zeros((batch, self.taps.shape[1] - 1, self.channels), dtype=self.dtype, device=dev)
        self.q = torch.empty((batch, heads, dk), dtype=self.dtype, device=dev)

    @staticmethod
    def _check(weights: dict, heads: int, groups: int, dk: int, dv: int) -> None:
        if groups < 1 or heads % groups:
            raise ValueError(f"{groups} groups do not divide {heads} heads")
        HV, C = heads * dv, heads * dv + 2 * groups * dk
        if groups > 1 and HV // groups % 128:
            raise ValueError(f"{groups} groups of {HV // groups} columns cut the output norm's blocks of 128")
        hidden = weights["in_proj"].shape[1]
        if hidden % 16 or HV % 16:
            raise ValueError(f"hidden size {hidden} and {HV} values: multiples of 16 are projected in 8 bits")
        for name, shape in (("in_proj", (HV + C + heads, hidden)), ("out_proj", (weights["out_proj"].shape[0], HV)), ("norm", (hidden,)),
                            ("out_norm", (HV,)), ("conv_bias", (C,)), ("dt_bias", (heads,)), ("A", (heads,)), ("D", (heads,))):
            w = weights.get(name)
            if w is not None and w.shape != shape:
                raise ValueError(f"{name}: {list(w.shape)}, not {list(shape)}")
        taps = weights["taps"].shape
        if len(taps) != 2 or taps[0] != C or not 2 <= taps[1] <= 4:
            raise ValueError(f"taps: {list(taps)}, not [{C}][2 to 4]")

    def _project_in(self, x: Tensor, residual: Tensor):
        u, s, residual = ops.norm(x, self.norm, self.eps, residual=residual, out_dtype=ops.F8)
        N = self.in_proj.shape[0]
        # rows of whole 64 bytes, so that z, xBC and dt are read where they lie
        wide = torch.empty((x.shape[0], -(-N // 32) * 32), dtype=self.dtype, device=x.device)[:, :N]
        ops.matmul_fp8(u, s, self.in_proj, self.in_scale, out=wide)
        HV, C = self.inner, self.channels
        return wide[:, :HV], wide[:, HV:HV + C], wide[:, HV + C:], residual

    def _project_out(self, y: Tensor, z: Tensor, **skip) -> Tensor:
        u, s, _ = ops.norm(y, self.out_norm, self.eps, group=self.inner // self.groups, gate=z, out_dtype=ops.F8, **skip)
        return ops.matmul_fp8(u, s, self.out_proj, self.out_scale, out_dtype=self.dtype)

    def prefill(self, x: Tensor, residual: Tensor, offsets: Tensor | None = None) -> tuple[Tensor, Tensor]:
        """Packed prompts x [T][hidden] (one sequence per request, continuing
        where the convolution's states and `layer.S` stand) with the residual
        stream [T][hidden]: (out [T][hidden], the residual stream with x added).
        Leaves every request's state and sketch ready for `step`.  The states
        are those of the last flush: a window must not be open."""
        if self.layer.n:
            raise ValueError(f"prefill with {self.layer.n} tokens in the replay buffer: their updates are not in the state yet")
        HV, GK = self.inner, self.groups * self.dk
        z, xbc, dt, residual = self._project_in(x, residual)
        xbc, _ = ops.conv(xbc, self.taps, self.conv_bias, offsets=offsets, batch=self.batch, state=self.conv_state,
                          state_out=self.conv_state)
        y, _ = ops.scan(self.layer.cfg, self.groups, xbc[:, :HV], xbc[:, HV:HV + GK], xbc[:, HV + GK:], dt, self.dt_bias, self.A,
                        D=self.D, offsets=offsets, S=self.layer.S, S_out=self.layer.S)
        self.layer.init_sketch()
        return self._project_out(y, z), residual

    def step(self, x: Tensor, residual: Tensor) -> tuple[Tensor, Tensor]:
        """One token of every request, x and residual [batch][hidden]: (out, the
        residual stream with x added)."""
        lay = self.layer
        z, xbc, dt, residual = self._project_in(x, residual)
        n = lay.n
        ops.conv_token(lay.cfg, self.groups, xbc, self.taps, self.conv_bias, self.conv_state, dt, self.dt_bias, self.A,
                       lay.ring, n, self.q)
        o = lay.read(self.q)
        return self._project_out(o.view(self.batch, self.inner), z, skip=lay.rv[:, :, n], D=self.D), residual
