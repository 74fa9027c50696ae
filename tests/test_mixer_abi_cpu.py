"""The mixer operators' C ABI: the library exports what the header declares,
and invalid calls are refused on the host.  No compute call is made; the fake
addresses are never launched on (every case fails its checks), and the cases
are skipped where a GPU is visible."""
import ctypes
import os
import re

import pytest
import torch

from paper_2609_33051_amd import binding as B
from paper_2609_33051_amd import build as builder
from paper_2609_33051_amd import ops

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "sketchssm_mixer.h")
cpu_only = pytest.mark.skipif(torch.cuda.is_available(), reason="host checks use fake addresses; run on CPU only")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        builder.build()
    return B.load()


def at(k):  # fake, 16-byte aligned, 4 GiB apart
    return (k + 1) << 32


def cfg(**kw):
    d = dict(kind="mamba2", batch=2, heads=8, dk=128, dv=64, rank=16, window=16, io="bf16")
    d.update(kw)
    return B.make_config(*(d[x] for x in ("kind", "batch", "heads", "dk", "dv", "rank", "window", "io")))


def test_header_and_exports(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(sketchssm_\w+)\s*\(", text))
    assert names == set(B.MIXER_FUNCTIONS)
    for n in names:
        assert hasattr(lib, n)


def conv(lib, C=1024, w=4, io=1, silu=1, batch=2, T=64, off=at(1), x=at(2), ldx=1024, taps=at(3), bias=at(4), s_in=at(5), s_out=at(6),
         y=at(7), ldy=1024):
    return lib.sketchssm_conv(B.ConvConfig(C, w, io, silu), batch, T, off, x, ldx, taps, bias, s_in, s_out, y, ldy, None)


@cpu_only
def test_conv_refusals(lib):
    assert conv(lib, io=2) == -1 and conv(lib, C=0) == -1 and conv(lib, silu=2) == -1
    assert conv(lib, C=1020, ldx=1024) == -2 and conv(lib, w=1) == -2 and conv(lib, w=5) == -2
    assert conv(lib, batch=0) == -1 and conv(lib, T=-1) == -1 and conv(lib, T=1 << 31) == -2
    assert conv(lib, off=None, T=65) == -1
    assert conv(lib, ldx=1016) == -1 and conv(lib, ldy=1025) == -3
    assert conv(lib, x=None) == -1 and conv(lib, taps=None) == -1 and conv(lib, y=None) == -1
    assert conv(lib, x=at(2) + 8) == -3 and conv(lib, bias=at(4) + 4) == -3 and conv(lib, off=at(1) + 2) == -3
    assert conv(lib, y=at(2)) == -1 and "overlap" in B.sketchssm_last_error()
    assert conv(lib, y=at(5)) == -1 and conv(lib, s_out=at(2) + 1024) == -1
    assert conv(lib, s_in=at(5), s_out=at(5) + 2048) == -1


def token(lib, c=None, G=4, w=4, x=at(2), ldx=1536, taps=at(3), bias=None, state=at(4), dt=at(5) + 2, lddt=8, dt_bias=None, A=at(6), n=0,
          q=at(7), ring=None):
    ring = ring or B.make_ring(k=at(8), v=at(9), beta=at(10), log_decay=at(11))
    return lib.sketchssm_conv_token(c or cfg(), G, w, x, ldx, taps, bias, state, dt, lddt, dt_bias, A, ring, n, q, None)


@cpu_only
def test_conv_token_refusals(lib):
    assert token(lib, c=cfg(kind="gdn", dv=128)) == -2 and token(lib, c=cfg(dk=96)) == -2 and token(lib, c=cfg(batch=0)) == -1
    assert token(lib, G=3) == -1 and token(lib, G=0) == -1 and token(lib, w=5) == -2
    assert token(lib, n=16) == -4 and token(lib, n=-1) == -4
    for name in ("x", "taps", "state", "dt", "A", "q"):
        assert token(lib, **{name: None}) == -1, name
    assert token(lib, x=at(2) + 8) == -3 and token(lib, dt=at(5) + 1) == -3 and token(lib, state=at(4) + 2) == -3
    assert token(lib, ldx=1528) == -1 and token(lib, ldx=1537) == -3 and token(lib, lddt=7) == -1
    assert token(lib, ring=B.make_ring(k=at(8), v=at(9), beta=at(10))) == -1
    assert token(lib, q=at(2) + 16) == -1 and "overlap" in B.sketchssm_last_error()
    assert token(lib, dt=at(4)) == -1


@cpu_only
def test_conv_wide_and_token_overlaps(lib):
    wide = (1 << 31) - 8
    assert conv(lib, C=wide, ldx=1 << 31, ldy=1 << 31) == -2 and "2^30" in B.sketchssm_last_error()
    assert token(lib, c=cfg(heads=1 << 24, batch=1), G=1, ldx=1 << 31, lddt=1 << 24) == -2
    assert token(lib, q=at(4)) == -1 and "written overlap" in B.sketchssm_last_error()
    assert token(lib, ring=B.make_ring(k=at(8), v=at(8) + 64, beta=at(10), log_decay=at(11))) == -1
    assert token(lib, ring=B.make_ring(k=at(8), v=at(9), beta=at(10), log_decay=at(10))) == -1


def scan(lib, c=None, G=4, T=64, off=at(1), x=at(2), ldx=512, b=at(3), ldb=512, cc=at(4), ldc=512, dt=at(5), lddt=8, bias=None, A=at(6),
         D=None, s_in=None, s_out=at(7), y=at(8), ldy=512, ws=None, nws=0):
    return lib.sketchssm_scan(c or cfg(), G, T, off, x, ldx, b, ldb, cc, ldc, dt, lddt, bias, A, D, s_in, s_out, y, ldy, ws, nws, None)


@cpu_only
def test_scan_refusals(lib):
    assert scan(lib, c=cfg(kind="kda", dv=128)) == -2 and scan(lib, c=cfg(dv=32)) == -2
    assert scan(lib, G=5) == -1 and scan(lib, T=-1) == -1 and scan(lib, off=None, T=63) == -1
    for name in ("x", "b", "cc", "dt", "A", "s_out", "y"):
        assert scan(lib, **{name: None}) == -1, name
    assert scan(lib, x=at(2) + 2) == -3 and scan(lib, dt=at(5) + 1) == -3 and scan(lib, A=at(6) + 2) == -3
    assert scan(lib, ldx=504) == -1 and scan(lib, ldb=513) == -3 and scan(lib, lddt=7) == -1
    assert scan(lib, y=at(2)) == -1 and scan(lib, s_out=at(3)) == -1 and scan(lib, y=at(7)) == -1
    assert scan(lib, s_in=at(7) + 1024) == -1 and "overlap" in B.sketchssm_last_error()
    # one long sequence is split over workgroups: its workspace is required
    need = lib.sketchssm_scan_workspace(cfg(batch=1), 4, 1 << 16)
    assert need > 0
    assert scan(lib, c=cfg(batch=1), T=1 << 16) == -1 and "workspace" in B.sketchssm_last_error()
    assert scan(lib, c=cfg(batch=1), T=1 << 16, ws=at(20), nws=need - 1) == -1
    assert scan(lib, c=cfg(batch=1), T=1 << 16, ws=at(8), nws=need) == -1
    assert lib.sketchssm_scan_workspace(cfg(batch=1), 4, 64) == 0


@cpu_only
def test_scan_workspace_and_wide_strides(lib):
    for ld in ("ldx", "ldb", "ldc", "ldy"):
        assert scan(lib, **{ld: 1 << 24}) == -2 and "stride" in B.sketchssm_last_error()
    # sized before the lengths are known: more tokens never need less than their shares do
    for H, G in ((2, 1), (8, 4), (128, 8)):
        c = B.make_config("mamba2", 1, H, 128, 64, 16, 16, "bf16")
        assert lib.sketchssm_scan_workspace(c, G, 128) == 0 and lib.sketchssm_scan_workspace(c, G, 129) > 0
        for T in (129, 1000, 4096, 16384, 1 << 20):
            parts = G * -(-(H // G) // 2)
            assert lib.sketchssm_scan_workspace(c, G, T) <= (T // 64 + 1) * H * (128 * 64 + 1) * 4
            assert lib.sketchssm_scan_workspace(c, G, T) <= -(-1024 * H // parts + H) * (128 * 64 + 1) * 4


def norm_args(**kw):
    d = dict(rows=4, columns=512, group=512, x_dtype=1, io_dtype=1, out_dtype=2, eps=1e-5, x=at(1), ldx=512, weight=at(2), out=at(3),
             ld_out=512, scales=at(4), ld_scales=4)
    d.update(kw)
    a = B.NormArgs()
    for k, v in d.items():
        setattr(a, k, v)
    return a


@cpu_only
def test_norm_refusals(lib):
    n = lambda **kw: lib.sketchssm_norm(norm_args(**kw), None)  # noqa: E731
    res = dict(residual=at(5), ld_residual=512)
    gate = dict(gate=at(6), ld_gate=512)
    skip = dict(gate, skip=at(7), ld_skip=512, skip_head=64, skip_width=64, D=at(8))
    assert n(io_dtype=3) == -1 and n(x_dtype=2) == -1 and n(out_dtype=0) == -1 and n(rows=-1) == -1 and n(group=0) == -1
    assert n(group=384) == -1 and n(columns=516, group=516, ldx=520, ld_out=528) == -2
    assert n(columns=65536, group=65536, ldx=65536, ld_out=65536) == -2 and n(group=64) == -2
    assert n(eps=-1.0) == -1 and n(eps=float("nan")) == -1
    assert n(**res, **gate) == -1 and n(residual_out=at(9), ld_residual_out=512) == -1
    assert n(**{**skip, "gate": None}) == -1 and n(**{**skip, "D": None}) == -1 and n(**{**skip, "skip_width": 60}) == -1
    assert n(**{**skip, "skip_head": 56}) == -1 and n(**{**skip, "ld_skip": 504}) == -1
    assert n(ldx=504) == -1 and n(ldx=516) == -3 and n(ld_out=500) == -1 and n(ld_scales=3) == -1
    assert n(x=None) == -1 and n(weight=None) == -1 and n(scales=None) == -1 and n(x=at(1) + 8) == -3
    assert n(out=at(1)) == -1 and n(scales=at(3)) == -1
    assert n(**res, residual_out=at(1) + 64, ld_residual_out=512) == -1 and "overlap" in B.sketchssm_last_error()
    assert n(rows=0) == 0


def matmul(lib, M=4, N=256, K=256, a=at(1), lda=256, sa=at(2), ldsa=4, w=at(3), ldw=256, sw=at(4), out=1, y=at(5), ldy=256, ws=at(6),
           nws=1 << 30):
    return lib.sketchssm_matmul_fp8(M, N, K, a, lda, sa, ldsa, w, ldw, sw, out, y, ldy, ws, nws, None)


@cpu_only
def test_matmul_refusals(lib):
    assert matmul(lib, M=-1) == -1 and matmul(lib, N=0) == -1 and matmul(lib, K=0) == -1 and matmul(lib, K=250) == -2
    assert matmul(lib, out=2) == -1 and matmul(lib, lda=240) == -1 and matmul(lib, ldw=264) == -3
    assert matmul(lib, ldsa=3) == -1 and matmul(lib, ldy=255) == -1
    for name in ("a", "sa", "w", "sw", "y"):
        assert matmul(lib, **{name: None}) == -1, name
        assert matmul(lib, **{name: at(9) + 8}) == -3, name
    assert matmul(lib, y=at(3)) == -1 and "overlap" in B.sketchssm_last_error()
    assert matmul(lib, M=0) == 0


@cpu_only
def test_matmul_extreme_sizes(lib):
    assert lib.sketchssm_matmul_fp8_workspace(0, 256, 8192) == 0 and lib.sketchssm_matmul_fp8_workspace(-1, 256, 8192) == 0
    assert lib.sketchssm_matmul_fp8_workspace(1, (1 << 31) - 1, 256) == 0
    assert matmul(lib, M=1, N=(1 << 31) - 1, ldy=1 << 31) == -2
    assert matmul(lib, lda=1 << 24) == -2 and matmul(lib, ldw=1 << 24) == -2 and "stride" in B.sketchssm_last_error()
    # K split over workgroups: the workspace is required
    need = lib.sketchssm_matmul_fp8_workspace(16, 256, 8192)
    assert need > 0
    big = dict(M=16, K=8192, lda=8192, ldw=8192, ldsa=16)
    assert matmul(lib, **big, nws=need - 1) == -1 and "workspace" in B.sketchssm_last_error()
    assert matmul(lib, **big, ws=None) == -1 and matmul(lib, **big, ws=at(1)) == -1


@cpu_only
def test_ops_refuse_cpu_tensors(lib):
    x = torch.zeros(4, 64)
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        ops.conv(x, torch.zeros(64, 4))
    with pytest.raises((ValueError, RuntimeError, AssertionError)):
        ops.norm(x, torch.ones(64), 1e-5)


def test_quantize_weight():
    """Values over their block's scale: the largest of every block is 448, and
    a value is off by at most half a step (2^-4 of it, or half the smallest subnormal)."""
    from paper_2609_33051_amd.mixer import quantize_weight
    g = torch.Generator().manual_seed(3)
    w = torch.randn((200, 144), generator=g)
    w[:128, 128:] = 0.0
    q, s = quantize_weight(w)
    assert q.shape == w.shape and s.shape == (2, 2) and q.dtype is torch.float8_e4m3fn
    wide = s.repeat_interleave(128, 0)[:200].repeat_interleave(128, 1)[:, :144]
    assert (q.float() * wide - w).abs().le(w.abs() * 2.0 ** -4 * 1.001 + wide * 2.0 ** -10 * 1.001).all()
    assert q[:128, :128].float().abs().max() == 448.0 and s[0, 1] == 2.0 ** -64


def test_struct_sizes_match_c():
    """The ctypes mirror of skssm_norm_args has the C layout (offsets of its last fields, natural alignment)."""
    assert ctypes.sizeof(B.NormArgs) % 8 == 0 and B.NormArgs.eps.offset == 32 and B.NormArgs.x.offset == 40
    assert B.NormArgs.ld_scales.offset == ctypes.sizeof(B.NormArgs) - 8


@pytest.mark.parametrize("rows,columns", [(2, 8), (3, 1), (5, 100)])
def test_scale_rows_that_overlap_are_refused(rows, columns):
    """Rows of scales that share memory (broadcast, or a stride below their length): a stride
    of the row's length in their place would leave the array."""
    one = torch.ones((1, columns))
    for x in (one.expand(rows, columns), torch.ones(rows * columns).as_strided((rows, columns), (columns - 1, 1))):
        with pytest.raises(ValueError, match="scales"):
            ops._rows("scales", x, rows, columns, -1)
    assert ops._rows("scales", torch.ones((rows, columns + 3))[:, :columns], rows, columns, -1) == columns + 3
    assert ops._rows("scales", one, 1, columns, -1) >= columns
    assert ops._rows("scales", torch.ones((rows, 0)), rows, 0, -1) >= 0


@cpu_only
def test_launches_of_too_many_threads_are_refused(lib):
    """A launch holds fewer than 2^32 threads: sizes past that are refused before any launch, by the
    kernel's own workgroups (64 threads of a norm's narrow group, 256 of a convolution's or a product's tiles)."""
    def refused(rc):
        return rc == -2 and "one launch" in B.sketchssm_last_error()
    far = lambda k: (k + 1) << 44  # noqa: E731
    # a norm by groups of 64 columns, 8192 columns: a workgroup of 64 threads a group
    for kw in (dict(rows=1 << 19, columns=8192, group=64), dict(rows=1 << 23, columns=8192, group=64), dict(rows=1 << 26, columns=64, group=64),
               dict(rows=1 << 22, columns=32768, group=32768)):
        n = kw["columns"]
        for out in (dict(out_dtype=1, scales=None), dict(scales=far(4), ld_scales=kw["rows"])) if n == kw["group"] else (dict(out_dtype=1, scales=None),):
            assert refused(lib.sketchssm_norm(norm_args(**kw, **out, ldx=n, ld_out=n, x=far(1), weight=far(2), out=far(3)), None)), (kw, out)
    # a convolution: 64 lanes of 16 bytes a column of workgroups, 48 tokens a workgroup, and its states
    arrays = dict(x=far(1), taps=far(2), bias=far(3), s_in=far(4), s_out=far(5), y=far(6))
    assert refused(conv(lib, C=8, T=1 << 30, ldx=8, ldy=8, off=None, batch=1, **arrays))
    assert refused(conv(lib, C=8, T=0, ldx=8, ldy=8, batch=1 << 26, **arrays))
    assert refused(conv(lib, C=8, T=0, ldx=8, ldy=8, batch=1 << 26, **{**arrays, "s_in": far(5)}))
    assert refused(conv(lib, C=1 << 23, T=1 << 16, ldx=1 << 23, ldy=1 << 23, batch=1, **arrays))
    # a product of one row and 2^30 columns: 2^24 tiles of 64 columns
    assert refused(matmul(lib, M=1, N=1 << 30, K=16, lda=16, ldw=16, ldsa=1, out=0, ldy=1 << 30, a=far(1), sa=far(2), w=far(3), sw=far(4), y=far(5),
                          ws=far(6)))


def test_scan_workspace_of_many_heads_and_tokens(lib):
    """The shares of 2^30 tokens and 2^22 heads pass 32 bits: no sequence is split, and nothing is divided by their remainder."""
    for heads, T in ((1 << 22, 1 << 30), (1 << 13, 1 << 30), ((1 << 22) - 1, (1 << 30) - 1), (1 << 10, 1 << 30), (513, 1 << 20)):
        c = B.make_config("mamba2", 1, heads, 128, 64, 16, 16, "bf16")
        assert lib.sketchssm_scan_workspace(c, heads, T) == 0, (heads, T)
    c = B.make_config("mamba2", 1, 2, 128, 64, 16, 16, "bf16")
    assert lib.sketchssm_scan_workspace(c, 1, 1 << 30) > 0


@cpu_only
def test_outputs_over_parameters_are_refused(lib):
    """No output may lie over an array that other workgroups still read: taps, biases, offsets, A, D, weights."""
    def refused(rc):
        return rc == -1 and "overlap" in B.sketchssm_last_error()
    # convolution: y [64][1024] bf16, new states [2][3][1024] bf16
    for p in (dict(taps=at(7) + 1024), dict(bias=at(7) + 1024), dict(off=at(7) + 1024), dict(taps=at(6)), dict(bias=at(6) + 64), dict(off=at(6) + 64)):
        assert refused(conv(lib, **p)), p
    # one token: the ring's slots, q and the state
    for where in (at(4), at(7), at(8), at(9), at(10), at(11)):
        for name in ("taps", "bias", "dt_bias", "A"):
            assert refused(token(lib, **{name: where})), (name, where)
    # scan: y, S_out (and, where there is one, the workspace)
    for where in (at(7), at(8)):
        for name in ("off", "bias", "A", "D"):
            assert refused(scan(lib, **{name: where})), (name, where)
    need = lib.sketchssm_scan_workspace(cfg(batch=1), 4, 1 << 16)
    for name in ("off", "bias", "A", "D"):
        assert refused(scan(lib, c=cfg(batch=1), T=1 << 16, ws=at(20), nws=need, **{name: at(20) + 64})), name
    # norm: the output, its scales and the residual's sum
    res = dict(residual=at(5), ld_residual=512, residual_out=at(9), ld_residual_out=512)
    gate = dict(gate=at(6), ld_gate=512, skip=at(7), ld_skip=512, skip_head=64, skip_width=64)
    for where in (at(3), at(4), at(9)):
        assert refused(lib.sketchssm_norm(norm_args(weight=where, **res), None)), where
    for where in (at(3), at(4)):
        assert refused(lib.sketchssm_norm(norm_args(D=where, **gate), None)), where


def test_ops_refuse_counts_below_one(monkeypatch):
    """No group of no columns (it was taken for all of them), no batch below one, no offsets without an entry."""
    with pytest.raises(ValueError, match="offsets"):
        ops._offsets(torch.zeros(0, dtype=torch.int32), None, -1)
    for batch in (0, -1):
        with pytest.raises(ValueError, match="batch"):
            ops._offsets(None, batch, -1)
    assert ops._offsets(None, None, -1) == (1, None) and ops._offsets(None, 5, -1) == (5, None)
    # norm, as far as the call into the library: its group as it was given
    seen = []

    class Library:
        def sketchssm_norm(self, a, stream):
            seen.append(a.group)
            return 0
    monkeypatch.setattr(ops, "_device", lambda x: -1)
    monkeypatch.setattr(ops, "_stream", lambda dev: 0)
    monkeypatch.setattr(B, "_lib", Library())
    x, w = torch.zeros((2, 64)), torch.ones(64)
    for group in (None, 0, 32):
        ops.norm(x, w, 1e-5, group=group)
    assert seen == [64, 0, 32]  # (the library refuses 0)
