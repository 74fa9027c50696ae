"""Refusals of include/sketchssm_attention.h on the CPU: every check comes before any launch, so the pointers here are
numbers that are never read.  And what the attention layer refuses when it is made."""
import ctypes
import math

import pytest
import torch

from paper_2609_33051_amd import binding as B
from paper_2609_33051_amd import build
from paper_2609_33051_amd.attention import Attention, rotary_angles

EINVAL, EUNSUPPORTED, EALIGN = -1, -2, -3
M = 1 << 32  # addresses far apart


@pytest.fixture(scope="module")
def lib():
    import os
    if not os.path.exists(build.LIB):
        build.build()
    return B.load()


def fields(obj, kw):
    for k, v in kw.items():
        assert hasattr(obj, k), k
        setattr(obj, k, v)
    return obj


def cache(**kw):
    return fields(B.Cache(M, 10, 8, 64, 128), kw)


def seq(**kw):
    return fields(B.NewTokens(100, 2 * M, 3 * M, 4 * M, 5, 4, 5), kw)


def rot(**kw):
    return fields(B.Rotation(5 * M, None, 1000, 128, 0), kw)


def append_args(**kw):
    D = 128
    return fields(B.AppendArgs(B.BF16, 32, 6 * M, 8 * D, D, 7 * M, 8 * D, D, 8 * M, 32 * D, D, 9 * M, 32 * D, D), kw)


def attention_args(**kw):
    D = 128
    return fields(B.AttentionArgs(B.BF16, B.BF16, 32, 0.1, 6 * M, 32 * D, D, 7 * M, 32 * D, None, 0, 8 * M, 1 << 31), kw)


def says(lib, rc, code, text):
    assert rc == code, (rc, lib.sketchssm_last_error())
    assert text in lib.sketchssm_last_error().decode()


def test_every_function_is_exported_and_bound(lib):
    import re
    text = open(build.INCLUDE + "/sketchssm_attention.h").read()
    named = set(re.findall(r"\b(sketchssm_\w+)\(", text)) - {"sketchssm_last_error"}
    assert named - {"sketchssm_matmul_fp8"} == set(B.ATTENTION_FUNCTIONS)
    for f in B.ATTENTION_FUNCTIONS:
        assert getattr(lib, f).argtypes is not None


def test_struct_sizes():
    """The binding's blocks are laid out as the header's: 8-byte fields aligned, no tail beyond them."""
    assert ctypes.sizeof(B.Cache) == 24 and ctypes.sizeof(B.NewTokens) == 48 and ctypes.sizeof(B.Rotation) == 32
    assert ctypes.sizeof(B.AppendArgs) == 8 + 4 * 24 and ctypes.sizeof(B.AttentionArgs) == 16 + 9 * 8


def test_cache_bytes(lib):
    for D in (64, 96, 128, 192, 256):
        for page in (16, 64, 1024):
            assert lib.sketchssm_cache_bytes(B.Cache(None, 7, 3, page, D)) == 7 * 3 * (page // 16) * 17 * D
    big = B.Cache(None, 1 << 20, 8, 64, 128)
    assert lib.sketchssm_cache_bytes(big) == (1 << 20) * 8 * 4 * 17 * 128
    for kw, code, text in ((dict(dim=100), EUNSUPPORTED, "channels"), (dict(dim=32), EUNSUPPORTED, "channels"), (dict(page=8), EUNSUPPORTED, "pages of"),
                           (dict(page=48), EUNSUPPORTED, "power of two"), (dict(page=2048), EUNSUPPORTED, "power"), (dict(pages=0), EINVAL, "0 pages"),
                           (dict(kv_heads=0), EINVAL, "0 heads"), (dict(kv_heads=1 << 17), EUNSUPPORTED, "65536"),
                           (dict(pages=2 ** 31 - 1, kv_heads=1 << 16), EUNSUPPORTED, "too many")):
        assert lib.sketchssm_cache_bytes(cache(**kw)) == 0
        assert text in lib.sketchssm_last_error().decode()
        says(lib, lib.sketchssm_attention(cache(**kw), seq(), attention_args(), None), code, text)
        says(lib, lib.sketchssm_cache_append(cache(**kw), seq(), rot(), append_args(), None), code, text)
        says(lib, lib.sketchssm_cache_read(cache(**kw), seq(), B.BF16, 6 * M, 7 * M, None), code, text)


TOKENS = ((dict(batch=0), EINVAL, "batch"), (dict(tokens=-1), EINVAL, "tokens"), (dict(tokens=1 << 31), EUNSUPPORTED, "2^30"),
          (dict(offsets=None, tokens=101), EINVAL, "equal"), (dict(offsets=2 * M + 2), EALIGN, "offsets"), (dict(columns=0), EINVAL, "columns"),
          (dict(ld_table=4), EINVAL, "columns"), (dict(columns=1 << 25, ld_table=1 << 25), EUNSUPPORTED, "2^30"), (dict(lengths=None), EINVAL, "lengths"),
          (dict(table=None), EINVAL, "table"), (dict(table=4 * M + 1), EALIGN, "table"), (dict(lengths=3 * M + 3), EALIGN, "lengths"))


@pytest.mark.parametrize("kw,code,text", TOKENS)
def test_new_tokens(lib, kw, code, text):
    says(lib, lib.sketchssm_cache_append(cache(), seq(**kw), rot(), append_args(), None), code, text)
    says(lib, lib.sketchssm_cache_read(cache(), seq(**kw), B.BF16, 6 * M, 7 * M, None), code, text)
    says(lib, lib.sketchssm_attention(cache(), seq(**kw), attention_args(), None), code, text)


ROTATIONS = ((dict(places=0), EINVAL, "places"), (dict(rotated=0), EINVAL, "rotated"), (dict(rotated=33), EINVAL, "even"), (dict(rotated=130), EINVAL, "130"),
             (dict(interleaved=2), EINVAL, "interleaved"), (dict(angles=5 * M + 4), EALIGN, "aligned"), (dict(positions=M + 2), EALIGN, "positions"))


@pytest.mark.parametrize("kw,code,text", ROTATIONS)
def test_rotations(lib, kw, code, text):
    says(lib, lib.sketchssm_cache_append(cache(), seq(), rot(**kw), append_args(), None), code, text)
    says(lib, lib.sketchssm_rotary(B.BF16, 10, 4, 128, rot(**kw), 6 * M, 512, 128, 7 * M, 512, 128, None), code, text)


def test_rotary(lib):
    call = lambda io=B.BF16, T=10, H=4, D=128, r=rot(), x=6 * M, ldx=512, xh=128, y=7 * M, ldy=512, yh=128: lib.sketchssm_rotary(  # noqa: E731
        io, T, H, D, r, x, ldx, xh, y, ldy, yh, None)
    for kw, code, text in ((dict(io=2), EINVAL, "io_dtype"), (dict(T=-1), EINVAL, "tokens"), (dict(H=0), EINVAL, "heads"), (dict(D=12), EUNSUPPORTED, "12"),
                           (dict(D=520), EUNSUPPORTED, "512"), (dict(r=None), EINVAL, "angles"), (dict(r=rot(angles=None)), EINVAL, "angles"),
                           (dict(x=None), EINVAL, "x is required"), (dict(y=None), EINVAL, "y is required"), (dict(x=6 * M + 8), EALIGN, "aligned"),
                           (dict(ldx=500), EINVAL, "stride"), (dict(ldx=513), EALIGN, "stride"), (dict(xh=120), EINVAL, "head stride"),
                           (dict(xh=129), EALIGN, "head stride"), (dict(ldy=1 << 31), EUNSUPPORTED, "2^30"), (dict(y=6 * M + 1024), EINVAL, "overlaps"),
                           (dict(y=6 * M, ldy=520), EINVAL, "overlaps"), (dict(y=5 * M + 16), EINVAL, "overlaps")):
        says(lib, call(**kw), code, text)
    assert call(T=0) == 0 and call(T=0, x=None, y=None) == 0


def test_append(lib):
    call = lambda r=rot(), **kw: lib.sketchssm_cache_append(cache(), seq(), r, append_args(**kw), None)  # noqa: E731
    says(lib, lib.sketchssm_cache_append(None, seq(), rot(), append_args(), None), EINVAL, "cache is NULL")
    says(lib, lib.sketchssm_cache_append(cache(), None, rot(), append_args(), None), EINVAL, "seq is NULL")
    says(lib, lib.sketchssm_cache_append(cache(), seq(), rot(), None, None), EINVAL, "args is NULL")
    says(lib, lib.sketchssm_cache_append(cache(data=None), seq(), rot(), append_args(), None), EINVAL, "data")
    says(lib, lib.sketchssm_cache_append(cache(data=M + 8), seq(), rot(), append_args(), None), EALIGN, "aligned")
    for kw, code, text in ((dict(io_dtype=7), EINVAL, "io_dtype"), (dict(r=None), EINVAL, "without angles"), (dict(q_out=None), EINVAL, "q_out"),
                           (dict(heads=0), EINVAL, "heads"), (dict(k=None), EINVAL, "k is required"), (dict(v=None), EINVAL, "v is required"),
                           (dict(ldk=1000), EINVAL, "k stride"), (dict(v_head=64), EINVAL, "v head"), (dict(ldq=32 * 128 + 4), EALIGN, "q stride"),
                           (dict(v=7 * M + 2), EALIGN, "aligned"), (dict(q_out=6 * M), EINVAL, "overlaps"), (dict(k=M + 1024), EINVAL, "overlaps"),
                           (dict(q=M + 1024), EINVAL, "overlaps"), (dict(q_out=M + 1024), EINVAL, "overlap"), (dict(q_out=8 * M + 16), EINVAL, "overlaps"),
                           (dict(q_out=3 * M), EINVAL, "overlaps"), (dict(q_out=5 * M), EINVAL, "overlaps")):
        says(lib, call(**kw), code, text)
    # queries, keys and values side by side: the queries may be turned where they lie, but not into a row's keys or values
    W = 48 * 128
    wide = dict(ldq=W, ld_qout=W, ldk=W, ldv=W, q=6 * M, q_out=6 * M, k=6 * M + 32 * 256, v=6 * M + 40 * 256)
    for kw in (dict(k=6 * M + 31 * 256), dict(v=6 * M + 41 * 256), dict(q=6 * M + 256), dict(ldk=W + 8)):
        says(lib, call(**{**wide, **kw}), EINVAL, "overlaps")
    assert lib.sketchssm_cache_append(cache(), seq(tokens=0), rot(), append_args(k=None, v=None, q=None), None) == 0


def test_read(lib):
    call = lambda k=6 * M, v=7 * M, io=B.BF16: lib.sketchssm_cache_read(cache(), seq(), io, k, v, None)  # noqa: E731
    for kw, code, text in ((dict(io=3), EINVAL, "io_dtype"), (dict(k=6 * M + 4), EALIGN, "aligned"), (dict(k=M), EINVAL, "overlaps"),
                           (dict(v=3 * M), EINVAL, "overlaps"), (dict(v=6 * M + 64), EINVAL, "overlap")):
        says(lib, call(**kw), code, text)
    assert call(None, None) == 0 and lib.sketchssm_cache_read(cache(), seq(tokens=0), B.BF16, None, None, None) == 0


def test_attention(lib):
    call = lambda **kw: lib.sketchssm_attention(cache(), seq(), attention_args(**kw), None)  # noqa: E731
    says(lib, lib.sketchssm_attention(cache(), seq(), None, None), EINVAL, "args is NULL")
    f8 = dict(out_dtype=B.E4M3, scales=9 * M, ld_scales=100)
    for kw, code, text in ((dict(io_dtype=2), EINVAL, "io_dtype"), (dict(out_dtype=B.F32), EINVAL, "out_dtype"), (dict(heads=12), EINVAL, "divide"),
                           (dict(heads=0), EINVAL, "divide"), (dict(heads=1 << 27), EUNSUPPORTED, "2^30 rows"), (dict(scale=0.0), EINVAL, "scale"), (dict(scale=-1.0), EINVAL, "scale"),
                           (dict(scale=math.inf), EINVAL, "scale"), (dict(scale=math.nan), EINVAL, "scale"), (dict(q=None), EINVAL, "q is required"),
                           (dict(ldq=32 * 128 - 8), EINVAL, "q stride"), (dict(q_head=132), EALIGN, "q head"), (dict(ld_out=100), EINVAL, "out stride"),
                           (dict(ld_out=32 * 128 + 4), EALIGN, "out stride"), (dict(ld_out=1 << 31), EUNSUPPORTED, "2^30"), (dict(out=None), EINVAL, "out"),
                           (dict(out=7 * M + 8), EALIGN, "aligned"), (dict(workspace=None), EINVAL, "workspace of 0"), (dict(workspace_bytes=1000), EINVAL, "workspace of 1000"),
                           (dict(out=6 * M), EINVAL, "overlaps"), (dict(out=M), EINVAL, "overlaps"), (dict(workspace=6 * M), EINVAL, "overlaps"),
                           (dict(workspace=7 * M), EINVAL, "overlap"), (dict(f8, scales=None), EINVAL, "scales"), (dict(f8, ld_scales=99), EINVAL, "scales stride"),
                           (dict(f8, scales=9 * M + 2), EALIGN, "scales"), (dict(f8, scales=7 * M), EINVAL, "overlap")):
        says(lib, call(**kw), code, text)
    for D, H, G, good in ((96, 8, 2, False), (192, 8, 2, False), (64, 6, 2, False), (64, 8, 2, True), (128, 8, 8, True), (256, 3, 1, True)):
        c, a = cache(dim=D, kv_heads=G), attention_args(heads=H, q_head=D, ldq=H * D, ld_out=H * D, **f8)
        a.out = None  # a check after the one looked for
        rc = lib.sketchssm_attention(c, seq(), a, None)
        assert rc == (EINVAL if good else EUNSUPPORTED), (D, H, G, lib.sketchssm_last_error())
    assert lib.sketchssm_attention(cache(), seq(tokens=0), attention_args(q=None, out=None, workspace=None, workspace_bytes=0), None) == 0


def test_workspace(lib):
    """None where nothing can be split: no keys for two rounds, or rows that fill the chip's workgroups; single tokens are
    split however many there are.  The sizes stay within what a
    chip's workgroups leave, whatever the batch."""
    w = lambda c=cache(), H=32, batch=4, T=4, columns=5: lib.sketchssm_attention_workspace(c, H, batch, T, columns)  # noqa: E731
    assert w() > 0 and w(columns=2) == 0 and w(T=200000) == 0
    assert w(H=12) == 0 and w(batch=0) == 0 and w(T=0) == 0 and w(columns=0) == 0
    for D in (64, 96, 128, 192, 256):
        for batch, T in ((1, 1), (64, 64), (1000, 1000), (3, 300)):
            n = w(cache(dim=D), 32, batch, T, 4096)
            assert 0 < n <= 256 * 4 * 2 * 32 * (D + 2) * 4 + (batch + 4) * 4
    assert w(T=1, batch=1, columns=4) < w(T=64, batch=64, columns=4096)


# ---- the layer and its table


def make(heads=8, kv_heads=2, dim=128, hidden=64, rotation=None, **kw):
    w = dict(norm=torch.ones(hidden), qkv_proj=torch.zeros((heads + 2 * max(kv_heads, 0)) * dim, hidden), out_proj=torch.zeros(hidden, heads * dim))
    w.update(kw)
    return Attention(w, heads, kv_heads, dim, 4, 16, rotation, device="cpu")


@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 2, 128), (8, 8, 128), (4, 2, 64), (3, 1, 256)])
def test_layers_that_run_are_taken(heads, kv_heads, dim):
    m = make(heads, kv_heads, dim)
    assert m.cache.shape == (4, kv_heads, 1, 17 * dim) and m.cache.dtype is torch.uint8


def test_layer_refusals():
    for kw, text in ((dict(heads=8, kv_heads=3), "divide"), (dict(kv_heads=0), "divide"), (dict(dim=96), "channels"), (dict(heads=6, kv_heads=2, dim=64), "even"),
                     (dict(hidden=72), "16"), (dict(qkv_proj=torch.zeros(100, 64)), "qkv_proj"), (dict(out_proj=torch.zeros(64, 128)), "out_proj"),
                     (dict(norm=torch.ones(32)), "norm"), (dict(rotation=torch.zeros(10, 130)), "rotation"), (dict(rotation=torch.zeros(10)), "rotation"),
                     (dict(rotation=torch.zeros(10, 3)), "rotation")):
        with pytest.raises(ValueError, match=text):
            make(**kw)
    with pytest.raises(B.SketchSSMError, match="pages"):
        w = dict(norm=torch.ones(64), qkv_proj=torch.zeros(12 * 128, 64), out_proj=torch.zeros(64, 1024))
        Attention(w, 8, 2, 128, 4, 24, device="cpu")


def test_rotary_angles():
    """Against complex powers, far places included; interpolated and by parts against the definition, frequency by frequency."""
    t = rotary_angles(200000, 64, 1e6, device="cpu")
    assert t.shape == (200000, 64) and t.dtype is torch.float32
    for p in (0, 1, 77, 199999):
        for i in (0, 1, 13, 31):
            a = p * 1e6 ** (-2 * i / 64)
            # fp32's rounding of the result; the angle in 64 bits is p 2^-53 off
            assert abs(float(t[p, i]) - math.cos(a)) <= 2.0 ** -24 + p * 2.0 ** -50 and abs(float(t[p, 32 + i]) - math.sin(a)) <= 2.0 ** -24 + p * 2.0 ** -50
    s = rotary_angles(1000, 32, factor=4.0, device="cpu")
    # angles over four: rows 4 p are those of p unscaled, but for the last place of an angle of up to 250
    assert torch.allclose(s[::4], rotary_angles(250, 32, device="cpu"), rtol=0, atol=2.0 ** -23)
    y = rotary_angles(5000, 64, 10000.0, factor=8.0, original=2048, device="cpu")
    m = 1 + 0.1 * math.log(8.0)
    for i in range(32):
        f = 10000.0 ** (-2 * i / 64)
        turns = 2048 * f / (2 * math.pi)
        k = min(max((turns - 1.0) / 31.0, 0.0), 1.0)
        a = 4999 * (k * f + (1 - k) * f / 8.0)
        assert abs(float(y[4999, i]) - m * math.cos(a)) <= 2.0 ** -23 and abs(float(y[4999, 32 + i]) - m * math.sin(a)) <= 2.0 ** -23
    assert float(rotary_angles(3, 8, factor=8.0, original=10, magnitude=1.0, device="cpu")[0, 0]) == 1.0
    for kw in (dict(places=0, dim=4), dict(places=3, dim=5), dict(places=3, dim=4, base=0.0), dict(places=3, dim=4, factor=0.5), dict(places=3, dim=4, original=0),
               dict(places=3, dim=4, original=9, low=3.0, high=2.0)):
        with pytest.raises(ValueError):
            rotary_angles(device="cpu", **kw)
