"""The operators around the recurrence of a Mamba-2 mixer layer, on torch
tensors (include/sketchssm_mixer.h through `binding`): the short causal
convolution and the selective scan of packed prompts, one token of every
request into the decode path's replay buffer, root-mean-square norms that end
in 8 bits, and products of 8-bit matrices.  And those of a softmax attention
layer between mixer layers (include/sketchssm_attention.h): rotary positions,
a paged cache of keys and values in 4 bits, attention over it.

torch supplies device memory and the current stream; every computation is a
call into libsketchssm.so.  Tensors are on the current device; matrices are
read where they lie as long as their rows are contiguous (any row stride of
whole 16-byte pieces).  Outputs and workspaces are allocated where the caller
gives none.  A tensor of the wrong type, shape, device or layout raises
ValueError; what the library itself refuses raises SketchSSMError.  Results
carry no gradient history: there is no backward pass.

Types: io is bfloat16 or float32; parameters (taps, biases, weights, A, D) and
scales are float32, 8-bit values torch.float8_e4m3fn, offsets int32.
"""
from __future__ import annotations

import torch
from torch import Tensor

from . import binding as B

F8 = torch.float8_e4m3fn
_F32 = torch.float32
_IO = {torch.float32: B.F32, torch.bfloat16: B.BF16}


# The current device and its current stream's handle: as torch.cuda.current_device()
# and current_stream(), of which the latter takes 2.9 us (a whole call here, launch
# included, takes 6 to 10).
try:
    from torch._C import _cuda_getCurrentRawStream as _stream
    from torch._C import _cuda_getDevice as _current
except ImportError:  # a build of torch without these
    _current = torch.cuda.current_device

    def _stream(dev: int) -> int:
        return torch.cuda.current_stream(dev).cuda_stream


def _io(x: Tensor) -> int:
    io = _IO.get(x.dtype)
    if io is None:
        raise ValueError(f"{x.dtype}: bfloat16 or float32 is read")
    return io


def _matrix(name: str, x: Tensor, shape: tuple, dtype, dev: int) -> int:
    """The row stride of a matrix whose rows are contiguous."""
    s = x.stride()
    if x.shape == shape and x.dtype is dtype and x.get_device() == dev and s[1] == 1 and s[0] >= shape[1] and shape[0] > 1:
        return s[0]
    if x.shape != shape or x.dtype is not dtype or x.get_device() != dev:
        raise ValueError(f"{name}: a {dtype} tensor {list(shape)} on cuda:{dev} is needed, not {_said(x)}")
    if s[1] != 1 and shape[1] > 1:
        raise ValueError(f"{name}: its rows are not contiguous ({_said(x)})")
    if shape[0] > 1 and shape[1] == 1 and s[0] > 0:
        return s[0]
    if shape[0] > 1:
        raise ValueError(f"{name}: its rows overlap ({_said(x)})")
    return -(-shape[1] // 16) * 16  # at most one row: any stride


def _flat(name: str, x: Tensor | None, shape: tuple, dtype, dev: int) -> int | None:
    """The address of a contiguous tensor (None passes)."""
    if x is None:
        return None
    if x.shape == shape and x.dtype is dtype and x.is_contiguous() and x.get_device() == dev:
        return x.data_ptr()
    raise ValueError(f"{name}: a contiguous {dtype} tensor {list(shape)} on cuda:{dev} is needed, not {_said(x)}")


def _said(x: Tensor) -> str:
    return f"{x.dtype} {list(x.shape)} strides {list(x.stride())} on {x.device}"


def _device(x: Tensor) -> int:
    dev = x.get_device()
    if dev < 0 or dev != _current():
        raise ValueError(f"{x.device}: tensors on the current GPU are read")
    return dev


def _offsets(offsets: Tensor | None, batch: int | None, dev: int) -> tuple[int, int | None]:
    """(sequences, address of their offsets or None)"""
    if batch is not None and batch < 1:
        raise ValueError(f"a batch of {batch}")
    if offsets is None:
        return (1 if batch is None else batch), None
    n = offsets.numel() - 1
    if n < 1:
        raise ValueError(f"offsets: {n + 1} entries, one more than the sequences are needed")
    if batch is not None and batch != n:
        raise ValueError(f"offsets of {n} sequences for a batch of {batch}")
    return n, _flat("offsets", offsets, (n + 1,), torch.int32, dev)


def conv(x: Tensor, taps: Tensor, bias: Tensor | None = None, *, offsets: Tensor | None = None, batch: int | None = None,
         state: Tensor | None = None, state_out: Tensor | None = None, silu: bool = True,
         out: Tensor | None = None) -> tuple[Tensor, Tensor]:
    """The depthwise causal convolution of packed prompts: (y, the sequences'
    new states).  x [T][C] io, taps [C][w] with w 2..4, bias [C]; sequence b is
    rows offsets[b] .. offsets[b+1]-1 (None: `batch` equal sequences, one by
    default); state [batch][w-1][C] holds the inputs before each sequence
    (None: zeros) and may be `state_out` itself."""
    dev = _device(x)
    io = _io(x)
    if x.dim() != 2 or taps.dim() != 2:
        raise ValueError("x [T][C] and taps [C][w] are needed")
    T, C = x.shape
    w = taps.shape[1]
    n, off = _offsets(offsets, batch, dev)
    ldx = _matrix("x", x, (T, C), x.dtype, dev)
    shape = (n, w - 1, C)
    if out is None:
        out = x.new_empty((T, C))
    if state_out is None:
        state_out = x.new_empty(shape)
    rc = (B._lib or B.load()).sketchssm_conv(B.ConvConfig(C, w, io, 1 if silu else 0), n, T, off, x.data_ptr(), ldx,
                                 _flat("taps", taps, (C, w), _F32, dev), _flat("bias", bias, (C,), _F32, dev),
                                 _flat("state", state, shape, x.dtype, dev), _flat("state_out", state_out, shape, x.dtype, dev),
                                 out.data_ptr(), _matrix("out", out, (T, C), x.dtype, dev), _stream(dev))
    if rc:
        B._check(rc)
    return out, state_out


def conv_token(cfg: B.Config, groups: int, x: Tensor, taps: Tensor, bias: Tensor | None, state: Tensor, dt: Tensor,
               dt_bias: Tensor | None, A: Tensor, ring: B.Ring, n_buffered: int, q: Tensor) -> None:
    """One token of every request into slot n_buffered of the replay buffer and
    into q, ready for the read of that slot: the convolution with SiLU over x
    [B][H V + 2 G K] (the channels of x, B and C), whose state [B][w-1][C]
    moves on in place; beta = softplus(dt + dt_bias) and log decay beta A."""
    dev = _device(x)
    _io(x)
    Bt, H, K, V = cfg.batch, cfg.heads, cfg.dk, cfg.dv
    C, w, t = H * V + 2 * groups * K, taps.shape[-1], x.dtype
    if _IO[t] != cfg.io_dtype:
        raise ValueError(f"x is {t}: not the io type of the configuration")
    ldx, lddt = _matrix("x", x, (Bt, C), t, dev), _matrix("dt", dt, (Bt, H), t, dev)
    rc = (B._lib or B.load()).sketchssm_conv_token(cfg, groups, w, x.data_ptr(), ldx, _flat("taps", taps, (C, w), _F32, dev),
                                       _flat("bias", bias, (C,), _F32, dev), _flat("state", state, (Bt, w - 1, C), t, dev),
                                       dt.data_ptr(), lddt, _flat("dt_bias", dt_bias, (H,), _F32, dev),
                                       _flat("A", A, (H,), _F32, dev), ring, n_buffered,
                                       _flat("q", q, (Bt, H, K), t, dev), _stream(dev))
    if rc:
        B._check(rc)


def scan(cfg: B.Config, groups: int, x: Tensor, b: Tensor, c: Tensor, dt: Tensor, dt_bias: Tensor | None, A: Tensor, *,
         D: Tensor | None = None, offsets: Tensor | None = None, S: Tensor | None = None, S_out: Tensor | None = None,
         out: Tensor | None = None, workspace: Tensor | None = None) -> tuple[Tensor, Tensor]:
    """The selective scan of packed prompts: (y [T][H V], the states each
    sequence ends in).  x [T][H V], b and c [T][G K], dt [T][H] io; A, D and
    dt_bias [H]; cfg gives batch, heads, dk, dv and the io type.  S (None:
    zeros) and S_out are states [B][H][V K] in the library's tile-major layout,
    as `SketchSSMLayer.S` holds them; S_out may be S."""
    dev = _device(x)
    _io(x)
    Bt, H, K, V = cfg.batch, cfg.heads, cfg.dk, cfg.dv
    t, T, GK = x.dtype, x.shape[0], groups * K
    if _IO[t] != cfg.io_dtype:
        raise ValueError(f"x is {t}: not the io type of the configuration")
    n, off = _offsets(offsets, Bt, dev)
    ldx = _matrix("x", x, (T, H * V), t, dev)
    shape = (Bt, H, V * K)
    if out is None:
        out = x.new_empty((T, H * V))
    if S_out is None:
        S_out = x.new_empty(shape, dtype=_F32)
    lib = B._lib or B.load()
    need = lib.sketchssm_scan_workspace(cfg, groups, T)
    if workspace is None and need:
        workspace = x.new_empty(need, dtype=torch.uint8)
    rc = lib.sketchssm_scan(cfg, groups, T, off, x.data_ptr(), ldx, b.data_ptr(), _matrix("b", b, (T, GK), t, dev), c.data_ptr(),
                            _matrix("c", c, (T, GK), t, dev), dt.data_ptr(), _matrix("dt", dt, (T, H), t, dev),
                            _flat("dt_bias", dt_bias, (H,), _F32, dev), _flat("A", A, (H,), _F32, dev),
                            _flat("D", D, (H,), _F32, dev), _flat("S", S, shape, _F32, dev),
                            _flat("S_out", S_out, shape, _F32, dev), out.data_ptr(), _matrix("out", out, (T, H * V), t, dev),
                            *_space(workspace, dev), _stream(dev))
    if rc:
        B._check(rc)
    return out, S_out


def _space(workspace: Tensor | None, dev: int) -> tuple[int | None, int]:
    if workspace is None:
        return None, 0
    if workspace.get_device() != dev or not workspace.is_contiguous():
        raise ValueError(f"workspace: a contiguous tensor on cuda:{dev} is needed, not {_said(workspace)}")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def norm(x: Tensor, weight: Tensor, eps: float, *, group: int | None = None, residual: Tensor | None = None,
         residual_out: Tensor | None = None, gate: Tensor | None = None, skip: Tensor | None = None, D: Tensor | None = None,
         out_dtype=None, out: Tensor | None = None,
         scales: Tensor | None = None) -> tuple[Tensor, Tensor | None, Tensor | None]:
    """Root-mean-square norm of x, of x + residual, or of (x + D skip)
    silu(gate), over groups of columns (all of them by default), times weight:
    (out, scales, residual_out).

    out_dtype None: the io type (gate's or residual's, else x's); F8: blocks of
    128 columns over their scale, scales [ceil(N / 128)][M] (what matmul_fp8
    reads).  x may be float32 beside bfloat16 gates and residuals.  With
    `residual` the sum is returned too, in the io type (residual_out; it may be
    x or residual).  skip is [M][heads][width] (strided as the replay buffer's
    slots are) with D [heads]."""
    dev = _device(x)
    if x.dim() != 2:
        raise ValueError("x [M][N] is needed")
    M, N = x.shape
    other = gate if gate is not None else residual
    t = x.dtype if other is None else other.dtype
    if out_dtype is None:
        out_dtype = t
    f8 = out_dtype is F8
    io = _IO.get
    a = B.NormArgs(M, N, N if group is None else group, io(x.dtype, -1), io(t, -1), B.E4M3 if f8 else io(out_dtype, -1), 0, eps, x.data_ptr(),
                   _matrix("x", x, (M, N), x.dtype, dev))
    a.weight = _flat("weight", weight, (N,), _F32, dev)
    if residual is not None:
        a.residual, a.ld_residual = residual.data_ptr(), _matrix("residual", residual, (M, N), t, dev)
        if residual_out is None:
            residual_out = residual.new_empty((M, N))
    if residual_out is not None:
        a.residual_out, a.ld_residual_out = residual_out.data_ptr(), _matrix("residual_out", residual_out, (M, N), t, dev)
    if gate is not None:
        a.gate, a.ld_gate = gate.data_ptr(), _matrix("gate", gate, (M, N), t, dev)
    if skip is not None:
        if (skip.dim() != 3 or skip.dtype is not t or skip.get_device() != dev or skip.shape[0] != M
                or skip.shape[1] * skip.shape[2] != N or skip.stride(2) != 1):
            raise ValueError(f"skip: a {t} tensor [{M}][heads][width] of {N} values a row is needed, not {_said(skip)}")
        a.skip_width, a.skip, a.skip_head = skip.shape[2], skip.data_ptr(), skip.stride(1)
        a.ld_skip = skip.stride(0) if M > 1 else max(skip.stride(0), skip.stride(1) * skip.shape[1])
        a.D = _flat("D", D, (skip.shape[1],), _F32, dev)
    elif D is not None:
        raise ValueError("D without skip")
    if out is None:
        out, a.ld_out = x.new_empty((M, N), dtype=out_dtype), N
    else:
        a.ld_out = _matrix("out", out, (M, N), out_dtype, dev)
    a.out = out.data_ptr()
    if f8:
        if scales is None:
            scales, a.ld_scales = x.new_empty((-(-N // 128), M), dtype=_F32), M
        else:
            a.ld_scales = _rows("scales", scales, -(-N // 128), M, dev)
        a.scales = scales.data_ptr()
    elif scales is not None:
        raise ValueError("scales without an 8-bit output")
    rc = (B._lib or B.load()).sketchssm_norm(a, _stream(dev))
    if rc:
        B._check(rc)
    return out, scales, residual_out


def _rows(name: str, x: Tensor, rows: int, columns: int, dev: int) -> int:
    """The row stride of a float32 matrix of scales."""
    if (x.dim() != 2 or x.shape[0] != rows or x.shape[1] != columns or x.dtype is not _F32 or x.get_device() != dev
            or x.stride(1) != 1 and columns > 1 or x.stride(0) < columns and rows > 1):
        raise ValueError(f"{name}: a {_F32} tensor [{rows}][{columns}] with contiguous rows that do not overlap on cuda:{dev} is needed, "
                         f"not {_said(x)}")
    return x.stride(0) if rows > 1 else columns


def matmul_fp8(a: Tensor, a_scale: Tensor, w: Tensor, w_scale: Tensor, *, out_dtype=torch.bfloat16, out: Tensor | None = None,
               workspace: Tensor | None = None) -> Tensor:
    """y = a w^T with block scales: a [M][K] and w [N][K] e4m3, a_scale
    [ceil(K / 128)][M], w_scale [ceil(N / 128)][ceil(K / 128)]; y [M][N] in
    bfloat16 or float32."""
    dev = _device(a)
    if a.dim() != 2 or w.dim() != 2:
        raise ValueError("a [M][K] and w [N][K] are needed")
    M, K = a.shape
    N = w.shape[0]
    kb = -(-K // 128)
    if out is None:
        out = a.new_empty((M, N), dtype=out_dtype)
    t = out.dtype
    if out.shape != (M, N) or t not in _IO or out.get_device() != dev or out.stride(1) != 1 and N > 1:
        raise ValueError(f"out: a bfloat16 or float32 tensor [{M}][{N}] with contiguous rows is needed, not {_said(out)}")
    lib = B._lib or B.load()
    need = lib.sketchssm_matmul_fp8_workspace(M, N, K)
    if workspace is None and need:
        workspace = a.new_empty(need, dtype=torch.uint8)
    rc = lib.sketchssm_matmul_fp8(M, N, K, a.data_ptr(), _matrix("a", a, (M, K), F8, dev), a_scale.data_ptr(),
                                  _rows("a_scale", a_scale, kb, M, dev), w.data_ptr(), _matrix("w", w, (N, K), F8, dev),
                                  _flat("w_scale", w_scale, (-(-N // 128), kb), _F32, dev), _IO[t], out.data_ptr(),
                                  out.stride(0) if M > 1 else N, *_space(workspace, dev), _stream(dev))
    if rc:
        B._check(rc)
    return out


# ---- the softmax attention layer's operators


def _heads(name: str, x: Tensor, shape: tuple, dtype, dev: int) -> tuple[int, int]:
    """(token stride, head stride) of an array [T][heads][dim] whose channels are contiguous."""
    if x.shape != shape or x.dtype is not dtype or x.get_device() != dev:
        raise ValueError(f"{name}: a {dtype} tensor {list(shape)} on cuda:{dev} is needed, not {_said(x)}")
    T, H, D = shape
    t, h, c = x.stride()
    if c != 1 or H > 1 and h < D:
        raise ValueError(f"{name}: its heads are not contiguous or overlap ({_said(x)})")
    if H == 1:
        h = -(-D // 16) * 16  # one head: any stride
    row = (H - 1) * h + D
    if T > 1 and t < row:
        raise ValueError(f"{name}: its rows overlap ({_said(x)})")
    return (t if T > 1 else -(-row // 16) * 16), h


def _rotation(angles: Tensor, positions: Tensor | None, interleaved: bool, tokens: int, dev: int) -> B.Rotation:
    shape = angles.shape
    if len(shape) != 2:
        raise ValueError("rotation [places][rotated] is needed")
    return B.Rotation(_flat("rotation", angles, shape, _F32, dev), _flat("positions", positions, (tokens,), torch.int32, dev), *shape,
                      1 if interleaved else 0)


def rotary(x: Tensor, rotation: Tensor, positions: Tensor | None = None, *, interleaved: bool = False, out: Tensor | None = None) -> Tensor:
    """x [T][heads][dim] io (dim a multiple of 8, up to 512) with the leading channels of every head rotated in
    pairs: (i, i + R / 2), or (2 i, 2 i + 1) if interleaved.  rotation
    [places][R] holds each place's cosines and then its sines
    (`attention.rotary_angles` makes one); positions [T] int32 names each
    token's row (None: row t).  A position outside the table turns into NaN.
    `out` may be x."""
    dev = _device(x)
    io = _io(x)
    if x.dim() != 3:
        raise ValueError("x [T][heads][dim] is needed")
    T, H, D = shape = x.shape
    if out is None:
        out, t, h = x.new_empty(shape), H * D, D
    else:
        t, h = _heads("out", out, shape, x.dtype, dev)
    rc = (B._lib or B.load()).sketchssm_rotary(io, T, H, D, _rotation(rotation, positions, interleaved, T, dev), x.data_ptr(),
                                               *_heads("x", x, shape, x.dtype, dev), out.data_ptr(), t, h, _stream(dev))
    if rc:
        B._check(rc)
    return out


def new_cache(pages: int, kv_heads: int, page: int, dim: int, device="cuda") -> Tensor:
    """An empty cache of keys and values in 4 bits: [pages][kv_heads][page / 16][17 dim] bytes
    (records of 16 tokens of a head, as include/sketchssm_attention.h lays them out)."""
    if not (B._lib or B.load()).sketchssm_cache_bytes(B.Cache(None, pages, kv_heads, page, dim)):
        raise B.SketchSSMError(-2, B.sketchssm_last_error())
    return torch.zeros((pages, kv_heads, page // 16, 17 * dim), dtype=torch.uint8, device=device)


def _cache(cache: Tensor, dev: int) -> B.Cache:
    if cache.dim() != 4 or cache.shape[3] % 17:
        raise ValueError(f"cache: [pages][kv_heads][page / 16][17 dim] bytes are needed, not {_said(cache)}")
    P, G, n, D = shape = cache.shape
    return B.Cache(_flat("cache", cache, shape, torch.uint8, dev), P, G, 16 * n, D // 17)


def _tokens(table: Tensor, lengths: Tensor, tokens: int, offsets: Tensor | None, dev: int) -> B.NewTokens:
    n = lengths.numel()
    off = None if offsets is None else _offsets(offsets, n, dev)[1]
    shape, s = table.shape, table.stride()
    if len(shape) != 2 or table.dtype is not torch.int32 or table.get_device() != dev or shape[0] != n or s[1] != 1 and shape[1] > 1:
        raise ValueError(f"table: an int32 tensor [{n}][columns] with contiguous rows on cuda:{dev} is needed, not {_said(table)}")
    return B.NewTokens(tokens, off, _flat("lengths", lengths, (n,), torch.int32, dev), table.data_ptr(), s[0] if n > 1 else shape[1], n, shape[1])


def cache_append(cache: Tensor, table: Tensor, lengths: Tensor, k: Tensor, v: Tensor, *, offsets: Tensor | None = None,
                 rotation: Tensor | None = None, positions: Tensor | None = None, interleaved: bool = False, q: Tensor | None = None,
                 q_out: Tensor | None = None) -> Tensor | None:
    """The new tokens' keys and values k, v [T][kv_heads][dim] io into the
    cache, in 4 bits; keys are rotated first (`rotation`, as in `rotary`; by
    their place in the sequence unless `positions` names rows), and so are the
    queries q [T][heads][dim] where given: q_out (a new tensor; it may be q).

    Sequence b's new tokens are rows offsets[b] .. offsets[b+1]-1 (None: T /
    batch each), its lengths[b] tokens end with them, and its places page j ..
    page (j + 1) - 1 are in page table[b][j] of the cache.  lengths, table and
    offsets are int32.  A token whose place is below 0 (lengths[b] less than
    its new tokens) is a padding row and not appended; one whose page is not
    in the cache is not written.  A page that is written is one sequence's, and
    stands in its row of the table once."""
    dev = _device(k)
    io = _io(k)
    c = _cache(cache, dev)
    if k.dim() != 3:
        raise ValueError("k [T][kv_heads][dim] is needed")
    T, t = k.shape[0], k.dtype
    shape = (T, c.kv_heads, c.dim)
    a = B.AppendArgs(io, 0, k.data_ptr(), *_heads("k", k, shape, t, dev), v.data_ptr(), *_heads("v", v, shape, t, dev))
    if q is not None:
        if q.dim() != 3:
            raise ValueError("q [T][heads][dim] is needed")
        if rotation is None:
            raise ValueError("q without a rotation")
        shape = (T, q.shape[1], c.dim)
        a.heads = H = q.shape[1]
        a.q, a.ldq, a.q_head = q.data_ptr(), *_heads("q", q, shape, t, dev)
        if q_out is None:
            q_out = q.new_empty(shape)
            a.q_out, a.ld_qout, a.qout_head = q_out.data_ptr(), H * c.dim, c.dim
        else:
            a.q_out, a.ld_qout, a.qout_head = q_out.data_ptr(), *_heads("q_out", q_out, shape, t, dev)
    elif q_out is not None:
        raise ValueError("q_out without q")
    rot = None if rotation is None else _rotation(rotation, positions, interleaved, T, dev)
    if rot is None and positions is not None:
        raise ValueError("positions without a rotation")
    rc = (B._lib or B.load()).sketchssm_cache_append(c, _tokens(table, lengths, T, offsets, dev), rot, a, _stream(dev))
    if rc:
        B._check(rc)
    return q_out


def cache_read(cache: Tensor, table: Tensor, lengths: Tensor, tokens: int, *, offsets: Tensor | None = None, dtype=torch.bfloat16,
               k: Tensor | None = None, v: Tensor | None = None) -> tuple[Tensor, Tensor]:
    """What the cache holds for its sequences' last tokens (`tokens` in all,
    indexed as in cache_append): (k, v) [tokens][kv_heads][dim], rotated keys and
    values as the 4 bits stand for them (bfloat16 holds them exactly).  Rows of
    places below 0 are 0, of pages that are not in the cache NaN."""
    dev = _device(cache)
    c = _cache(cache, dev)
    if dtype not in _IO:
        raise ValueError(f"{dtype}: bfloat16 or float32 is written")
    shape = (tokens, c.kv_heads, c.dim)
    if k is None and v is None:
        k, v = cache.new_empty((2, *shape), dtype=dtype).unbind()
    elif k is None:
        k = torch.empty_like(v)
    elif v is None:
        v = torch.empty_like(k)
    rc = (B._lib or B.load()).sketchssm_cache_read(c, _tokens(table, lengths, tokens, offsets, dev), _IO[dtype], _flat("k", k, shape, dtype, dev),
                                                   _flat("v", v, shape, dtype, dev), _stream(dev))
    if rc:
        B._check(rc)
    return k, v


def attention(cache: Tensor, table: Tensor, lengths: Tensor, q: Tensor, *, offsets: Tensor | None = None, scale: float | None = None,
              out: Tensor | None = None, out_dtype=None, scales: Tensor | None = None,
              workspace: Tensor | None = None) -> tuple[Tensor, Tensor | None]:
    """Causal softmax attention of the new tokens' queries q [T][heads][dim] io
    over their sequences in the cache (tokens, table and lengths as in
    cache_append, which comes first): (out [T][heads][dim], scales).  heads /
    kv_heads consecutive heads share a key head; scale is dim^-1/2 unless given.
    out_dtype None: the io type; F8: blocks of 128 columns over their scale,
    scales [heads dim / 128][T] (what matmul_fp8 reads).  Padding rows are 0.

    One form is taken for the whole call, by the new tokens a sequence has on
    average: prompts and single tokens over long contexts are faster as two
    calls.  Weights keep 24 bits in float32; in bfloat16 at least 16 for F8 and
    for single tokens (of up to 16 heads a key head), 8 for prompts."""
    dev = _device(q)
    io = _io(q)
    c = _cache(cache, dev)
    if q.dim() != 3:
        raise ValueError("q [T][heads][dim] is needed")
    T, H, D = q.shape
    if D != c.dim:
        raise ValueError(f"q has heads of {D} channels, the cache of {c.dim}")
    if out_dtype is None:
        out_dtype = q.dtype
    f8 = out_dtype is F8
    a = B.AttentionArgs(io, B.E4M3 if f8 else _IO.get(out_dtype, -1), H, D ** -0.5 if scale is None else scale, q.data_ptr(),
                        *_heads("q", q, q.shape, q.dtype, dev))
    if out is None:
        out, a.ld_out = q.new_empty((T, H, D), dtype=out_dtype), H * D
    else:
        a.ld_out, head = _heads("out", out, q.shape, out_dtype, dev)
        if head != D and H > 1:
            raise ValueError(f"out: its heads are not contiguous ({_said(out)})")
    a.out = out.data_ptr()
    if f8:
        if H * D % 128:
            raise ValueError(f"{H} heads of {D} channels are not whole blocks of 128")
        if scales is None:
            scales, a.ld_scales = q.new_empty((H * D // 128, T), dtype=_F32), T
        else:
            a.ld_scales = _rows("scales", scales, H * D // 128, T, dev)
        a.scales = scales.data_ptr()
    elif scales is not None:
        raise ValueError("scales without an 8-bit output")
    lib = B._lib or B.load()
    tok = _tokens(table, lengths, T, offsets, dev)
    need = lib.sketchssm_attention_workspace(c, H, tok.batch, T, tok.columns)
    if workspace is None and need:
        workspace = q.new_empty(need, dtype=torch.uint8)
    a.workspace, a.workspace_bytes = _space(workspace, dev)
    rc = lib.sketchssm_attention(c, tok, a, _stream(dev))
    if rc:
        B._check(rc)
    return out, scales
