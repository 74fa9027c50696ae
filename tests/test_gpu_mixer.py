"""The mixer layer's operators on the GPU against their 64-bit definitions.

Bounds are derived, not fitted.  A sum of n fp32 products is within n 2^-24 of the
sum of their magnitudes; a value stored in bf16 (eight significant bits) within 2^-8 of itself; silu is a
few units more (its exponential and reciprocal); with bf16 inputs the scan
rounds one operand of every term (2^-8 of the sum of magnitudes), and what enters the
state keeps 16 bits (2^-16); e4m3 is within 2^-4 of a value, or half its
smallest subnormal; the 8-bit matrix instruction under a bf16 output is within
2^-11 of the largest product of a block."""
import pytest
import torch

import mixer_reference as R
from paper_2609_33051_amd import binding as B
from paper_2609_33051_amd import ops

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def case(*a):
    print("[case]", *a, flush=True)


def rnd(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda shape, dtype=torch.float32, scale=1.0: (torch.randn(shape, device="cuda", generator=g) * scale).to(dtype)


def silu_bound(s, mag, w, dtype):
    """|error| of silu(sum): the sum's, through a slope of at most 1.1, the exponential's and reciprocal's, the rounding."""
    y = R.silu(s)
    return 1.1 * (w + 2) * R.U32 * mag + y.abs() * (s.abs() + 16) * 2 * R.U32 + y.abs() * R.unit(dtype) + 1e-37


# ---- convolution


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("w", [2, 3, 4])
@pytest.mark.parametrize("lengths", [[1], [0, 5, 0], [2, 1, 3, 0, 1], [31, 1, 32, 33, 0, 64], [300], [7, 40, 8, 1, 90, 16]])
def test_conv(io, w, lengths):
    case("conv", io, w, lengths)
    dt, r, T, C = DT[io], rnd(w + sum(lengths)), sum(lengths), 264
    wide = r((T, C + 24), dt)
    wide[:, C:] = float("nan")  # what lies beside a row is not read
    x, taps, bias = wide[:, :C], r((C, w)), r((C,))
    state = r((len(lengths), w - 1, C), dt)
    off = R.offsets(lengths)
    for st, b, act in ((state, bias, True), (None, None, False), (state, None, True)):
        y, new = ops.conv(x, taps, b, offsets=off, state=st, silu=act)
        want, mag, s, states = R.conv(x, taps, b, lengths, st, act)
        bound = silu_bound(s, mag, w, dt) if act else (w + 2) * R.U32 * mag + want.abs() * R.unit(dt)
        R.close(y, want, bound, "y")
        assert torch.equal(new.double(), states)
    # in place of the old states
    new2 = state.clone()
    y2, _ = ops.conv(x, taps, bias, offsets=off, state=new2, state_out=new2)
    y1, new1 = ops.conv(x, taps, bias, offsets=off, state=state)
    assert torch.equal(y1, y2) and torch.equal(new1, new2)


@pytest.mark.parametrize("io,C", [("bf16", 64), ("f32", 1032)])
def test_conv_many_tokens(io, C):
    """Enough tokens for the wide kernel; boundaries inside its workgroups and at their edges."""
    case("conv many", io, C)
    lengths = [16, 0, 5000, 15, 17, 4000, 1, 7999, 33] if C == 64 else [3000, 1, 31, 6000, 0, 16]
    dt, r, T = DT[io], rnd(C), sum(lengths)
    x, taps, bias, state = r((T, C), dt), r((C, 4)), r((C,)), r((len(lengths), 3, C), dt)
    y, new = ops.conv(x, taps, bias, offsets=R.offsets(lengths), state=state)
    want, mag, s, states = R.conv(x, taps, bias, lengths, state)
    R.close(y, want, silu_bound(s, mag, 4, dt), "y")
    assert torch.equal(new.double(), states)


def test_conv_equal_lengths_and_no_tokens():
    case("conv equal lengths")
    r = rnd(4)
    x, taps, bias, state = r((60, 64), torch.bfloat16), r((64, 4)), r((64,)), r((5, 3, 64), torch.bfloat16)
    a, sa = ops.conv(x, taps, bias, batch=5, state=state)
    b, sb = ops.conv(x, taps, bias, offsets=R.offsets([12] * 5), state=state)
    assert torch.equal(a, b) and torch.equal(sa, sb)
    y, s = ops.conv(x[:0], taps, bias, offsets=R.offsets([0] * 5), state=state)
    assert y.shape == (0, 64) and torch.equal(s, state)


def test_conv_many_columns_and_nan_stay_apart():
    """Channels over several workgroups; a NaN reaches its own channel and the w - 1 tokens after it, and no other sequence."""
    case("conv columns")
    r = rnd(11)
    lengths = [50, 40]
    x, taps = r((90, 4352), torch.bfloat16), r((4352, 4))
    x[48, 100] = float("nan")
    y, st = ops.conv(x, taps, offsets=R.offsets(lengths))
    bad = torch.isnan(y)
    assert int(bad.sum()) == 2 and bool(bad[48:50, 100].all())
    assert int(torch.isnan(st).sum()) == 1


# ---- one token into the replay buffer


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("Bt,H,G,K,V,W,w,n", [(1, 128, 8, 128, 64, 16, 4, 0), (3, 7, 1, 128, 64, 12, 3, 11), (2, 20, 4, 64, 64, 8, 2, 3),
                                              (5, 32, 32, 128, 128, 32, 4, 31), (203, 128, 8, 128, 64, 4, 4, 2),
                                              (513, 8, 1, 128, 128, 2, 2, 1)])
def test_conv_token(io, Bt, H, G, K, V, W, w, n):
    case("token", io, Bt, H, G, K, V, W, w, n)
    dt, r = DT[io], rnd(Bt + H + n)
    C = H * V + 2 * G * K
    wide = r((Bt, 64 + C + -(-H // 8) * 8), dt)
    x, raw = wide[:, 64:64 + C], wide[:, 64 + C:64 + C + H]
    taps, bias, state, dt_bias, A = r((C, w)), r((C,)), r((Bt, w - 1, C), dt), r((H,)) - 4.0, -torch.exp(r((H,)))
    cfg = B.make_config("mamba2", Bt, H, K, V, 16, W, io)
    rk, rv = torch.full((Bt, H, W, K), 7.0, dtype=dt, device="cuda"), torch.full((Bt, H, W, V), 7.0, dtype=dt, device="cuda")
    rb, rl = torch.full((Bt, H, W), 7.0, device="cuda"), torch.full((Bt, H, W), 7.0, device="cuda")
    q = torch.empty((Bt, H, K), dtype=dt, device="cuda")
    ring = B.make_ring(k=rk, v=rv, beta=rb, log_decay=rl)
    old = state.clone()
    ops.conv_token(cfg, G, x, taps, bias, state, raw, dt_bias, A, ring, n, q)
    want, mag, s, new = R.conv(x, taps, bias, [1] * Bt, old)
    bound = silu_bound(s, mag, w, dt)
    got = torch.cat([rv[:, :, n].reshape(Bt, -1), rk[:, ::H // G, n].reshape(Bt, -1), q[:, ::H // G].reshape(Bt, -1)], 1)
    R.close(got, want, bound, "v, k, q")
    for t in (rk[:, :, n], q):  # every head of a group has the group's
        assert torch.equal(t.reshape(Bt, G, H // G, K), t.reshape(Bt, G, H // G, K)[:, :, :1].expand(Bt, G, H // G, K))
    assert torch.equal(state.double(), new)
    step = R.softplus(raw.double() + dt_bias.double())
    rel = (16 + (raw.double() + dt_bias.double()).abs() * 2) * R.U32
    R.close(rb[:, :, n], step, step * rel, "beta")
    R.close(rl[:, :, n], step * A.double(), step * A.double().abs() * (rel + R.U32), "log decay")
    others = [j for j in range(W) if j != n]
    for t in (rk, rv, rb, rl):  # other slots are left alone
        assert bool((t[:, :, others] == 7.0).all())


# ---- scan


def scan_case(seed, lengths, H, G, K, V, io, initial=True, skip=True, bias=True, dt_shift=-4.0):
    dt, r, T = DT[io], rnd(seed), sum(lengths)
    C = H * V + 2 * G * K
    wide = r((T, C + 8), dt)
    wide[:, C:] = float("nan")
    a = dict(x=wide[:, :H * V], b=wide[:, H * V:H * V + G * K], c=wide[:, H * V + G * K:C])
    raw = r((T, H + 3), dt)
    a["dt"] = raw[:, 1:H + 1]
    a["dt_bias"] = r((H,)) + dt_shift if bias else None
    a["A"] = -torch.exp(r((H,)))
    a["D"] = r((H,)) if skip else None
    S = r((len(lengths), H, V, K)) if initial else None
    return a, S


def scan_check(a, S, lengths, H, G, K, V, io, in_place=False, offsets=True):
    dt = DT[io]
    cfg = B.make_config("mamba2", len(lengths), H, K, V, 16, 16, io)
    off = R.offsets(lengths) if offsets else None
    T = sum(lengths)
    S0 = None if S is None else R.tiles(S).contiguous()
    kw = dict(S_out=S0) if in_place else {}
    y, St = ops.scan(cfg, G, a["x"], a["b"], a["c"], a["dt"], a["dt_bias"], a["A"], D=a["D"], offsets=off, S=S0, **kw)
    cpu = {k: None if v is None else v.cpu() for k, v in a.items()}
    wy, my, wS, mS = R.scan(cpu["x"], cpu["b"], cpu["c"], cpu["dt"], cpu["dt_bias"], cpu["A"], cpu["D"], lengths,
                            None if S is None else S.cpu(), H, G)
    # decays: each step's softplus and product are a few units off, over the tokens a term
    # survives; terms that survive many tokens have small log decays (their sum is bounded
    # by 100, beyond which the term is nothing): at most 100 units of 2^-21 or so
    acc = (T + 64) * R.U32 + 100 * 2.0 ** -22
    op = R.U16 if io == "bf16" else 0.0
    R.close(y.cpu(), wy, my * (1.02 * op + acc) + wy.abs() * R.unit(dt) + 1e-30, "y")
    R.close(St.cpu(), R.tiles(wS), R.tiles(mS) * ((2.0 ** -16 if io == "bf16" else 0.0) + acc) + 1e-30, "S")
    return y, St


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,K,V", [(2, 1, 64, 64), (4, 2, 128, 64), (3, 3, 128, 128)])
@pytest.mark.parametrize("lengths", [[1], [0, 3, 0, 17], [63, 64, 65], [16, 130, 1, 0, 32]])
def test_scan(io, H, G, K, V, lengths):
    case("scan", io, H, G, K, V, lengths)
    for initial in (True, False):
        a, S = scan_case(H + K + sum(lengths), lengths, H, G, K, V, io, initial, skip=initial, bias=initial,
                         dt_shift=-4.0)
        scan_check(a, S, lengths, H, G, K, V, io)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("lengths", [[700], [1, 900, 0, 255, 257], [256, 256, 256], [513, 300]])
def test_scan_split_over_workgroups(io, lengths):
    """Few items and long sequences: segments, some of them of one sequence, states in place and apart."""
    case("scan split", io, lengths)
    H, G, K, V = 2, 1, 128, 64
    assert B.load().sketchssm_scan_workspace(B.make_config("mamba2", len(lengths), H, K, V, 16, 16, io), G, sum(lengths)) > 0
    a, S = scan_case(sum(lengths), lengths, H, G, K, V, io)
    y1, S1 = scan_check(a, S, lengths, H, G, K, V, io)
    y2, S2 = scan_check(a, S, lengths, H, G, K, V, io, in_place=True)
    assert torch.equal(y1, y2) and torch.equal(S1, S2)
    a, S = scan_case(sum(lengths) + 1, lengths, H, G, K, V, io, initial=False)
    scan_check(a, None, lengths, H, G, K, V, io)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_scan_forgets(io):
    """Steps from nothing to far beyond what fp32 can decay by, in one chunk: the
    decays between later tokens are not blurred by the sum before them."""
    case("scan forgets", io)
    lengths, H, G, K, V = [100], 2, 1, 64, 64
    a, S = scan_case(5, lengths, H, G, K, V, io, bias=False)
    a["dt"] = torch.full((100, 2), -9.0, dtype=DT[io], device="cuda")
    a["dt"][::7] = 80.0
    a["dt"][50:60] = 3000.0
    a["A"] = torch.tensor([-0.5, -30.0], device="cuda")
    a["x"] = (a["x"].float() * torch.where(a["dt"][:, :1].float() > 0, 1e-3, 1.0)).to(DT[io]).contiguous()
    scan_check(a, S, lengths, H, G, K, V, io)
    a["A"] = torch.zeros(2, device="cuda")  # no decay at all
    a["dt"] = torch.full((100, 2), -60.0, dtype=DT[io], device="cuda")
    scan_check(a, S, lengths, H, G, K, V, io)


def test_scan_equal_lengths_and_no_tokens():
    case("scan equal lengths")
    H, G, K, V = 4, 1, 128, 64
    a, S = scan_case(3, [40, 40], H, G, K, V, "bf16")
    y1, S1 = scan_check(a, S, [40, 40], H, G, K, V, "bf16")
    y2, S2 = scan_check(a, S, [40, 40], H, G, K, V, "bf16", offsets=False)
    assert torch.equal(y1, y2) and torch.equal(S1, S2)
    none = {k: v if v is None or k in ("dt_bias", "A", "D") else v[:0] for k, v in a.items()}
    scan_check(none, S, [0, 0], H, G, K, V, "bf16")


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("lengths", [[129], [128], [150] * 6, [65, 0, 64, 1]])
def test_scan_short_segments(io, lengths):
    """Segments of one chunk or a few, by offsets and by equal lengths, in a workspace of the size asked for."""
    case("scan short segments", io, lengths)
    H, G, K, V = 3, 1, 128, 64
    a, S = scan_case(len(lengths) + sum(lengths), lengths, H, G, K, V, io)
    y1, S1 = scan_check(a, S, lengths, H, G, K, V, io)
    y2, S2 = scan_check(a, S, lengths, H, G, K, V, io, in_place=True)
    assert torch.equal(y1, y2) and torch.equal(S1, S2)
    if len(set(lengths)) == 1:
        y3, S3 = scan_check(a, S, lengths, H, G, K, V, io, offsets=False)
        assert torch.equal(y1, y3) and torch.equal(S1, S3)


@pytest.mark.parametrize("lengths", [[(7 * i) % 11 for i in range(256)], [(5 * i) % 9 for i in range(300)], [4] * 33])
def test_scan_many_sequences(lengths):
    """Every sequence is scanned once, whatever order the workgroups take them in: equal lengths, empty ones, more than are sorted."""
    case("scan many sequences", len(lengths))
    H, G, K, V = 2, 1, 64, 64
    a, S = scan_case(len(lengths), lengths, H, G, K, V, "bf16")
    scan_check(a, S, lengths, H, G, K, V, "bf16")


def test_scan_many_short_segments():
    """One head pair over 9000 tokens: tens of states to join."""
    case("scan many segments")
    H, G, K, V = 2, 1, 64, 64
    a, S = scan_case(44, [9000], H, G, K, V, "bf16")
    scan_check(a, S, [9000], H, G, K, V, "bf16")


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_scan_nan_stays_in_its_head_and_sequence(io):
    case("scan nan", io)
    H, G, K, V = 4, 2, 128, 64
    lengths = [50, 90, 30]
    a, S = scan_case(8, lengths, H, G, K, V, io)
    cfg = B.make_config("mamba2", 3, H, K, V, 16, 16, io)
    go = lambda: ops.scan(cfg, G, a["x"], a["b"], a["c"], a["dt"], a["dt_bias"], a["A"], D=a["D"], offsets=R.offsets(lengths),  # noqa: E731
                          S=R.tiles(S).contiguous())
    y0, S0 = go()
    a["x"][120, 2 * V + 5] = float("nan")  # second sequence, head 2
    y1, S1 = go()
    keep = torch.ones((170, H * V), dtype=torch.bool, device="cuda")
    keep[50:140, 2 * V:3 * V] = False
    assert torch.equal(y0[keep], y1[keep]) and not bool(torch.isnan(y1[keep]).any())
    assert bool(torch.isnan(y1[120:140, 2 * V + 5]).all()) and bool(torch.isnan(S1[1, 2]).any())
    ok = torch.ones((3, H), dtype=torch.bool, device="cuda")
    ok[1, 2] = False
    assert torch.equal(S0[ok], S1[ok])


def test_scan_leads_into_the_sketch():
    """The scan's states are what the flush and the sketch read: one more token by the exact recurrence equals a scan of one more token."""
    case("scan into update")
    lengths, H, G, K, V = [33, 20], 4, 4, 128, 64
    a, S = scan_case(21, lengths, H, G, K, V, "f32", initial=False, skip=False)
    cfg = B.make_config("mamba2", 2, H, K, V, 0, 1, "f32")
    off = R.offsets([32, 19])
    part = torch.tensor([i for i in range(53) if i not in (32, 52)], device="cuda")
    cut = {k: v if v is None or k in ("dt_bias", "A") else v[part].contiguous() for k, v in a.items()}
    _, S1 = ops.scan(cfg, G, cut["x"], cut["b"], cut["c"], cut["dt"], cut["dt_bias"], cut["A"], offsets=off)
    y2, S2 = ops.scan(cfg, G, a["x"], a["b"], a["c"], a["dt"], a["dt_bias"], a["A"], offsets=R.offsets(lengths))
    last = torch.tensor([32, 52], device="cuda")
    beta = R.softplus(a["dt"][last].double() + a["dt_bias"].double()).float()
    k, q = (a[z][last].reshape(2, H, 1, K).contiguous() for z in "bc")
    v = a["x"][last].reshape(2, H, 1, V).contiguous()
    ring = B.make_ring(k=k, v=v, beta=beta.reshape(2, H, 1), log_decay=(beta * a["A"]).reshape(2, H, 1).contiguous())
    o = torch.empty((2, H, V), device="cuda")
    B.sketchssm_update(cfg, S1, None, ring, 0, q, None, o)
    torch.cuda.synchronize()
    assert float((S1 - S2).norm() / S2.norm()) < 1e-5
    assert float((o.reshape(2, -1) - y2[last]).norm() / y2[last].norm()) < 1e-5


# ---- norm


def check_norm(M, N, group, io, form, f8, x_f32=False, seed=0):
    dt, r = DT[io], rnd(M + N + seed)
    x = r((M, N + 8), torch.float32 if x_f32 else dt, 2.0)[:, :N]
    weight = r((N,)) * 0.2 + 1.0
    kw = {}
    if form == "residual":
        kw["residual"] = r((M, N), dt, 3.0)
    if form.startswith("gated"):
        kw["gate"] = r((M, 2 * N), dt)[:, N:]
    if form == "gated_skip":
        kw["skip"] = r((M, N // 64, 3, 64), dt)[:, :, 1]
        kw["D"] = r((N // 64,))
    out, scales, res = ops.norm(x, weight, 1e-5, group=group, out_dtype=ops.F8 if f8 else None if form != "plain" else dt, **kw)
    y, u = R.norm(x, weight, 1e-5, group, **kw)
    # u: a few operations, the gate's exponential; the mean of squares of `group` values as a tree
    mag = x.double().abs() + (kw["residual"].double().abs() if form == "residual" else 0.0)
    if form == "gated_skip":
        mag = mag + (kw["skip"].double() * kw["D"].double()[:, None]).abs().flatten(1)
    if form.startswith("gated"):
        z = kw["gate"].double()
        mag = mag * R.silu(z).abs() * (1 + (z.abs() + 16) / 2)
    factor = (y / torch.where(u == 0, torch.ones_like(u), u)).abs().amax(-1, keepdim=True)
    off = mag * factor * 4 * R.U32 + y.abs() * 64 * R.U32
    if form == "residual":
        R.close(res, u, u.abs() * R.unit(dt) + mag * 2 * R.U32, "residual")
    if not f8:
        R.close(out, y, off * 2 + y.abs() * R.unit(dt) * 1.01, "out")
        return
    s = R.blocks(y)
    most = torch.nn.functional.pad(off, (0, -N % 128)).reshape(M, -1, 128).amax(-1).t()
    R.close(scales, s, most / 448.0 + s * 4 * R.U32, "scales")
    wide = scales.double().repeat_interleave(128, 0)[:N].t()
    R.close(out.float().double() * wide, y, y.abs() * 2.0 ** -4 * 1.001 + wide * 2.0 ** -10 * 1.001 + 2 * off, "values")


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("form", ["plain", "residual", "gated", "gated_skip"])
@pytest.mark.parametrize("M,N,group", [(1, 64, 64), (3, 8, 8), (2, 520, 520), (5, 1024, 256), (4, 2056, 2056), (2, 8192, 1024),
                                       (3, 4160, 4160), (1, 16384, 16384)])
def test_norm(io, form, M, N, group):
    if form == "gated_skip" and N % 64:
        N, group = 64 * (N // 64 + 1), 64 * (N // 64 + 1)
    case("norm", io, form, M, N, group)
    for f8 in (True, False):
        check_norm(M, N, group, io, form, f8)
        if io == "bf16":
            check_norm(M, N, group, io, form, f8, x_f32=form != "plain", seed=1)


@pytest.mark.parametrize("N,group", [(20480, 20480), (32768, 32768), (40960, 20480)])
def test_norm_widest_groups(N, group):
    case("norm widest", N, group)
    for form in ("plain", "residual", "gated_skip"):
        for f8 in (True, False):
            check_norm(2, N, group, "bf16", form, f8)


def test_norm_zero_rows_and_extremes():
    """Rows of zeros give zeros and the smallest scale; rows whose values span
    the exponent range keep theirs; a NaN or an infinity stays in its row and group."""
    case("norm extremes")
    x = torch.randn((6, 512), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    x[0] = 0.0
    x[1, :128] = 0.0
    x[2] *= 1e15
    x[3] *= 1e-15
    x[4, 3] = float("nan")
    x[5, 300] = float("inf")
    w = torch.ones(512, device="cuda")
    out, s, _ = ops.norm(x, w, 1e-30, group=256, out_dtype=ops.F8)
    v = out.float()
    assert bool((v[0] == 0).all()) and bool((s[:, 0] == 2.0 ** -64).all())
    assert bool((v[1, :128] == 0).all()) and float(s[0, 1]) == 2.0 ** -64
    y, _ = R.norm(x[:4], w, 1e-30, 256)
    wide = s.double().repeat_interleave(128, 0).t()[:4]
    R.close(v[:4].double() * wide, y, y.abs() * 2.0 ** -4 * 1.01 + wide * 2.0 ** -10 * 1.01, "values")
    assert bool(torch.isnan(v[4, :256]).all()) and not bool(torch.isnan(v[4, 256:]).any())
    assert not bool(torch.isnan(v[5, :256]).any()) and bool(torch.isnan(s[:2, 4]).all())


def test_norm_in_place_residual():
    case("norm residual in place")
    r = rnd(9)
    x, res, w = r((7, 1024), torch.bfloat16), r((7, 1024), torch.bfloat16), r((1024,))
    a, s, ra = ops.norm(x, w, 1e-5, residual=res, out_dtype=ops.F8)
    stream = res.clone()
    b, t, rb = ops.norm(x, w, 1e-5, residual=stream, residual_out=stream, out_dtype=ops.F8)
    assert rb is stream and torch.equal(ra, rb) and torch.equal(a.float(), b.float()) and torch.equal(s, t)


# ---- 8-bit products


def fp8(r, shape, scale=130.0):
    return r(shape, scale=scale).clamp(-448, 448).to(ops.F8)


@pytest.mark.parametrize("M", [1, 15, 17, 33, 64, 77, 128, 129, 300])
@pytest.mark.parametrize("N,K", [(1, 16), (17, 144), (128, 128), (130, 64), (200, 1040), (513, 384), (1024, 2048)])
def test_matmul(M, N, K):
    case("matmul", M, N, K)
    r = rnd(M + N + K)
    kb, nb = -(-K // 128), -(-N // 128)
    a, w = fp8(r, (M, K)), fp8(r, (N, K))
    sa, sw = torch.exp(r((kb, M))), torch.exp(r((nb, kb)))
    y, mag, top = R.matmul(a, sa, w, sw)
    bound = (128 + K / 128 + 4) * R.U32 * mag
    R.close(ops.matmul_fp8(a, sa, w, sw, out_dtype=torch.float32), y, bound, "f32")
    R.close(ops.matmul_fp8(a, sa, w, sw), y, bound + top * 2.0 ** -11 + y.abs() * R.U16, "bf16")


@pytest.mark.parametrize("M,N,K", [(4096, 4096, 256), (4000, 4600, 272), (130, 70000, 144), (5100, 3600, 128)])
def test_matmul_many_tiles(M, N, K):
    """Enough tiles for the widest kernel, with rows, columns and a block past
    its tiles' ends; some rows of every tile of rows are checked over all columns."""
    case("matmul many", M, N, K)
    r = rnd(M)
    kb, nb = -(-K // 128), -(-N // 128)
    a, w = fp8(r, (M, K)), fp8(r, (N, K))
    sa, sw = torch.exp(r((kb, M))), torch.exp(r((nb, kb)))
    y = ops.matmul_fp8(a, sa, w, sw)
    yf = ops.matmul_fp8(a, sa, w, sw, out_dtype=torch.float32)
    rows = torch.tensor(sorted({m for t in range(0, M, 256) for m in (t, t + 77, t + 255)} & set(range(M)) | {M - 1}), device="cuda")
    want, mag, top = R.matmul(a.float()[rows].to(ops.F8), sa[:, rows], w, sw)
    bound = (128 + K / 128 + 4) * R.U32 * mag
    R.close(yf[rows], want, bound, "f32")
    R.close(y[rows], want, bound + top * 2.0 ** -11 + want.abs() * R.U16, "bf16")
    assert bool(torch.isfinite(y).all())


@pytest.mark.parametrize("M,N,K", [(5, 96, 256), (140, 272, 320), (600, 400, 272)])
def test_matmul_strides_and_neighbours(M, N, K):
    """Strided rows of every matrix; what lies between them is neither read (NaN) nor written."""
    case("matmul strides", M, N, K)
    r = rnd(K)
    kb, nb = -(-K // 128), -(-N // 128)
    nan = lambda rows, cols: torch.full((rows, cols), float("nan"), device="cuda").to(ops.F8)  # noqa: E731
    A, W = nan(M, K + 48), nan(N, K + 32)
    A[:, :K], W[:, :K] = fp8(r, (M, K)), fp8(r, (N, K))
    a, w = A[:, :K], W[:, :K]
    sa = torch.full((kb, M + 5), float("nan"), device="cuda")
    sa[:, :M] = torch.exp(r((kb, M)))
    sw = torch.exp(r((nb, kb)))
    y, mag, top = R.matmul(a, sa[:, :M], w, sw)
    for dt, ld in ((torch.float32, N + 7), (torch.bfloat16, N + 8), (torch.bfloat16, N + 3)):
        out = torch.full((M, ld), 5.0, dtype=dt, device="cuda")
        ops.matmul_fp8(a, sa[:, :M], w, sw, out=out[:, :N])
        low = top * 2.0 ** -11 if dt is torch.bfloat16 else 0.0
        R.close(out[:, :N], y, (128 + K / 128 + 4) * R.U32 * mag + low + y.abs() * R.unit(dt), "y")
        assert bool((out[:, N:] == 5.0).all())


@pytest.mark.parametrize("M", [3, 70, 200])
def test_matmul_nan_stays_in_its_row_and_column(M):
    case("matmul nan", M)
    r = rnd(M)
    N, K = 300, 208  # a short last block
    a, w = fp8(r, (M, K)), fp8(r, (N, K))
    sa, sw = torch.exp(r((2, M))), torch.exp(r((3, 2)))
    y0 = ops.matmul_fp8(a, sa, w, sw)
    a2, w2 = a.clone(), w.clone()
    a2[1, 207] = float("nan")
    w2[37, 200] = float("nan")
    y1 = ops.matmul_fp8(a2, sa, w2, sw)
    bad = torch.zeros((M, N), dtype=torch.bool, device="cuda")
    bad[1], bad[:, 37] = True, True
    assert torch.equal(torch.isnan(y1), bad) and torch.equal(y0[~bad], y1[~bad])


# ---- streams, refusals, the layer


def test_ops_run_on_the_current_stream():
    """Inputs made on a side stream, every operator on it: results as on the default one."""
    case("stream")
    r = rnd(2)
    x, w = r((40, 1024), torch.bfloat16), torch.ones(1024, device="cuda")
    wt, sw = fp8(r, (256, 1024)), torch.ones((2, 8), device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        late = x.clone()
        for _ in range(20):
            late = late * 1.0
        q, sc, _ = ops.norm(late, w, 1e-5, out_dtype=ops.F8)
        y = ops.matmul_fp8(q, sc, wt, sw)
    s.synchronize()
    q2, sc2, _ = ops.norm(x, w, 1e-5, out_dtype=ops.F8)
    assert torch.equal(y, ops.matmul_fp8(q2, sc2, wt, sw))


def test_ops_refusals():
    case("refusals")
    dev = "cuda"
    x, taps = torch.zeros((8, 64), device=dev), torch.zeros((64, 4), device=dev)
    bad = [lambda: ops.conv(x.half(), taps), lambda: ops.conv(x.t(), taps), lambda: ops.conv(x, taps.double()),
           lambda: ops.conv(x, taps, offsets=torch.zeros(2, dtype=torch.int64, device=dev)),
           lambda: ops.conv(x, taps, state=torch.zeros((1, 3, 32), device=dev)),
           lambda: ops.conv(x.cpu(), taps), lambda: ops.norm(x, torch.ones(32, device=dev), 1e-5),
           lambda: ops.norm(x, torch.ones(64, device=dev), 1e-5, D=torch.ones(1, device=dev)),
           lambda: ops.norm(x, torch.ones(64, device=dev), 1e-5, residual=torch.zeros((8, 32), device=dev)),
           lambda: ops.matmul_fp8(x, x, x, x)]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            print("not refused:", i)
    for f in (lambda: ops.conv(x, taps[:, :1].contiguous()), lambda: ops.norm(x, torch.ones(64, device=dev), -1.0),
              lambda: ops.conv(x[:, 1:33], taps[:32].contiguous()), lambda: ops.conv(x, taps, out=x)):
        with pytest.raises(B.SketchSSMError):
            f()


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_mixer_layer_decodes_what_it_prefilled(io):
    """prefill of n + m tokens equals prefill of n and m steps (full-rank sketch:
    exact reads), over a flush, with an empty and a one-token prompt among the requests.
    Both sides quantise the same activations; where two roundings fall apart, a value
    moves by one step of e4m3 (2^-3 of it) in one of some hundred terms."""
    from paper_2609_33051_amd.mixer import Mamba2Mixer
    case("layer", io)
    r = rnd(31)
    Bt, H, G, K, V, hidden, W, m = 3, 4, 2, 128, 64, 256, 4, 6
    C = H * V + 2 * G * K
    weights = dict(norm=torch.ones(hidden), in_proj=r((H * V + C + H, hidden)) * hidden ** -0.5, taps=r((C, 4)) * 0.5,
                   conv_bias=r((C,)) * 0.1, dt_bias=r((H,)) - 3.0, A=-torch.exp(r((H,))), D=r((H,)), out_norm=torch.ones(H * V),
                   out_proj=r((hidden, H * V)) * (H * V) ** -0.5)
    om = torch.eye(K).expand(H, K, K).contiguous()
    make = lambda: Mamba2Mixer(weights, Bt, H, G, K, V, K, W, om, om, io=io)  # noqa: E731
    lengths = [40, 0, 1]
    full = [n + m for n in lengths]
    X = [r((n, hidden), DT[io]) for n in full]
    Y = [r((n, hidden), DT[io]) for n in full]
    a, b = make(), make()
    o1, r1 = a.prefill(torch.cat(X), torch.cat(Y), R.offsets(full))
    b.prefill(torch.cat([x[:n] for x, n in zip(X, lengths)]), torch.cat([x[:n] for x, n in zip(Y, lengths)]), R.offsets(lengths))
    ends = R.offsets(full).tolist()
    for t in range(m):
        o2, r2 = b.step(torch.stack([X[i][lengths[i] + t] for i in range(Bt)]), torch.stack([Y[i][lengths[i] + t] for i in range(Bt)]))
        at = torch.tensor([ends[i] + lengths[i] + t for i in range(Bt)], device="cuda")
        assert torch.equal(r1[at], r2)
        assert float((o1[at].float() - o2.float()).norm() / o1[at].float().norm()) < (2e-2 if io == "bf16" else 1e-2)
    assert b.layer.n == m % W
