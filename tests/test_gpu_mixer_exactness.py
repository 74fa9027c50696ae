"""What the mixer layer's operators keep in 32 bits, held to it.

Bounds are derived from counts of operations and unit roundoffs (2^-24, and 2^-8
for a value stored in bf16).  A scan's decays are products of softplus, step and
exponent, each a few units off, over the tokens a term survives."""
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


def scan_inputs(seed, lengths, H, G, K, V, io, dt_shift=-4.0, initial=True):
    dt, r, T = DT[io], rnd(seed), sum(lengths)
    a = dict(x=r((T, H * V), dt), b=r((T, G * K), dt), c=r((T, G * K), dt), dt=r((T, -(-H // 8) * 8), dt)[:, :H], dt_bias=r((H,)) + dt_shift,
             A=-torch.exp(r((H,))), D=r((H,)))
    return a, r((len(lengths), H, V, K)) if initial else None


def run_scan(a, S, lengths, H, G, K, V, io):
    cfg = B.make_config("mamba2", len(lengths), H, K, V, 16, 16, io)
    return ops.scan(cfg, G, a["x"], a["b"], a["c"], a["dt"], a["dt_bias"], a["A"], D=a["D"], offsets=R.offsets(lengths),
                    S=None if S is None else R.tiles(S).contiguous())


def definition(a, S, lengths, H, G):
    c = {k: v.cpu() for k, v in a.items()}
    return R.scan(c["x"], c["b"], c["c"], c["dt"], c["dt_bias"], c["A"], c["D"], lengths, None if S is None else S.cpu(), H, G)


def skip_terms(a, H):
    """|D x| of every output"""
    x = a["x"].cpu().double()
    return (x.reshape(x.shape[0], H, -1) * a["D"].cpu().double()[:, None]).abs().reshape(x.shape)


# ---- scan: the skip term


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,K,V", [(2, 1, 64, 64), (6, 2, 128, 64), (3, 3, 128, 128)])
def test_scan_skip_is_not_rounded(io, H, G, K, V):
    """D between two bf16 values and steps of nothing: y is D x rounded once, by its own type.
    The operands that are rounded to bf16 belong to the other terms alone."""
    case("scan skip", io, H, G, K, V)
    lengths = [70, 1, 130]
    a, S = scan_inputs(H + K, lengths, H, G, K, V, io, dt_shift=-40.0, initial=False)
    a["D"] = torch.linspace(1.5039, 1.9961, H, device="cuda")  # a bf16's neighbours here lie 2^-7 apart
    y, _ = run_scan(a, S, lengths, H, G, K, V, io)
    want, mag, _, _ = definition(a, S, lengths, H, G)
    skip = skip_terms(a, H)
    R.close(y.cpu(), want, (mag - skip) * 0.01 + skip * 4 * R.U32 + want.abs() * R.unit(DT[io]), "y")


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("lengths", [[700], [1, 90, 0, 255]])
def test_scan_rounds_only_what_the_state_and_scores_take(io, lengths):
    """Ordinary steps and a large D: the operands' 2^-8 is of the recurrence's terms, not of D x."""
    case("scan terms", io, lengths)
    H, G, K, V = 4, 2, 128, 64
    a, S = scan_inputs(sum(lengths), lengths, H, G, K, V, io)
    a["D"] = a["D"] * 40.0
    y, _ = run_scan(a, S, lengths, H, G, K, V, io)
    want, mag, _, _ = definition(a, S, lengths, H, G)
    skip = skip_terms(a, H)
    acc = (sum(lengths) + 64) * R.U32 + 100 * 2.0 ** -22
    op = 1.02 * R.U16 if io == "bf16" else 0.0
    R.close(y.cpu(), want, (mag - skip) * (op + acc) + skip * (4 * R.U32 + acc) + want.abs() * R.unit(DT[io]) + 1e-30, "y")


def test_prompt_and_token_apply_the_same_skip():
    """The decode path adds D x in fp32 in front of the gated norm; the scan's own D does the same."""
    case("scan skip and norm skip")
    lengths, H, G, K, V = [50], 4, 1, 64, 64
    a, S = scan_inputs(3, lengths, H, G, K, V, "bf16", dt_shift=-40.0, initial=False)
    a["D"] = torch.tensor([1.5039, 0.7519, 1.9961, 3.0078], device="cuda")
    y, _ = run_scan(a, S, lengths, H, G, K, V, "bf16")
    want = (a["x"].float().reshape(50, H, V) * a["D"][:, None]).reshape(50, H * V)
    assert float((y.float() - want).norm() / want.norm()) < 2.0 ** -9  # rms of one rounding: 2^-8 / sqrt(3) at the most, less over a binade


# ---- 8-bit products whose K axis is split


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(5, 130, 8208), (77, 513, 4112), (40, 17, 6160), (77, 4096, 8192), (1, 256, 16400), (16, 1028, 2064),
                                   (64, 66, 4096), (200, 384, 8080), (33, 1, 12304)])
def test_matmul_split(M, N, K, out):
    """Parts of unequal length, a short last block, N that is no multiple of four, more than two parts; an output
    between guard columns, a workspace of the size asked for, NaN before the call, with a guard behind it."""
    case("matmul split", M, N, K, out)
    r = rnd(M + N + K)
    kb, nb = -(-K // 128), -(-N // 128)
    f8 = lambda shape: r(shape, scale=130.0).clamp(-448, 448).to(ops.F8)  # noqa: E731
    a, w = f8((M, K)), f8((N, K))
    sa, sw = torch.exp(r((kb, M))), torch.exp(r((nb, kb)))
    need = B.load().sketchssm_matmul_fp8_workspace(M, N, K)
    assert need >= 2 * M * N * 4  # the split is taken
    space = torch.full((need // 4 + 64,), float("nan"), device="cuda")
    space[need // 4:] = 3.0
    y, mag, top = R.matmul(a, sa, w, sw)
    bound = (128 + K / 128 + 8) * R.U32 * mag
    if out == "bf16":
        bound = bound + top * 2.0 ** -11 + y.abs() * R.U16
    for ld in (N, N + 3, -(-N // 16) * 16 + 16):
        wide = torch.full((M, ld), 5.0, dtype=DT[out], device="cuda")
        ops.matmul_fp8(a, sa, w, sw, out=wide[:, :N], workspace=space[:need // 4])
        R.close(wide[:, :N], y, bound, f"y, rows of {ld}")
        assert bool((wide[:, N:] == 5.0).all()) and bool((space[need // 4:] == 3.0).all())
    again = torch.empty((M, N), dtype=DT[out], device="cuda")
    ops.matmul_fp8(a, sa, w, sw, out=again)
    assert torch.equal(again, wide[:, :N])  # parts are joined in order


# ---- the state's 24 bits, and heads shared out over the XCDs


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,K,V", [(2, 1, 64, 64), (4, 2, 128, 64), (3, 3, 128, 128)])
@pytest.mark.parametrize("lengths", [[64], [37, 0, 20], [130, 5]])
def test_scan_state_keeps_24_bits(io, H, G, K, V, lengths):
    """Slow decays, so that every token's share of the state lasts: the state is as close as fp32 sums are, value by
    value and in the norm (two bf16 parts of x dt 2^{..} are 2e-6 off in the norm)."""
    case("scan state", io, H, G, K, V, lengths)
    a, S = scan_inputs(H + K + sum(lengths), lengths, H, G, K, V, io, initial=False)
    a["A"] = a["A"] * 0.1
    _, St = run_scan(a, S, lengths, H, G, K, V, io)
    _, _, want, mag = definition(a, S, lengths, H, G)
    acc = (sum(lengths) + 64) * R.U32 + 100 * 2.0 ** -22
    R.close(St.cpu(), R.tiles(want), R.tiles(mag) * acc + 1e-30, "S")
    n = [i for i, k in enumerate(lengths) if k]
    got, ref = St.cpu().double()[n], R.tiles(want)[n]
    assert float((got - ref).norm() / ref.norm()) < 1e-6


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,K,V", [(16, 8, 128, 64), (32, 2, 128, 64), (16, 8, 64, 64), (8, 8, 128, 128), (24, 8, 64, 64)])
def test_scan_heads_over_the_dies(io, H, G, K, V):
    """Parts of heads in multiples of eight, which are dealt out in runs; with later segments."""
    case("scan heads", io, H, G, K, V)
    lengths = [260, 3, 0, 150]
    assert B.load().sketchssm_scan_workspace(B.make_config("mamba2", 4, H, K, V, 16, 16, io), G, sum(lengths)) > 0
    a, S = scan_inputs(H + G + K, lengths, H, G, K, V, io)
    y, St = run_scan(a, S, lengths, H, G, K, V, io)
    wy, my, wS, mS = definition(a, S, lengths, H, G)
    skip = skip_terms(a, H)
    acc = (sum(lengths) + 64) * R.U32 + 100 * 2.0 ** -22
    op = 1.02 * R.U16 if io == "bf16" else 0.0
    R.close(y.cpu(), wy, (my - skip) * (op + acc) + skip * (4 * R.U32 + acc) + wy.abs() * R.unit(DT[io]) + 1e-30, "y")
    R.close(St.cpu(), R.tiles(wS), R.tiles(mS) * acc + 1e-30, "S")


# ---- exponentials of the gates


def test_step_sizes_are_fp32():
    """softplus of a step down to 2^-100 and less, without a bias (whose sum would be rounded first): its exponential is
    within 2 units (1 ulp) of the instruction and 2 of its argument's low part, the reciprocal within 2, the series, its
    factors and the last sum within 6; log decay adds a product."""
    case("softplus")
    Bt, H, K, V, W = 512, 8, 64, 64, 4
    r = torch.linspace(-84.0, 84.0, Bt * H, device="cuda").reshape(Bt, H)
    C = H * V + 2 * K
    z = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    cfg = B.make_config("mamba2", Bt, H, K, V, 16, W, "f32")
    rk, rv, rb, rl, q, A = z(Bt, H, W, K), z(Bt, H, W, V), z(Bt, H, W), z(Bt, H, W), z(Bt, H, K), -torch.linspace(0.5, 8.0, H, device="cuda")
    ops.conv_token(cfg, 1, z(Bt, C), z(C, 4), None, z(Bt, 3, C), r, None, A, B.make_ring(k=rk, v=rv, beta=rb, log_decay=rl), 1, q)
    want = torch.log1p(torch.exp(r.double())).where(r < 0, r.double() + torch.log1p(torch.exp(-r.double())))
    R.close(rb[:, :, 1], want, want * 12 * R.U32, "beta")
    R.close(rl[:, :, 1], want * A.double(), (want * A.double()).abs() * 13 * R.U32, "log decay")
    assert float(((rb[:, :, 1] - want) / want).square().mean().sqrt()) < 2 * R.U32


def test_silu_is_fp32():
    """The convolution's and the gate's silu in fp32, to |z| = 80: z sigma(z) of an exact z, its exponential within 4
    units, the sum, the reciprocal and two products within 6; where sigma is less than 2^-126 nothing is asked."""
    case("silu")
    n = 1 << 14
    x = torch.linspace(-80.0, 80.0, n, device="cuda").reshape(n // 64, 64)
    taps = torch.zeros((64, 4), device="cuda")
    taps[:, 3] = 1.0
    y, _ = ops.conv(x, taps)
    z = x.double()
    want = z / (1 + torch.exp(-z))
    R.close(y, want, want.abs() * 10 * R.U32, "conv")
    one = torch.ones((n // 64, 64), device="cuda")
    out, _, _ = ops.norm(one, torch.ones(64, device="cuda"), 1e-30, gate=x, group=8)
    u = want.reshape(-1, 8, 8)
    y = (u / (u.square().mean(-1, keepdim=True) + 1e-30).sqrt()).reshape(x.shape)
    R.close(out, y, y.abs() * 32 * R.U32, "norm")


@pytest.mark.parametrize("lengths", [[(97 * i) % 400 for i in range(64)], [(89 * i) % 400 for i in range(65)], [192] * 3, [0, 600, 0, 600, 1, 600],
                                     [575, 1], [1, 575], [191, 192, 192]])
def test_scan_orders_sequences_by_length(lengths):
    """Every sequence is scanned once where workgroups start longest first: ties, empty ones, both sides of the rule."""
    case("scan order", len(lengths), sum(lengths))
    H, G, K, V = 2, 1, 64, 64
    a, S = scan_inputs(len(lengths), lengths, H, G, K, V, "bf16")
    y, St = run_scan(a, S, lengths, H, G, K, V, "bf16")
    wy, my, wS, mS = definition(a, S, lengths, H, G)
    skip = skip_terms(a, H)
    acc = (max(lengths) + 64) * R.U32 + 100 * 2.0 ** -22
    R.close(y.cpu(), wy, (my - skip) * (1.02 * R.U16 + acc) + skip * (4 * R.U32 + acc) + wy.abs() * R.U16 + 1e-30, "y")
    R.close(St.cpu(), R.tiles(wS), R.tiles(mS) * acc + 1e-30, "S")


@pytest.mark.parametrize("M,N,K", [(1, 66000, 144), (64, 65540, 128), (65, 65601, 272), (128, 65536, 256), (129, 65536, 256), (257, 40001, 144)])
def test_matmul_of_few_rows_and_many_columns(M, N, K):
    """A vocabulary's columns for a decode batch: both sides of the rule that gives the widest tiles to more rows."""
    case("matmul columns", M, N, K)
    r = rnd(M + N)
    kb, nb = -(-K // 128), -(-N // 128)
    f8 = lambda shape: r(shape, scale=130.0).clamp(-448, 448).to(ops.F8)  # noqa: E731
    a, w = f8((M, K)), f8((N, K))
    sa, sw = torch.exp(r((kb, M))), torch.exp(r((nb, kb)))
    y = ops.matmul_fp8(a, sa, w, sw)
    rows = torch.tensor(sorted({0, M // 2, M - 1}), device="cuda")
    want, mag, top = R.matmul(a.float()[rows].to(ops.F8), sa[:, rows], w, sw)
    R.close(y[rows], want, (128 + K / 128 + 4) * R.U32 * mag + top * 2.0 ** -11 + want.abs() * R.U16, "bf16")
    assert bool(torch.isfinite(y).all())
