"""Plain 64-bit definitions of the attention layer's operators, with the sums of
magnitudes that bound what rounding can do to a result."""
import torch

U32, U16 = 2.0 ** -24, 2.0 ** -8  # the unit roundoff: fp32 has 24 significant bits, bf16 eight
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def unit(dtype):
    return U16 if dtype is torch.bfloat16 else U32


def rotated(x, angles, positions, interleaved):
    """x [T][H][D] in 32 bits, each product and sum rounded (the operators' definition), rows of angles [places][R]."""
    R, x = angles.shape[1], x.float()
    cs = angles[positions.long()]
    co, si = cs[:, None, :R // 2], cs[:, None, R // 2:]
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if interleaved else (x[..., :R // 2], x[..., R // 2:R])
    u, w = a * co - b * si, b * co + a * si
    y = torch.stack([u, w], -1).flatten(-2) if interleaved else torch.cat([u, w], -1)
    return torch.cat([y, x[..., R:]], -1)


def held(x):
    """The 4-bit numbers nearest to x [..][D] over each block's power of two, by trying all of them; ties to the
    even code.  A block that is not finite, or past 7 2^124, is NaN."""
    v = x.double().unflatten(-1, (-1, 32))
    top = v.abs().amax(-1, keepdim=True)
    e = torch.full_like(top, -64.0)
    for k in range(-64, 125):
        e = torch.where(top > 7.0 * 2.0 ** (k - 1), torch.full_like(e, float(k)), e) if k > -64 else e
    two = ((e.long() + 1023) << 52).view(torch.float64)  # 2^e, exactly
    a = v.abs() / two
    best, off = torch.zeros_like(a), a.clone()
    for i in (2, 4, 6, 1, 3, 5, 7):  # even codes first
        d = (a - GRID[i]).abs()
        best, off = torch.where(d < off, GRID[i], best), torch.minimum(d, off)
    y = best * torch.sign(v) * two
    bad = ~torch.isfinite(v).all(-1, keepdim=True) | (top > 7.0 * 2.0 ** 124)
    return torch.where(bad, torch.full_like(y, float("nan")), y).flatten(-2)


def attention(q, k, v, n, scale):
    """One sequence: q [n][H][D], k and v [length][G][D] as the cache holds them.  (out, sum of p |v|, largest sum of |q k| of a row) in 64 bits."""
    H, D = q.shape[1:]
    L, G = k.shape[:2]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    mag, most = torch.zeros_like(out), torch.zeros(q.shape[:2], dtype=torch.float64, device=q.device)
    if not n or not L:
        return out, mag, most
    place = torch.arange(L - n, L, device=q.device)
    hide = torch.arange(L, device=q.device)[None] > place[:, None]
    for h in range(H):
        g = h // (H // G)
        s = q[:, h].double() @ k[:, g].double().t() * scale
        w = (q[:, h].double().abs() @ k[:, g].double().abs().t() * scale).masked_fill(hide, 0.0)
        s = s.masked_fill(hide, float("-inf"))
        seen = (~hide).any(1)
        x = torch.softmax(s[seen], -1)
        out[seen, h], mag[seen, h], most[seen, h] = x @ v[:, g].double(), x @ v[:, g].double().abs(), w[seen].amax(-1)
    return out, mag, most


def bound(out, mag, most, length, D, dtype):
    """|error| of an attention output.  A score is off by its D products' roundings (and the exponent's few): eps of
    every weight; with bf16 io a weight is rounded to bf16; the weights' sum is off by as much again; the sums over
    the keys have `length` terms."""
    eps = (D + 16) * U32 * most[..., None] + 32 * U32 + (U16 if dtype is torch.bfloat16 else 4 * U32)
    return 2 * eps * mag + (length + 8) * U32 * mag + out.abs() * unit(dtype) + 1e-37


def close(got, want, bound, what):
    got, want = got.double(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    off = torch.where(torch.isnan(want), torch.zeros_like(want), (got - want).abs())
    worst = (off / torch.where(torch.isnan(want), torch.ones_like(want), bound)).max() if off.numel() else 0.0
    assert bool((off <= torch.where(torch.isnan(want), torch.full_like(off, float("inf")), bound)).all()), f"{what}: {float(worst):.3g} of the bound"


def angles(places, R, device="cuda", base=1e4):
    f = base ** (-torch.arange(0, R, 2, dtype=torch.float64, device=device) / R)
    a = torch.arange(places, dtype=torch.float64, device=device)[:, None] * f
    return torch.cat([torch.cos(a), torch.sin(a)], 1).float()


def table(lengths, page, device="cuda", seed=0, spare=2, columns=None):
    """(table with impossible entries where no token lies, pages in the pool)"""
    need = [-(-max(n, 0) // page) for n in lengths]
    total = sum(need) + spare
    g = torch.Generator().manual_seed(seed)
    order = torch.randperm(total, generator=g).tolist()
    t = torch.full((len(lengths), columns or max(1, max(need))), 1 << 30, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        t[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    return t.to(device), total


def offsets(counts, device="cuda"):
    return torch.tensor([0] + torch.tensor(counts).cumsum(0).tolist(), dtype=torch.int32, device=device)
