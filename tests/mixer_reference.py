"""Plain 64-bit definitions of the mixer layer's operators, with the sums of
magnitudes that bound what rounding can do to a result."""
import torch

F8 = torch.float8_e4m3fn
U32, U16 = 2.0 ** -24, 2.0 ** -8  # the unit roundoff: fp32 has 24 significant bits, bf16 eight


def unit(dtype):
    return U16 if dtype is torch.bfloat16 else U32


def silu(z):
    return z / (1.0 + torch.exp(-z))


def softplus(r):
    return torch.clamp_min(r, 0.0) + torch.log1p(torch.exp(-r.abs()))


def conv(x, taps, bias, lengths, state, act=True):
    """(y, magnitude of the sum behind y, new states)"""
    T, C = x.shape
    w = taps.shape[1]
    ys, mags, new, at = [], [], [], 0
    for b, n in enumerate(lengths):
        past = torch.zeros((w - 1, C), dtype=torch.float64, device=x.device) if state is None else state[b].double()
        z = torch.cat([past, x[at:at + n].double()])
        t = taps.double()
        s = sum(z[j:j + n] * t[:, j] for j in range(w))
        m = sum((z[j:j + n] * t[:, j]).abs() for j in range(w))
        if bias is not None:
            s, m = s + bias.double(), m + bias.double().abs()
        ys.append(s)
        mags.append(m)
        new.append(z[n:])
        at += n
    s, m = torch.cat(ys), torch.cat(mags)
    return (silu(s) if act else s), m, s, torch.stack(new)


def scan(x, b, c, dt, dt_bias, A, D, lengths, S, heads, groups):
    """The recurrence, token by token: (y, sum of |terms| of y, final S [B][H][V][K], sum of |terms| of S)."""
    T = x.shape[0]
    H, G = heads, groups
    V, K = x.shape[1] // H, b.shape[1] // G
    y = torch.zeros((T, H, V), dtype=torch.float64, device=x.device)
    m = torch.zeros_like(y)
    Sf, Mf, at = [], [], 0
    for i, n in enumerate(lengths):
        s = torch.zeros((H, V, K), dtype=torch.float64, device=x.device) if S is None else S[i].double().clone()
        a = s.abs()
        for t in range(at, at + n):
            r = dt[t].double() + (0.0 if dt_bias is None else dt_bias.double())
            step = softplus(r)
            dec = torch.exp(step * A.double())[:, None, None]
            xv = x[t].double().reshape(H, V)
            bv, cv = (z[t].double().reshape(G, K).repeat_interleave(H // G, 0) for z in (b, c))
            up = (step[:, None] * xv)[:, :, None] * bv[:, None, :]
            s = dec * s + up
            a = dec * a + up.abs()
            d = 0.0 if D is None else D.double()[:, None] * xv
            y[t] = (s * cv[:, None, :]).sum(-1) + d
            m[t] = (a * cv.abs()[:, None, :]).sum(-1) + (0.0 if D is None else d.abs())
        at += n
        Sf.append(s)
        Mf.append(a)
    return y.reshape(T, H * V), m.reshape(T, H * V), torch.stack(Sf), torch.stack(Mf)


def tiles(X):
    B, H, V, K = X.shape
    return X.reshape(B, H, V // 16, 16, K // 16, 4, 4).permute(0, 1, 2, 4, 5, 3, 6).reshape(B, H, V * K)


def norm(x, weight, eps, group, residual=None, gate=None, skip=None, D=None):
    """(y, u)"""
    u = x.double()
    if residual is not None:
        u = u + residual.double()
    if skip is not None:
        u = u + (skip.double() * D.double()[:, None]).flatten(1)
    if gate is not None:
        u = u * silu(gate.double())
    v = u.reshape(u.shape[0], -1, group)
    return (v / torch.sqrt(v.square().mean(-1, keepdim=True) + eps)).reshape(u.shape) * weight.double(), u


def blocks(y):
    """Scales [blocks][rows] of 128 columns each."""
    M, N = y.shape
    nb = -(-N // 128)
    p = torch.nn.functional.pad(y, (0, nb * 128 - N)).reshape(M, nb, 128)
    return (p.abs().amax(-1) / 448.0).clamp_min(2.0 ** -64).t()


def matmul(a, sa, w, sw):
    """(y, sum of |terms|, sum over blocks of the largest |term|)"""
    M, K = a.shape
    N = w.shape[0]
    col, row = torch.arange(K, device=a.device) // 128, torch.arange(N, device=a.device) // 128
    x = a.double() * sa.double().t()[:, col]
    z = w.double() * sw.double()[row][:, col]
    top = sum((x[:, None, k:k + 128] * z[None, :, k:k + 128]).abs().amax(-1) for k in range(0, K, 128))
    return x @ z.t(), x.abs() @ z.abs().t(), top


def offsets(lengths, device="cuda"):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device=device)


def close(got, want, bound, what):
    """Every value within its bound (and NaN where the definition has NaN)."""
    g, w = got.double(), want.double()
    bad = ~((g - w).abs() <= bound) & ~(torch.isnan(g) & torch.isnan(w)) & ~(g == w)
    if bool(bad.any()):
        i = tuple(int(k) for k in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside, first at {i}: {float(g[i])!r} for "
                             f"{float(w[i])!r}, bound {float(torch.as_tensor(bound).expand_as(w)[i]):.3g}")
