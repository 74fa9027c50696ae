"""Timed cases of the operators around the recurrence in a Mamba-2 mixer layer:
the short causal convolution and the selective scan (prompts and single
tokens), the norms that end in 8 bits, and the projections in 8 bits.

`own = False` computes each operator in plain torch operations in 32 bits,
`own = True` calls `paper_2609_33051_amd.ops`.  `listed()` names twelve cases,
`draw(rng)` makes more of the same ranges; `prepare` makes the inputs on the
GPU, `run` is one call, `work` the bytes and operations it cannot do without,
`exact` its definition in 64 bits.

The calls (`op`):
  conv    a batch of prompts, packed: the depthwise causal convolution with
          SiLU, from the sequences' states to their new ones
  token   one token of every request: the convolution, the gates, and the
          token's place in the decode path's replay buffer
  scan    the prompts' scan: outputs of every token and the state each sequence ends in
  norm    root-mean-square norm of the sum with the residual, or of the gated
          output by groups (with the skip term on the decode path)
  matmul  a projection: 8-bit activations with a scale per row and 128
          columns, 8-bit weights with a scale per 128 x 128

Fields: T packed tokens, B sequences (`ragged` > 0: their lengths are drawn
from that number, with an empty one among them where there are several), H
heads, G groups, K and V channels, w taps; M rows, N columns; io type.
"""
import math

import numpy as np
import torch

own = False

CHUNK = 64
F8 = torch.float8_e4m3fn


def _conv(name, T, B, H, G, K, V, w=4, io="bf16", ragged=0, initial=True):
    return dict(name=name, op="conv", T=T, B=B, H=H, G=G, K=K, V=V, w=w, io=io, ragged=ragged, initial=initial)


def _token(name, B, H, G, K, V, W, w=4, io="bf16", n=0):
    return dict(name=name, op="token", B=B, H=H, G=G, K=K, V=V, W=W, w=w, io=io, n=n)


def _scan(name, T, B, H, G, K, V, io="bf16", ragged=0, initial=False):
    return dict(name=name, op="scan", T=T, B=B, H=H, G=G, K=K, V=V, io=io, ragged=ragged, initial=initial)


def _norm(name, M, N, form, group=0, io="bf16", out="fp8", V=64):
    return dict(name=name, op="norm", M=M, N=N, form=form, group=group or N, io=io, out=out, V=V)


def _matmul(name, M, N, K, io="bf16"):
    return dict(name=name, op="matmul", M=M, N=N, K=K, io=io)


def listed():
    return [
        # a batch of prompts through the layer's convolution (8192 + 2 * 8 * 128 channels): the large streaming case
        _conv("conv_prompts", 16384, 8, 128, 8, 128, 64, ragged=3),
        # a few short prompts, fp32, three taps, no states before them
        _conv("conv_short_f32", 777, 5, 20, 4, 64, 64, w=3, io="f32", ragged=5, initial=False),
        # one request's next token, where latency counts
        _token("token_b1", 1, 128, 8, 128, 64, 16, n=5),
        # the benchmark's decode batch
        _token("token_b256", 256, 128, 8, 128, 64, 16, n=11),
        # one long prompt: few (sequence, head) items, a long axis
        _scan("scan_one_prompt", 16384, 1, 128, 8, 128, 64),
        # many prompts of uneven length that continue earlier states
        _scan("scan_ragged", 12000, 37, 128, 8, 128, 64, ragged=7, initial=True),
        # a small fp32 layer, odd lengths
        _scan("scan_short_f32", 1001, 3, 20, 4, 64, 64, io="f32", ragged=9, initial=True),
        # the layer's input norm over a prompt batch, with the residual, for the input projection
        _norm("norm_residual_prompts", 8192, 4096, "residual"),
        # the decode batch's gated norm, with the skip term, for the output projection
        _norm("norm_gated_b256", 256, 8192, "gated_skip", group=1024),
        # the input projection over a prompt batch (the largest case)
        _matmul("matmul_prompts", 8192, 18560, 4096),
        # the input projection of one token: the weights' bytes
        _matmul("matmul_b1", 1, 18560, 4096),
        # the output projection of an odd decode batch
        _matmul("matmul_b77", 77, 4096, 8192),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _count(rng, hi):
    """1 to hi over its logarithm: powers of two, or odd."""
    v = _log(rng, 1, hi)
    return max(1, min(hi, 1 << round(math.log2(v)) if rng.random() < 0.3 else int(v) | 1))


_LARGEST = None


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    """One more case of these ranges, of no more work than the largest listed one."""
    global _LARGEST
    if _LARGEST is None:
        _LARGEST = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(("conv", "token", "scan", "scan", "norm", "norm", "matmul", "matmul"))
        io = rng.choice(("bf16", "bf16", "bf16", "f32"))
        K, V = rng.choice(((64, 64), (128, 64), (128, 64), (128, 128)))
        H, G = rng.choice(((4, 1), (7, 1), (16, 2), (20, 4), (32, 1), (32, 8), (48, 4), (128, 8)))
        if op == "conv":
            T = _count(rng, 16384)
            B = min(_count(rng, 64), T)
            c = _conv(None, T, B, H, G, K, V, rng.choice((2, 3, 4, 4)), io, rng.randrange(1, 1000), rng.random() < 0.5)
        elif op == "token":
            W = rng.choice((4, 8, 12, 16, 16, 32))
            c = _token(None, _count(rng, 512), H, G, K, V, W, rng.choice((2, 3, 4, 4)), io, rng.randrange(W))
        elif op == "scan":
            T = _count(rng, 16384)
            B = min(_count(rng, 64), T)
            c = _scan(None, T, B, H, G, K, V, io, rng.randrange(1, 1000), rng.random() < 0.5)
            if B * int(_lengths(c).max()) * H > 16384 * 128 or io == "f32" and T * H > 4096 * 128:
                continue
        elif op == "norm":
            M = _count(rng, 8192)
            form = rng.choice(("plain", "residual", "residual", "gated", "gated_skip"))
            if form.startswith("gated"):
                c = _norm(None, M, H * V, form, H * V // G, io, rng.choice(("fp8", "fp8", "io")), V)
            else:
                c = _norm(None, M, 8 * (int(_log(rng, 8, 1024)) | 1) if rng.random() < 0.5 else
                          rng.choice((64, 512, 1024, 2048, 4096, 5120, 8192)), form, 0, io,
                          rng.choice(("fp8", "fp8", "io")))
        else:
            N = int(_log(rng, 16, 18560)) | 1 if rng.random() < 0.3 else rng.choice((128, 1024, 2048, 4096, 5120, 8192, 18560))
            c = _matmul(None, _count(rng, 8192), N, rng.choice((64, 144, 512, 1024, 2048, 2896, 4096, 5120, 8192)), io)
        c.pop("name")
        if _cost(c) <= _LARGEST:
            return c


# ---- inputs


def _dt(c):
    return torch.bfloat16 if c["io"] == "bf16" else torch.float32


def _lengths(c):
    """The sequences' lengths: equal ones, or B uneven ones that add up to T."""
    if not c["ragged"]:
        return np.full(c["B"], c["T"] // c["B"], dtype=np.int64)
    g = np.random.default_rng(c["ragged"])
    share = g.gamma(2.0, size=c["B"])
    if c["B"] > 2:
        share[g.integers(0, c["B"])] = 0.0
    ends = np.floor(np.cumsum(share) / share.sum() * c["T"] + 0.5).astype(np.int64)
    ends[-1] = c["T"]
    return np.diff(ends, prepend=0)


def _offsets(c):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(_lengths(c))]).astype(np.int32)).cuda()


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, shape, dtype=torch.float32, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _channels(c):
    return c["H"] * c["V"] + 2 * c["G"] * c["K"]


def _inputs(c, seed):
    """The arrays a call reads, from the seed alone."""
    g, dt, op = _gen(seed), _dt(c), c["op"]
    st = {}
    if op in ("conv", "token"):
        C, w = _channels(c), c["w"]
        st["taps"] = _randn(g, (C, w), scale=w ** -0.5)
        st["bias"] = _randn(g, (C,), scale=0.1)
        st["state"] = _randn(g, (c["B"], w - 1, C), dt) if op == "token" or c["initial"] else None
        H = c["H"]
        # the projection's output holds the gate z, the convolution's channels and the step sizes side by side
        rows = c["T"] if op == "conv" else c["B"]
        wide = _randn(g, (rows, H * c["V"] + C + -(-H // 8) * 8), dt)
        st["x"] = wide[:, H * c["V"]:H * c["V"] + C]
        if op == "token":
            st["dt"] = wide[:, H * c["V"] + C:H * c["V"] + C + H]
    if op == "scan":
        H, G, K, V = c["H"], c["G"], c["K"], c["V"]
        wide = torch.nn.functional.silu(_randn(g, (c["T"], _channels(c)))).to(dt)  # the convolution's output
        st["x"], st["b"], st["c"] = wide[:, :H * V], wide[:, H * V:H * V + G * K], wide[:, H * V + G * K:]
        st["dt"] = _randn(g, (c["T"], H), dt)
        st["D"] = _randn(g, (H,)).add_(1.0)
        st["S"] = _randn(g, (c["B"], H, V, K), scale=0.1) if c["initial"] else None
    if op in ("token", "scan"):
        # step sizes about 1e-3 to 1e-1, decays A = -exp(U[0, 2])
        H = c["H"]
        st["dt_bias"] = torch.rand((H,), generator=g, device="cuda") * 4.0 - 6.5
        st["A"] = -torch.exp(2.0 * torch.rand((H,), generator=g, device="cuda"))
    if op == "norm":
        M, N, form = c["M"], c["N"], c["form"]
        st["weight"] = _randn(g, (N,), scale=0.2).add_(1.0)
        st["x"] = _randn(g, (M, N), torch.float32 if form == "gated_skip" else dt, 2.0)
        if form == "residual":
            st["residual"] = _randn(g, (M, N), dt, 3.0)
        if form.startswith("gated"):
            st["gate"] = _randn(g, (M, 2 * N), dt)[:, :N]
        if form == "gated_skip":
            st["skip"] = _randn(g, (M, N // c["V"], 3, c["V"]), dt)[:, :, 1]  # a slot of the replay buffer
            st["D"] = _randn(g, (N // c["V"],)).add_(1.0)
    if op == "matmul":
        M, N, K = c["M"], c["N"], c["K"]
        kb, nb = -(-K // 128), -(-N // 128)
        st["a"] = (torch.randn((M, K), generator=g, device="cuda") * 130.0).clamp_(-448.0, 448.0).to(F8)
        st["w"] = (torch.randn((N, K), generator=g, device="cuda") * 130.0).clamp_(-448.0, 448.0).to(F8)
        st["a_scale"] = torch.exp(_randn(g, (kb, M), scale=0.5)) / 130.0
        st["w_scale"] = torch.exp(_randn(g, (nb, kb), scale=0.3)) / 130.0 / math.sqrt(K)
    return st


def prepare(case, seed):
    c = case
    st = _inputs(c, seed)
    st["case"] = c
    op = c["op"]
    if op in ("conv", "scan"):
        st["offsets"] = _offsets(c)
        if op == "scan":
            st["pad"] = _padding(c)
    if op in ("token", "scan"):
        from paper_2609_33051_amd import binding
        W = c.get("W", 16)
        st["cfg"] = binding.make_config("mamba2", c["B"], c["H"], c["K"], c["V"], 16, W, c["io"])
    if op == "scan" and c["initial"]:
        st["S"] = _tiles(st["S"])
    if op == "token":
        B, H, K, V, W = (c[x] for x in ("B", "H", "K", "V", "W"))
        dt = _dt(c)
        st["rk"] = torch.zeros((B, H, W, K), dtype=dt, device="cuda")
        st["rv"] = torch.zeros((B, H, W, V), dtype=dt, device="cuda")
        st["rbeta"] = torch.zeros((B, H, W), device="cuda")
        st["rla"] = torch.zeros((B, H, W), device="cuda")
        st["q"] = torch.zeros((B, H, K), dtype=dt, device="cuda")
        st["ring"] = binding.make_ring(k=st["rk"], v=st["rv"], beta=st["rbeta"], log_decay=st["rla"])
    return st


# ---- the operators


def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["op"]](state, state["case"])


def _own_conv(st, c):
    from paper_2609_33051_amd import ops
    y, state = ops.conv(st["x"], st["taps"], st["bias"], offsets=st["offsets"], state=st["state"])
    return {"y": y, "state": state}


def _own_token(st, c):
    from paper_2609_33051_amd import ops
    n = c["n"]
    ops.conv_token(st["cfg"], c["G"], st["x"], st["taps"], st["bias"], st["state"], st["dt"], st["dt_bias"], st["A"],
                   st["ring"], n, st["q"])
    return _slot(st, n)


def _slot(st, n):
    return {"k": st["rk"][:, :, n], "v": st["rv"][:, :, n], "beta": st["rbeta"][:, :, n], "log_decay": st["rla"][:, :, n],
            "q": st["q"], "state": st["state"]}


def _own_scan(st, c):
    from paper_2609_33051_amd import ops
    y, S = ops.scan(st["cfg"], c["G"], st["x"], st["b"], st["c"], st["dt"], st["dt_bias"], st["A"], D=st["D"],
                    offsets=st["offsets"], S=st["S"])
    return {"y": y, "S": S}


def _own_norm(st, c):
    from paper_2609_33051_amd import ops
    out, scales, res = ops.norm(st["x"], st["weight"], 1e-5, group=c["group"], residual=st.get("residual"),
                                gate=st.get("gate"), skip=st.get("skip"), D=st.get("D"),
                                out_dtype=F8 if c["out"] == "fp8" else _dt(c))
    return {"out": out, "scales": scales, "residual": res}


def _own_matmul(st, c):
    from paper_2609_33051_amd import ops
    return ops.matmul_fp8(st["a"], st["a_scale"], st["w"], st["w_scale"], out_dtype=_dt(c))


def _windows(x, state, off, w):
    """For every token the w inputs up to it, from the state before the sequence's start: [T][w][C] in 32 bits."""
    T = x.shape[0]
    B = off.numel() - 1
    t = torch.arange(T, device=x.device)
    seq = torch.searchsorted(off[1:].long(), t, right=True)
    at = t[:, None] - (w - 1) + torch.arange(w, device=x.device)[None, :]
    before = at - off[seq].long()[:, None]  # < 0: before the start
    past = torch.zeros((B, w - 1, x.shape[1]), device=x.device) if state is None else state.float()
    return torch.where((before < 0)[..., None], past[seq[:, None], (before + w - 1).clamp(0, w - 2)], x.float()[at.clamp_min(0)])


def _silu(x):
    return x / (1.0 + torch.exp(-x))


def _softplus(x):
    return torch.clamp_min(x, 0.0) + torch.log1p(torch.exp(-torch.abs(x)))


def _plain_conv(st, c):
    x, off, w = st["x"], st["offsets"], c["w"]
    y = _silu((_windows(x, st["state"], off, w) * st["taps"].t()).sum(1) + st["bias"]).to(x.dtype)
    # the last w - 1 inputs of state and sequence together
    B, C = c["B"], x.shape[1]
    lo, hi = off[:-1].long(), off[1:].long()
    at = hi[:, None] - (w - 1) + torch.arange(w - 1, device=x.device)[None, :]
    before = at - lo[:, None]
    past = torch.zeros((B, w - 1, C), dtype=x.dtype, device=x.device) if st["state"] is None else st["state"]
    old = torch.gather(past, 1, (before + w - 1).clamp(0, w - 2)[..., None].expand(B, w - 1, C))
    return {"y": y, "state": torch.where((before < 0)[..., None], old, x[at.clamp_min(0)])}


def _plain_token(st, c):
    B, H, G, K, V, n = (c[x] for x in ("B", "H", "G", "K", "V", "n"))
    x, s = st["x"], st["state"]
    full = torch.cat([s, x[:, None]], 1)
    y = _silu((full.float() * st["taps"].t()).sum(1) + st["bias"]).to(x.dtype)
    s.copy_(full[:, 1:])
    beta = _softplus(st["dt"].float() + st["dt_bias"])
    st["rv"][:, :, n] = y[:, :H * V].reshape(B, H, V)
    st["rk"][:, :, n] = y[:, H * V:H * V + G * K].reshape(B, G, 1, K).expand(B, G, H // G, K).reshape(B, H, K)
    st["q"].copy_(y[:, H * V + G * K:].reshape(B, G, 1, K).expand(B, G, H // G, K).reshape(B, H, K))
    st["rbeta"][:, :, n] = beta
    st["rla"][:, :, n] = beta * st["A"]
    return _slot(st, n)


def _padding(c):
    """Where the packed tokens lie in equal rows of whole chunks: (place of each
    row's tokens in the packed arrays, whether there is one, place of each packed token)."""
    n = _lengths(c)
    L = max(1, -(-int(n.max()) // CHUNK)) * CHUNK
    start = np.cumsum(n) - n
    at = np.minimum(start[:, None] + np.arange(L)[None], c["T"] - 1)
    there = np.arange(L)[None] < n[:, None]
    back = np.flatnonzero(there.reshape(-1))
    return torch.from_numpy(at).cuda(), torch.from_numpy(there).cuda(), torch.from_numpy(back).cuda()


def _decays(g):
    """exp(sum_{s < j <= t} g_j) for t >= s, else 0, over g's last axis; by sums of masked copies, without differences."""
    n = g.shape[-1]
    m = torch.tril(torch.ones((n, n), dtype=torch.bool, device=g.device), -1)
    x = torch.where(m, g[..., :, None].expand(*g.shape, n), torch.zeros((), device=g.device)).cumsum(-2)
    return torch.where(torch.tril(torch.ones_like(m)), torch.exp(x), torch.zeros((), device=g.device))


def _plain_scan(st, c):
    B, H, G, K, V, T = (c[x] for x in ("B", "H", "G", "K", "V", "T"))
    at, there, back = st["pad"]
    L, n = CHUNK, at.shape[1] // CHUNK
    dt = torch.where(there[..., None], _softplus(st["dt"].float() + st["dt_bias"])[at], torch.zeros((), device=at.device))
    x = st["x"].float()[at].reshape(B, n, L, H, V)
    b = st["b"].float()[at].reshape(B, n, L, G, K)
    q = st["c"].float()[at].reshape(B, n, L, G, K)
    dt = dt.reshape(B, n, L, H)
    g = (dt * st["A"]).permute(0, 1, 3, 2).contiguous()             # B n H L
    total = g.cumsum(-1)
    xd = (x * dt[..., None]).permute(0, 1, 3, 2, 4).contiguous()    # B n H L V
    b, q = (z.permute(0, 1, 3, 2, 4).contiguous() for z in (b, q))  # B n G L K
    heads = lambda z: z[:, :, :, None].expand(B, n, G, H // G, *z.shape[3:]).reshape(B, n, H, *z.shape[3:])  # noqa: E731
    y = torch.matmul(heads(torch.matmul(q, b.transpose(-1, -2).contiguous())) * _decays(g), xd)
    ends = torch.exp(total[..., -1:] - total)                       # B n H L
    S = torch.matmul((xd * ends[..., None]).transpose(-1, -2).contiguous(), heads(b))  # B n H V K
    first = torch.zeros((B, 1, H, V, K), device=at.device) if st["S"] is None else _rows(st["S"], K, V)[:, None]
    S = torch.cat([first, S], 1).transpose(1, 2).reshape(B, H, n + 1, V * K)
    pass_on = _decays(torch.nn.functional.pad(total[..., -1].transpose(1, 2), (1, 0)))  # B H n+1 n+1
    S = torch.matmul(pass_on, S).reshape(B, H, n + 1, V, K).transpose(1, 2)
    y = y + torch.matmul(heads(q) * torch.exp(total)[..., None], S[:, :-1].transpose(-1, -2).contiguous())
    y = y + x.permute(0, 1, 3, 2, 4) * st["D"][:, None, None]
    y = y.transpose(2, 3).reshape(B * n * L, H * V)[back].to(st["x"].dtype)
    return {"y": y, "S": _tiles(S[:, -1])}


def _tiles(X):
    """States [B][H][V][K] in the library's tile-major layout."""
    B, H, V, K = X.shape
    return X.reshape(B, H, V // 16, 16, K // 16, 4, 4).permute(0, 1, 2, 4, 5, 3, 6).reshape(B, H, V * K)


def _rows(S, K, V):
    B, H = S.shape[:2]
    return S.reshape(B, H, V // 16, K // 16, 4, 16, 4).permute(0, 1, 2, 5, 3, 4, 6).reshape(B, H, V, K)


def _normed(st, c, f):
    """(norm of the sum or of the gated value, the sum) with the inputs as f makes them."""
    u = f(st["x"])
    if c["form"] == "residual":
        u = u + f(st["residual"])
    if c["form"] == "gated_skip":
        u = u + (f(st["skip"]) * f(st["D"])[:, None]).reshape(u.shape)
    if c["form"].startswith("gated"):
        u = u * _silu(f(st["gate"]))
    v = u.reshape(u.shape[0], -1, c["group"])
    return (v / torch.sqrt((v * v).mean(-1, keepdim=True) + 1e-5)).reshape(u.shape) * f(st["weight"]), u


def _quantised(y):
    """(values over their block's scale, scales [blocks][rows])"""
    M, N = y.shape
    nb = -(-N // 128)
    p = torch.nn.functional.pad(y, (0, nb * 128 - N)).reshape(M, nb, 128)
    s = (p.abs().amax(-1) / 448.0).clamp_min(2.0 ** -64)
    return (p / s[..., None]).reshape(M, -1)[:, :N], s.t().contiguous()


def _plain_norm(st, c):
    y, u = _normed(st, c, lambda z: z.float())
    res = u.to(_dt(c)) if c["form"] == "residual" else None
    if c["out"] == "fp8":
        y, s = _quantised(y)
        return {"out": y.to(F8), "scales": s, "residual": res}
    return {"out": y.to(_dt(c)), "scales": None, "residual": res}


def _plain_matmul(st, c):
    N, K = c["N"], c["K"]
    col = torch.arange(K, device="cuda") // 128
    row = torch.arange(N, device="cuda") // 128
    a = st["a"].float() * st["a_scale"].t()[:, col]
    w = st["w"].float() * st["w_scale"][row][:, col]
    return torch.matmul(a, w.t()).to(_dt(c))


_PLAIN = {"conv": _plain_conv, "token": _plain_token, "scan": _plain_scan, "norm": _plain_norm, "matmul": _plain_matmul}
_OWN = {"conv": _own_conv, "token": _own_token, "scan": _own_scan, "norm": _own_norm, "matmul": _own_matmul}


# ---- what a call cannot do without


def work(case):
    c, op = case, case["op"]
    e = 2 if c["io"] == "bf16" else 4
    if op == "conv":
        C, w = _channels(c), c["w"]
        states = c["B"] * (w - 1) * C * e
        return {"bytes": float(2 * c["T"] * C * e + states * (2 if c["initial"] else 1) + 4 * C * (w + 1)),
                "flops": float(2 * w * c["T"] * C)}
    if op == "token":
        B, H, K, V, w, C = c["B"], c["H"], c["K"], c["V"], c["w"], _channels(c)
        return {"bytes": float(B * (C * e * (2 * w - 1) + H * e + H * (V + 2 * K) * e + 8 * H) + 4 * C * (w + 1) + 8 * H),
                "flops": float(2 * w * B * C)}
    if op == "scan":
        T, B, H, G, K, V = (c[x] for x in ("T", "B", "H", "G", "K", "V"))
        return {"bytes": float(T * (2 * H * V + 2 * G * K + H) * e + 4 * B * H * V * K * (2 if c["initial"] else 1)),
                "flops": float(4 * T * H * V * K)}
    if op == "norm":
        M, N, form = c["M"], c["N"], c["form"]
        b = e + (1 if c["out"] == "fp8" else e) + {"plain": 0, "residual": 2 * e, "gated": e, "gated_skip": e + 4}[form]
        return {"bytes": float(M * N * b + 4 * N + (4 * M * -(-N // 128) if c["out"] == "fp8" else 0)), "flops": float(4 * M * N)}
    M, N, K = c["M"], c["N"], c["K"]
    kb = -(-K // 128)
    return {"bytes": float(M * K + N * K + e * M * N + 4 * kb * (M + -(-N // 128))), "flops": float(2.0 * M * N * K)}


# ---- the definitions in 64 bits


def exact(case, seed):
    return _EXACT[case["op"]](_inputs(case, seed), case)


def _sigmoid64(x):
    return torch.where(x >= 0, 1.0 / (1.0 + torch.exp(-x.abs())), torch.exp(-x.abs()) / (1.0 + torch.exp(-x.abs())))


def _exact_conv(st, c):
    w, C = c["w"], _channels(c)
    ends = np.cumsum(_lengths(c))
    ys, states = [], []
    for i in range(c["B"]):
        lo = 0 if i == 0 else int(ends[i - 1])
        part = st["x"][lo:int(ends[i])].double()
        past = torch.zeros((w - 1, C), dtype=torch.float64, device="cuda") if st["state"] is None else st["state"][i].double()
        z = torch.cat([past, part])
        m = part.shape[0]
        acc = st["bias"].double()[None] + sum(z[j:j + m] * st["taps"][:, j].double() for j in range(w))
        ys.append(acc * _sigmoid64(acc))
        states.append(z[m:])
    return {"y": torch.cat(ys), "state": torch.stack(states)}


def _exact_token(st, c):
    B, H, G, K, V, w = (c[x] for x in ("B", "H", "G", "K", "V", "w"))
    z = torch.cat([st["state"].double(), st["x"].double()[:, None]], 1)
    acc = st["bias"].double() + sum(z[:, j] * st["taps"][:, j].double() for j in range(w))
    y = acc * _sigmoid64(acc)
    r = st["dt"].double() + st["dt_bias"].double()
    beta = torch.maximum(r, torch.zeros_like(r)) + torch.log1p(torch.exp(-r.abs()))
    k, q = (y[:, H * V + i * G * K:H * V + (i + 1) * G * K].reshape(B, G, K).repeat_interleave(H // G, 1) for i in (0, 1))
    return {"k": k, "v": y[:, :H * V].reshape(B, H, V), "beta": beta, "log_decay": beta * st["A"].double(), "q": q, "state": z[:, 1:]}


def _exact_scan(st, c):
    """The recurrence, token by token, all sequences side by side."""
    B, H, G, K, V, T = (c[x] for x in ("B", "H", "G", "K", "V", "T"))
    n = torch.from_numpy(_lengths(c)).cuda()
    start = n.cumsum(0) - n
    S = torch.zeros((B, H, V, K), dtype=torch.float64, device="cuda") if st["S"] is None else st["S"].double()
    y = torch.zeros((T, H, V), dtype=torch.float64, device="cuda")
    D = st["D"].double()
    order = torch.argsort(n, descending=True, stable=True)  # the sequences still running lead
    S, start = S[order].contiguous(), start[order]
    lengths = n[order].tolist()
    live = B
    for t in range(lengths[0]):
        while lengths[live - 1] <= t:
            live -= 1
        i = start[:live] + t
        r = st["dt"][i].double() + st["dt_bias"].double()
        dt = torch.maximum(r, torch.zeros_like(r)) + torch.log1p(torch.exp(-r.abs()))
        x = st["x"][i].double().reshape(live, H, V)
        b, q = (st[z][i].double().reshape(live, G, K).repeat_interleave(H // G, 1) for z in "bc")
        s = S[:live]
        s.mul_(torch.exp(dt * st["A"].double())[..., None, None])
        s.addcmul_((dt[..., None] * x)[..., None], b[:, :, None, :])
        y[i] = (s * q[:, :, None, :]).sum(-1) + D[:, None] * x
    back = torch.empty_like(S)
    back[order] = S
    return {"y": y.reshape(T, H * V), "S": _tiles(back)}


def _exact_norm(st, c):
    x = st["x"].double()
    if c["form"] == "residual":
        x = x + st["residual"].double()
    res = x if c["form"] == "residual" else None
    if c["form"] == "gated_skip":
        x = x + (st["D"].double()[None, :, None] * st["skip"].double()).flatten(1)
    if c["form"].startswith("gated"):
        z = st["gate"].double()
        x = x * z * _sigmoid64(z)
    parts = [p * torch.rsqrt(p.square().mean(1, keepdim=True) + 1e-5) for p in x.split(c["group"], 1)]
    y = torch.cat(parts, 1) * st["weight"].double()
    if c["out"] != "fp8":
        return {"out": y, "scales": None, "residual": res}
    blocks = y.split(128, 1)
    s = torch.stack([torch.maximum(p.abs().max(1).values / 448.0, torch.full((), 2.0 ** -64, dtype=torch.float64, device="cuda"))
                     for p in blocks])
    return {"out": torch.cat([p / s[i][:, None] for i, p in enumerate(blocks)], 1), "scales": s, "residual": res}


def _exact_matmul(st, c):
    y = torch.zeros((c["M"], c["N"]), dtype=torch.float64, device="cuda")
    wide = st["w_scale"].double().repeat_interleave(128, 0)[:c["N"]]
    for i, k in enumerate(range(0, c["K"], 128)):
        p = torch.mm(st["a"][:, k:k + 128].double(), st["w"][:, k:k + 128].double().t())
        y += p * st["a_scale"][i].double()[:, None] * wide[:, i][None, :]
    return y


_EXACT = {"conv": _exact_conv, "token": _exact_token, "scan": _exact_scan, "norm": _exact_norm, "matmul": _exact_matmul}
