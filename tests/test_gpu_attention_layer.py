"""The attention layer's operators in a row, as a model uses them: prompts in one call or in pieces, single tokens,
captured steps, another stream, and a mixer layer beside the attention layer."""
import pytest
import torch

import attention_reference as R
from paper_2609_33051_amd import ops
from paper_2609_33051_amd.attention import Attention, rotary_angles
from paper_2609_33051_amd.mixer import Mamba2Mixer

pytestmark = pytest.mark.gpu

# Two sides of the same layer round the same values at the same places, but where they differ by a little one may fall on
# the other side of a border.  e4m3: values are 2^-3 apart at most and differ by 2^-7 (bf16's rounding, either side), so one in sixteen
# moves, by 2^-3: rms 2^-5 for each of the two arrays in 8 bits.  4 bits: numbers are a third of themselves apart or less (from
# 2 up, where half of a block's weight is), values 2^-7: one in 40, rms 1/19 for keys and for values.  Queries, keys, values and outputs in bf16: 2^-8 each.
APART = 2 * 2.0 ** -5 + 2 / 19 + 4 * 2.0 ** -8


def case(*a):
    print("[case]", *a, flush=True)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def layer(seed, hidden, H, G, D, pages, page, rotated=None, io="bf16", **kw):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    w = dict(norm=1 + 0.1 * r(hidden), qkv_proj=r((H + 2 * G) * D, hidden) * hidden ** -0.5, out_proj=r(hidden, H * D) * (H * D) ** -0.5)
    ang = None if rotated == 0 else rotary_angles(4096, rotated or D)
    return Attention(w, H, G, D, pages, page, ang, io=io, **kw), w


def dequantised(q, s):
    n, k = q.shape
    return q.double() * s.double().repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)[:, :k]


def plain(m, x, res, lengths, io):
    """The layer over whole sequences in 64 bits, with the roundings of its 8-bit and 4-bit arrays: out, one sequence after the other."""
    dt = torch.bfloat16 if io == "bf16" else torch.float32

    def eight(y):
        b = y.reshape(y.shape[0], -1, 128)
        s = (b.abs().amax(-1, keepdim=True) / 448.0).clamp_min(2.0 ** -64)
        return ((b / s).float().to(ops.F8).double() * s).reshape(y.shape)

    outs, at = [], 0
    H, G, D = m.heads, m.kv_heads, m.dim
    for n in lengths:
        u = x[at:at + n].double() + res[at:at + n].double()
        u = eight(u / torch.sqrt((u * u).mean(-1, keepdim=True) + m.eps) * m.norm.double())
        qkv = (u @ dequantised(m.qkv_proj, m.qkv_scale).t()).to(dt).view(n, H + 2 * G, D)
        pos = torch.arange(n, device="cuda")
        t = (lambda z: R.rotated(z, m.rotation, pos, m.interleaved)) if m.rotation is not None else (lambda z: z.float())  # noqa: E731
        y, _, _ = R.attention(t(qkv[:, :H]).to(dt), R.held(t(qkv[:, H:H + G])), R.held(qkv[:, H + G:]), n, D ** -0.5)
        outs.append(eight(y.reshape(n, H * D)) @ dequantised(m.out_proj, m.out_scale).t())
        at += n
    return torch.cat(outs)


@pytest.mark.parametrize("io,H,G,D,rotated,page", [("bf16", 8, 2, 128, None, 16), ("bf16", 8, 2, 64, 32, 64), ("bf16", 4, 1, 256, 64, 32), ("f32", 8, 4, 128, 0, 16),
                                                   ("f32", 4, 2, 64, 64, 16)])
def test_prompts_pieces_and_tokens(io, H, G, D, rotated, page):
    """Ragged prompts in one call, then tokens one by one, against the whole sequences in 64 bits; and the same prompts in two calls."""
    case("layer", io, H, G, D, rotated, page)
    hidden, lengths, more = 256, [37, 1, 130, 16], 4
    full = [n + more for n in lengths]
    tab, pool = R.table(full, page)
    m, _ = layer(1, hidden, H, G, D, pool, page, rotated, io)
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(2)
    x, res = (torch.randn((sum(full), hidden), generator=g, device="cuda").to(dt) for _ in range(2))
    want = plain(m, x, res, full, io)
    starts = [sum(full[:b]) for b in range(4)]
    rows = torch.cat([torch.arange(s, s + n) for s, n in zip(starts, lengths)]).cuda()
    got = torch.zeros((sum(full), hidden), dtype=dt, device="cuda")
    got[rows], r1 = m.prefill(x[rows], res[rows], tab, i32(lengths), R.offsets(lengths))
    assert torch.equal(r1, (x[rows].float() + res[rows].float()).to(dt))
    for t in range(more):
        at = torch.tensor([s + n + t for s, n in zip(starts, lengths)]).cuda()
        got[at], _ = m.step(x[at], res[at], tab, i32([n + t + 1 for n in lengths]))
    err = (got.double() - want).norm() / want.norm()
    assert float(err) <= APART, float(err)
    # the prompts in two pieces: the same cache and, for the second piece, the same outputs within bf16 and 8-bit roundings
    m2, _ = layer(1, hidden, H, G, D, pool, page, rotated, io)
    half = [n // 2 for n in lengths]
    a = torch.cat([torch.arange(s, s + n) for s, n in zip(starts, half)]).cuda()
    b = torch.cat([torch.arange(s + h, s + n) for s, n, h in zip(starts, lengths, half)]).cuda()
    m2.prefill(x[a], res[a], tab, i32(half), R.offsets(half))
    out2, _ = m2.prefill(x[b], res[b], tab, i32(lengths), R.offsets([n - h for n, h in zip(lengths, half)]))
    err = (out2.double() - got[b].double()).norm() / got[b].double().norm()
    assert float(err) <= APART, float(err)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_captured_steps(io):
    """A captured step whose lengths move on the device: every replay against the eager step, with other work between; two graphs in turn."""
    case("graph", io)
    hidden, H, G, D, page, B = 256, 8, 2, 128, 16, 5
    start = [3, 40, 0, 700, 15]
    tab, pool = R.table([n + 40 for n in start], page)
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    (m, _), (e, _) = (layer(4, hidden, H, G, D, pool, page, None, io) for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(5)
    T = sum(start)
    x0 = torch.randn((T, hidden), generator=g, device="cuda").to(dt)
    for z in (m, e):
        z.prefill(x0, x0, tab, i32(start), R.offsets(start))
    x, res, lengths = torch.zeros((B, hidden), dtype=dt, device="cuda"), torch.zeros((B, hidden), dtype=dt, device="cuda"), i32(start)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):  # once before the capture
        m.step(x, res, tab, i32([0] * B))
    torch.cuda.current_stream().wait_stream(s)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            lengths += 1
            out, _ = m.step(x, res, tab, lengths)
        graphs.append((graph, out))
    lengths.copy_(i32(start))
    for t in range(8):
        new = torch.randn((B, hidden), generator=g, device="cuda").to(dt)
        x.copy_(new)
        res.copy_(new)
        graph, out = graphs[t % 2]
        graph.replay()
        want, _ = e.step(new, new, tab, i32([n + t + 1 for n in start]))
        torch.cuda.synchronize()
        assert torch.equal(out, want), t
    assert torch.equal(m.cache, e.cache)


def test_another_stream_and_padded_batches():
    """Calls on a side stream; a batch with padding rows (length 0) gives the others the same bits."""
    case("stream")
    hidden, H, G, D, page = 128, 4, 2, 128, 16
    lengths = [20, 300, 7]
    tab, pool = R.table(lengths, page)
    (a, _), (b, _) = (layer(6, hidden, H, G, D, pool, page) for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(7)
    x = torch.randn((sum(lengths), hidden), generator=g, device="cuda").bfloat16()
    want, _ = a.prefill(x, x, tab, i32(lengths), R.offsets(lengths))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got, _ = b.prefill(x, x, tab, i32(lengths), R.offsets(lengths))
        tok = torch.randn((3, hidden), generator=g, device="cuda").bfloat16()
        got1, _ = b.step(tok, tok, tab, i32([20, 300, 7]))
    s.synchronize()
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)
    wide = torch.full((6, tab.shape[1]), -1, dtype=torch.int32, device="cuda")
    wide[[0, 2, 5]] = tab
    pad = torch.zeros((6, hidden), dtype=torch.bfloat16, device="cuda")
    pad[[0, 2, 5]] = tok
    got6, _ = a.step(pad, pad, wide, i32([20, 0, 300, 0, 0, 7]))
    assert torch.equal(got6[[0, 2, 5]], got1) and not bool(got6[[1, 3, 4]].any()) and torch.equal(a.cache, b.cache)


def test_beside_a_mixer_layer():
    """A mixer layer and an attention layer in a row: a prompt, then tokens through both; the last tokens as if they had been in the prompt."""
    case("hybrid")
    H, G, K, V, hidden, B, n, more = 4, 2, 128, 64, 256, 3, 24, 2
    g = torch.Generator(device="cuda").manual_seed(10)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    C = H * V + 2 * G * K
    w = dict(norm=torch.ones(hidden), in_proj=r(H * V + C + H, hidden) * hidden ** -0.5, taps=r(C, 4) * 0.5, conv_bias=r(C) * 0.1, dt_bias=r(H) - 3.0,
             A=-torch.exp(r(H)), D=r(H), out_norm=torch.ones(H * V), out_proj=r(hidden, H * V) * (H * V) ** -0.5)
    om = torch.eye(K).expand(H, K, K).contiguous()  # exact reads
    mixers = [Mamba2Mixer(w, B, H, G, K, V, K, 4, om, om, baseline=True) for _ in range(2)]
    page = 16
    tab, pool = R.table([n + more] * B, page)
    (a, _), (b, _) = (layer(8, hidden, 8, 2, 64, pool, page) for _ in range(2))
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn((B, n + more, hidden), generator=g, device="cuda").bfloat16()

    def through(mixer, att, z, k):
        flat = z.reshape(-1, hidden).contiguous()
        h, r = mixer.prefill(flat, torch.zeros_like(flat))
        return att.prefill(h, r, tab, i32([k] * B))[0].view(B, -1, hidden)

    whole = through(mixers[0], a, x, n + more)
    through(mixers[1], b, x[:, :n], n)
    for t in range(more):
        h, r = mixers[1].step(x[:, n + t].contiguous(), torch.zeros((B, hidden), dtype=torch.bfloat16, device="cuda"))
        out, _ = b.step(h, r, tab, i32([n + t + 1] * B))
        err = (out.double() - whole[:, n + t].double()).norm() / whole[:, n + t].double().norm()
        # the mixer layer has two more arrays in 8 bits, and its scan rounds scores and state to bf16 where the token's read does not
        assert float(err) <= APART + 2 * 2.0 ** -5 + 4 * 2.0 ** -8, float(err)
