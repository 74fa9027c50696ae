"""Attention's forms that a call takes by its sizes alone: loads past the caches, two tiles of rows a wave with the keys split, 8-bit
outputs from all of them.  Each against its 64-bit definition, with the kernel that ran named by a captured call, so that the sizes
here stay sizes that take the form."""
import ctypes
import re

import pytest
import torch

import attention_reference as R
from paper_2609_33051_amd import ops
from test_gpu_attention import DT, F8, built, case, check, i32, rnd

pytestmark = pytest.mark.gpu


class _Dim(ctypes.Structure):
    _fields_ = [(x, ctypes.c_uint32) for x in "xyz"]


class _Launch(ctypes.Structure):  # hipKernelNodeParams
    _fields_ = [("block", _Dim), ("extra", ctypes.c_void_p), ("func", ctypes.c_void_p), ("grid", _Dim), ("args", ctypes.c_void_p), ("shared", ctypes.c_uint)]


def kernels(f):
    """The kernels that f launches, in order, as attention_kernel<t,128,1,1,0,0> (t bf16, f fp32): f is captured, not run."""
    hip = ctypes.CDLL([line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64" in line][0])
    hip.hipKernelNameRefByPtr.restype = ctypes.c_char_p
    hip.hipKernelNameRefByPtr.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
    f()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        f()
    raw, n = ctypes.c_void_p(graph.raw_cuda_graph()), ctypes.c_size_t()
    assert hip.hipGraphGetNodes(raw, None, ctypes.byref(n)) == 0
    nodes = (ctypes.c_void_p * n.value)()
    assert hip.hipGraphGetNodes(raw, nodes, ctypes.byref(n)) == 0
    out = []
    for node in nodes:
        p = _Launch()
        assert hip.hipGraphKernelNodeGetParams(ctypes.c_void_p(node), ctypes.byref(p)) == 0
        kernel, args = re.search(r"([a-z_]+_kernel)I(.*?)EEv", hip.hipKernelNameRefByPtr(p.func, None).decode()).groups()
        out.append(f"{kernel}<{','.join([args[0]] + re.findall('L[ib]([0-9]+)', args))}>")
    return out


def pool(r, lengths, G, D, page, dt, pages, columns, fill=255):
    """As `built`, with the sequences' pages anywhere in a pool of `pages`."""
    cache, tab, ln, ks, vs = built(r, lengths, G, D, page, dt, fill=fill)
    at = torch.randperm(pages, generator=torch.Generator().manual_seed(pages))[:cache.shape[0]].cuda()
    wide = torch.empty((pages, *cache.shape[1:]), dtype=torch.uint8, device="cuda")
    wide.fill_(fill)
    wide[at] = cache
    t = torch.full((len(lengths), columns), -1, dtype=torch.int32, device="cuda")
    here = tab < cache.shape[0]
    t[:, :tab.shape[1]] = torch.where(here, at[torch.where(here, tab, torch.zeros_like(tab)).long()].int(), torch.full_like(tab, -1))
    return wide, t, ln, ks, vs


def single(got, q, ks, vs, lengths, dt, what):
    D = q.shape[2]
    for b, n in enumerate(lengths):
        o, mag, most = R.attention(q[b:b + 1], ks[b], vs[b], 1, D ** -0.5)
        R.close(got[b:b + 1], o, R.bound(o, mag, most, max(n, 1), D, dt), f"{what} {b}")


@pytest.mark.parametrize("io,H,G,page,lengths", [("bf16", 32, 8, 64, [1, 3000, 0, 64, 65, 17, 1999, 500]), ("f32", 16, 8, 64, [700, 2, 1533, 31]), ("bf16", 4, 4, 16, [900, 33]),
                                                 ("bf16", 7, 1, 1024, [1023, 1025, 5000])])
def test_loads_past_the_caches(io, H, G, page, lengths):
    """128 channels, more bytes within the tables' reach than the last-level cache holds."""
    case("past the caches", io, H, G, page, lengths)
    r, dt, D = rnd(page + H), DT[io], 128
    record = G * (page // 16) * 17 * D
    pages = (280 << 20) // record
    columns = -(-(300 << 20) // (record * len(lengths)))
    cache, tab, ln, ks, vs = pool(r, lengths, G, D, page, dt, pages, columns)
    assert cache.numel() > 256 << 20
    q = r((len(lengths), H, D), dt)
    took = kernels(lambda: ops.attention(cache, tab, ln, q))
    assert took[0] == f"attention_kernel<{'t' if io == 'bf16' else 'f'},128,1,1,0,1>", took
    got, _ = ops.attention(cache, tab, ln, q)
    single(got, q, ks, vs, lengths, dt, "sequence")
    near, _ = ops.attention(*built(rnd(page + H), lengths, G, D, page, dt)[:3], q)  # the same from a small pool
    for b, n in enumerate(lengths):
        o, mag, most = R.attention(q[b:b + 1], ks[b], vs[b], 1, D ** -0.5)
        R.close(near[b:b + 1], o, R.bound(o, mag, most, max(n, 1), D, dt), f"small pool {b}")


TWO = [("bf16", 64, 8, 2, 64, [300, 77], [8300, 12077]), ("bf16", 96, 7, 1, 32, [405, 0, 33], [9001, 0, 12000]), ("bf16", 128, 8, 2, 128, [301, 77], [301, 12077]),
       ("bf16", 128, 20, 4, 16, [50, 61, 7], [7000, 61, 5003]), ("f32", 64, 8, 2, 64, [300, 77], [8300, 12077]), ("f32", 64, 6, 1, 16, [211], [16384])]


@pytest.mark.parametrize("io,D,H,G,page,new,lengths", TWO)
def test_two_tiles_a_wave_split(io, D, H, G, page, new, lengths):
    """Few new tokens over many keys: tiles of 32 rows whose keys lie in several workgroups, the last ones not full."""
    case("two tiles", io, D, H, G, page, new, lengths)
    dt = DT[io]
    cache, tab, ln, _, _ = built(rnd(0), lengths, G, D, page, dt)
    q = torch.zeros((sum(new), H, D), dtype=dt, device="cuda")
    off = R.offsets(new)
    took = kernels(lambda: ops.attention(cache, tab, ln, q, offsets=off))
    kind = "t" if io == "bf16" else "f"
    assert took == [f"attention_kernel<{kind},{D},2,1,0,0>", f"join_kernel<{kind},{D},2,0>"], took
    del cache
    check(io, H, G, D, page, new, lengths, seed=D)


EIGHT = [
    ("bf16", 8, 2, 128, [1, 1, 1], [3, 40, 4000], "attention_kernel<t,128,1,1,1,0>"), ("bf16", 8, 2, 64, [1, 1], [1, 700], "attention_kernel<t,64,1,1,1,0>"),
    ("bf16", 8, 2, 128, [301, 77], [301, 12077], "attention_kernel<t,128,2,1,1,0>"), ("bf16", 8, 2, 64, [300], [8300], "attention_kernel<t,64,2,1,1,0>"),
    ("f32", 8, 2, 64, [300], [8300], "attention_kernel<f,64,2,1,1,0>"), ("bf16", 32, 8, 128, [1200, 900], [1200, 1000], "prompt_kernel<t,128,2,1>"),
    ("bf16", 64, 16, 64, [1100], [1111], "prompt_kernel<t,64,2,1>"), ("bf16", 16, 16, 256, [1100, 3000], [1200, 3000], "prompt_kernel<t,256,1,1>"),
    ("f32", 32, 8, 128, [1200, 900], [1200, 1000], "attention_kernel<f,128,1,0,1,0>")]


@pytest.mark.parametrize("io,H,G,D,new,lengths,kernel", EIGHT)
def test_scales_of_8_bits(io, H, G, D, new, lengths, kernel):
    """An 8-bit output's scales are in 32 bits, whatever io is: off by what the fp32 form is, and at most 2^-16 of each weight (as two bf16 parts would be),
    twice, for the sum of the weights."""
    case("scales", io, H, G, D, new, lengths)
    dt, r = DT[io], rnd(D)
    cache, tab, ln, ks, vs = built(r, lengths, G, D, 32, dt)
    q = r((sum(new), H, D), dt)
    off = R.offsets(new)
    call = lambda: ops.attention(cache, tab, ln, q, offsets=off, out_dtype=F8)  # noqa: E731
    took = kernels(call)
    assert took[0] == kernel, took
    got, scales = call()
    at = 0
    for b, n in enumerate(new):
        o, mag, most = R.attention(q[at:at + n], ks[b], vs[b], n, D ** -0.5)
        bd = (R.bound(o, mag, most, lengths[b], D, torch.float32) + 2 * 2.0 ** -16 * mag).reshape(n, -1, 128)
        o = o.reshape(n, -1, 128)
        top = (o.abs().amax(-1) / 448.0).clamp_min(2.0 ** -64)
        s = scales[:, at:at + n].t().double()
        R.close(s, top, bd.amax(-1) / 448.0 + 4 * R.U32 * top, f"scales {b}")
        # e4m3: 2^-4 of a value, 2^-10 of the scale where it is below the normal ones
        y = got[at:at + n].float().double().reshape(n, -1, 128) * s[..., None]
        R.close(y, o, bd + o.abs() * 2.0 ** -4 + s[..., None] * 2.0 ** -10 + 8 * R.U32 * o.abs(), f"sequence {b}")
        at += n


@pytest.mark.parametrize("io,H,G,D,new,lengths,kernel", [(*e[:5], [min(n, 9000) for n in e[5]], e[6]) for e in EIGHT])
def test_weights_of_8_bits_are_not_bf16(io, H, G, D, new, lengths, kernel):
    """Every other key weighs w = (1 + 0.98 2^-8) / 2, which bf16 would take to 1/2, 0.98 2^-8 of it off; the others weigh 1.  With values 1 and 0 the outputs are
    a / (a + b w) of a keys and b, of which that rounding is w b / (a + b w) 0.98 2^-8, some 1/3 2^-8 and so 1.3e-3: more than the bound, which 16 bits of a weight keep."""
    case("not bf16", io, H, G, D, new, lengths)
    w = 0.5 * (1.0 + 0.98 * 2.0 ** -8)
    scale = float(torch.tensor(-torch.log(torch.tensor(w, dtype=torch.float64)).item(), dtype=torch.float32))
    T, dt = sum(lengths), DT[io]
    k, v = torch.zeros((T, G, D), dtype=dt, device="cuda"), torch.zeros((T, G, D), dtype=dt, device="cuda")
    at = 0
    for n in lengths:
        k[at + 1:at + n:2, :, 0] = -1.0
        v[at:at + n:2] = 1.0
        at += n
    tab, pages = R.table(lengths, 32)
    cache = ops.new_cache(pages, G, 32, D)
    ops.cache_append(cache, tab, i32(lengths), k, v, offsets=R.offsets(lengths))
    q = torch.zeros((sum(new), H, D), dtype=dt, device="cuda")
    q[..., 0] = 1.0
    _, scales = ops.attention(cache, tab, i32(lengths), q, offsets=R.offsets(new), scale=scale, out_dtype=F8)
    at = 0
    w = torch.exp(torch.tensor(-scale, dtype=torch.float64))
    for n, length in zip(new, lengths):
        seen = torch.arange(length - n + 1, length + 1, device="cuda", dtype=torch.float64)
        b = (seen / 2).floor()
        want = (seen - b) / (seen - b + b * w)
        # one product a score, a handful of roundings of the exponent; the sums; 16 bits of a weight
        bd = want * (2 * 32 * R.U32 + (length + 8) * R.U32 + 2 * 2.0 ** -16)
        assert bool((bd < 1.3e-3 * 2 / 3 * want).all())
        R.close(scales[:, at:at + n].t(), (want / 448.0)[:, None].expand(-1, H * D // 128), (bd + 4 * R.U32 * want)[:, None] / 448.0, "scales")
        at += n


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,D", [(8, 2, 128), (8, 2, 64), (6, 1, 256)])
def test_alone_and_in_company(io, H, G, D):
    """A token's output by itself, and beside others, a prompt among them: keys are split elsewhere and another form may be taken, so the bits may
    differ, by no more than either may be off."""
    case("alone", io, H, G, D)
    dt, r = DT[io], rnd(H + D)
    lengths = [1400, 1, 333, 4000]
    cache, tab, ln, ks, vs = built(r, lengths, G, D, 32, dt)
    q, prompt = r((4, H, D), dt), r((1400, H, D), dt)
    whole, _ = ops.attention(cache, tab, ln, q)
    # the first sequence's new tokens are all of its 1400
    mixed, _ = ops.attention(cache, tab, ln, torch.cat([prompt, q[1:]]), offsets=R.offsets([1400, 1, 1, 1]))
    for b in range(4):
        one, _ = ops.attention(cache, tab[b:b + 1], ln[b:b + 1], q[b:b + 1])
        o, mag, most = R.attention(q[b:b + 1], ks[b], vs[b], 1, D ** -0.5)
        bd = R.bound(o, mag, most, lengths[b], D, dt)
        R.close(one, o, bd, f"alone {b}")
        R.close(whole[b:b + 1], o, bd, f"beside {b}")
        if b:
            R.close(mixed[1399 + b:1400 + b], o, bd, f"mixed {b}")
    o, mag, most = R.attention(prompt, ks[0], vs[0], 1400, D ** -0.5)
    R.close(mixed[:1400], o, R.bound(o, mag, most, 1400, D, dt), "prompt")
