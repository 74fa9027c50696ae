"""The attention layer's operators on the GPU against their 64-bit definitions.
Rotations and the cache are compared bit for bit (every product and sum of
the definition is rounded on its own); attention within bounds that count its
roundings (attention_reference.bound)."""
import pytest
import torch

import attention_reference as R
from paper_2609_33051_amd import binding as B
from paper_2609_33051_amd import ops

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
F8 = torch.float8_e4m3fn
NAN = float("nan")


def case(*a):
    print("[case]", *a, flush=True)


def rnd(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda shape, dtype=torch.float32, scale=1.0: (torch.randn(shape, device="cuda", generator=g) * scale).to(dtype)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def same(a, b):
    return torch.equal(a.float().nan_to_num(nan=12345.0), b.float().nan_to_num(nan=12345.0))


# ---- rotation


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("T,H,D,rot", [(1, 1, 64, 64), (3, 7, 128, 128), (5, 3, 96, 24), (4, 2, 96, 96), (2, 40, 256, 64), (515, 3, 192, 48), (700, 2, 128, 20),
                                       (9, 2, 8, 6), (2, 3, 512, 512), (1030, 1, 24, 16)])
def test_rotary(io, interleaved, T, H, D, rot):
    case("rotary", io, interleaved, T, H, D, rot)
    r, dt = rnd(T + D), DT[io]
    wide = r((T, H + 1, D + 16), dt)
    wide[:, :, D:] = NAN  # what lies beside a head is not read
    x = wide[:, :H, :D]
    ang = R.angles(5000, rot)
    pos = torch.randint(0, 5000, (T,), device="cuda", dtype=torch.int32)
    want = R.rotated(x, ang, pos, interleaved).to(dt)
    assert torch.equal(ops.rotary(x, ang, pos, interleaved=interleaved), want)
    first = ops.rotary(x[:5], ang, interleaved=interleaved)  # row t
    assert torch.equal(first, R.rotated(x[:5], ang, torch.arange(min(T, 5), device="cuda"), interleaved).to(dt))
    y = wide.clone()
    assert ops.rotary(y[:, :H, :D], ang, pos, interleaved=interleaved, out=y[:, :H, :D]).data_ptr() == y.data_ptr()
    assert torch.equal(y[:, :H, :D], want) and bool(torch.isnan(y[:, :, D:]).all()) and torch.equal(y[:, H, :D], wide[:, H, :D])


def test_rotary_outside_its_table_and_copies():
    case("rotary outside")
    ang = R.angles(10, 32)
    x = rnd(1)((4, 2, 64), torch.bfloat16)
    x[0, 0, 40:44] = torch.tensor([-0.0, float("inf"), NAN, -1.0], dtype=torch.bfloat16)
    y = ops.rotary(x, ang, i32([9, 10, -1, 2 ** 31 - 1]))
    assert not bool(torch.isnan(y[0, :, :32]).any()) and bool(torch.isnan(y[1:, :, :32]).all())
    assert torch.equal(y[..., 32:].view(torch.int16), x[..., 32:].view(torch.int16))
    assert ops.rotary(x[:0], ang).shape == (0, 2, 64)


# ---- the cache


def built(r, lengths, G, D, page, dt, seed=0, scale=1.0, fill=255, columns=None):
    """(cache, table, lengths, keys and values per sequence as the cache has to hold them), appended in one call to
    a cache of bytes `fill`."""
    tab, pool = R.table(lengths, page, seed=seed, columns=columns)
    cache = ops.new_cache(pool, G, page, D)
    cache.fill_(fill)
    T = sum(lengths)
    k, v = r((T, G, D), dt, scale), r((T, G, D), dt, scale)
    ops.cache_append(cache, tab, i32(lengths), k, v, offsets=R.offsets(lengths))
    at, ks, vs = 0, [], []
    hk, hv = R.held(k), R.held(v)
    for n in lengths:
        ks.append(hk[at:at + n])
        vs.append(hv[at:at + n])
        at += n
    return cache, tab, i32(lengths), ks, vs


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("D,G,page,new,before", [
    (64, 1, 16, [1], [0]), (128, 8, 64, [1, 1, 1, 1], [0, 15, 16, 200]), (96, 3, 32, [40, 0, 7], [0, 5, 31]), (192, 2, 16, [17, 33], [15, 0]),
    (256, 2, 128, [3, 130], [127, 0]), (128, 2, 1024, [600, 1, 90], [3, 1023, 500])])
def test_append_and_read(io, D, G, page, new, before):
    case("append", io, D, G, page, new, before)
    dt, T, H = DT[io], sum(new), 2 * G
    r = rnd(T + D)
    lengths = [a + b for a, b in zip(new, before)]
    tab, pool = R.table(lengths, page, seed=T)
    cache = ops.new_cache(pool, G, page, D)
    start = torch.randint(0, 256, cache.shape, device="cuda", dtype=torch.uint8)
    cache.copy_(start)
    wide = r((T, (H + 2 * G) * D + 32), dt)
    q, k, v = (wide[:, i * D:j * D].unflatten(1, (-1, D)) for i, j in ((0, H), (H, H + G), (H + G, H + 2 * G)))
    pos = torch.cat([torch.arange(b, b + n) for n, b in zip(new, before)]).cuda().to(torch.int32)
    for rot, inter in ((D, False), (D // 2, True), (22, False), (0, False)):
        ang = R.angles(max(lengths), rot) if rot else None
        cache.copy_(start)
        got = ops.cache_append(cache, tab, i32(lengths), k, v, offsets=R.offsets(new), rotation=ang, interleaved=inter, q=q if rot else None)
        kt = R.rotated(k, ang, pos, inter) if rot else k.float()
        if rot:
            assert torch.equal(got, R.rotated(q, ang, pos, inter).to(dt))
        want = R.held(kt), R.held(v)
        for d in (torch.float32, torch.bfloat16):
            a, b = ops.cache_read(cache, tab, i32(lengths), T, offsets=R.offsets(new), dtype=d)
            assert same(a, want[0]) and same(b, want[1])
        # every other byte is as it was
        rec = torch.zeros((pool, page), dtype=torch.bool, device="cuda")
        seq = torch.repeat_interleave(torch.arange(len(new)), torch.tensor(new)).cuda()
        rec[tab[seq, pos.long() // page].long(), pos.long() % page] = True
        rec = rec.view(pool, 1, page // 16, 16).expand(pool, G, page // 16, 16)
        kept = torch.cat([rec.repeat_interleave(D // 2, -1),
                          rec.unflatten(-1, (4, 1, 1, 4)).expand(*rec.shape[:3], 4, 16, D // 32, 4).flatten(3), rec.repeat_interleave(D // 32, -1),
                          rec.repeat_interleave(D // 32, -1)], -1)
        assert torch.equal(torch.where(kept, torch.zeros_like(cache), cache), torch.where(kept, torch.zeros_like(start), start))
    if rot == 0 and T == len(new):  # one token each needs no offsets
        again = start.clone()
        ops.cache_append(again, tab, i32(lengths), k, v)
        assert torch.equal(again, cache)


def test_append_in_place_queries_and_rows():
    """q_out may be q; positions name other rows of the table than the places."""
    case("append in place")
    r = rnd(3)
    q, k, v = r((700, 6, 96), torch.bfloat16), r((700, 2, 96), torch.bfloat16), r((700, 2, 96), torch.bfloat16)
    tab, pool = R.table([700], 64)
    cache = ops.new_cache(pool, 2, 64, 96)
    ang, pos = R.angles(900, 96), torch.randint(0, 900, (700,), device="cuda", dtype=torch.int32)
    for inter in (False, True):
        mine = q.clone()
        assert ops.cache_append(cache, tab, i32([700]), k, v, rotation=ang, positions=pos, interleaved=inter, q=mine, q_out=mine) is mine
        assert torch.equal(mine, R.rotated(q, ang, pos, inter).bfloat16())
        a, b = ops.cache_read(cache, tab, i32([700]), 700)
        assert same(a, R.held(R.rotated(k, ang, pos, inter))) and same(b, R.held(v))


def test_cache_values():
    """Every border of the 4-bit grid, small, large and impossible blocks."""
    case("cache values")
    row = torch.zeros(33, 1, 64)
    t = torch.arange(0, 57) / 8.0  # 0 .. 7: every border and tie
    for i, e in enumerate((-70, -64, -63, -10, 0, 1, 60, 124)):
        row[i, 0, :32] = (t[25:57] * 2.0 ** e)
        row[i, 0, 32:57] = -(t[:25] * 2.0 ** e)
        row[i + 8, 0, :31] = t[:31] * 2.0 ** e  # with a larger one beside them
        row[i + 8, 0, 31] = 7.0 * 2.0 ** e
        row[i + 16, 0, :31] = torch.nextafter(t[:31], torch.tensor(100.0)) * 2.0 ** e
        row[i + 16, 0, 31] = torch.nextafter(torch.tensor(7.0), torch.tensor(8.0)) * 2.0 ** e if e < 124 else 0.0
    row[24, 0, 3], row[25, 0, 33], row[26, 0, 40] = float("inf"), NAN, float("-inf")
    row[27, 0, 0] = 3.4e38
    row[28] = -0.0
    row[29, 0, :] = 1e-40
    row = row.cuda()
    tab, pool = R.table([33], 16)
    cache = ops.new_cache(pool, 1, 16, 64)
    ops.cache_append(cache, tab, i32([33]), row, row.flip(-1).contiguous())
    a, b = ops.cache_read(cache, tab, i32([33]), 33, dtype=torch.float32)
    assert same(a, R.held(row)) and same(b, R.held(row.flip(-1)))
    assert bool(torch.isnan(a[24, 0, :32]).all()) and not bool(torch.isnan(a[24, 0, 32:]).any())
    fine = torch.isfinite(R.held(row)) & (row.abs() > 0)
    step = (a - row).abs()[fine] / row.abs().unflatten(-1, (-1, 32)).amax(-1, keepdim=True).expand(33, 1, 2, 32).flatten(-2)[fine]
    # in units of 2^e: from 4 to 6 the numbers are 2 apart, so a value v is off by |v - 4| <= 1 up to 5 and 6 - v <= 1 from there, at most a
    # fifth of v and of the block's largest; past 6 by v - 6 <= 1 of at most 7; below 4 by at most 1/2, with a largest of more than 3.5
    assert float(step[row.abs()[fine] > 1e-18].max()) <= 1 / 5 + 1e-6


def test_padding_rows_bad_pages_and_rows_behind():
    """Places below 0 are not appended; pages that are not there are not written and read as NaN; what lies behind the last sequence stays."""
    case("padding")
    r, G, D, page = rnd(8), 2, 64, 16
    lengths = i32([2, 0, 40, -3])
    n = [4, 3, 40, 2]
    T = sum(n) + 5
    tab = i32([[0, 9, 9], [9, 9, 9], [1, 7, 2], [3, 3, 3]])  # 7 is past the pool's 4 pages
    cache = ops.new_cache(4, G, page, D)
    k, v, q = r((T, G, D), torch.bfloat16), r((T, G, D), torch.bfloat16), r((T, 4, D), torch.bfloat16)
    off = R.offsets(n)
    qo = torch.full_like(q, 7.0)
    ops.cache_append(cache, tab, lengths, k, v, offsets=off, rotation=R.angles(40, 64), q=q, q_out=qo)
    assert bool((qo[sum(n):] == 7.0).all()) and torch.equal(qo[:2], q[:2]) and not torch.equal(qo[3], q[3])  # place 0 turns by nothing
    assert not bool(cache[3].any())
    kk, vv = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    ops.cache_read(cache, tab, lengths, T, offsets=off, k=kk, v=vv)
    for z, w in ((vv, R.held(v)),):
        assert not bool(z[:2].any()) and same(z[2:4], w[2:4]) and not bool(z[4:7].any())
        assert same(z[7:23], w[7:23]) and bool(torch.isnan(z[23:39]).all()) and same(z[39:47], w[39:47])
        assert not bool(z[47:49].any()) and bool((z[49:] == 7.0).all())
    out = torch.full_like(q, 7.0)
    ops.attention(cache, tab, lengths, qo, offsets=off, out=out)
    assert not bool(out[:2].any()) and not bool(out[4:7].any()) and not bool(out[47:49].any()) and bool((out[49:] == 7.0).all())
    assert bool(torch.isfinite(out[7:23]).all()) and bool(torch.isnan(out[23:47]).all()) and bool(torch.isfinite(out[2:4]).all())


# ---- attention


def check(io, H, G, D, page, new, lengths, seed=0, out="io", scale=None, qscale=1.0, columns=None, fill=255):
    dt = DT[io]
    r = rnd(seed + sum(lengths))
    T = sum(new)
    cache, tab, ln, ks, vs = built(r, lengths, G, D, page, dt, seed, fill=fill, columns=columns)
    wide = r((T, H * D + 32), dt, qscale)
    wide[:, H * D:] = NAN
    q = wide[:, :H * D].unflatten(1, (H, D))
    off = None if all(n == 1 for n in new) else R.offsets(new)
    sc = D ** -0.5 if scale is None else scale
    got, scales = ops.attention(cache, tab, ln, q, offsets=off, scale=scale, out_dtype=F8 if out == "f8" else None)
    at = 0
    for b, n in enumerate(new):
        o, mag, most = R.attention(q[at:at + n], ks[b], vs[b], n, sc)
        bd = R.bound(o, mag, most, max(lengths[b], 1), D, dt)
        if out == "io":
            R.close(got[at:at + n], o, bd, f"sequence {b}")
        else:
            s = scales[:, at:at + n].t()[..., None].double()                      # n, blocks, 1
            y = got[at:at + n].float().double().reshape(n, -1, 128) * s
            o, bd = o.reshape(n, -1, 128), bd.reshape(n, -1, 128)
            top = (o.abs().amax(-1, keepdim=True) / 448.0).clamp_min(2.0 ** -64)
            R.close(s, top, bd.amax(-1, keepdim=True) / 448.0 + 4 * R.U32 * top, f"scales {b}")
            R.close(y, o, bd + o.abs() * 2.0 ** -4 + s * 2.0 ** -10 + 8 * R.U32 * o.abs(), f"sequence {b}")
        at += n
    return got


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("H,G", [(1, 1), (8, 2), (7, 1), (20, 1)])
def test_single_tokens(io, D, H, G):
    case("tokens", io, D, H, G)
    check(io, H, G, D, 16, [1] * 9, [1, 2, 15, 16, 17, 31, 33, 64, 129], seed=D + H)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("D,H,G,page", [(128, 8, 2, 64), (64, 4, 4, 16), (256, 6, 1, 32), (96, 16, 2, 128), (192, 3, 3, 1024)])
def test_long_contexts(io, D, H, G, page):
    """Split over many workgroups, in uneven pieces."""
    case("long", io, D, H, G, page)
    check(io, H, G, D, page, [1, 1, 1], [5000, 1, 777], seed=H)
    check(io, H, G, D, page, [3], [3001], seed=H + 1)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("D,H,G,page,new,before", [
    (128, 4, 2, 16, [1, 0, 5, 33], [0, 7, 30, 100]), (64, 8, 1, 32, [70, 3], [0, 61]), (96, 6, 2, 16, [40, 1, 16], [9, 0, 16]),
    (192, 2, 2, 64, [65], [64]), (256, 4, 1, 16, [20, 9], [0, 50]), (128, 3, 1, 64, [7, 0, 0, 11], [90, 3, 0, 5])])
def test_prompts_split(io, D, H, G, page, new, before):
    """Few rows: pieces of sequences."""
    case("prompts", io, D, H, G, page, new, before)
    check(io, H, G, D, page, new, [a + b for a, b in zip(new, before)], seed=D)


@pytest.mark.parametrize("io,D,H,G,new,before", [
    ("bf16", 128, 32, 8, [1100, 1, 900, 0, 130], [0, 40, 300, 5, 64]), ("bf16", 64, 64, 16, [700, 333], [0, 77]), ("bf16", 96, 48, 16, [350, 501], [33, 0]),
    ("bf16", 256, 16, 16, [900, 3200], [10, 0]), ("bf16", 192, 32, 16, [1030, 1100], [0, 1]), ("f32", 128, 32, 16, [1000, 1100], [0, 200]),
    ("f32", 64, 32, 32, [2080, 1], [3, 0]), ("f32", 256, 32, 32, [700, 1400], [0, 64]), ("f32", 192, 32, 16, [2100], [17]), ("f32", 96, 32, 16, [2100], [0])])
def test_prompts_by_rows(io, D, H, G, new, before):
    """Enough rows for a workgroup of them a CU."""
    case("rows", io, D, H, G, new, before)
    check(io, H, G, D, 64, new, [a + b for a, b in zip(new, before)], seed=H)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("D,H,G,new,lengths", [(128, 8, 2, [1, 1, 1], [3, 40, 2000]), (64, 8, 2, [1, 1], [1, 700]), (256, 6, 2, [5, 2], [5, 300]), (64, 12, 2, [40], [64]),
                                               (128, 32, 8, [1200, 900], [1200, 1000]), (64, 64, 16, [1100], [1111]), (256, 16, 16, [1100, 3000], [1200, 3000])])
def test_into_8_bits(io, D, H, G, new, lengths):
    case("8 bits", io, D, H, G, new, lengths)
    check(io, H, G, D, 32, new, lengths, out="f8", seed=D)


def test_scales_and_peaks():
    """Large scores (one key takes all), tiny scales, a maximum that rises by little for long."""
    case("peaks")
    for io in ("bf16", "f32"):
        check(io, 4, 2, 128, 16, [1, 1], [900, 33], qscale=12.0, seed=1)
        check(io, 4, 2, 128, 16, [9], [300], scale=1e-6, seed=2)
        check(io, 4, 2, 64, 16, [1], [4000], scale=1.0, seed=3)
    r = rnd(5)
    k = (torch.ones(1600, 1, 64, device="cuda") * torch.linspace(0.0, 4.0, 1600, device="cuda")[:, None, None])
    tab, pool = R.table([1600], 64)
    cache, v, q = ops.new_cache(pool, 1, 64, 64), r((1600, 1, 64)), torch.ones(1, 1, 64, device="cuda")
    ops.cache_append(cache, tab, i32([1600]), k, v)
    for s in (0.1, 1.0):
        got, _ = ops.attention(cache, tab, i32([1600]), q, scale=s)
        o, mag, most = R.attention(q, R.held(k), R.held(v), 1, s)
        R.close(got, o, R.bound(o, mag, most, 1600, 64, torch.float32), "rising")


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_not_numbers_stay_where_they_are_seen(io):
    """A NaN in a key or value reaches the outputs of its head at tokens that see it, and no other; one behind the sequence reaches nothing."""
    case("nan", io)
    dt, r = DT[io], rnd(2)
    for L, n, G in ((50, 50, 2), (2100, 2100, 16)):
        k, v, q = r((L, G, 128), dt), r((L, G, 128), dt), r((n, 2 * G, 128), dt)
        k[40, 0, 5] = NAN
        v[45, 1, 70] = float("inf")
        tab, pool = R.table([L], 16)
        cache = ops.new_cache(pool, G, 16, 128)
        cache.fill_(255)
        ops.cache_append(cache, tab, i32([L]), k, v)
        bad = torch.isnan(ops.attention(cache, tab, i32([L]), q)[0])
        assert not bool(bad[:40].any()) and not bool(bad[:45, 2:4].any()) and not bool(bad[:, 4:].any())
        assert bool(bad[40:, :2].all()) and bool(bad[45:, 2:4, 64:96].all())
        q2 = q.clone()
        q2[7, 0, 3] = NAN
        assert bool(torch.isnan(ops.attention(cache, tab, i32([L]), q2)[0][7, 0]).all())
        assert torch.equal(torch.isnan(ops.attention(cache, tab, i32([L]), q2)[0])[8:40], bad[8:40])


@pytest.mark.parametrize("fill", [252, 254, 255])
@pytest.mark.parametrize("io,D,H,G,new,before", [("bf16", 128, 4, 2, [5, 1], [30, 17]), ("bf16", 128, 32, 8, [1100, 900], [5, 0]), ("bf16", 64, 64, 16, [700, 333], [0, 77]),
                                                 ("f32", 96, 32, 16, [2100], [3]), ("bf16", 256, 16, 16, [900, 3200], [10, 0])])
def test_anything_behind_a_sequence(fill, io, D, H, G, new, before):
    """Bytes that were never appended, with the largest exponents, infinities and NaN, behind the last token and in its page."""
    case("behind", fill, io, D, H, G, new, before)
    check(io, H, G, D, 32, new, [a + b for a, b in zip(new, before)], fill=fill, seed=fill)


@pytest.mark.parametrize("H,G,n", [(4, 2, 40), (32, 16, 2100)])
def test_a_page_that_is_not_there(H, G, n):
    """Rows before its first place are as they are, whatever bytes the cache begins with; the others are NaN."""
    case("no page", H, G, n)
    r = rnd(n)
    for fill in (0, 254):
        cache, tab, ln, ks, vs = built(r, [n], G, 128, 16, torch.bfloat16, fill=fill)
        k0 = torch.full_like(cache[0], fill)
        spare = [p for p in range(cache.shape[0]) if p not in tab.tolist()[0]][0]
        cache[spare] = cache[0]  # page 0 holds bytes that were never appended
        tab[tab == 0] = spare
        cache[0] = k0
        tab[0, 1] = -1  # places 16 .. 31
        q = r((n, H, 128), torch.bfloat16)
        got, _ = ops.attention(cache, tab, ln, q, offsets=R.offsets([n]))
        o, mag, most = R.attention(q[:16], ks[0][:16], vs[0][:16], 16, 128 ** -0.5)
        R.close(got[:16], o, R.bound(o, mag, most, 16, 128, torch.bfloat16), "before")
        assert bool(torch.isnan(got[16:]).all())


def test_equal_calls_and_equal_forms():
    """Equal calls give equal bits; offsets of ones are no offsets; a token's output does not hang on who shares its call."""
    case("equal")
    r, G, D = rnd(4), 2, 128
    lengths = [1, 400, 33, 1500]
    cache, tab, ln, _, _ = built(r, lengths, G, D, 64, torch.bfloat16)
    q = r((4, 8, D), torch.bfloat16)
    a, _ = ops.attention(cache, tab, ln, q)
    b, _ = ops.attention(cache, tab, ln, q)
    c, _ = ops.attention(cache, tab, ln, q, offsets=R.offsets([1] * 4))
    assert torch.equal(a, b) and torch.equal(a, c)
    # strided queries, a given output and workspace
    wide = torch.full((4, 8, D + 8), NAN, dtype=torch.bfloat16, device="cuda")
    wide[..., :D] = q
    out = torch.full((4, 8 * D + 64), 7.0, dtype=torch.bfloat16, device="cuda")
    need = B.load().sketchssm_attention_workspace(B.Cache(cache.data_ptr(), cache.shape[0], G, 64, D), 8, 4, 4, tab.shape[1])
    ops.attention(cache, tab, ln, wide[..., :D], out=out[:, :8 * D].unflatten(1, (8, D)), workspace=torch.empty(need, dtype=torch.uint8, device="cuda"))
    assert torch.equal(out[:, :8 * D].unflatten(1, (8, D)), a) and bool((out[:, 8 * D:] == 7.0).all())


def test_a_wide_table():
    """A table for contexts far longer than any there is."""
    case("wide table")
    check("bf16", 4, 1, 128, 16, [1, 1], [70, 3], columns=5000)
    check("bf16", 4, 1, 128, 1024, [2, 0], [2, 0], columns=1000)


@pytest.mark.parametrize("columns,page,length", [(1, 128, 129), (1, 128, 140), (8, 16, 200), (2, 16, 33), (3, 1024, 4000)])
def test_lengths_past_the_table(columns, page, length):
    """Tokens past the table's last column read as NaN, also where its places are whole rounds of steps."""
    case("past", columns, page, length)
    r = rnd(columns)
    cap = columns * page
    cache, tab, _, _, _ = built(r, [cap, 5], 2, 64, page, torch.bfloat16)
    assert tab.shape[1] == columns
    q = r((4, 4, 64), torch.bfloat16)
    out, _ = ops.attention(cache, tab, i32([length, 5]), q, offsets=R.offsets([2, 2]))
    seen = torch.isnan(out).all(-1)
    assert bool(seen[1].all()) and not bool(torch.isnan(out[2:]).any()) and bool(seen[0].all()) == (length - 2 >= cap)


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("B,longest,H,G,D", [(300, 40, 4, 2, 64), (700, 9, 2, 1, 128), (65, 900, 8, 1, 128), (130, 300, 6, 2, 96), (257, 260, 4, 4, 256)])
def test_many_sequences(io, B, longest, H, G, D):
    """More sequences than lanes and than threads; workgroups whose share is parts of several."""
    case("many", io, B, longest, H, G, D)
    g = torch.Generator().manual_seed(B)
    lengths = [int(x) for x in torch.randint(0, longest + 1, (B,), generator=g)]
    new = [min(1, n) for n in lengths] if B != 130 else [min(n, int(x)) for n, x in zip(lengths, torch.randint(0, 4, (B,), generator=g))]
    check(io, H, G, D, 16, new, lengths, seed=B)


@pytest.mark.parametrize("io,D,H,G", [("bf16", 128, 32, 8), ("bf16", 96, 64, 16), ("f32", 128, 32, 16), ("bf16", 256, 16, 8)])
def test_padding_rows_of_prompts(io, D, H, G):
    """Places below 0 among rows enough for a workgroup of them a CU: zeros, and the rows behind them as without."""
    case("padding of prompts", io, D, H, G)
    dt, r = DT[io], rnd(D)
    lengths, pad = [1300, 700], [37, 1000]
    cache, tab, ln, ks, vs = built(r, lengths, G, D, 64, dt)
    q = r((sum(lengths) + sum(pad), H, D), dt)
    n = [a + b for a, b in zip(lengths, pad)]
    got, _ = ops.attention(cache, tab, ln, q, offsets=R.offsets(n))
    at = 0
    for b in range(2):
        assert not bool(got[at:at + pad[b]].any())
        o, mag, most = R.attention(q[at + pad[b]:at + n[b]], ks[b], vs[b], lengths[b], D ** -0.5)
        R.close(got[at + pad[b]:at + n[b]], o, R.bound(o, mag, most, lengths[b], D, dt), f"sequence {b}")
        at += n[b]


def test_a_cache_past_4_gib():
    """Pages whose bytes lie past 2^32 of the cache's start, written, read and attended to."""
    case("4 GiB")
    r, G, D, page, pages = rnd(6), 8, 256, 1024, 2100
    cache = torch.empty((pages, G, page // 16, 17 * D), dtype=torch.uint8, device="cuda")
    assert cache.numel() > 1 << 32
    lengths, new = [1500, 40], [1500, 40]
    tab = i32([[2099, 2050], [2098, -1]])
    k, v, q = r((1540, G, D), torch.bfloat16), r((1540, G, D), torch.bfloat16), r((1540, G, D), torch.bfloat16)
    ops.cache_append(cache, tab, i32(lengths), k, v, offsets=R.offsets(new))
    a, b = ops.cache_read(cache, tab, i32(lengths), 1540, offsets=R.offsets(new))
    hk, hv = R.held(k), R.held(v)
    assert same(a, hk) and same(b, hv)
    one, _ = ops.attention(cache, tab, i32(lengths), q[[1499, 1539]])
    for got, rows in ((ops.attention(cache, tab, i32(lengths), q, offsets=R.offsets(new))[0], None), (one, True)):
        for s, at, L in ((0, 0, 1500), (1, 1500, 40)):
            qs = q[at:at + L] if rows is None else q[at + L - 1:at + L]
            g = got[at:at + L] if rows is None else got[s:s + 1]
            o, mag, most = R.attention(qs, hk[at:at + L], hv[at:at + L], qs.shape[0], D ** -0.5)
            R.close(g, o, R.bound(o, mag, most, L, D, torch.bfloat16), f"sequence {s}")


def test_outputs_between_the_queries_rows():
    """Queries turned, and outputs written, where others' rows lie between; the same on a table with unused columns of anything."""
    case("between")
    r, H, G, D = rnd(12), 4, 2, 64
    lengths = [30, 5]
    cache, tab, ln, ks, vs = built(r, lengths, G, D, 16, torch.bfloat16)
    wide = r((35, 2 * H * D), torch.bfloat16)
    q, out = wide[:, :H * D].unflatten(1, (H, D)), wide[:, H * D:].unflatten(1, (H, D))
    want, _ = ops.attention(cache, tab, ln, q.clone(), offsets=R.offsets(lengths))
    ops.attention(cache, tab, ln, q, offsets=R.offsets(lengths), out=out)
    assert torch.equal(out, want)
    more = torch.full((2, 200), -(1 << 31), dtype=torch.int32, device="cuda")
    more[:, :tab.shape[1]] = tab
    assert torch.equal(ops.attention(cache, more, ln, wide[:, :H * D].unflatten(1, (H, D)), offsets=R.offsets(lengths))[0], want)


def test_refused_before_any_launch():
    """What the calls on tensors refuse: wrong types, shapes, devices and layouts."""
    case("refusals")
    r = rnd(1)
    tab, pool = R.table([20], 16)
    cache = ops.new_cache(pool, 2, 16, 64)
    k, q, ln = r((20, 2, 64), torch.bfloat16), r((20, 4, 64), torch.bfloat16), i32([20])
    ang = R.angles(20, 64)
    good = dict(cache=cache, table=tab, lengths=ln)
    for kw in (dict(cache=cache.float()), dict(cache=cache[..., :-1]), dict(cache=cache.cpu()), dict(cache=cache[:, :, :, ::2]), dict(table=tab.long()), dict(table=tab.cpu()),
               dict(table=tab[0]), dict(lengths=ln.long()), dict(lengths=i32([20, 1])), dict(offsets=R.offsets([20]).long()), dict(offsets=R.offsets([10, 10]))):
        with pytest.raises(ValueError):
            ops.attention(*{**good, **{x: y for x, y in kw.items() if x != "offsets"}}.values(), q, offsets=kw.get("offsets"))
        with pytest.raises(ValueError):
            ops.cache_append(*{**good, **{x: y for x, y in kw.items() if x != "offsets"}}.values(), k, k, offsets=kw.get("offsets"))
        with pytest.raises(ValueError):
            ops.cache_read(*{**good, **{x: y for x, y in kw.items() if x != "offsets"}}.values(), 20, offsets=kw.get("offsets"))
    for f in (lambda: ops.attention(cache, tab, ln, q.half()), lambda: ops.attention(cache, tab, ln, q[..., :32]), lambda: ops.attention(cache, tab, ln, q.cpu()),
              lambda: ops.attention(cache, tab, ln, q.transpose(1, 2)), lambda: ops.attention(cache, tab, ln, q, out=q[:, :2]), lambda: ops.attention(cache, tab, ln, q[0]),
              lambda: ops.attention(cache, tab, ln, q, scales=torch.zeros(2, 20, device="cuda")), lambda: ops.attention(cache, tab, ln, q, out=torch.zeros_like(q).float()),
              lambda: ops.cache_append(cache, tab, ln, k, k[:, :1]), lambda: ops.cache_append(cache, tab, ln, k, k.float()), lambda: ops.cache_append(cache, tab, ln, k, k, q=q),
              lambda: ops.cache_append(cache, tab, ln, k, k, positions=i32(list(range(20)))), lambda: ops.cache_append(cache, tab, ln, k, k, q_out=q),
              lambda: ops.cache_append(cache, tab, ln, k, k, rotation=ang, positions=i32([0, 1])), lambda: ops.cache_append(cache, tab, ln, k, k, rotation=ang.double()),
              lambda: ops.cache_read(cache, tab, ln, 20, dtype=torch.float16), lambda: ops.cache_read(cache, tab, ln, 20, k=q), lambda: ops.rotary(q, ang[0]),
              lambda: ops.rotary(q, ang, positions=i32([1])), lambda: ops.rotary(q[0], ang), lambda: ops.rotary(q, ang, out=q[:, :, :32])):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: ops.attention(cache, tab, ln, q, scale=-1.0), lambda: ops.attention(cache, tab, ln, q[:, :3]), lambda: ops.rotary(q, R.angles(20, 66)),
              lambda: ops.rotary(q[:, :2], ang, out=q[:, 1:3]), lambda: ops.attention(cache, tab, ln, q, scale=float("inf")), lambda: ops.new_cache(4, 2, 24, 64), lambda: ops.new_cache(4, 2, 16, 80)):
        with pytest.raises(B.SketchSSMError):
            f()


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("H,G,D,n,before", [(4, 2, 128, 1, 1100), (8, 2, 64, 3, 700), (32, 16, 128, 2100, 200), (16, 16, 256, 2100, 100)])
def test_first_scores_that_overflow(io, H, G, D, n, before):
    """Products of the first 64 keys and every query below -3.4e38 weigh nothing, and the others as without them."""
    case("overflow", io, H, G, D, n, before)
    dt, r = DT[io], rnd(before)
    L = n + before
    q = (r((n, H, D), torch.bfloat16).abs().clamp_min(0.25) * 1024).to(dt)  # without low parts, whose signs would differ
    k, v = r((L, G, D), dt, 2.0 ** -10), r((L, G, D), dt)
    k[:64] = -2.0 ** 124
    tab, pool = R.table([L], 32)
    cache = ops.new_cache(pool, G, 32, D)
    ops.cache_append(cache, tab, i32([L]), k, v)
    got, _ = ops.attention(cache, tab, i32([L]), q, offsets=R.offsets([n]))
    o, mag, most = R.attention(q, R.held(k[64:]), R.held(v[64:]), n, D ** -0.5)
    R.close(got, o, R.bound(o, mag, most, L, D, dt), "out")


@pytest.mark.parametrize("B,T,H,G,D,length", [(16383, 65536, 8, 1, 64, 4096), (16381, 65536, 16, 2, 128, 3000), (5000, 20000, 4, 4, 64, 700), (40, 1500, 32, 8, 128, 900)])
def test_offsets_that_do_not_rise(B, T, H, G, D, length):
    """Nothing is written beside the outputs, whatever the offsets say (sums of rows and rounds past 2^31 among them), and the next call is right."""
    case("wild offsets", B, T, H, G, D, length)
    r = rnd(B)
    cache, tab, ln, ks, vs = built(r, [length], G, D, 64, torch.bfloat16)
    q = r((T, H, D), torch.bfloat16)
    room = torch.full((T + 64, H, D), 7.0, dtype=torch.bfloat16, device="cuda")
    want = ops.attention(cache, tab, ln, q[:1])[0]
    off = torch.zeros(B + 1, dtype=torch.int32)
    off[1::2] = 1 << 30
    off[2::6] = -5
    ops.attention(cache, tab.expand(B, -1).contiguous(), ln.expand(B).contiguous(), q, offsets=off.cuda(), out=room[32:32 + T])
    torch.cuda.synchronize()
    assert bool((room[:32] == 7).all()) and bool((room[32 + T:] == 7).all())
    assert torch.equal(ops.attention(cache, tab, ln, q[:1])[0], want)


@pytest.mark.parametrize("B,H,G,D,longest", [(1, 32, 8, 128, 9000), (5, 16, 1, 64, 700), (40, 8, 4, 256, 500), (3, 7, 1, 96, 3000), (70, 12, 6, 192, 200)])
def test_single_tokens_keep_16_bits_of_a_weight(B, H, G, D, longest):
    """A bf16 output of single tokens is off by its own rounding and 2^-16 of the weights: each is two bf16 parts, the second half a step (2^-8) of the first off by
    2^-8 of itself; twice, for the sum of the weights."""
    case("two parts", B, H, G, D, longest)
    r = rnd(longest)
    lengths = [longest - (b * 37) % (longest // 2) for b in range(B)]
    cache, tab, ln, ks, vs = built(r, lengths, G, D, 64, torch.bfloat16)
    q = r((B, H, D), torch.bfloat16)
    got, _ = ops.attention(cache, tab, ln, q)
    for b in range(B):
        o, mag, most = R.attention(q[b:b + 1], ks[b], vs[b], 1, D ** -0.5)
        fp32 = R.bound(o, mag, most, lengths[b], D, torch.float32)
        R.close(got[b:b + 1], o, fp32 + 2 * 2.0 ** -16 * mag + (o.abs() + fp32 + 2.0 ** -15 * mag) * R.U16, f"sequence {b}")
