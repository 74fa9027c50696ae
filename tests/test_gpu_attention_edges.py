"""The ends of what the attention layer's operators take: lengths, scores and values as small and as large as they can be."""
import pytest
import torch

import attention_reference as R
from paper_2609_33051_amd import ops
from test_gpu_attention import DT, case, i32, rnd, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("length", [-(1 << 31), -(1 << 31) + 3, -(1 << 30), -(1 << 30) - 1, -1])
def test_the_smallest_lengths(io, length):
    """A token at a place below 0 is a padding row however far below: not appended, its query copied, read as 0, its attention 0."""
    case("smallest lengths", io, length)
    r, dt, G, D = rnd(3), DT[io], 2, 64
    new, lengths = [2, 5, 3], i32([2, length, 3])
    q, k, v = r((10, 4, D), dt), r((10, G, D), dt), r((10, G, D), dt)
    cache = ops.new_cache(4, G, 16, D)
    tab, off = i32([[0], [1], [2]]), R.offsets(new)
    got = ops.cache_append(cache, tab, lengths, k, v, offsets=off, rotation=R.angles(16, 32), q=q)
    pos = i32([0, 1, 0, 0, 0, 0, 0, 0, 1, 2])
    assert torch.equal(got[2:7], q[2:7]) and torch.equal(got[[0, 1, 7, 8, 9]], R.rotated(q, R.angles(16, 32), pos, False).to(dt)[[0, 1, 7, 8, 9]])
    assert not bool(cache[1].any()) and not bool(cache[3].any())
    a, b = ops.cache_read(cache, tab, lengths, 10, offsets=off)
    assert not bool(a[2:7].any()) and not bool(b[2:7].any()) and same(b[7:], R.held(v[7:]))
    out, _ = ops.attention(cache, tab, lengths, got, offsets=off)
    assert not bool(out[2:7].any()) and bool(torch.isfinite(out).all()) and bool(out[[0, 1, 7, 8, 9]].any(-1).all())


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("rising,D,H,G,new,lengths,last", [
    (False, 128, 8, 2, [1, 1], [5000, 900], 1), (True, 128, 8, 2, [1, 1], [4362, 4300], 1), (False, 64, 8, 2, [300, 77], [8300, 12077], 300),
    (True, 64, 8, 2, [300], [4500], 300), (True, 128, 32, 8, [4362], [4362], 200), (False, 256, 16, 16, [2100, 1000], [2100, 1000], 200)])
def test_scores_far_from_zero(io, rising, D, H, G, new, lengths, last):
    """Scores 1.5 2^22 + {0 .. 6}, whole in fp32, over maxima that differ from wave to wave or move on the way: their product with log2 e is
    rounded to whole numbers, by the same for all that a row's sums are made of.  What counts is how far scores lie apart, 6."""
    case("far scores", io, rising, D, H, G, new, lengths)
    dt, T = DT[io], sum(lengths)
    k, v = torch.zeros((T, G, D), dtype=dt, device="cuda"), torch.zeros((T, G, D), dtype=dt, device="cuda")
    k[..., :32] = 192.0
    grid = torch.tensor(R.GRID, device="cuda")
    at = 0
    for n in lengths:
        j = torch.arange(n, device="cuda")
        # rising: 4096 keys of 0, then 6, so that the weights' sum passes 2^16 some 150 keys later
        f = torch.where(j < 4096, 0.0, 6.0) if rising else grid[j // 32 % 8]
        k[at:at + n, :, 32] = f[:, None].to(dt)
        v[at:at + n] = (torch.where(j < 4096 + 128, 1.0, -1.0) if rising else torch.where(j // 32 % 3 == 0, 1.0, -1.0))[:, None, None].to(dt)
        at += n
    tab, pages = R.table(lengths, 32)
    cache = ops.new_cache(pages, G, 32, D)
    ops.cache_append(cache, tab, i32(lengths), k, v, offsets=R.offsets(lengths))
    q = torch.zeros((sum(new), H, D), dtype=dt, device="cuda")
    q[..., :32], q[..., 32] = 1024.0, 1.0
    got, _ = ops.attention(cache, tab, i32(lengths), q, offsets=R.offsets(new), scale=1.0)
    a, t = 0, 0
    for n, length in zip(new, lengths):
        a, t = a + length, t + n
        m = min(n, last)
        o, mag, most = R.attention(q[t - m:t], k[a - length:a], v[a - length:a], m, 1.0)
        R.close(got[t - m:t], o, R.bound(o, mag, torch.full_like(most, 6.0), length, D, dt), f"{length} keys")


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("out", ["io", "f8"])
@pytest.mark.parametrize("D,H,G,new,lengths", [(128, 8, 2, [1, 1], [9000, 700]), (64, 8, 2, [300], [8300]), (128, 32, 8, [1100, 900], [1200, 1000]), (256, 16, 16, [2100, 1000], [2100, 1000])])
def test_the_largest_values(io, out, D, H, G, new, lengths):
    """Values of up to 2^80 under scores that rise to ten (weights of up to 2^14 over a maximum that stays): sums stay in fp32's range."""
    case("largest values", io, out, D, H, G, new, lengths)
    dt, r, T = DT[io], rnd(D + len(new)), sum(lengths)
    k, v = torch.zeros((T, G, D), dtype=dt, device="cuda"), r((T, G, D), torch.float32).clamp(-4, 4) * 2.0 ** 78
    v = v.to(dt)
    at = 0
    for n in lengths:
        k[at:at + n, :, :2] = (torch.arange(n, device="cuda") * (10.0 / n)).to(dt)[:, None, None]
        at += n
    tab, pages = R.table(lengths, 32)
    cache = ops.new_cache(pages, G, 32, D)
    ops.cache_append(cache, tab, i32(lengths), k, v, offsets=R.offsets(lengths))
    q = torch.zeros((sum(new), H, D), dtype=dt, device="cuda")
    q[..., 0] = 1.0
    got, scales = ops.attention(cache, tab, i32(lengths), q, offsets=R.offsets(new), scale=1.0, out_dtype=torch.float8_e4m3fn if out == "f8" else None)
    hk, hv = R.held(k), R.held(v)
    a, t = 0, 0
    for n, length in zip(new, lengths):
        a, t = a + length, t + n
        m = min(n, 200)
        o, mag, most = R.attention(q[t - m:t], hk[a - length:a], hv[a - length:a], m, 1.0)
        bd = R.bound(o, mag, most, length, D, dt)
        if out == "io":
            R.close(got[t - m:t], o, bd, f"{length} keys")
            continue
        s = scales[:, t - m:t].t()[..., None].double()
        o, bd = o.reshape(m, -1, 128), bd.reshape(m, -1, 128)
        R.close(got[t - m:t].float().double().reshape(m, -1, 128) * s, o, bd + o.abs() * 2.0 ** -4 + s * 2.0 ** -10 + 8 * R.U32 * o.abs(), f"{length} keys")
