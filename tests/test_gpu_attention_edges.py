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
