"""The operators over the 8-bit cache at the ends of what their arguments may be, against tests/byte_cache_util.py."""

import pytest

from test_gpu_byte_cache import cache_of, data, ints

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("counts", [None, [70, 69, 1, 64, 5, 33]])
def test_lengths_at_the_end_of_their_range_store_nothing(counts):
    """Lengths within the count of -2^31, whose difference has no 32 bits."""
    low = -(1 << 31)
    k, _ = data(7, 6, 70, 2, 32, "f32")
    for lens in ([low] * 6, [low + 1] * 6, [low + (70 if counts is None else c) - 1 for c in counts or [0] * 6]):
        cache = cache_of(6, 2, 32, 128)
        buffers = (cache.k, cache.v, cache.k_scale, cache.v_scale, cache.k_tail, cache.v_tail)
        was = [t.clone() for t in buffers]
        cache.append(k, k, ints(lens), counts=None if counts is None else ints(counts))
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(was, buffers)), lens


@pytest.mark.parametrize("back", [201, 192, 128, 64, 0])
def test_tokens_taken_back(back):
    """Within the block that is not whole yet, or to whole blocks: what is left, and what comes after, is as if they had never been there."""
    import numpy as np
    from test_gpu_byte_cache import check_contents
    k, kn = data(11, 2, 400, 2, 64, "f16")
    q, _ = data(12, 2, 3, 2, 64, "f16")
    cache, other = cache_of(2, 2, 64, 400), cache_of(2, 2, 64, 400)
    cache.append(k[:, :215], k[:, :215], ints([215] * 2))
    if back:
        other.append(k[:, :back], k[:, :back], ints([back] * 2))
    assert torch.equal(cache.attention(q, ints([back] * 2)), other.attention(q, ints([back] * 2)))
    assert torch.equal(cache.read(ints([back] * 2), 220)[1], other.read(ints([back] * 2), 220)[1])
    new = k[:, 300:400]
    cache.append(new, new, ints([back + 100] * 2))
    other.append(new, new, ints([back + 100] * 2))
    for r in range(2):
        check_contents(cache, r, *[np.concatenate([kn[r, :back], kn[r, 300:]])] * 2, back + 100)
    assert torch.equal(cache.attention(q, ints([back + 100] * 2)), other.attention(q, ints([back + 100] * 2)))


@pytest.mark.parametrize("rows", [1, 40])
def test_a_bound_on_the_lengths_that_32_bits_do_not_hold(rows):
    k, _ = data(13, 1, 300, 1, 64, "bf16")
    q, _ = data(14, 1, rows, 1, 64, "bf16")
    cache = cache_of(1, 1, 64, 300)
    cache.append(k, k, ints([300]))
    want = cache.attention(q, ints([300]))
    for bound in (300, 320, 321, (1 << 31) - 1, 1 << 31, (1 << 32) + 1, (1 << 32) + 64, 1 << 70):
        assert torch.equal(cache.attention(q, ints([300]), max_len=bound), want), bound
