"""Pieces of a prompt with bf16 queries that fill the chip, and launches whose heads do not fill the XCDs evenly."""

import numpy as np
import pytest

from test_gpu_byte_cache import LENS28, cache_of, check_attention, data, ints

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [32, 64, 96, 128])
@pytest.mark.parametrize("rows,heads,kv,strided", [(100, 8, 8, False), (130, 4, 4, True), (50, 24, 8, False)])
def test_ragged_requests_with_limits(dim, rows, heads, kv, strided):
    limits = [[max(n - rows + i + 1 - 3 * (r % 2), 0) for i in range(rows)] for r, n in enumerate(LENS28)]
    check_attention("bf16", LENS28, rows, heads, kv, dim, row_limit=limits, strided=strided, seed=dim, room=70)


@pytest.mark.parametrize("dim", [64, 128])
def test_tags(dim):
    rows, rng = 100, np.random.default_rng(8)
    tags = [[int(x) for x in np.sort(rng.integers(0, 5, max(n, 1)))] for n in LENS28]
    check_attention("bf16", LENS28, rows, 8, 8, dim, tags=(tags, [[i % 6 - 1 for i in range(rows)] for _ in LENS28]), scale=-0.2, seed=3)
    check_attention("bf16", [200] * 28, rows, 8, 8, dim, max_len=230, seed=4)


def test_nan_stays_where_it_is():
    k, _ = data(96, 28, 190, 8, 64, "bf16")
    q, _ = data(97, 28, 100, 8, 64, "bf16")
    limit = ints([[64 if i < 30 else 128 if i < 60 else 190 for i in range(100)]] * 28)
    lens, out = ints([190] * 28), []
    for bad in (False, True):
        kk, vv, qq = k.clone(), k.flip(1).contiguous(), q.clone()
        if bad:
            kk[3, 100, 2, 5] = vv[4, 70, 1, 7] = vv[5, 150, 0, 9] = qq[6, 40, 3, 1] = float("nan")
            qq[7, 50, 4, 2] = float("inf")
        cache = cache_of(28, 8, 64, 200)
        cache.append(kk, vv, lens)
        out.append(cache.attention(qq, lens, row_limit=limit))
    moved = (out[0] != out[1]).any(dim=3)
    want = torch.zeros_like(moved)
    want[3, 30:, 2] = want[4, 30:, 1] = want[5, 60:, 0] = want[6, 40, 3] = want[7, 50, 4] = True
    assert torch.equal(moved, want)
    assert torch.isnan(out[1][3, 30:, 2]).all() and torch.isnan(out[1][6, 40, 3]).all() and torch.isnan(out[1][7, 50, 4]).all()
    assert torch.isnan(out[1][5, 60:, 0, 9]).all()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("req,rows,heads,kv", [(17, 130, 7, 7), (3, 33, 3, 3), (1, 200, 9, 9), (2, 65, 12, 6), (1, 300, 1, 1)])
def test_heads_that_are_no_multiple_of_eight(kind, req, rows, heads, kv):
    """119 heads of two groups of 128 columns, 9 (eight on an XCD each, one on all), 12, and one."""
    lens = [max(400 - 31 * r, 1) for r in range(req)]
    limits = [[max(n - rows + i + 1, 0) for i in range(rows)] for n in lens]
    check_attention(kind, lens, rows, heads, kv, 64, row_limit=limits, seed=rows)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_few_heads_of_long_caches_in_groups_and_splits(kind):
    check_attention(kind, [5001], 40, 1, 1, 64, seed=5)
    check_attention(kind, [3000, 100], 50, 10, 5, 32, seed=6)
