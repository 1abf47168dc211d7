"""Attention over the 8-bit cache where the value scales of its blocks lie far apart, against tests/byte_cache_util.py.

The rows: one token (or one of each wave's) takes half of the sum, thousands of others, all of them alike, the other half.  All
tokens lie in whole blocks, and all scores but that token's are 0, so that what is left of the errors is small enough to see what
the scales cost.  There are as many heads as it takes for every wave to go through several blocks."""

import math

import numpy as np
import pytest

import byte_cache_util as u
from test_gpu_byte_cache import DEV, TYPES, cache_of, ints

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def bounds(kind, out, mag, top, tokens, largest, blocks):
    """Largest error of (out, lse) for the tokens of whole blocks whose scores are products of few codes.

    A probability: its score is four fp32 factors (2^-24 each of the score, and of the exponent, below 48 in magnitude for the sum
    with the reference and, bf16 and half, the logarithm of the ratio: 2^-19 for those), the exponential 2^-22, as an operand 2^-11
    (bf16; a half has 11 bits, so it is off by up to torch.finfo(torch.float16).eps / 2) or 2^-22, but by half of the smallest half,
    2^-25, at least: over 2^7 (2^11 for pairs), 1/2 as the reference is rounded up and 1/4 as the value scale's reference is within
    4 times it, 2^-29 (2^-33) of the row's largest; in the outputs times 127 times a scale, at most the largest value.  Sums: 64
    additions in the matrix instruction, one per block of a wave, and at most 64 of waves and splits, of positive numbers: 2^-24 each, in the
    sums and, of the magnitudes, in the outputs."""
    prob = top * 2.0 ** -22 + 2.0 ** -22 + (2.0 ** -11 if kind == "bf16" else 2.0 ** -22) + (0 if kind == "f32" else 2.0 ** -19)
    least = tokens * 2.0 ** (-29 if kind == "bf16" else -33)
    adds = (64 + blocks + 64) * 2.0 ** -24
    total = prob + least + adds
    rounded = np.maximum(np.abs(out) * u.HALF_STEP[kind], u.SMALLEST[kind])
    p, t = prob[..., None], total[..., None]
    return (mag * (p + adds) + least * largest + np.abs(out) * t) * 1.01 + rounded, total + (top + 16) * 2.0 ** -23


def plain_cache(seed, req, heads, dim, v_scale, k_scale=2.0 ** -7, waves=1):
    """Codes of a cache whose keys are 0 but for one token, or one in the blocks of each of some waves (b mod `waves`)."""
    rng, n_blk = np.random.default_rng(seed), len(v_scale)
    k = np.zeros((req, heads, n_blk, 64, dim), dtype=np.int8)
    for w in range(waves):
        k[:, :, w + waves * int(rng.integers(n_blk // waves)), int(rng.integers(64)), 3] = 100
    v = rng.integers(-127, 128, (req, heads, n_blk, dim, 64), dtype=np.int8)
    nan = lambda *shape: np.full((req, heads, 2, *shape), np.nan, dtype=np.float16)  # noqa: E731
    scales = [np.broadcast_to(np.asarray(x, dtype=np.float32), (req, heads, n_blk)).copy() for x in (k_scale, v_scale)]
    return {"k": k, "v": v, "k_scale": scales[0], "v_scale": scales[1], "k_tail": nan(64, dim), "v_tail": nan(dim, 64)}


def made(plain, heads=None):
    """The cache; heads: that many of the one that there is."""
    from paper_2506_23431_amd import ByteCache
    tensors = {name: torch.from_numpy(x).to(DEV) for name, x in plain.items()}
    return ByteCache.from_tensors(**{name: t if heads is None else t.expand(-1, heads, *t.shape[2:]) for name, t in tensors.items()})


def held(plain, r, h):
    """Keys and values [token][1][dim] of one request and head in 64 bits."""
    k = plain["k"][r, h].astype(np.float64) * plain["k_scale"][r, h, :, None, None].astype(np.float64)
    v = plain["v"][r, h].astype(np.float64) * plain["v_scale"][r, h, :, None, None].astype(np.float64)
    return [x.reshape(-1, 1, x.shape[-1]) for x in (k, v.swapaxes(-1, -2))]


def queries(kind, req, rows, heads, dim, tokens):
    """Queries whose score with such a token is about ln(tokens) (scale 1): half of the sum of that many."""
    q = np.zeros((req, rows, heads, dim), dtype=np.float32)
    q[..., 3] = (math.log(tokens) / (100 * 2.0 ** -7)) * (1 - 0.01 * np.arange(rows)[:, None] / rows)
    t = torch.from_numpy(q).to(TYPES[kind])
    return t.to(DEV), t.float().numpy().astype(np.float64)


def check(kind, cache, q, qn, n, held_by, limits=None, blocks=None):
    """held_by: {(request, head): keys and values}; blocks: the most that one wave goes through, if known."""
    req, rows = qn.shape[:2]
    out, lse = cache.attention(q, ints([n] * req), scale=1.0, with_lse=True, max_len=n,
                               row_limit=None if limits is None else ints([limits] * req))
    out, lse = out.double().cpu().numpy(), lse.cpu().numpy()
    worst = [0.0, 0.0]
    sees = np.ones((rows, n), dtype=bool) if limits is None else np.arange(n)[None] < np.array(limits)[:, None]
    for (r, h), (k, v) in held_by.items():
        want, wl, mag, (_, top, _) = u.attend(qn[r][:, h:h + 1], k, v, sees, 1.0)
        largest = np.array([np.abs(v[s]).max() for s in sees])[:, None, None]
        tol, tl = bounds(kind, want, mag, top, n, largest, blocks or n // 64)
        worst = [max(worst[0], (np.abs(out[r][:, h:h + 1] - want) / tol).max()), max(worst[1], (np.abs(lse[r][:, h:h + 1] - wl) / tl).max())]
    print(f"[scales] {kind}: out at {worst[0]:.2f}, lse at {worst[1]:.2f} of the tolerance")
    assert worst[0] <= 1 and worst[1] <= 1, worst


def apart(order, power, n_blk):
    """Value scales: all blocks of one half 2^-power of those of the other one, or some here and there."""
    high, half = 0.7, n_blk // 2
    low = high * 2.0 ** -power
    if order == "mixed":
        return [high if x else low for x in np.random.default_rng(n_blk).integers(0, 2, n_blk)]
    return [low] * half + [high] * (n_blk - half) if order == "up" else [high] * half + [low] * (n_blk - half)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("order", ["up", "down", "mixed"])
@pytest.mark.parametrize("power", [0, 2, 6, 11, 13])
@pytest.mark.parametrize("rows,heads,dim", [(1, 1, 128), (1, 64, 128), (40, 64, 32)])
def test_flat_rows_over_value_scales_that_lie_apart(kind, order, power, rows, heads, dim):
    n = 8192
    plain = plain_cache(power, 1, heads, dim, apart(order, power, n // 64))
    q, qn = queries(kind, 1, rows, heads, dim, n)
    check(kind, made(plain), q, qn, n, {(0, h): held(plain, 0, h) for h in {0, heads // 2}})


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("order,power", [("down", 11), ("up", 13), ("mixed", 6)])
def test_long_flat_rows(kind, order, power):
    n, heads = 65536, 16
    plain = plain_cache(power, 1, heads, 64, apart(order, power, n // 64))
    q, qn = queries(kind, 1, 2, heads, 64, n)
    check(kind, made(plain), q, qn, n, {(0, h): held(plain, 0, h) for h in (0, 9)})


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("order,power", [("down", 11), ("mixed", 11), ("down", 10), ("mixed", 4)])
def test_every_wave_has_a_token_that_takes_half_of_its_sum(kind, order, power):
    """300 heads: no splits, eight waves of 128 blocks each."""
    n, heads, dim = 65536, 300, 32
    plain = plain_cache(power, 1, 1, dim, apart(order, power, n // 64), waves=8)
    cache = made(plain, heads)
    q, qn = queries(kind, 1, 2, heads, dim, n // 8)
    check(kind, cache, q, qn, n, {(0, 170): held(plain, 0, 0)}, blocks=n // 64 // 8)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("order,power", [("down", 11), ("up", 11), ("down", 13), ("mixed", 6)])
def test_pieces_that_fill_the_chip(kind, order, power):
    n = 4096
    plain = plain_cache(power, 28, 8, 64, apart(order, power, n // 64))
    q, qn = queries(kind, 28, 100, 8, 64, n)
    check(kind, made(plain), q, qn, n, {at: held(plain, *at) for at in ((0, 0), (27, 5))})


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("order", ["up", "down", "mixed"])
def test_stored_tokens_of_magnitudes_that_lie_apart(kind, order):
    """The same through append: values of one block 2^-11 of those of another one."""
    n, heads, dim = 8192, 64, 64
    rng = np.random.default_rng(5)
    v = (rng.standard_normal((1, n, 1, dim)) * np.repeat(apart(order, 11, n // 64), 64)[None, :, None, None]).astype(np.float32)
    k = np.zeros((1, n, 1, dim), dtype=np.float32)
    k[0, 4000, 0, 3] = 100 * 2.0 ** -7
    cache = cache_of(1, heads, dim, n)
    cache.append(*(torch.from_numpy(x).to(DEV).expand(1, n, heads, dim) for x in (k, v)), ints([n]))
    q, qn = queries(kind, 1, 3, heads, dim, n)
    check(kind, cache, q, qn, n, {(0, 63): [u.contents(x[0])[3] for x in (k, v)]})


@pytest.mark.parametrize("rows", [4, 40])
@pytest.mark.parametrize("kind,least,most", [("f32", -32, 32), ("bf16", -32, 32), ("f16", -32, 8)])
@pytest.mark.parametrize("order", ["up", "down", "mixed"])
def test_scales_at_the_ends_of_their_range(kind, least, most, order, rows):
    """Value scales of 2^-32 and 2^32 (half: what it holds) in one cache: rows that see all of it, and rows that see a half."""
    n, heads = 2048, 64
    scales = np.array(apart(order, most - least, n // 64)) / 0.7 * 2.0 ** most
    plain = plain_cache(1, 1, heads, 64, scales, k_scale=np.where(np.arange(n // 64) % 2, 2.0 ** -32, 2.0 ** 32))
    q, qn = queries(kind, 1, rows, heads, 64, n)
    seen = int(np.flatnonzero(plain["k"][0, 0].any(axis=(1, 2)))[0])       # the block of the token whose key is not 0
    down = 2.0 ** -7 / float(plain["k_scale"][0, 0, seen])
    if kind == "f16":                            # (queries stay halves)
        plain["k_scale"][:] = 2.0 ** -7
    else:
        q, qn = q * down, qn * down
    limits = [n if i % 2 else n // 2 for i in range(rows)]
    check(kind, made(plain), q, qn, n, {(0, h): held(plain, 0, h) for h in (0, 40)}, limits=limits)
