"""Probabilities of rows over the 8-bit cache, one by one: a block in which token j has a value in dim j only."""

import numpy as np
import pytest

from test_gpu_byte_cache import DEV, TYPES, ints

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,rows,heads", [("f32", 300, 64), ("f32", 12, 1024), ("f16", 300, 64), ("f16", 12, 1024), ("f16", 200, 128)])
def test_both_halves_of_a_probability_are_of_the_same_number(kind, rows, heads):
    """0.8 to 1.6 million probabilities.  Where the high half of a pair and the low one are not of the same number, but of two that differ
    by a rounding, and a border between two halves lies between them, the pair is off by a whole step of a half, 2^-11 to 2^-10 of
    the probability.

    The bound, relative: a score is four fp32 factors (2^-24 each) and half a step of 2^-21 of the row's largest query at most, times
    the codes; the exponential 2^-22; a pair of halves 2^-22; the sum of 64 such, each addition 2^-24; the quotient and
    the product with the code 2^-23, and half outputs' rounding 2^-11."""
    from paper_2506_23431_amd import ByteCache
    dim, rng = 64, np.random.default_rng(rows)
    plain = {"k": rng.integers(-127, 128, (1, heads, 1, 64, dim), dtype=np.int8),
             "v": np.broadcast_to(127 * np.eye(64, dtype=np.int8), (1, heads, 1, dim, 64)).copy(),
             "k_scale": np.full((1, heads, 1), 2.0 ** -7, dtype=np.float32),
             "v_scale": rng.uniform(0.5, 1, (1, heads, 1)).astype(np.float32),
             "k_tail": np.zeros((1, heads, 2, 64, dim), dtype=np.float16), "v_tail": np.zeros((1, heads, 2, dim, 64), dtype=np.float16)}
    cache = ByteCache.from_tensors(**{name: torch.from_numpy(x).to(DEV) for name, x in plain.items()})
    q = torch.from_numpy(rng.uniform(-0.5, 0.5, (1, rows, heads, dim)).astype(np.float32)).to(TYPES[kind])
    out = cache.attention(q.to(DEV), ints([64]), scale=1.0)[0].double().cpu().numpy()       # [row][head][token]
    k = plain["k"][0, :, 0].astype(np.float64) * 2.0 ** -7                                                    # [head][token][dim]
    qq = q[0].double().numpy().transpose(1, 0, 2)                                                            # [head][row][dim]
    score = np.matmul(qq, k.transpose(0, 2, 1))
    p = np.exp(score - score.max(-1, keepdims=True))
    want = p / p.sum(-1, keepdims=True) * 127 * plain["v_scale"][0].astype(np.float64)[:, :, None]
    off = np.abs(out.transpose(1, 0, 2) / want - 1)
    step = np.abs(k).sum(-1)[:, None] * np.abs(qq).max(-1, keepdims=True) * 2.0 ** -22
    one = np.abs(score) * 2.0 ** -22 + step + 2.0 ** -22 + 2.0 ** -22
    bound = one + one.max(-1, keepdims=True) + 64 * 2.0 ** -24 + 2.0 ** -23 + (2.0 ** -11 if kind == "f16" else 0)
    print(f"[probabilities] {kind} {rows} rows: {(off > bound).sum()} of {off.size} off, worst {off.max():.2e}, bound {bound.max():.2e}")
    assert (off <= bound).all()
