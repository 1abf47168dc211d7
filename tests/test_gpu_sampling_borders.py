"""The choice of tokens next to its borders, against the definition in 64-bit numpy."""

import math

import numpy as np
import pytest
import torch

from test_gpu_sampling import DEV, TYPES, stay

LAST = 1 - 2.0 ** -24                                        # the largest fp32 number below 1


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [32000, 131072, 160000, 1 << 20])
def test_many_tokens_alike(kind, vocab):
    """One token far above all others, which are alike or of three near values: the cut by sum lies among them, and the logarithm of the
    first one's probability, -log of what stays, tells how many stay.  Borders hold to 1e-10 of the sum, and a token stays or does
    not; then the logarithm's own rounding."""
    from paper_2506_23431_amd import sample
    for low, t, rank in ((-24.0, 1.0, 0), (-22.0, 1.0, 0), (-18.0, 1.0, vocab - 5), (-44.0, 2.0, 0), (-11.0, 1.0, 0), (-9.0, 0.5, vocab // 2)):
        for values in ((low,), (low, low - 0.125, low + 0.0625)):
            x = torch.full((1, vocab), low, device=DEV)
            for i, v in enumerate(values):
                x[0, i::len(values)] = v
            x[0, 0] = 0.0
            x = x.to(TYPES[kind])
            tail = np.sort(np.exp(x[0, 1:].double().cpu().numpy() / t))[::-1]
            tail = (tail[:rank - 1] if rank else tail).astype(np.longdouble)
            passed = np.concatenate([[0], np.cumsum(tail)])
            total = 1 + passed[-1]
            for part in (0.2, 0.5, 0.9):
                p = np.float32(1 - (1 - part) * passed[-1] / total)
                if p >= 1:
                    continue
                # tokens of the tail that stay: those with less than p of the sum in front of them
                want = float(np.log1p(passed[np.count_nonzero(1 + passed[:-1] < np.longdouble(p) * total)]))
                p = float(p)
                token, logprob = sample(x, torch.zeros(1, device=DEV), temperature=t, top_k=rank, top_p=p, with_logprob=True)
                assert token.item() == 0
                off = abs(-logprob.double().item() - want)
                assert off <= 1e-10 + (tail[0] + 1e-13) / (1 + math.expm1(want)) + 2.0 ** -24 * want, (low, t, rank, len(values), part, off)


@pytest.mark.gpu
@pytest.mark.parametrize("vocab", [900, 5000, 32000, 70001])
def test_random_numbers_of_one_and_above_are_the_last_below(vocab):
    """The last tokens hold less than 2^-24 of the sum: a number below 1 does not reach them."""
    from paper_2506_23431_amd import sample
    g = torch.Generator(device=DEV)
    g.manual_seed(vocab)
    x = torch.randn(3, vocab, generator=g, device=DEV)
    x[:, -vocab // 3:] -= 40.0
    last = torch.full((3,), LAST, device=DEV)
    for more in (dict(), dict(top_p=0.9999999), dict(min_p=1e-30), dict(top_k=vocab * 2 // 3 + 20), dict(top_k=vocab * 2 // 3 + 20, top_p=0.9999999)):
        want = sample(x, last, with_logprob=True, **more)
        if "top_p" not in more:
            rows = [stay(r.double().cpu().numpy(), 1.0, more.get("top_k", 0), 1.0, more.get("min_p", 0.0)) for r in x]
            assert want[0].tolist() == [idx[np.searchsorted(np.cumsum(e) / e.sum(), LAST, side="right")] for idx, e in rows]
        for bad in (1.0, 1.5, 3e38, math.inf):
            got = sample(x, torch.full((3,), bad, device=DEV), with_logprob=True, **more)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), (more, bad)
    # few by rank: one wave puts them in order; and more, all threads
    for few in (50, 400):
        y = x.clone()
        y[:, -few // 2:] = -30.0
        y[:, few // 2:-few // 2] = -60.0
        got = [sample(y, torch.full((3,), v, device=DEV), top_k=few) for v in (LAST, 1.0, math.inf)]
        assert (got[0] < few // 2).all() and torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])
