"""The paged cache and the choice of tokens where offsets leave 32 bits, and attention of prompts of thousands of rows."""

import math

import numpy as np
import pytest
import torch

from paged_cache_util import PAGE, TYPES, attend, tolerance
from test_gpu_paged_cache import DEV, f64, filled, i32, table

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_pages_whose_places_leave_32_bits(kind):
    """2.6e9 keys: what is stored in the last pages, read back and attended to is what the same calls give in a cache of few pages."""
    from paper_2506_23431_amd import PagedCache
    kv, dim, req, n_slot, n_page = 8, 128, 3, 5, 40000
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    large, small = PagedCache(n_page, kv, dim, TYPES[kind]), PagedCache(req * n_slot, kv, dim, TYPES[kind])
    few = torch.randperm(req * n_slot, generator=g, device=DEV).view(req, n_slot).int()
    few[:, :2] = few[:1, :2]
    many = n_page - 1 - few
    lens, shared = i32([300, 260, 131]), i32([130])
    new = 300
    k, v = (torch.randn(req, new, kv, dim, generator=g, device=DEV) for _ in range(2))
    q = torch.randn(req, new, 2 * kv, dim, generator=g, device=DEV)
    freqs = 10000.0 ** (-torch.arange(64, device=DEV, dtype=torch.float64) / 64)
    outs = []
    for cache, pages in ((large, many), (small, few)):
        # (the shared pages: every request stores the same there)
        turned = cache.append(k[:1].expand(req, -1, -1, -1), v[:1].expand(req, -1, -1, -1), pages, lens, counts=lens, freqs=freqs, q=q)
        outs.append([turned, *cache.read(pages, lens, new)] + [cache.attention(turned[:, :rows].contiguous(), pages, lens, shared=s)
                                                               for rows in (1, 5, 40) for s in (None, shared)])
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    assert not torch.equal(outs[0][1], torch.zeros_like(outs[0][1]))
    assert (large.k[:100] == 0).all() and (large.v[:100] == 0).all()


def test_logits_whose_places_leave_32_bits():
    from paper_2506_23431_amd import sample
    rows, vocab = 70000, 32000
    x = torch.empty(rows, vocab, dtype=torch.float16, device=DEV)
    g = torch.Generator(device=DEV)
    g.manual_seed(4)
    x.normal_(generator=g)
    u = torch.rand(rows, generator=g, device=DEV)
    for more in (dict(top_k=50, top_p=0.9), dict(top_p=0.9), dict(temperature=0.0)):
        token, logprob = sample(x, u, with_logprob=True, **more)
        for at in (slice(0, 3), slice(67108, 67112), slice(rows - 3, rows)):       # (2^31 / 32000 = 67108.9)
            want = sample(x[at].clone(), u[at].clone(), with_logprob=True, **more)
            assert torch.equal(token[at], want[0]) and torch.equal(logprob[at], want[1])


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("groups,per,rows,heads,kv,dim,shared", [(0, 2, 1999, 4, 2, 64, 0), (1, 2, 1500, 8, 2, 128, 777), (0, 1, 4000, 3, 3, 96, 0),
                                                                 (2, 2, 1025, 2, 1, 32, 100)])
def test_prompts(kind, groups, per, rows, heads, kv, dim, shared):
    """Causal rows of a whole input, all of its tokens new: some rows against the definition."""
    req = max(groups, 1) * per
    lens = [shared + rows - 7 * r for r in range(req)]
    n_slot = max(lens) // PAGE + 1
    pages, n_page = table(req, n_slot, groups, [shared] * groups, 6)
    cache, k, v = filled(kind, n_page, kv, dim, 7)
    g = torch.Generator(device=DEV)
    g.manual_seed(8)
    q = (2 * torch.randn(req, rows, heads, dim, generator=g, device=DEV)).to(TYPES[kind])
    limit = [[max(0, lens[r] - rows + 1 + i) for i in range(rows)] for r in range(req)]
    for bounds in (dict(), dict(max_shared=shared, max_behind=rows)):
        out, lse = cache.attention(q, pages, i32(lens), shared=i32([shared] * groups) if groups else None, row_limit=i32(limit), with_lse=True, **bounds)
        for r in range(req):
            at = np.arange(lens[r])
            lead = pages[r // per * per] if groups else pages[r]
            page = np.where(at < shared, lead.cpu().numpy()[at // PAGE], pages[r].cpu().numpy()[at // PAGE])
            kk, vv = f64(k)[page, at % PAGE], f64(v)[page, at % PAGE]
            some = [0, 1, 5, 63, 64, 500, rows // 2, rows - 130, rows - 2, rows - 1]
            sees = at[None] < np.array(limit[r])[some][:, None]
            want, want_lse, mag, scores = attend(f64(q[r, some]), kk, vv, sees, 1 / math.sqrt(dim))
            tol, tol_lse = tolerance(kind, want, mag, scores, dim, lens[r], np.abs(vv).max() / 512)
            assert (np.abs(f64(out[r, some]) - want) <= tol).all()
            seen = np.isfinite(want_lse)
            assert np.array_equal(np.isneginf(f64(lse[r, some])), ~seen)
            assert (np.abs(f64(lse[r, some])[seen] - want_lse[seen]) <= tol_lse[seen]).all()
