"""Attention over pages where probabilities and values are small: halves of 2^-33 of a row's largest probability, values next to the type's smallest number."""

import numpy as np
import pytest
import torch

from paged_cache_util import PAGE, TYPES, attend, tolerance
from test_gpu_paged_cache import DEV, f64, i32

pytestmark = pytest.mark.gpu


def check(kind, k, v, q, shared, scale):
    """All requests hold the same tokens k, v [token][head][dim], the first `shared` of them once."""
    from paper_2506_23431_amd import PagedCache
    req, rows, heads, dim = q.shape
    n, kv = k.shape[:2]
    blocks = -(-n // PAGE)
    whole = shared // PAGE
    pages = torch.arange(req * blocks, device=DEV).view(req, blocks).int()
    pages[:, :whole] = pages[:1, :whole]
    pool_k, pool_v = (torch.zeros(req * blocks, PAGE, kv, dim, device=DEV, dtype=TYPES[kind]) for _ in range(2))
    for r in range(req):
        for b in range(blocks):
            at = slice(b * PAGE, min((b + 1) * PAGE, n))
            page = pages[r, b].item()
            pool_k[page, : at.stop - at.start], pool_v[page, : at.stop - at.start] = k[at], v[at]
    out, lse = PagedCache.from_tensors(pool_k, pool_v).attention(q, pages, i32([n] * req), shared=i32([shared]) if shared else None, scale=scale, with_lse=True,
                                                                 max_shared=shared, max_behind=n - shared)
    for r in range(req):
        want, want_lse, mag, scores = attend(f64(q[r]), f64(k), f64(v), np.ones((rows, n), dtype=bool), scale)
        # (halves are 2^8 times what the running maximum makes them, so what a token loses is 2^-25 of 2^-8: a 512th of 2^-24)
        tol, tol_lse = tolerance(kind, want, mag, scores, dim, n, np.abs(f64(v)).max() / 512)
        off = np.abs(f64(out[r]) - want)
        assert (off <= tol).all(), (off / tol).max()
        assert (np.abs(f64(lse[r]) - want_lse) <= tol_lse).all()
    return out


WAYS = [(1, 1, 1, 0), (1, 1, 1, 2000), (3, 5, 2, 100), (2, 20, 3, 0), (2, 40, 2, 2000), (4, 1, 1, 1500)]


@pytest.mark.parametrize("req,rows,group,shared", WAYS)
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("strong", [0, 1234, 2999])
def test_one_strong_token_and_many_weak_ones(kind, req, rows, group, shared, strong):
    """Weak tokens of 2^-14 to 2^-30 of the strong one's probability, with values of one sign a thousand times its own."""
    n, kv, dim = 3000, 2, 64
    g = torch.Generator(device=DEV)
    g.manual_seed(strong + rows)
    for low, high in ((14, 22), (20, 24), (23.4, 23.6), (24, 30)):
        k = torch.zeros(n, kv, dim, device=DEV)
        k[:, :, 0] = -(low + (high - low) * torch.rand(n, kv, generator=g, device=DEV)) * 0.6931471805599453
        v = 500 + 500 * torch.rand(n, kv, dim, generator=g, device=DEV)
        k[strong], v[strong] = 0.0, 0.5
        q = torch.zeros(req, rows, kv * group, dim, device=DEV)
        q[..., 0] = 1.0
        check(kind, k.to(TYPES[kind]), v.to(TYPES[kind]), q.to(TYPES[kind]), shared, 1.0)


@pytest.mark.parametrize("req,rows,group,shared", WAYS)
@pytest.mark.parametrize("kind,least", [("f16", 2.0 ** -24), ("bf16", 2.0 ** -126)])
def test_values_next_to_the_smallest(kind, least, req, rows, group, shared):
    """Halves below the smallest normal one; bf16 numbers from the smallest normal one on."""
    n, kv, dim = 700, 2, 64
    g = torch.Generator(device=DEV)
    g.manual_seed(rows)
    k = torch.randn(n, kv, dim, generator=g, device=DEV).to(TYPES[kind])
    q = torch.randn(req, rows, kv * group, dim, generator=g, device=DEV).to(TYPES[kind])
    sign = torch.randint(0, 2, (n, kv, dim), generator=g, device=DEV) * 2.0 - 1
    for most in (1, 3, 40, 1500):
        # (all of one sign: what comes out is no smaller than what went in)
        v = (least * torch.randint(1, most + 1, (n, kv, dim), generator=g, device=DEV).double()).to(TYPES[kind])
        out = check(kind, k, v, q, min(shared, 500), 0.125)
        assert (out.double() >= least).all()
        if kind == "f16":
            check(kind, k, (v.double() * sign).to(TYPES[kind]), q, min(shared, 500), 0.125)
