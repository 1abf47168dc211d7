"""Attention over the 8-bit cache with queries whose channels differ much, against tests/byte_cache_util.py: what a query holds has to
reach its scores, whatever its largest channel is."""

import numpy as np
import pytest

import byte_cache_util as u
from test_gpu_byte_cache import DEV, TYPES, cache_of, data, fill, ints

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("loud", [30, 1000, 20000])
@pytest.mark.parametrize("req,rows,heads,kv,dim", [(2, 1, 2, 2, 64), (1, 4, 4, 1, 96), (1, 40, 2, 2, 128), (2, 70, 3, 1, 32), (28, 100, 8, 8, 64)])
def test_a_loud_channel_leaves_the_others_their_bits(kind, loud, req, rows, heads, kv, dim):
    """One channel of the queries `loud` times the others, where the keys are next to nothing.  Steps of the row's largest / 2^22, so
    off by half of that, whatever the type (u.tolerance has a term for coarser steps of bf16 queries: the sum of |k| times the row's
    largest / 65024, which is replaced)."""
    lens = [333, 64][:req] if req < 28 else [400 - 7 * r for r in range(req)]
    k, kn = data(1, req, max(lens), kv, dim, "f32")
    k[..., 5] *= 1e-3
    kn[..., 5] *= np.float32(1e-3)
    v, vn = data(2, req, max(lens), kv, dim, "f32")
    q = np.random.default_rng(3).standard_normal((req, rows, heads, dim)).astype(np.float32) * 2
    q[..., 5] = np.copysign(loud * 2.0, q[..., 5])
    q = torch.from_numpy(q).to(TYPES[kind])
    qn = q.float().numpy().astype(np.float64)
    cache = cache_of(req, kv, dim, max(lens))
    fill(cache, k, v, lens)
    out, lse = cache.attention(q.to(DEV), ints(lens), with_lse=True)
    out, lse = out.double().cpu().numpy(), lse.cpu().numpy()
    for r in range(req) if req < 28 else (0, 13, 27):
        n = lens[r]
        kk, vv = u.contents(kn[r, :n])[3], u.contents(vn[r, :n])[3]
        want, wl, mag, (dot, top, flat) = u.attend(qn[r], kk, vv, np.ones((rows, n), dtype=bool), dim ** -0.5)
        if kind == "bf16":
            flat = flat * 65024 * 2.0 ** -22
        tol, tl = u.tolerance(kind, want, mag, (dot, top, flat), dim, n, np.abs(vv).max())
        worst = (np.abs(out[r] - want) / tol).max(), (np.abs(lse[r] - wl) / tl).max()
        print(f"[queries] {kind} {loud}: out at {worst[0]:.2f}, lse at {worst[1]:.2f} of the tolerance")
        assert max(worst) <= 1, worst


@pytest.mark.parametrize("case", [0, 2, 3])
def test_a_loud_channel_of_a_decoder_leaves_the_others_their_bits(case):
    """One channel per head whose keys are 0, so that nothing that queries hold there reaches a score: queries 2^10 times as large in
    it move the logits by rounding only, a tenth of the tolerance against the oracle at most, over halves and over codes."""
    import pd_inputs as pi
    from parity_util import TOL, make_decoder
    from test_gpu_byte_context import CASES, run
    cfg = CASES[case]
    ctx, logits = pi.make_context(cfg), {}
    # (rotary positions turn a channel with its partner, half a head away: both)
    channels = [h * cfg.head_dim + c for h in range(cfg.n_head) for c in (5, 5 + cfg.head_dim // 2)]
    for loud in (0, 10):
        w = pi.make_weights(cfg, threads=4)
        for layer in w["layers"]:
            layer["wqkv"][[cfg.d_model + c for c in channels]] = 0
            layer["wqkv"][channels] += np.uint16(loud << 7)              # the exponent of bf16 (weights that are 0 are not there)
            assert (layer["wqkv"][channels] & 0x7f80).all()
        dec = make_decoder(cfg, w)
        for on in (False, True):
            dec.use_byte_context(on)
            logits[loud, on] = run(dec, cfg, ctx)
        dec.close()
    moved = [max(np.nanmax(np.abs(a - b)) for a, b in zip(logits[0, on], logits[10, on])) for on in (False, True)]
    print(f"[queries] {cfg.name}: a loud channel moves the logits by {moved[0]:.2e} over halves, {moved[1]:.2e} over codes")
    assert max(moved) <= TOL[cfg.dtype] / 10
