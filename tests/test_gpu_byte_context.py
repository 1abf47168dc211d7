"""Decode steps over a context in 8 bits (pd_byte_context) against the oracle on a context that is quantised in 64 bits by the
rule of include/pd.h (tests/byte_cache_util.py)."""

import numpy as np
import pytest

import byte_cache_util as u
import pd_inputs as pi
from pd_inputs.configs import WorkloadConfig, DTYPE_BF16, DTYPE_F32, FFN_SWIGLU, NORM_RMSNORM, POS_ROPE
from parity_util import TOL, compare_teacher_forced, make_decoder, oracle_run

pytestmark = pytest.mark.gpu

BASE = dict(dtype=DTYPE_BF16, n_layer=2, d_ff=256, vocab=503, norm_init="random", qkv_std=0.1)
CASES = [
    # two whole blocks and 22 tokens; two requests
    WorkloadConfig(name="byte-64", seed=301, d_model=128, n_head=2, head_dim=64, batch=2, ctx_len=150, n_sub=5, delta_t=2,
                   sub_tokens=7, **BASE),
    # the context is whole blocks only, heads of 32
    WorkloadConfig(name="byte-32", seed=302, d_model=96, n_head=3, head_dim=32, batch=3, ctx_len=128, n_sub=4, delta_t=1,
                   sub_tokens=5, **BASE),
    # rotary positions, heads of 128, one block and a long rest
    WorkloadConfig(name="byte-128", seed=303, d_model=256, n_head=2, head_dim=128, batch=1, ctx_len=127, n_sub=3, delta_t=3,
                   sub_tokens=6, ffn_kind=FFN_SWIGLU, norm_kind=NORM_RMSNORM, pos_kind=POS_ROPE, **BASE),
    # heads of 96, more than 16 rows per request (two groups of rows)
    WorkloadConfig(name="byte-96", seed=304, d_model=192, n_head=2, head_dim=96, batch=2, ctx_len=200, n_sub=20, delta_t=1,
                   sub_tokens=24, **BASE),
    # a long context, split over work-groups, and generated tokens that reach into their own blocks of halves
    WorkloadConfig(name="byte-long", seed=305, d_model=128, n_head=1, head_dim=128, batch=1, ctx_len=2111, n_sub=8, delta_t=2,
                   sub_tokens=16, **BASE),
]


def quantised(kv):
    """The oracle's context keys and values [H][L][hd] per layer, whole blocks of 64 tokens as codes times scales."""
    out = []
    for per_layer in kv:
        layers = []
        for x in per_layer:
            whole = x.shape[1] // u.BLOCK * u.BLOCK
            y = np.array(x, dtype=np.float64)
            y[:, :whole] = u.contents(y[:, :whole].transpose(1, 0, 2).astype(np.float32))[3].transpose(1, 0, 2)
            layers.append(y)
        out.append(layers)
    return tuple(out)


def contexts_of(cfg, w, ctx):
    from oracle.model import OracleModel
    model = OracleModel(cfg, w)
    return [quantised(model.prefill(ctx[b])) for b in range(cfg.batch)]


@pytest.mark.parametrize("cfg", CASES, ids=lambda c: c.name)
def test_steps_match_the_oracle_on_the_quantised_context(cfg):
    from paper_2506_23431_amd import binding
    w, ctx = pi.make_weights(cfg, threads=4), pi.make_context(cfg)
    plain = oracle_run(cfg, w, ctx)
    force = np.full((max(o["steps"] for o in plain), cfg.batch, cfg.n_sub), -1, dtype=np.int32)
    for b, o in enumerate(plain):
        for t, emitted in enumerate(o["emitted"]):
            for i, tok in emitted.items():
                force[t, b, i - 1] = tok
    outs = oracle_run(cfg, w, ctx, force=force, context_kv=contexts_of(cfg, w, ctx))
    dec = make_decoder(cfg, w)
    dec.use_byte_context()
    got = compare_teacher_forced(cfg, w, ctx, dec, outs, force=force, tol=TOL[cfg.dtype])
    assert dec.get_info(binding.PD_INFO_BYTE_BLOCKS) == cfg.ctx_len // 64
    # the codes are what is read: the oracle on the context as it was is further away
    moved = max(np.abs(np.asarray(p["logits"]) - np.asarray(q["logits"])).max()
                for a, b in zip(plain, outs) for p, q in zip(a["trace"], b["trace"]) if len(p["rows"]))
    print(f"[byte context] {cfg.name}: codes move the logits by up to {moved:.3e}, library off by {got['worst']:.3e}")
    assert moved > 2 * got["worst"]
    dec.close()


def run(dec, cfg, ctx, **kw):
    dec.prefill_context(ctx, cfg.n_sub, cfg.delta_t, cfg.sub_tokens, cfg.time_steps)
    return steps(dec, cfg)


def steps(dec, cfg):
    rng = np.random.default_rng(7)
    out = []
    for _ in range(cfg.time_steps):
        force = rng.integers(0, cfg.vocab, (cfg.batch, cfg.n_sub)).astype(np.int32)
        out.append(dec.decode_step(force=force, want_logits=True)[1].cpu().numpy())
    return out


def same(a, b):
    return all(np.array_equal(x, y, equal_nan=True) for x, y in zip(a, b))


def test_switched_on_and_off_before_and_after_the_context_pass():
    from paper_2506_23431_amd import binding
    cfg = CASES[0]
    w, ctx = pi.make_weights(cfg, threads=4), pi.make_context(cfg)
    dec = make_decoder(cfg, w)
    halves = run(dec, cfg, ctx)
    assert dec.get_info(binding.PD_INFO_BYTE_BLOCKS) == 0
    dec.use_byte_context()                       # the contexts are there already
    dec.reset_decode()
    codes = steps(dec, cfg)
    assert not same(halves, codes)
    assert same(codes, run(dec, cfg, ctx))       # and after another pass over them
    other = np.ascontiguousarray(ctx[:, ::-1])
    moved = run(dec, cfg, other)                 # codes follow the context
    assert not same(codes, moved) and same(codes, run(dec, cfg, ctx))
    dec.use_byte_context(False)
    assert same(halves, run(dec, cfg, ctx))
    dec.close()


def test_a_captured_step_ends_with_the_switch():
    """Steps replayed from a graph read the codes while they are on, and the halves again after."""
    import torch
    from paper_2506_23431_amd import binding
    cfg = CASES[0]
    w, ctx = pi.make_weights(cfg, threads=4), pi.make_context(cfg)
    args = (ctx, cfg.n_sub, cfg.delta_t, cfg.sub_tokens, cfg.time_steps)
    with torch.cuda.stream(torch.cuda.Stream()):
        dec = make_decoder(cfg, w)
        dec.set_option(binding.PD_OPT_USE_GRAPH, 1)
        seen = []
        for on in (False, True, False, True):
            dec.use_byte_context(on)
            dec.prefill_context(*args)
            dec.decode_steps(cfg.time_steps - 1)
            seen.append(dec.decode_step(want_logits=True)[1].cpu().numpy())
        assert same([seen[0]], [seen[2]]) and same([seen[1]], [seen[3]]) and not same([seen[0]], [seen[1]])
        dec.close()


def test_replayed_steps_and_splits_and_events():
    import torch
    from paper_2506_23431_amd import binding
    cfg = CASES[4]
    w, ctx = pi.make_weights(cfg, threads=4), pi.make_context(cfg)
    dec = make_decoder(cfg, w)
    dec.use_byte_context()
    args = (ctx, cfg.n_sub, cfg.delta_t, cfg.sub_tokens, cfg.time_steps)
    want = dec.generate(*args)
    with torch.cuda.stream(torch.cuda.Stream()):
        dec.set_option(binding.PD_OPT_USE_GRAPH, 1)
        for _ in range(3):
            assert all(np.array_equal(a, b) for a, b in zip(want, dec.generate(*args)))
        dec.set_option(binding.PD_OPT_USE_GRAPH, 0)
    for mode in (1, 2, 3):
        dec.set_option(binding.PD_OPT_PROFILE, mode)
        assert all(np.array_equal(a, b) for a, b in zip(want, dec.generate(*args)))
        us, n = dec.profile_read()
        assert (n > 0 and 0 < us < 1e4) if mode < 3 else n == 0
    dec.set_option(binding.PD_OPT_PROFILE, 0)
    base = run(dec, cfg, ctx)
    for splits in (1, 3, 8):
        dec.set_option(binding.PD_OPT_ATTN_SPLITS, splits)
        got = run(dec, cfg, ctx)
        worst = max(np.nanmax(np.abs(a - b)) for a, b in zip(base, got))
        assert worst < 2e-3, (splits, worst)     # rounding order only: a tenth of the tolerance against the oracle
    dec.close()


def test_switched_on_again_while_steps_are_under_way():
    """Another buffer takes the codes; the steps that read the first one, on a stream of their own, keep it until they are done."""
    import torch
    cfg = CASES[4]
    w, ctx = pi.make_weights(cfg, threads=4), pi.make_context(cfg)
    args = (ctx, cfg.n_sub, cfg.delta_t, cfg.sub_tokens, cfg.time_steps)
    dec = make_decoder(cfg, w)
    dec.use_byte_context()
    dec.prefill_context(*args)
    dec.decode_steps(cfg.time_steps - 1)
    want = dec.decode_step(want_logits=True)[1].cpu().numpy()
    side = torch.cuda.Stream()
    for _ in range(3):
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            dec.reset_decode()
            dec.decode_steps(cfg.time_steps - 1)
        dec.use_byte_context()
        torch.full((dec.lib.pd_byte_context_bytes(dec.ctx),), 77, dtype=torch.uint8, device="cuda:0")   # (takes the freed memory)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            got = dec.decode_step(want_logits=True)[1].cpu().numpy()
        assert np.array_equal(want, got, equal_nan=True)
    dec.close()


def test_teacher_forced_pass_does_not_see_the_codes():
    cfg = CASES[0]
    w, ctx = pi.make_weights(cfg, threads=4), pi.make_context(cfg)
    targets = [[[cfg.bos_id, 5, 6, 7], [cfg.bos_id, 9]] for _ in range(cfg.batch)]
    results = []
    for on in (False, True):
        dec = make_decoder(cfg, w)
        dec.use_byte_context(on)
        dec.prefill_context(ctx, cfg.n_sub, cfg.delta_t, cfg.sub_tokens, cfg.time_steps)
        results.append([x.cpu().numpy() for x in dec.teacher_forced(targets)[0]])
        dec.close()
    assert same(*results)


def test_refusals():
    import ctypes as C
    from paper_2506_23431_amd import PdError
    cfg = CASES[0]
    w = pi.make_weights(cfg, threads=4)
    dec = make_decoder(cfg, w)
    need = dec.lib.pd_byte_context_bytes(dec.ctx)
    assert need >= 2 * cfg.n_layer * cfg.batch * cfg.d_model * (cfg.ctx_len // 64) * 64
    assert dec.lib.pd_byte_context(dec.ctx, C.c_void_p(256), need - 1, None) == -3
    assert dec.lib.pd_byte_context(dec.ctx, C.c_void_p(257), need, None) == -1
    assert dec.lib.pd_byte_context(None, None, 0, None) == -1 and dec.lib.pd_byte_context_bytes(None) == 0
    dec.use_byte_context(False)                  # nothing to switch off
    dec.close()
    f32 = WorkloadConfig(name="byte-f32", seed=9, dtype=DTYPE_F32, n_layer=1, d_model=32, n_head=2, head_dim=16, d_ff=32,
                         vocab=37, batch=1, ctx_len=70, n_sub=2, delta_t=1, sub_tokens=2)
    dec = make_decoder(f32, pi.make_weights(f32))
    with pytest.raises(PdError, match="matrix-core"):
        dec.use_byte_context()
    assert dec.lib.pd_byte_context(dec.ctx, C.c_void_p(256), 1 << 30, None) == -1
    dec.close()


def test_an_encoder_decoder_context_refuses():
    import ctypes as C
    from paper_2506_23431_amd import PdError
    from test_gpu_encdec import CASES as MODELS, make
    _, _, dec = make(MODELS["encdec-sequential"])
    with pytest.raises(PdError, match="decoder-only"):
        dec.use_byte_context()
    assert dec.lib.pd_byte_context(dec.ctx, C.c_void_p(256), 1 << 30, None) == -1
    dec.use_byte_context(False)
    dec.close()
