"""An 8-bit context beside layers that keep pairs of halves."""

import pytest

import pd_inputs as pi
from parity_util import make_decoder
from test_gpu_byte_context import CASES, run, same

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pairs", [0, 1, 2])
def test_layers_of_pairs_stay_as_they_are(pairs):
    """Steps say that they read codes where a layer does, and only there do they give anything else."""
    from paper_2506_23431_amd import binding
    cfg = CASES[0]
    w, ctx = pi.make_weights(cfg, threads=4), pi.make_context(cfg)
    dec = make_decoder(cfg, w, kv_pair_layers=pairs)
    assert dec.get_info(binding.PD_INFO_KV_PAIR_LAYERS) == pairs
    halves = run(dec, cfg, ctx)
    dec.use_byte_context()
    codes = run(dec, cfg, ctx)
    assert dec.get_info(binding.PD_INFO_BYTE_BLOCKS) == (cfg.ctx_len // 64 if pairs < cfg.n_layer else 0)
    assert same(halves, codes) == (pairs == cfg.n_layer)
    dec.use_byte_context(False)
    assert dec.get_info(binding.PD_INFO_BYTE_BLOCKS) == 0 and same(halves, run(dec, cfg, ctx))
    dec.close()


def test_a_named_workload_at_full_width():
    """cfg2, all six layers of width 768 behind 1024 input tokens: the first steps against the oracle on the quantised context."""
    import numpy as np
    from parity_util import TOL, compare_teacher_forced, oracle_run
    from test_gpu_byte_context import contexts_of
    cfg, steps = pi.get_config("cfg2"), 12
    w, ctx = pi.make_weights(cfg), pi.make_context(cfg)
    force = pi.make_forced_tokens(cfg, steps)
    outs = oracle_run(cfg, w, ctx, force=force, steps=steps, context_kv=contexts_of(cfg, w, ctx),
                      log=lambda m: print(m, flush=True))
    dec = make_decoder(cfg, w)
    dec.use_byte_context()
    got = compare_teacher_forced(cfg, w, ctx, dec, outs, force=force, steps=steps, tol=TOL[cfg.dtype])
    print(f"[byte context] cfg2: library off by {got['worst']:.3e}")
    dec.close()
