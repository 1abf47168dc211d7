"""Decode steps with drawn tokens in the encoder-decoder form, and of a vocabulary whose rows of logits do not fit LDS: tokens by the rules from the logits of
their step, logits those of the same tokens forced, nothing drawn for subsequences that were not fed."""

import numpy as np
import pytest
import torch

import pd_inputs as pi
from parity_util import make_decoder
from test_gpu_encdec import CASES, make
from test_gpu_sample_step import config
from test_gpu_sampling import DEV, stay
from pd_inputs.configs import DTYPE_BF16

pytestmark = pytest.mark.gpu


def compare(cfg, ctx, drawn, forced, settings, steps):
    shape = (cfg.batch, cfg.n_sub)
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    for dec in (drawn, forced):
        dec.prefill_context(ctx, cfg.n_sub, cfg.delta_t, cfg.sub_tokens, cfg.time_steps)
    n_drawn, done = 0, False
    for _ in range(steps):
        u = torch.rand(shape, generator=g, device=DEV)
        toks, logits, logprob, done = drawn.sample_step(u, **settings)
        want_toks, want, ended = forced.decode_step(force=toks, want_logits=True)
        assert np.array_equal(want_toks, toks) and ended == done
        fed = ~torch.isnan(want[..., 0])
        assert torch.equal(fed, ~torch.isnan(logits[..., 0])) and torch.equal(want[fed], logits[fed])
        assert (logprob[~fed] == 0).all() and (torch.from_numpy(toks).to(DEV)[~fed] == -1).all()
        x = logits.double().cpu().numpy()
        for b, i in np.argwhere(toks >= 0):
            idx, e = stay(x[b, i], settings["temperature"], settings.get("top_k", 0), settings.get("top_p", 1.0), settings.get("min_p", 0.0))
            run = np.cumsum(e) / e.sum()
            at = min(np.searchsorted(run, u[b, i].item(), side="right"), len(idx) - 1)
            assert np.abs(run - u[b, i].item()).min() < 1e-9 or toks[b, i] == idx[at]
            n_drawn += 1
    assert n_drawn > 0
    drawn.close()
    forced.close()
    return done


@pytest.mark.parametrize("name", ["encdec-hd64", "encdec-hd128-packed", "encdec-manyrows", "encdec-sequential"])
def test_encoder_decoder(name):
    cfg = CASES[name]
    _, ctx, drawn = make(cfg)
    _, _, forced = make(cfg)
    assert compare(cfg, ctx, drawn, forced, dict(temperature=0.7, top_k=40, top_p=0.95), cfg.time_steps + 1)


@pytest.mark.parametrize("settings", [dict(temperature=0.8, top_p=0.9), dict(temperature=0.8, top_k=50, top_p=0.95, min_p=0.01), dict(temperature=1.0)])
def test_rows_that_do_not_fit(settings):
    cfg = config(DTYPE_BF16, vocab=50265, batch=2)
    w, ctx = pi.make_weights(cfg, threads=4), pi.make_context(cfg)
    compare(cfg, ctx, make_decoder(cfg, w), make_decoder(cfg, w), settings, 8)
