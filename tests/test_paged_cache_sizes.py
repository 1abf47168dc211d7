"""Sizes beyond what a launch holds, and whose products leave 64 bits, are refused by the operators over a paged cache and the choice of tokens (no GPU call is
reached)."""

import ctypes as C

import pytest

from test_library import lib  # noqa: F401
from test_paged_cache_refusals import STRIDES, a_cache, append, attend, read, sampled, workspace

MOST = (1 << 31) - 1


@pytest.mark.parametrize("sizes", [dict(n_req=4, n_row=MOST, n_head=MOST - 1), dict(n_req=1 << 24, n_row=1 << 20, n_head=1 << 20),
                                   dict(n_req=1 << 24, n_row=1 << 10, n_head=1 << 30), dict(n_req=1 << 23, n_row=2, n_head=2),
                                   dict(n_req=1 << 24, n_row=1, n_head=4)])
def test_attention(lib, sizes):  # noqa: F811
    assert workspace(lib, a_cache(), **sizes) == 0
    assert len(lib.pd_last_error()) > 0
    assert attend(lib, a_cache(), **sizes) == -1


def test_attention_joined_by_too_large_a_launch(lib):  # noqa: F811
    """2^24 work-groups put the partial results of 8 rows and heads each together."""
    for n_req, least in ((1 << 22, 1), (1 << 23, 0)):
        assert min(workspace(lib, a_cache(head_dim=128, n_kv_head=1), n_slot=8192, n_req=n_req, n_group=1, n_head=16, n_row=1), 1) == least


def test_no_rows_of_many_requests_are_fine(lib):  # noqa: F811
    assert workspace(lib, a_cache(), n_req=1 << 24, n_row=0) > 0
    assert attend(lib, a_cache(n_kv_head=1 << 20), n_req=1 << 24, n_row=0, n_head=1 << 20, q=None) == 0


def test_append(lib):  # noqa: F811
    for sizes in (dict(n_req=1 << 24), dict(n_req=1 << 24, n_slot=1 << 24, n_new=1 << 30), dict(n_slot=1 << 24, n_new=1 << 29),
                  dict(n_req=1 << 23, q=4096, qs=STRIDES, n_head=2, out_q=4096)):
        assert append(lib, a_cache(), **sizes) == -1
    assert append(lib, a_cache(n_kv_head=1 << 20), n_req=1 << 24, n_slot=1 << 24, n_new=(1 << 30) - 64) == -1      # 2^24 * 2^24 * 2^18 work-groups


def test_read(lib):  # noqa: F811
    for sizes in (dict(n_req=1 << 23), dict(n_req=1 << 24, n_tok=MOST), dict(n_req=1, n_tok=1 << 29), dict(first=4096, n_req=1, n_tok=MOST)):
        assert read(lib, a_cache(), **sizes) == -1
    assert read(lib, a_cache(n_kv_head=1 << 20), n_req=1 << 24, n_tok=MOST - 63) == -1                             # 2^24 * 2^25 * 2^18


def test_sample(lib):  # noqa: F811
    for n in (1 << 22, 1 << 24, MOST):
        assert sampled(lib, n_row=n) == -1
    assert C.c_char_p(lib.pd_last_error()).value
