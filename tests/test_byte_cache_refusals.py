"""What the operators over the 8-bit cache refuse, at the C boundary (no GPU call is reached)."""

import ctypes as C

import pytest

from test_library import lib  # noqa: F401


def a_cache(**over):
    from paper_2506_23431_amd.binding import PdByteCache
    f = dict(k=4096, v=4096, k_scale=4096, v_scale=4096, k_tail=4096, v_tail=4096, n_req=2, n_kv_head=2, head_dim=64, n_block=4)
    f.update(over)
    return PdByteCache(**f)


BAD_CACHES = [dict(k=None), dict(v_scale=None), dict(v_tail=None), dict(head_dim=0), dict(head_dim=48), dict(head_dim=160),
              dict(n_req=0), dict(n_kv_head=-1), dict(n_block=0), dict(n_block=(1 << 24) + 1), dict(k=4097), dict(v_tail=4104),
              dict(k_scale=4098), dict(n_req=1 << 20, n_kv_head=1 << 20)]
STRIDES = (C.c_int64 * 3)(1024, 128, 64)


def append(lib, cache, **over):  # noqa: F811
    f = dict(k=4096, v=4096, type=0, ks=STRIDES, vs=STRIDES, n_new=3, counts=None, lens=4096)
    f.update(over)
    return lib.pd_byte_append(C.byref(cache) if cache else None, f["k"], f["v"], f["type"], f["ks"], f["vs"], f["n_new"],
                              f["counts"], f["lens"], None)


def read(lib, cache, **over):  # noqa: F811
    f = dict(first=None, n_tok=3, lens=4096, k=4096, v=4096, type=0)
    f.update(over)
    return lib.pd_byte_read(C.byref(cache) if cache else None, f["first"], f["n_tok"], f["lens"], f["k"], f["v"], f["type"], None)


def attend(lib, cache, **over):  # noqa: F811
    f = dict(q=4096, type=0, qs=STRIDES, n_head=2, n_row=1, lens=4096, row_limit=None, key_tag=None, row_tag=None, scale=0.125,
             max_len=0, out=8192, lse=None, ws=None, bytes=0)
    f.update(over)
    return lib.pd_byte_attention(C.byref(cache) if cache else None, f["q"], f["type"], f["qs"], f["n_head"], f["n_row"],
                                 f["lens"], f["row_limit"], f["key_tag"], f["row_tag"], f["scale"], f["max_len"], f["out"],
                                 f["lse"], f["ws"], f["bytes"], None)


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_bad_caches(lib, bad):  # noqa: F811
    c = a_cache(**bad)
    assert append(lib, c) == read(lib, c) == attend(lib, c) == -1
    assert len(lib.pd_last_error()) > 0
    assert lib.pd_byte_attention_workspace_bytes(C.byref(c), 2, 1, 0) == 0


def test_no_cache(lib):  # noqa: F811
    assert append(lib, None) == read(lib, None) == attend(lib, None) == -1
    assert lib.pd_byte_attention_workspace_bytes(None, 2, 1, 0) == 0


@pytest.mark.parametrize("bad", [dict(k=None), dict(v=None), dict(lens=None), dict(ks=None), dict(vs=None), dict(type=3),
                                 dict(type=-1), dict(n_new=-1), dict(n_new=257), dict(k=4098), dict(type=1, v=4097)])
def test_append(lib, bad):  # noqa: F811
    assert append(lib, a_cache(), **bad) == -1


def test_nothing_to_do_is_fine(lib):  # noqa: F811
    assert append(lib, a_cache(), n_new=0, k=None, lens=None) == 0
    assert read(lib, a_cache(), n_tok=0, k=None) == 0
    assert attend(lib, a_cache(), n_row=0, q=None) == 0


@pytest.mark.parametrize("bad", [dict(k=None), dict(v=None), dict(lens=None), dict(type=3), dict(n_tok=-1), dict(k=4100)])
def test_read(lib, bad):  # noqa: F811
    assert read(lib, a_cache(), **bad) == -1


@pytest.mark.parametrize("bad", [dict(q=None), dict(out=None), dict(lens=None), dict(qs=None), dict(type=3), dict(n_head=3),
                                 dict(n_head=0), dict(n_head=-2), dict(n_row=-1), dict(max_len=-1), dict(n_row=1 << 30),
                                 dict(key_tag=4096), dict(row_tag=4096), dict(key_tag=4098, row_tag=4096), dict(out=8196),
                                 dict(q=4097, type=1), dict(scale=float("nan")), dict(scale=float("inf"))])
def test_attention(lib, bad):  # noqa: F811
    assert attend(lib, a_cache(), **bad) == -1


def test_attention_workspace(lib):  # noqa: F811
    """A long cache and few rows are split: without room for the parts the call is refused."""
    c = a_cache(n_req=1, n_kv_head=1, n_block=1000)
    need = lib.pd_byte_attention_workspace_bytes(C.byref(c), 4, 2, 0)
    assert need > 1 << 16
    assert attend(lib, c, n_head=4, n_row=2) == -3
    assert attend(lib, c, n_head=4, n_row=2, ws=4096, bytes=need - 1) == -3
    assert attend(lib, c, n_head=4, n_row=2, ws=4100, bytes=need) == -1
    assert b"aligned" in lib.pd_last_error()
    # a bound on the lengths makes it less, rows that fill the chip make it nothing
    assert lib.pd_byte_attention_workspace_bytes(C.byref(c), 4, 2, 64) == 16
    assert lib.pd_byte_attention_workspace_bytes(C.byref(c), 4, 100000, 0) == 16
