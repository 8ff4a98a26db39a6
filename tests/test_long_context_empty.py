"""Sizes of the workspaces over a long context for empty batches and for what is refused (on the host;
nothing is launched)."""

import ctypes

import pytest

from paper_2603_04427_gb300 import binding as tb
from paper_2603_04427_gb300 import build as tbuild


@pytest.fixture(scope="module")
def lib():
    tbuild.build()
    return tb.load_library()


def _desc(batch=2, **kw):
    return tb.tk_cache_desc(batch, 8, 2, 32, 128, kw.get("capacity", 1 << 20), 0, 0, 0, kw.get("fmt", tb.TK_BF16))


@pytest.mark.parametrize("n_q,fmt", [(1, tb.TK_BF16), (1, tb.TK_I8), (16, tb.TK_BF16), (128, tb.TK_BF16), (128, tb.TK_I4)])
@pytest.mark.parametrize("max_len", [0, 100, 1 << 20])
def test_weights_of_an_empty_batch(lib, n_q, fmt, max_len):
    """Some size, as for any other call, whatever form a batch would take."""
    assert lib.tk_attn_weights_workspace_size(ctypes.byref(_desc(0, fmt=fmt)), n_q, max_len) >= 256


@pytest.mark.parametrize("n_q,max_len", [(0, 0), (0, 1 << 20), (-1, 100), (1, -1)])
@pytest.mark.parametrize("batch", [0, 2])
def test_weights_of_no_queries(lib, batch, n_q, max_len):
    """Refused where the size is asked for, as by the call itself."""
    assert lib.tk_attn_weights_workspace_size(ctypes.byref(_desc(batch)), n_q, max_len) == 0
    assert f"n_q={n_q}" in tb.tk_last_error()


def test_the_others_of_an_empty_batch(lib):
    assert lib.tk_cache_evict_workspace_size(ctypes.byref(_desc(0)), 64) >= 256
