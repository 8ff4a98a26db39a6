"""The workspace of the attention weights: one for a longer context serves every shorter one."""

import ctypes

import pytest
import torch

from _helpers import require_gpu
from _long_context import Cache
from paper_2603_04427_gb300 import binding as tb

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean():
    require_gpu()
    tb.tk_get_device_error()
    yield
    assert tb.tk_get_device_error() == 0


def _size(desc, n_q, max_len):
    return int(tb.load_library().tk_attn_weights_workspace_size(ctypes.byref(desc), n_q, max_len))


@pytest.mark.parametrize("B,h_kv", [(1, 1), (2, 8), (3, 5), (40, 8)])
@pytest.mark.parametrize("r,G,n_q,fmt", [
    (64, 4, 32, tb.TK_BF16), (32, 8, 64, tb.TK_BF16), (128, 1, 33, tb.TK_BF16),      # products on tcgen05
    (32, 4, 8, tb.TK_BF16), (64, 2, 3, tb.TK_BF16), (128, 8, 64, tb.TK_I8),          # on mma.sync
    (16, 8, 1, tb.TK_BF16), (32, 1, 1, tb.TK_I4)])                                   # one query: fused, or scores kept
def test_a_shorter_context_needs_no_more(B, h_kv, r, G, n_q, fmt):
    desc = tb.tk_cache_desc(B, G * h_kv, h_kv, r, 64, 1 << 22, 0, 0, 0, fmt)
    before = 0
    for n in list(range(0, 20000)) + list(range(20000, 1 << 22, 4999)):
        need = _size(desc, n_q, n)
        assert need >= before, (n, need, before)
        before = need


@pytest.mark.parametrize("r,n,long,short", [(64, 32, 1280, 1152), (64, 32, 1280, 1000), (32, 8, 9729, 9728)])
def test_a_workspace_of_a_longer_context_is_taken(r, n, long, short):
    """The weights with it are those with one of the call's own size, bit for bit."""
    cap = (long + 15) // 16 * 16
    x = Cache([short, short // 2], 32, 8, r, 64, cap, 0, "bf16", seed=r)
    q = torch.randn(2, 32, n, r, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(torch.bfloat16)
    a, b = tb.slot_weights(x.c), tb.slot_weights(x.c)
    tb.tk_attn_weights(x.c, q, x.seq, short, a, tb.attn_weights_workspace(x.c, long, n))
    tb.tk_attn_weights(x.c, q, x.seq, short, b, tb.attn_weights_workspace(x.c, short, n))
    torch.cuda.synchronize()
    assert torch.equal(a, b) and a.sum() > 0
