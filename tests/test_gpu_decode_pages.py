"""Bad page ids of a decode over pages smaller than its 64-token chunks are recorded wherever
they stand in a chunk, and those past the context are not looked at."""

import pytest
import torch

from _helpers import require_gpu
from paper_2603_04427_gb300 import binding as tb
from paper_2603_04427_gb300 import inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", [0, 1, 3])
def test_every_page_of_a_chunk_is_checked(bad):
    require_gpu()
    tb.tk_get_device_error()
    table = torch.tensor([[0, 1, 2, 3, 4, -1]])
    cache = tb.ThinKeyCache.allocate(1, 2, 1, 32, 64, page_size=16, num_pages=5, page_table=table)
    q, out = inputs.normal_bf16((1, 2, 32), 1, device="cuda"), torch.empty(1, 2, 64, device="cuda")
    ws, lens = tb.decode_workspace(cache.desc, 96), torch.tensor([70], dtype=torch.int32, device="cuda")
    tb.tk_attn_decode(cache, q, lens, 96, out, ws)
    assert tb.tk_get_device_error() == 0
    cache.page_table[0, bad] = 5
    tb.tk_attn_decode(cache, q, lens, 96, out, ws)
    assert tb.tk_get_device_error() == 1
