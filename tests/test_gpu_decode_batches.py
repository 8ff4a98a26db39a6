"""Decode batches of 33 to 128 sequences, whose first chunks are prefetched by lengths and page tables
that an earlier kernel on the stream may still be writing: the result goes by the written ones."""

import math

import pytest
import torch

from _helpers import f64, parity, require_gpu
from _long_context import Cache, i32
from oracle import attention as oa
from paper_2603_04427_gb300 import binding as tb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,ps,k", [(33, 0, "bf16"), (100, 16, "int8"), (128, 64, "bf16")])
def test_lengths_and_tables_written_right_before(B, ps, k):
    require_gpu()
    tb.tk_get_device_error()
    lens = [(41 * b) % 320 for b in range(B)]
    x = Cache(lens, 4, 2, 32, 64, 320, ps, k, seed=B)
    g = torch.Generator().manual_seed(1)
    q = torch.randn(B, 4, 32, generator=g).to(torch.bfloat16).cuda()
    out, ws = torch.empty(B, 4, 64, device="cuda"), tb.decode_workspace(x.c.desc, 320)
    true_lens, true_table = x.seq.clone(), None if not ps else x.c.page_table.clone()
    for stale in (0, 320, 7):
        # what the prefetch may see: other lengths, pages out of range
        x.seq.fill_(stale)
        if ps:
            x.c.page_table.fill_(1 << 20)
        torch.cuda.synchronize()
        if ps:
            x.c.page_table.copy_(true_table)
        x.seq.copy_(true_lens)
        tb.tk_attn_decode(x.c, q, x.seq, 320, out, ws)
        torch.cuda.synchronize()
        keys, vals, qq, got = x.keys64(), x.values(), f64(q), f64(out)
        for b in range(0, B, 3):
            for h in range(2):
                rows = x.rows(b, h)
                if len(rows):
                    ref = oa.attention_head(qq[b, 2 * h:2 * h + 2], keys[rows], vals[rows], 1 / math.sqrt(32))
                    parity(got[b, 2 * h:2 * h + 2], ref)
                else:
                    assert (got[b, 2 * h:2 * h + 2] == 0).all()
    assert tb.tk_get_device_error() == 0
    # a step that appends: the lengths are those before it
    if k == "bf16":
        new_k, new_v = (torch.randn(B, 2, w, generator=g).to(torch.bfloat16).cuda() for w in (32, 64))
        fits = i32([n for n in lens])
        tb.tk_attn_decode_append(x.c, q, new_k, new_v, fits, 320, out, ws)
        b = 5
        rows = x.rows(b, 1, lens[b] + 1)
        keys, vals = x.keys64(), x.values()
        parity(f64(out)[b, 2:], oa.attention_head(f64(q)[b, 2:], keys[rows], vals[rows], 1 / math.sqrt(32)))
        assert tb.tk_get_device_error() == 0
