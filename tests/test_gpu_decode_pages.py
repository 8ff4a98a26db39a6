"""Entries out of range in the tables of a decode over pages or blocks smaller than its 64-token chunks:
recorded wherever they stand in a chunk, read as the first one of the cache, and not looked at past
the context."""

import math

import numpy as np
import pytest
import torch

from _helpers import f64, parity, require_gpu
from _long_context import Cache, bits, i32
from oracle import attention as oa
from paper_2603_04427_gb300 import binding as tb

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean():
    require_gpu()
    tb.tk_get_device_error()
    yield
    assert tb.tk_get_device_error() == 0


def _q(B, hq, r):
    return torch.randn(B, hq, r, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).cuda()


@pytest.mark.parametrize("ps", [16, 32, 64])
@pytest.mark.parametrize("k", ["bf16", "int8"])
def test_every_page_of_a_context(ps, k):
    """Each entry in turn, of a context of 197 tokens on pages of which the last one is partly filled."""
    x = Cache([197, 70], 4, 2, 32, 64, 256, ps, k, seed=ps)
    x.c.k.nan_to_num_(0.0) if k == "bf16" else x.c.k_scale.nan_to_num_(0.0, 0.0)
    x.c.v.nan_to_num_(0.0)
    table = x.c.page_table
    table[:, -(-197 // ps):] = -1                     # past the longest context
    q, out, ws = _q(2, 4, 32), torch.empty(2, 4, 64, device="cuda"), tb.decode_workspace(x.c.desc, 256)
    tb.tk_attn_decode(x.c, q, x.seq, 256, out, ws)
    assert tb.tk_get_device_error() == 0
    for b, n in ((0, 197), (1, 70)):
        for j in range(-(-n // ps)):
            good, bad = table[b, j].clone(), x.c.desc.num_pages if j % 2 else -7
            table[b, j] = 0
            tb.tk_attn_decode(x.c, q, x.seq, 256, out, ws)
            want = out.clone()
            assert tb.tk_get_device_error() == 0
            table[b, j] = bad
            tb.tk_attn_decode(x.c, q, x.seq, 256, out, ws)
            assert tb.tk_get_device_error() == 1, (b, j)
            assert torch.equal(bits(out), bits(want)), (b, j)
            table[b, j] = good


@pytest.mark.parametrize("block", [16, 32, 64, 128])
def test_every_entry_of_a_table_of_blocks(block):
    x = Cache([16 * block, 9 * block], 4, 2, 32, 64, 16 * block, 0, "bf16", seed=block)
    n = 9
    table = torch.stack([torch.randperm(9, generator=torch.Generator().manual_seed(p)) + 16 * p for p in range(4)])
    lens = [n * block, (n - 1) * block + 1, 5 * block - 3, 1]
    table[2, 5:], table[3, 1:] = -1, 1 << 30          # past the blocks that are read
    sel = tb.BlockSelection(block, table.to(torch.int32).cuda(), i32(lens))
    q, out, ws = _q(2, 4, 32), torch.empty(2, 4, 64, device="cuda"), tb.decode_blocks_workspace(x.c, sel)
    tb.tk_attn_decode_blocks(x.c, q, sel, out, ws)
    assert tb.tk_get_device_error() == 0
    flat_k, flat_v = x.keys64(), x.values()
    for p in range(4):
        t = np.arange(lens[p])
        rows = table[p].numpy()[t // block] * block + t % block
        parity(f64(out).reshape(4, 2, 64)[p],
               oa.attention_head(f64(q).reshape(4, 2, 32)[p], flat_k[rows], flat_v[rows], 1 / math.sqrt(32)))
    total = 4 * 16
    for p in range(4):
        for j in range(-(-lens[p] // block)):
            good = sel.table[p, j].clone()
            sel.table[p, j] = 0
            tb.tk_attn_decode_blocks(x.c, q, sel, out, ws)
            want = out.clone()
            sel.table[p, j] = total if j % 2 else -1
            tb.tk_attn_decode_blocks(x.c, q, sel, out, ws)
            assert tb.tk_get_device_error() == 1, (p, j)
            assert torch.equal(bits(out), bits(want)), (p, j)
            sel.table[p, j] = good


def test_an_appending_decode_checks_its_pages():
    """The step's own token is on the last page: a bad entry before it, in the same chunk, is recorded
    once more than the append alone would."""
    x = Cache([50], 2, 1, 32, 64, 64, 16, "bf16", seed=9)
    q, ws = _q(1, 2, 32), tb.decode_workspace(x.c.desc, 64)
    kn, vn = torch.ones(1, 1, 32, device="cuda").bfloat16(), torch.ones(1, 1, 64, device="cuda").bfloat16()
    out = torch.empty(1, 2, 64, device="cuda")
    tb.tk_attn_decode_append(x.c, q, kn, vn, x.seq, 64, out, ws)
    assert tb.tk_get_device_error() == 0
    for j in range(1, 3):
        good = x.c.page_table[0, j].clone()
        x.c.page_table[0, j] = 1 << 20
        tb.tk_attn_decode_append(x.c, q, kn, vn, x.seq, 64, out, ws)
        assert tb.tk_get_device_error() == 1, j
        x.c.page_table[0, j] = good
