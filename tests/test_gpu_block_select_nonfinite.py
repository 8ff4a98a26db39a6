"""The choice of blocks where scores are infinite or NaN, for every number of query heads of a kv head,
against the float64 oracle: such a block counts as the largest, and of more of them than there is
room for the earlier ones are taken, beside the first and the last blocks of the context."""

import numpy as np
import pytest
import torch

from _helpers import f64, require_gpu
from _long_context import Cache
from oracle import long_context as lc
from paper_2603_04427_gb300 import binding as tb

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.fixture(autouse=True)
def _clean():
    require_gpu()
    tb.tk_get_device_error()
    yield
    assert tb.tk_get_device_error() == 0


def _cache(G, blocks, r=32, lens=None, k="bf16", seed=0):
    return Cache(lens or [blocks * 16, blocks * 16 - 9], 2 * G, 2, r, 64, blocks * 16, 0, k, seed=seed)


def _boxes(x, seed):
    g = torch.Generator().manual_seed(seed)
    n = x.rows_total // 16
    mid, half = torch.randn(n, x.r, generator=g), 0.5 + torch.rand(n, x.r, generator=g)
    return torch.stack([mid - half, mid + half], 1).to(torch.bfloat16)


def _queries(x, seed):
    return torch.randn(x.B, x.h_q, x.r, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def _check(x, box, q, n, first=1, last=1):
    sel = tb.BlockSelection.allocate(x.c, n, 16, ids=True)
    tb.tk_block_select(x.c, q.cuda(), box.cuda().view(tb._bounds_shape(x.c, 16)), x.seq, max(x.lens), sel, first, last)
    torch.cuda.synchronize()
    flat, qq, G = f64(box).reshape(-1, 2, x.r), f64(q), x.h_q // x.h_kv
    table, lens = sel.table.cpu().numpy().reshape(x.B, x.h_kv, n), sel.lens.cpu().numpy().reshape(x.B, x.h_kv)
    for b in range(x.B):
        for g in range(x.h_kv):
            rows = x.rows(b, g)[::16] // 16
            scores = lc.block_scores(qq[b, g * G:(g + 1) * G], flat[rows, 0], flat[rows, 1])
            pick = lc.block_select(scores, n, first, last).astype(np.int64)
            pad = np.full(n - len(pick), -1)
            assert sel.ids[b, g].tolist() == pick.tolist() + pad.tolist(), (b, g)
            assert table[b, g].tolist() == rows[pick].tolist() + pad.tolist()
            assert lens[b, g] == (len(pick) - 1) * 16 + x.lens[b] - (len(rows) - 1) * 16
    return sel


@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("r", [16, 64])
@pytest.mark.parametrize("first,last", [(1, 1), (0, 2), (3, 1)])
def test_more_unbounded_blocks_than_there_is_room_for(G, r, first, last):
    """Bounds as a NaN in a key leaves them, -inf and +inf in one element, in half of the blocks: all
    query heads score such a block NaN."""
    x = _cache(G, 40, r)
    box = _boxes(x, G)
    odd = torch.randperm(len(box), generator=torch.Generator().manual_seed(r))[:len(box) // 2]
    box[odd, 0, odd % r] = -INF
    box[odd, 1, odd % r] = INF
    _check(x, box, _queries(x, r), 8, first, last)


@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_unbounded_and_infinite_blocks_rank_alike(G):
    """NaN scores, infinite ones and finite ones together, with room for some, all and more than all."""
    x = _cache(G, 40)
    box = _boxes(x, 3 + G)
    box[2::5, 0, 3], box[2::5, 1, 3] = -INF, INF        # NaN
    box[4::10, 1, 5] = INF                              # infinite for the heads whose q is positive there
    box[9::10, 0, 7] = NAN
    for n in (3, 8, 20, 30):
        _check(x, box, _queries(x, 5), n)


@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_nan_queries(G):
    """A NaN in one query head, in all of one kv head, in all: no block can be ranked, the earlier ones
    are taken and the last one of the context is among them."""
    x = _cache(G, 40)
    box, q = _boxes(x, 11), _queries(x, 12)
    for heads in (slice(0, 1), slice(0, G), slice(0, 2 * G)):
        q[0, heads, 9] = NAN
        q[1, heads, 4] = INF
        sel = _check(x, box, q, 8)
        assert sel.ids[0, 0].tolist() == [0, 1, 2, 3, 4, 5, 6, 39]


@pytest.mark.parametrize("G", [2, 8])
@pytest.mark.parametrize("blocks", [700, 3000])
def test_many_unbounded_blocks_of_a_long_context(G, blocks):
    """More of them than are ranked by comparing all, over several blocks of threads."""
    x = _cache(G, blocks, 16, [blocks * 16 - 5])
    box = _boxes(x, blocks)
    odd = torch.randperm(len(box), generator=torch.Generator().manual_seed(G))[:len(box) * 2 // 3]
    box[odd, 0, 1], box[odd, 1, 1] = -INF, INF
    _check(x, box, _queries(x, 2), 100)


@pytest.mark.parametrize("G", [1, 8])
@pytest.mark.parametrize("k", ["bf16", "int8"])
def test_from_keys_with_nans(G, k):
    """The bounds and the choice of a cache with a NaN in most of its blocks' keys (or key scales)."""
    x = _cache(G, 30, 32, k=k, seed=4)
    for t in range(5, 29 * 16 - 9, 20):
        if k == "bf16":
            x.c.k[:, :, t, t % 32] = NAN
        else:
            x.c.k_scale[:, :, t] = NAN
    box = tb.block_bounds(x.c, 16)
    tb.tk_block_bounds(x.c, box, x.seq, block=16)
    _check(x, box.cpu().view(-1, 2, 32), _queries(x, 6), 7)


@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_zero_queries_and_infinite_bounds(G):
    """0 times infinity is no score: such a block counts as the largest, although every finite one
    scores 0."""
    x = _cache(G, 40)
    box = _boxes(x, 21)
    box[7::9, 0, 3] = -INF
    box[8::9, 1, 4] = NAN
    q = torch.zeros(x.B, x.h_q, x.r, dtype=torch.bfloat16)
    for n in (4, 8, 20):
        _check(x, box, q, n)
    q[:, G:] = _queries(x, 22)[:, G:]                   # of one kv head alone
    _check(x, box, q, 8)


@pytest.mark.parametrize("G", [1, 2, 4, 8])
def test_zero_bounds_and_infinite_queries(G):
    """Blocks whose bounds are all zero, with queries of infinities and NaNs: nothing can be ranked."""
    x = _cache(G, 40)
    box = torch.zeros_like(_boxes(x, 1))
    q = _queries(x, 23)
    q[0, :, 2], q[1, 0, 3] = INF, NAN
    _check(x, box, q, 8)
    box[11, 1, 2] = 1.0
    _check(x, box, q, 8)
