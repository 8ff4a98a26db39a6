"""tk_block_tables with more rows than one per thread of a block on every SM, four of them a thread: against the
oracle, exact."""

import numpy as np
import pytest
import torch

from _helpers import require_gpu
from oracle import rope
from paper_2603_04427_gb300 import binding as tb

pytestmark = pytest.mark.gpu

I32 = dict(dtype=torch.int32, device="cuda")


def _many(B):
    """Rows past which a thread fills four: one per thread of a block on every SM."""
    return torch.cuda.get_device_properties(0).multi_processor_count * (128 if B <= 128 else 512)


def _state(rng, B, ps, max_pages, top, spare):
    """Random lengths up to `top`, their pages random ids, a free stack of `spare` others."""
    lens = rng.integers(0, top + 1, B)
    held = -(-lens // ps)
    P = int(held.sum()) + spare + 3
    ids = rng.permutation(P)
    table = np.full((B, max_pages), -1)
    at = np.cumsum(held) - held
    for b in range(B):
        table[b, :held[b]] = ids[at[b]:at[b] + held[b]]
    free = np.full(P, -5)
    free[:spare] = ids[held.sum():held.sum() + spare]
    return lens, table, free


def _check(lens, new, table, free, count, ps, rows, per, in_place):
    t = lambda x: torch.tensor(np.asarray(x), **I32)  # noqa: E731
    pool = tb.PagePool(ps, t(table), t(free), t([count]), t(lens), torch.zeros(1, **I32))
    slots, pos = torch.full((rows + 4,), 77, **I32), torch.full((rows + 4,), 77, **I32)
    offs, refused = torch.full((len(lens) + 1,), 77, **I32), torch.full((1,), 77, **I32)
    own = {} if in_place else dict(seq_lens_out=torch.empty(len(lens), **I32), free_count_out=torch.empty(1, **I32))
    tb.tk_block_tables(pool, t(new), slots[:rows], pos[:rows], tokens_per_seq=per, offsets=offs, refused=refused, **own)
    assert tb.tk_get_device_error() == 0 and pool.workspace.item() == 0
    ref = rope.block_tables(lens, new, table, free, count, ps, rows, per)
    got = dict(page_table=pool.page_table, free_pages=pool.free_pages, slots=slots[:rows], positions=pos[:rows],
               offsets=offs, refused=refused, seq_lens=own.get("seq_lens_out", pool.seq_lens),
               free_count=own.get("free_count_out", pool.free_count))
    for k, v in got.items():
        assert np.array_equal(v.cpu().numpy().reshape(-1), np.asarray(ref[k]).reshape(-1)), k
    assert slots[rows:].tolist() == [77] * 4 and pos[rows:].tolist() == [77] * 4
    return ref


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("B,ps", [(1, 16), (5, 64), (128, 16), (129, 32), (700, 16), (1025, 256), (4096, 16)])
@pytest.mark.parametrize("spare", [1.0, 0.2])
def test_packed(B, ps, spare, in_place):
    """Ragged prompts whose rows outnumber the threads, 1 to 3 rows past a multiple of four."""
    require_gpu()
    rng = np.random.default_rng(B + ps)
    mean = _many(B) * 5 // 4 // B + 1
    new = rng.integers(mean // 2, mean * 2, B)
    if B > 1:
        new[rng.random(B) < 0.1] = 0
        new[rng.random(B) < 0.1] = -1
        new[0] = mean
    max_pages = (3 * ps + 2 * mean) // ps + 1
    need = int((-(-np.maximum(new, 0) // ps)).sum() * spare)
    lens, table, free = _state(rng, B, ps, max_pages, 3 * ps, need)
    rows = max(int(np.maximum(new, 0).sum()), _many(B))
    rows += 4 - rows % 4 + 1 + B % 3
    assert rows > _many(B) and rows % 4
    ref = _check(lens, new, table, free, need, ps, rows, 0, in_place)
    if spare < 1 and B > 1:
        assert ref["refused"] > 0
    # a slot map that ends inside the prompts
    short = max(_many(B) + 1 + B % 3, int(np.maximum(new, 0).sum() * 0.9))
    _check(lens, new, table, free, need, ps, short, 0, in_place)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("B,per", [(127, 201), (126, 163), (3, 8191), (4095, 33), (2999, 37), (513, 1023)])
def test_padded(B, per, in_place):
    """Rows of each sequence padded: threads' four rows cross from one sequence to the next."""
    require_gpu()
    rng = np.random.default_rng(B + per)
    ps = 16
    new = rng.integers(-1, per + 2, B)
    max_pages = (2 * ps + per) // ps + 1
    need = int((-(-np.maximum(new, 0) // ps)).sum())
    lens, table, free = _state(rng, B, ps, max_pages, 2 * ps, need)
    assert B * per > _many(B)
    _check(lens, new, table, free, need, ps, B * per, per, in_place)
    new[:] = 1                                     # one token in each sequence's rows
    _check(lens, new, table, free, need, ps, B * per, per, in_place)
