"""tk_block_tables: what a step leaves behind in the arrays that it reads and writes."""

import threading

import numpy as np
import pytest
import torch

from _helpers import require_gpu
from oracle import rope
from paper_2603_04427_gb300 import binding as tb

pytestmark = pytest.mark.gpu

I32 = dict(dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("length,new", [(-4, 1), (49, 1), (49, 0), (-(2 ** 31), 0), (2 ** 31 - 1, 1), (20, -2)])
def test_ill_formed_request_keeps_its_length(length, new, in_place):
    """It is refused and flagged at every step, its length stays as it is, and finishing it frees nothing: the
    ids in its row may belong to others."""
    require_gpu()
    lens, table = [20, length, 3], [[0, 1, -1], [2, 3, 4], [5, -1, -1]]
    pool = tb.PagePool(16, torch.tensor(table, **I32), torch.tensor([6, 7, -1, -1, -1, -1, -1, -1], **I32),
                       torch.tensor([2], **I32), torch.tensor(lens, **I32), torch.zeros(1, **I32))
    slots, pos, refused = torch.empty(16, **I32), torch.empty(16, **I32), torch.empty(1, **I32)
    own = {} if in_place else dict(seq_lens_out=torch.empty(3, **I32), free_count_out=torch.empty(1, **I32))
    after = pool.seq_lens if in_place else own["seq_lens_out"]
    free = pool.free_count if in_place else own["free_count_out"]

    def step(counts):
        tb.tk_block_tables(pool, torch.tensor(counts, **I32), slots, pos, refused=refused, **own)
        assert tb.tk_get_device_error() == 1 and refused.item() == 1

    step([1, new, 14])
    assert after.tolist() == [21, length, 17] and free.item() == 1
    if not -1 < length < 49:                         # finished, and still ill-formed
        step([0, -1, 0])
        assert after.tolist()[1] == length
        assert free.item() == (1 if in_place else 2)
        assert pool.free_pages[:2].tolist() == [6, 7] and bool((pool.free_pages[2:] == -1).all())
    assert pool.page_table[1].tolist() == table[1]


def test_batches_of_several_sizes_from_several_threads():
    """Three host threads, each with a pool, a stream and a large batch of its own: every call is launched."""
    require_gpu()
    failed = []

    def work(B):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                pool = tb.PagePool.allocate(B, 4, 16, B)
                new, slots, pos = torch.zeros(B, **I32), torch.empty(B, **I32), torch.empty(B, **I32)
                call = tb.prepare_block_tables(pool, new, slots, pos, tokens_per_seq=1, stream=s)
                for i in range(20000):
                    call()
                    if i % 500 == 0:
                        s.synchronize()
                s.synchronize()
                assert bool((slots == -1).all())
        except Exception as e:
            failed.append(f"batch {B}: {e}")

    threads = [threading.Thread(target=work, args=(B,)) for B in (4096, 1700, 2500)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
    assert tb.tk_get_device_error() == 0


def test_lengths_in_place_over_many_blocks():
    """The lengths and the free count that every block reads are overwritten by the same call: with hundreds of
    blocks, each of many runs from the same state gives the oracle's step."""
    require_gpu()
    rng = np.random.default_rng(2)
    B, ps, max_pages = 4096, 16, 8
    lens = rng.integers(0, 4 * ps, B)
    held = -(-lens // ps)
    new = rng.integers(-1, 60, B)
    P = int(held.sum()) + 8000
    ids = rng.permutation(P)
    table = np.full((B, max_pages), -1)
    at = np.cumsum(held) - held
    for b in range(B):
        table[b, :held[b]] = ids[at[b]:at[b] + held[b]]
    free = np.full(P, -5)
    free[:8000] = ids[held.sum():]
    rows = int(np.maximum(new, 0).sum())
    assert rows > torch.cuda.get_device_properties(0).multi_processor_count * 512
    ref = rope.block_tables(lens, new, table, free, 8000, ps, rows, 0)
    start = [torch.tensor(x, **I32) for x in (table, free, [8000], lens)]
    pool = tb.PagePool(ps, *(x.clone() for x in start), torch.zeros(1, **I32))
    now = (pool.page_table, pool.free_pages, pool.free_count, pool.seq_lens)
    counts, slots, pos = torch.tensor(new, **I32), torch.empty(rows, **I32), torch.empty(rows, **I32)
    want = [torch.tensor(np.asarray(ref[k]).reshape(-1), **I32)
            for k in ("page_table", "free_pages", "free_count", "seq_lens", "slots", "positions")]
    for i in range(50):
        for x, x0 in zip(now, start):
            x.copy_(x0)
        slots.fill_(77)
        tb.tk_block_tables(pool, counts, slots, pos)
        for x, y in zip((*now, slots, pos), want):
            assert torch.equal(x.view(-1), y), i
    assert tb.tk_get_device_error() == 0 and pool.workspace.item() == 0
