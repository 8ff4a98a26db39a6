"""tk_block_tables on the GPU against the oracle that serves request after request: exact."""

import numpy as np
import pytest
import torch

from _helpers import require_gpu
from oracle import rope
from paper_2603_04427_gb300 import binding as tb

pytestmark = pytest.mark.gpu

I32 = dict(dtype=torch.int32, device="cuda")


def _state(rng, B, ps, max_pages, ctx, spare, owned_elsewhere=3):
    """Random lengths whose pages are random ids, a free stack of `spare` others."""
    lens = rng.integers(0, min(ctx, max_pages * ps) + 1, B)
    held = -(-lens // ps)
    P = int(held.sum()) + spare + owned_elsewhere
    ids = rng.permutation(P)
    table = np.full((B, max_pages), -1)
    at = 0
    for b in range(B):
        table[b, :held[b]] = ids[at:at + held[b]]
        at += held[b]
    free = np.full(P, -5)
    free[:spare] = ids[at:at + spare]
    return lens, table, free, spare


def _run(lens, new, table, free, count, ps, rows, per, in_place, extra=True):
    t = lambda x: torch.tensor(np.asarray(x), **I32)  # noqa: E731
    pool = tb.PagePool(ps, t(table), t(free), t([count]), t(lens), torch.zeros(1, **I32))
    slots, pos = torch.full((rows,), 77, **I32), torch.full((rows,), 77, **I32)
    offs = torch.full((len(lens) + 1,), 77, **I32) if extra else None
    refused = torch.full((1,), 77, **I32) if extra else None
    out = None if in_place else torch.empty_like(pool.seq_lens)
    cnt = None if in_place else torch.empty(1, **I32)
    for _ in range(1 if in_place else 2):     # with outputs of their own a call can be repeated
        tb.tk_block_tables(pool, t(new), slots, pos, tokens_per_seq=per, offsets=offs, refused=refused,
                           seq_lens_out=out, free_count_out=cnt)
    assert pool.workspace.item() == 0
    got = dict(page_table=pool.page_table, free_pages=pool.free_pages,
               free_count=pool.free_count if in_place else cnt, seq_lens=pool.seq_lens if in_place else out,
               slots=slots, positions=pos)
    if extra:
        got.update(offsets=offs, refused=refused)
    return {k: v.cpu().numpy() for k, v in got.items()}


def _check(lens, new, table, free, count, ps, rows, per, in_place=False, extra=True):
    got = _run(lens, new, table, free, count, ps, rows, per, in_place, extra)
    assert tb.tk_get_device_error() == 0
    ref = rope.block_tables(lens, new, table, free, count, ps, rows, per)
    for k, v in got.items():
        assert np.array_equal(v.reshape(-1), np.asarray(ref[k]).reshape(-1)), k
    return ref


@pytest.mark.parametrize("B", [1, 3, 64, 511, 513, 1025, 4096])
@pytest.mark.parametrize("ps", [16, 64, 256])
@pytest.mark.parametrize("spare", [1.0, 0.6])
def test_decode_steps(B, ps, spare):
    """One token a request, some finished, some idle; with too few pages the later ones are refused."""
    require_gpu()
    rng = np.random.default_rng(B + ps)
    new = rng.choice([1, 1, 1, 0, -1], B)
    lens, table, free, count = _state(rng, B, ps, 5, 5 * ps, int(B * spare / ps) + 1)
    _check(lens, new, table, free, count, ps, B, 1, in_place=B % 2 == 1)
    _check(lens, new, table, free, count, ps, B + 5, 0)


@pytest.mark.parametrize("B,ps,top,rows_of", [
    (1, 16, 1000, 1.0), (7, 32, 300, 1.2), (40, 16, 700, 0.7), (300, 64, 500, 1.0), (600, 16, 90, 1.1), (1500, 128, 70, 1.0)])
@pytest.mark.parametrize("spare", [1.0, 0.5, 0.0])
def test_packed_prompts(B, ps, top, rows_of, spare):
    require_gpu()
    rng = np.random.default_rng(B)
    new = rng.integers(0, top, B)
    new[rng.random(B) < 0.15] = -1
    new[rng.random(B) < 0.1] = 0
    need = int((-(-np.maximum(new, 0) // ps)).sum() * spare)
    lens, table, free, count = _state(rng, B, ps, 60, 10 * ps, need)
    rows = max(1, int(np.maximum(new, 0).sum() * rows_of))
    ref = _check(lens, new, table, free, count, ps, rows, 0, in_place=True)
    if spare == 1.0 and rows_of >= 1.0 and top <= 500:
        assert ref["refused"] == 0
    _check(lens, new, table, free, count, ps, rows, 0, extra=False)


@pytest.mark.parametrize("T", [1, 5, 16, 33])
def test_padded_rows(T):
    """Requests longer than their rows, or than the table's row, are refused on their own."""
    require_gpu()
    rng = np.random.default_rng(T)
    B, ps = 130, 16
    lens, table, free, count = _state(rng, B, ps, 4, 4 * ps, 200)
    new = rng.integers(-1, T + 3, B)
    ref = _check(lens, new, table, free, count, ps, B * T, T)
    assert ref["refused"] > 0


def test_boundaries():
    """Lengths of zero, exact pages, a full row, nothing free, everything finished."""
    require_gpu()
    table = np.array([[4, 2, -1], [7, -1, -1], [0, 1, 3], [-1, -1, -1]])
    free = np.array([5, 6, 8, -9, -9, -9, -9, -9, -9])
    for new in ([0, 0, 0, 0], [1, 1, 0, 16], [0, 0, 1, 1], [-1, -1, -1, -1], [16, -1, -1, 48], [-1, 33, 0, 48], [0, 0, 0, 49]):
        for count in (0, 1, 3):
            _check([32, 16, 48, 0], new, table, free, count, 16, max(1, sum(max(n, 0) for n in new)), 0)
    # finished requests of length 0 give nothing back; a slot map without rows still serves lengths
    _check([0, 0], [-1, -1], table[:2], free, 3, 16, 1, 0)
    _check([16, 15], [0, -1], table[:2], free, 3, 16, 0, 0)


def test_empty_batch():
    require_gpu()
    got = _run([], [], np.zeros((0, 4)), np.array([2, 0, 1]), 2, 16, 0, 0, False)
    assert got["free_count"][0] == 2 and got["offsets"].tolist() == [0] and got["refused"][0] == 0
    assert tb.tk_get_device_error() == 0


def test_returned_pages_out_of_range_are_flagged():
    """A finished request whose row holds a bad page id: flagged, the sound pages come back."""
    require_gpu()
    got = _run([40, 5], [-1, 0], np.array([[0, 9, 1], [2, -1, -1]]), np.array([3, -1, -1, -1]), 1, 16, 1, 0, False)
    assert tb.tk_get_device_error() == 1
    assert got["free_count"][0] == 4 and got["free_pages"].tolist() == [3, 0, -1, 1]


def test_many_steps_keep_every_page_once():
    require_gpu()
    rng = np.random.default_rng(9)
    B, ps, max_pages, P = 24, 16, 12, 130
    pool = tb.PagePool.allocate(B, max_pages, ps, P)
    lens = np.zeros(B, np.int64)
    table, free, count = np.full((B, max_pages), -1), np.arange(P - 1, -1, -1), P
    served = 0
    for step in range(40):
        new = np.where(rng.random(B) < 0.15, -1, np.where(lens == 0, rng.integers(0, 150, B), rng.integers(0, 3, B)))
        rows = int(np.maximum(new, 0).sum()) + 1
        slots, pos = torch.empty(rows, **I32), torch.empty(rows, **I32)
        tb.tk_block_tables(pool, torch.tensor(new, **I32), slots, pos)
        ref = rope.block_tables(lens, new, table, free, count, ps, rows, 0)
        lens, table, free, count = (ref[k] for k in ("seq_lens", "page_table", "free_pages", "free_count"))
        assert np.array_equal(pool.seq_lens.cpu().numpy(), lens) and pool.free_count.item() == count
        assert np.array_equal(slots.cpu().numpy(), ref["slots"])
        owned = [int(table[b, i]) for b in range(B) for i in range(-(-int(lens[b]) // ps))]
        assert sorted(owned + [int(x) for x in pool.free_pages[:count].tolist()]) == list(range(P))
        served += ref["refused"]
    assert tb.tk_get_device_error() == 0 and served > 0     # the pool ran short at times


@pytest.mark.parametrize("what", ["length", "beyond", "count", "free", "page", "stack"])
def test_bad_values_are_flagged_and_contained(what):
    """Out-of-range values set the error word; the other requests are served and nothing else is written."""
    require_gpu()
    lens, new, count = [20, 5, 3], [1, 1, 14], 2
    table, free = np.array([[0, 1, -1], [2, -1, -1], [3, -1, -1]]), np.array([4, 5, -1, -1, -1, -1])
    if what == "length":
        lens[1] = -4
    elif what == "beyond":
        lens[1] = 49
    elif what == "count":
        new[1] = -2
    elif what == "free":
        count = 7
    elif what == "page":
        table[1, 0] = 6
    else:
        free[1] = -3
    got = _run(lens, new, table, free, count, 16, 16, 0, False)
    assert tb.tk_get_device_error() == 1 and tb.tk_get_device_error() == 0
    assert got["slots"][0] == 16 + 4                        # the sound first request
    if what in ("length", "beyond", "count"):
        assert got["refused"][0] == 1 and got["offsets"].tolist() == [0, 1, 1, 15]
    if what == "page":
        assert got["slots"][1] == -1 and got["seq_lens"].tolist() == [21, 6, 17]
    if what == "stack":
        assert got["slots"][15] == -1 and got["page_table"][2].tolist() == [3, -1, -1]


def test_prepared_graph_replays():
    """A decode step recorded once, replayed in place: lengths grow by one a replay."""
    require_gpu()
    B, ps = 3, 16
    s = torch.cuda.Stream()
    pool = tb.PagePool.allocate(B, 4, ps, 12)
    new, slots, pos = torch.ones(B, **I32), torch.empty(B, **I32), torch.empty(B, **I32)
    s.wait_stream(torch.cuda.current_stream())
    step = tb.prepare_block_tables(pool, new, slots, pos, tokens_per_seq=1, stream=s, graph=True)   # runs once
    for _ in range(40):
        step()
    s.synchronize()
    assert pool.seq_lens.tolist() == [41] * B and pos.tolist() == [40] * B
    owned = pool.page_table[:, :3].flatten().tolist()
    assert sorted(owned + pool.free_pages[:pool.free_count.item()].tolist()) == list(range(12))
    assert slots.tolist() == [p * ps + 8 for p in pool.page_table[:, 2].tolist()]
    assert tb.tk_get_device_error() == 0


@pytest.mark.parametrize("graph", [False, True])
def test_decode_right_behind_the_tables(graph):
    """The decode reads lengths and page table ahead of its wait (a prefetch): with the tables just written by the
    kernel before it, its result is still that of a call on settled tables."""
    require_gpu()
    B, hq, hkv, r, dv, ps, mp = 4, 8, 2, 32, 64, 16, 8
    num_pages = B * mp
    pool = tb.PagePool.allocate(B, mp, ps, num_pages)
    c = tb.ThinKeyCache.allocate(B, hq, hkv, r, dv, page_size=ps, num_pages=num_pages, page_table=pool.page_table)
    c.k.copy_(torch.randn(c.k.shape, device="cuda"))
    c.v.copy_(torch.randn(c.v.shape, device="cuda"))
    q = torch.randn(B, hq, r, device="cuda").to(torch.bfloat16)
    new = torch.tensor([1, 1, 1, 1], **I32)
    slots, pos = torch.empty(B, **I32), torch.empty(B, **I32)
    out, ref = torch.empty(B, hq, dv, device="cuda"), torch.empty(B, hq, dv, device="cuda")
    ws = tb.decode_workspace(c.desc, mp * ps)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        tables = tb.prepare_block_tables(pool, new, slots, pos, tokens_per_seq=1, stream=s)

        def step():
            tables()
            tb.tk_attn_decode(c, q, pool.seq_lens, mp * ps, out, ws)

        step()
        if graph:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                step()
        for i in range(3 * ps * mp // 4):
            new.fill_(-1 if i == 40 else 1)             # once everybody leaves and the pages come back
            g.replay() if graph else step()
            s.synchronize()
            tb.tk_attn_decode(c, q, pool.seq_lens, mp * ps, ref, ws)
            assert torch.equal(out, ref), i
    assert tb.tk_get_device_error() == 0
