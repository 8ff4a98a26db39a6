"""Eviction against the oracle: everything is moved, nothing computed, so all of it has to be equal."""

import numpy as np
import pytest
import torch

from _helpers import require_gpu
from _long_context import Cache, bits, i32
from oracle import long_context as lc
from paper_2603_04427_gb300 import binding as tb

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean():
    require_gpu()
    tb.tk_get_device_error()
    yield
    assert tb.tk_get_device_error() == 0


def _weights(x, seed, kind="normal"):
    g = torch.Generator().manual_seed(seed)
    w = torch.exp(2 * torch.randn(x.rows_total, generator=g))
    if kind == "ties":
        w = (w * 2).floor() / 2
    elif kind == "equal":
        w = torch.ones_like(w)
    elif kind == "odd":
        w[torch.rand(x.rows_total, generator=g) < 0.3] = float("nan")
        w[torch.rand(x.rows_total, generator=g) < 0.1] = float("-inf")
        w[torch.rand(x.rows_total, generator=g) < 0.1] = float("inf")
        w[torch.rand(x.rows_total, generator=g) < 0.1] = -0.0
        w[torch.rand(x.rows_total, generator=g) < 0.1] = 0.0
    elif kind == "rising":
        w = torch.arange(x.rows_total).float()
    elif kind == "falling":
        w = -torch.arange(x.rows_total).float()
    return w.view(x.c.v.shape[:-1]).cuda()


def _check(x, w, keep, recent, in_place=False, kept=True, max_len=None, pool=None, valid=None):
    c = x.c
    old = {n: t.clone() for n, t in (("k", c.k), ("v", c.v), ("ks", c.k_scale), ("w", w)) if t is not None}
    w_out = w if in_place else torch.full_like(w, 5.0)
    out0 = w_out.clone()
    seq_out = x.seq if in_place else torch.full_like(x.seq, -9)
    where = torch.full((x.B, x.h_kv, keep), -7, dtype=torch.int32, device="cuda") if kept else None
    tb.tk_cache_evict(c, x.seq, max(x.lens) if max_len is None else max_len, w, keep, recent,
                      tb.cache_evict_workspace(c, keep), w_out, seq_out, where, pool)
    torch.cuda.synchronize()
    flat = lambda t: bits(t).reshape(x.rows_total, -1).numpy()  # noqa: E731
    want = {n: flat(t).copy() for n, t in old.items() if n != "w"}
    want_w, wv = flat(out0).copy(), old["w"].cpu().numpy().astype(np.float64).reshape(-1)
    for b in range(x.B):
        if valid is not None and not valid[b]:
            continue
        for g in range(x.h_kv):
            rows = x.rows(b, g)
            order = lc.evict(wv[rows], keep, recent)
            for n in want:
                want[n][rows[:len(order)]] = flat(old[n])[rows[order]]
            want_w[rows[:len(order)]] = flat(old["w"])[rows[order]]
            if kept:
                full = np.full(keep, -1)
                full[:len(order)] = order
                assert np.array_equal(where[b, g].cpu().numpy(), full), (b, g)
    for n, t in (("k", c.k), ("v", c.v), ("ks", c.k_scale)):
        if t is not None:
            assert np.array_equal(flat(t), want[n]), n
    assert np.array_equal(flat(w_out), want_w)
    lens = [min(L, keep) for L in x.lens] if valid is None else None
    if lens is not None:
        assert seq_out.tolist() == lens
    return seq_out


@pytest.mark.parametrize("k,r,dv,ps", [
    ("bf16", 16, 64, 0), ("bf16", 32, 128, 64), ("bf16", 128, 128, 16), ("int8", 16, 64, 0), ("int8", 64, 128, 32),
    ("int4", 32, 64, 0), ("int4", 128, 128, 128)])
@pytest.mark.parametrize("keep,recent", [(64, 16), (65, 0), (100, 100), (1, 0), (1, 1), (37, 36)])
def test_evict(k, r, dv, ps, keep, recent):
    lens = [0, 1, keep - 1, keep, keep + 1, keep + recent, 2 * keep + 3, 600, 1024]
    x = Cache([min(L, 1024) for L in lens], 4, 2, r, dv, 1024, ps, k, seed=r + keep)
    _check(x, _weights(x, keep + recent), keep, recent, in_place=ps == 0)


@pytest.mark.parametrize("kind", ["ties", "equal", "odd", "rising", "falling"])
def test_evict_kinds_of_weights(kind):
    x = Cache([500, 333, 64, 700], 2, 2, 32, 64, 704, 0, "bf16", seed=5)
    _check(x, _weights(x, 6, kind), 200, 50, in_place=True)
    x = Cache([500, 333, 64, 700], 2, 2, 32, 64, 704, 16, "int8", seed=6)
    _check(x, _weights(x, 7, kind), 100, 0)


@pytest.mark.parametrize("lens,keep,recent", [
    ([1500, 1401], 1400, 1300),        # the recent ones overlap their places in many rounds
    ([3000, 2999], 2998, 2998),
    ([5000, 4097], 2048, 1000), ([20000, 4097], 4096, 128), ([140000], 1000, 100), ([70000], 60000, 30000)])
def test_evict_long(lens, keep, recent):
    cap = -(-max(lens) // 16) * 16
    x = Cache(lens, 1, 1, 16, 64, cap, 0, "bf16", seed=8)
    _check(x, _weights(x, 9), keep, recent, in_place=True)


def test_evict_with_ties_across_a_cluster():
    x = Cache([40000], 1, 1, 16, 64, 40000, 16, "bf16", seed=9)
    _check(x, _weights(x, 10, "equal"), 20000, 7)
    x = Cache([40000], 1, 1, 16, 64, 40000, 16, "bf16", seed=9)
    _check(x, _weights(x, 10, "ties"), 1234, 7, kept=False)


def test_evict_again_and_again():
    """Steps that append and evict: the recent ones keep their order, so that the last appended
    tokens are always the ones that stay."""
    keep, recent, step = 48, 20, 5
    x = Cache([keep] * 2, 2, 1, 32, 64, 64, 0, "bf16", seed=10)
    mark = [list(range(keep)) for _ in range(2)]            # the token in each slot
    count = keep
    w = tb.slot_weights(x.c)
    w[:, :, :keep] = torch.rand(2, 1, keep, generator=torch.Generator().manual_seed(1)).cuda()
    ws, kept = tb.cache_evict_workspace(x.c, keep), torch.empty(2, 1, keep, dtype=torch.int32, device="cuda")
    for _ in range(12):
        new = torch.randn(2, 1, step, 32).to(torch.bfloat16).cuda()
        val = torch.randn(2, 1, step, 64).to(torch.bfloat16).cuda()
        tb.tk_kv_append(x.c, new, val, x.seq)
        w[:, :, keep:keep + step] = 0.0                       # no attention yet: only their age keeps them
        x.seq += step
        tb.tk_cache_evict(x.c, x.seq, keep + step, w, keep, recent, ws, kept=kept)
        for b in range(2):
            mark[b] += list(range(count, count + step))
            mark[b] = [mark[b][i] for i in kept[b, 0].tolist()]
            assert mark[b][keep - recent:] == list(range(count + step - recent, count + step))
        count += step
    assert x.seq.tolist() == [keep, keep]


@pytest.mark.parametrize("ps,keep", [(16, 40), (64, 128), (32, 33)])
def test_pages_go_back(ps, keep):
    lens = [300, 10, 0, keep, keep + 1, 512]
    x = Cache(lens, 2, 2, 32, 64, 512, ps, "bf16", seed=11)
    P = x.c.desc.num_pages
    pool = tb.PagePool(ps, x.c.page_table, torch.full((P,), -3, dtype=torch.int32, device="cuda"), i32([2]), x.seq, i32([0]))
    _check(x, _weights(x, 12), keep, 5, in_place=True, pool=pool)
    back = [int(p) for b in range(6) if lens[b] > keep for p in x.table[b][-(-keep // ps):-(-lens[b] // ps)]]
    assert pool.free_count.item() == 2 + len(back)
    assert pool.free_pages[2:2 + len(back)].tolist() == back and (pool.free_pages[2 + len(back):] == -3).all()
    assert x.seq.tolist() == [min(L, keep) for L in lens]


def test_pages_of_many_sequences_and_a_full_stack():
    B, ps = 600, 16
    lens = [(b * 7) % 65 for b in range(B)]
    x = Cache(lens, 1, 1, 16, 64, 64, ps, "bf16", seed=12)
    P = x.c.desc.num_pages
    pool = tb.PagePool(ps, x.c.page_table, torch.full((P,), -3, dtype=torch.int32, device="cuda"), i32([0]), x.seq, i32([0]))
    _check(x, _weights(x, 13), 20, 4, in_place=True, pool=pool)
    back = [int(p) for b in range(B) if lens[b] > 20 for p in x.table[b][2:-(-lens[b] // ps)]]
    assert pool.free_pages[:pool.free_count.item()].tolist() == back
    x.seq.copy_(i32(lens))
    pool.free_count.fill_(P - 1)                              # one more fits
    tb.tk_cache_evict(x.c, x.seq, 64, _weights(x, 14), 20, 4, tb.cache_evict_workspace(x.c, 20), pool=pool)
    assert pool.free_count.item() == P and pool.free_pages[P - 1].item() == back[0]
    assert tb.tk_get_device_error() == 1


def test_bad_lengths_leave_a_sequence_alone():
    x = Cache([100, 100, 100], 2, 2, 32, 64, 112, 0, "bf16", seed=13)
    x.seq = i32([-4, 100, 113])
    out = _check(x, _weights(x, 14), 50, 10, valid=[False, True, False], kept=False, max_len=112)
    assert out.tolist() == [-4, 50, 113]
    assert tb.tk_get_device_error() == 1
    x.seq = i32([100, 70, 90])                               # beyond the caller's bound
    x.lens = [100, 70, 90]
    out = _check(x, _weights(x, 15), 50, 10, valid=[False, True, False], kept=False, max_len=80)
    assert out.tolist() == [100, 50, 90]
    assert tb.tk_get_device_error() == 1


def test_bad_pages_are_not_touched():
    x = Cache([64, 64], 1, 1, 32, 64, 64, 16, "bf16", seed=14)
    x.c.page_table[0, 3] = 77
    x.c.page_table[1, 0] = -1
    k0, v0 = x.c.k.clone(), x.c.v.clone()
    tb.tk_cache_evict(x.c, x.seq, 64, _weights(x, 16), 24, 8, tb.cache_evict_workspace(x.c, 24))
    assert tb.tk_get_device_error() == 1
    own = set(x.table.reshape(-1).tolist())
    for p in range(x.c.desc.num_pages):
        if p not in own:
            assert torch.equal(bits(k0[p]), bits(x.c.k[p])) and torch.equal(bits(v0[p]), bits(x.c.v[p]))


def test_evict_in_a_graph():
    x = Cache([200, 150], 2, 1, 32, 64, 208, 0, "bf16", seed=15)
    y = Cache([200, 150], 2, 1, 32, 64, 208, 0, "bf16", seed=15)
    w = _weights(x, 17)
    s = torch.cuda.Stream()
    a, b = torch.zeros_like(w), torch.zeros_like(w)
    ka, kb = (torch.zeros(2, 1, 96, dtype=torch.int32, device="cuda") for _ in range(2))
    la, lb = i32([0, 0]), i32([0, 0])
    ws = tb.cache_evict_workspace(x.c, 96)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        call = tb.prepare_cache_evict(x.c, x.seq, 208, w, 96, 30, ws, a, la, ka, stream=s, graph=True)
        w2 = _weights(x, 18)
        w.copy_(w2)
        call()
    s.synchronize()
    for weights in (_weights(y, 17), w2):
        tb.tk_cache_evict(y.c, y.seq, 208, weights, 96, 30, ws, b, lb, kb)
    torch.cuda.synchronize()
    assert torch.equal(ka, kb) and torch.equal(la, lb) and torch.equal(bits(a), bits(b))
    assert torch.equal(bits(x.c.k), bits(y.c.k)) and torch.equal(bits(x.c.v), bits(y.c.v))
