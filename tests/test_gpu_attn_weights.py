"""Accumulated attention weights against the float64 oracle.

Tolerance, derived: with A = scale log2e max |q_i| . |k_i| (the largest sum of magnitudes of a score),
a score of r / 16 steps is off by at most (r / 16) 17 2^-23 A on the tensor cores, and by 3 2^-24 A
for the scale, its product and the difference with the maximum; two such errors meet in a weight
(its own and, averaged, those of the sum), ln 2 each, with 2^-22 for each exponential and 2^-24
for each of the log2(L) + 16 levels of a sum of positive terms.  Where a row is one number,
maximum + log2 of the sum, that rounds by 2^-24 (A + log2 L): the difference's 2^-24 A, and ln 2
log2(L) 2^-24 among the levels."""

import math

import numpy as np
import pytest
import torch

from _helpers import f64, require_gpu
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


def _queries(B, hq, n, r, seed, size=1.0):
    return (size * torch.randn(B, hq, n, r, generator=torch.Generator().manual_seed(seed))).to(torch.bfloat16).cuda()


def _tol(x, q, scale):
    live = np.concatenate([x.rows(b, g) for b in range(x.B) for g in range(x.h_kv)])
    A = abs(scale) * 1.4427 * np.abs(f64(q)).max((0, 1, 2)) @ np.abs(x.keys64()[live]).max(0)
    dx = (x.r / 16 * 17 * 2.0 ** -23 + 3 * 2.0 ** -24) * A
    return 2 * math.log(2) * dx + 2 * 2.0 ** -22 + (math.log2(max(x.lens) + 2) + 16) * 2.0 ** -24


def _check(x, q, old=None, decay=1.0, scale=None, max_len=None, w0=0.75):
    n = q.shape[2]
    max_len = max(x.lens) if max_len is None else max_len
    w = tb.slot_weights(x.c)
    w.fill_(w0)
    for b in range(x.B):                     # slots without a weight hold NaNs
        for g in range(x.h_kv):
            rows = x.rows(b, g)
            first = 0 if old is None else min(max(old[b], 0), len(rows))
            w.view(-1)[torch.from_numpy(rows[first:]).cuda()] = float("nan")
    before = w.clone()
    tb.tk_attn_weights(x.c, q, x.seq, max_len, w, tb.attn_weights_workspace(x.c, max_len, n),
                       None if old is None else i32(old), decay, scale)
    torch.cuda.synchronize()
    s = 1 / math.sqrt(x.r) if scale is None else scale
    got, keys, qq = w.cpu().numpy().astype(np.float64).reshape(-1), x.keys64(), f64(q)
    want, G, live = before.cpu().numpy().astype(np.float64).reshape(-1), x.h_q // x.h_kv, np.zeros(x.rows_total, bool)
    add = np.zeros(x.rows_total)
    for b in range(x.B):
        for g in range(x.h_kv):
            rows = x.rows(b, g)
            live[rows] = True
            first = 0 if old is None else min(max(old[b], 0), len(rows))
            want[rows[first:]] = 0
            want[rows[:first]] *= decay
            add[rows] = lc.attn_weights(qq[b, g * G:(g + 1) * G], keys[rows], s, n)
    want[live] += add[live]
    err = np.abs(got - want)[live]
    bound = _tol(x, q, s) * add[live] + 2.0 ** -23 * np.abs(want[live]) + 1e-37
    assert np.all(np.isfinite(got[live])) and (err <= bound).all(), (err / bound).max()
    assert torch.equal(bits(w).view(-1)[~torch.from_numpy(live)], bits(before).view(-1)[~torch.from_numpy(live)])
    return w


@pytest.mark.parametrize("k,r,G,ps", [
    ("bf16", 16, 1, 0), ("bf16", 32, 4, 64), ("bf16", 64, 8, 16), ("bf16", 128, 2, 0), ("int8", 16, 8, 16),
    ("int8", 32, 4, 0), ("int8", 64, 1, 256), ("int8", 128, 4, 32), ("int4", 32, 2, 0), ("int4", 64, 4, 64),
    ("int4", 128, 8, 128)])
@pytest.mark.parametrize("n", [1, 3, 17])
def test_weights(k, r, G, ps, n):
    lens = [0, 1, 2, 15, 16, 17, 255, 1000, 1300]
    x = Cache(lens, 2 * G, 2, r, 64, 1536, ps, k, seed=r + G + n)
    q = _queries(x.B, x.h_q, n, r, n)
    _check(x, q)
    _check(x, q, [max(0, L - n) for L in lens], 0.9)


@pytest.mark.parametrize("G,n", [(1, 512), (8, 64), (4, 33), (2, 100), (1, 7)])
def test_many_queries(G, n):
    x = Cache([5, 700, 64], 2 * G, 2, 32, 64, 704, 0, "bf16", seed=n)
    _check(x, _queries(3, 2 * G, n, 32, n), [0, 650, 64], 0.5)


@pytest.mark.parametrize("r,G,n,ps,cap", [
    (16, 4, 32, 0, 1312), (16, 8, 40, 64, 1536), (32, 8, 64, 16, 1536), (32, 2, 64, 0, 1312),
    (64, 4, 12, 0, 1312), (128, 4, 8, 16, 1536), (64, 4, 32, 16, 1536), (64, 1, 65, 64, 1536), (64, 8, 64, 128, 1536), (64, 2, 200, 256, 1536),
    (128, 2, 32, 0, 1328), (128, 8, 64, 32, 1536), (128, 4, 33, 128, 1536), (128, 4, 100, 0, 1504)])
def test_tiles_of_many_queries(r, G, n, ps, cap):
    """Rows of bf16 keys enough for products of 128 x 128 tiles.  Contexts of less than a tile,
    of one, and that end inside one; rows that see nothing; row tiles that are not full."""
    lens = [0, 1, 63, 127, 128, 129, 640, 1000, 1300]
    x = Cache(lens, 2 * G, 2, r, 64, cap, ps, "bf16", seed=r + n)
    q = _queries(x.B, x.h_q, n, r, G)
    _check(x, q)
    _check(x, q, [max(0, L - n) for L in lens], 0.9, scale=-0.2)
    w = _check(x, q, scale=0.0)
    assert torch.isfinite(w.view(-1)[torch.from_numpy(x.rows(8, 1)).cuda()]).all()


@pytest.mark.parametrize("B,G,n,L,ps", [(1, 4, 32, 40001, 64), (40, 4, 16, 1500, 0), (2, 8, 64, 9001, 16)])
def test_tiles_of_many_queries_in_long_ranges(B, G, n, L, ps):
    """Rings and score buffers that are used more than once, more pairs than processors."""
    lens = [L - 37 * i for i in range(B)]
    x = Cache(lens, 4 * G, 4, 64, 64, (L + 255) // 256 * 256, ps, "bf16", seed=n + B)
    _check(x, _queries(B, 4 * G, n, 64, B, size=2.0))


def test_tiles_of_many_queries_infinities_nans_and_bad_pages():
    x = Cache([300, 300], 4, 2, 64, 64, 304, 16, "bf16", seed=31)
    q, ws = _queries(2, 4, 40, 64, 13), tb.attn_weights_workspace(x.c, 300, 40)
    keys = x.c.k.view(-1, 64)
    saved = keys.clone()
    _check(x, q)
    keys[int(x.rows(0, 0)[50]), 3] = float("nan")
    keys[int(x.rows(1, 1)[60]), 3] = float("inf")
    w = tb.slot_weights(x.c)
    tb.tk_attn_weights(x.c, q, x.seq, 300, w, ws)
    flat = w.view(-1).cpu().numpy()
    assert all(np.isfinite(flat[x.rows(b, g)]).all() == (b != g) for b in range(2) for g in range(2))
    keys.copy_(saved)
    # a key that scores -inf has no weight, and the others have theirs
    keys[int(x.rows(0, 0)[7]), 0] = float("-inf")
    tb.tk_attn_weights(x.c, q.abs(), x.seq, 300, w, ws)
    got = w.view(-1).cpu().numpy()[x.rows(0, 0)]
    assert got[7] == 0 and np.isfinite(got).all() and abs(got.sum() / 80 - 1) < 1e-5
    keys.copy_(saved)
    x.c.page_table[0, 1] = 1 << 20
    w.zero_()
    tb.tk_attn_weights(x.c, q, x.seq, 300, w, ws)
    assert tb.tk_get_device_error() == 1
    other = np.ones(w.numel(), bool)
    other[np.concatenate([x.rows(0, g)[i] for g in range(2) for i in (slice(16), slice(32, None))] + [x.rows(1, 0), x.rows(1, 1)])] = False
    assert (w.view(-1).cpu().numpy()[other] == 0).all()


def test_tiles_of_many_queries_the_same_bits_again_and_through_a_graph():
    x = Cache([3000, 777], 8, 2, 64, 64, 3008, 0, "bf16", seed=14)
    q = _queries(2, 8, 24, 64, 12)
    s = torch.cuda.Stream()
    ws = tb.attn_weights_workspace(x.c, 3000, 24)
    a, b = tb.slot_weights(x.c), tb.slot_weights(x.c)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        call = tb.prepare_attn_weights(x.c, q, x.seq, 3000, a, ws, x.seq, stream=s, graph=True)
        for _ in range(3):
            call()
    s.synchronize()
    for _ in range(4):
        tb.tk_attn_weights(x.c, q, x.seq, 3000, b, ws, x.seq)
    torch.cuda.synchronize()
    assert torch.equal(bits(a), bits(b)) and a.sum() > 0


@pytest.mark.parametrize("k,r,G", [("bf16", 32, 4), ("bf16", 64, 8), ("bf16", 32, 1), ("int8", 64, 2)])
def test_scores_kept_in_the_workspace(k, r, G):
    """Keys beyond what the L2 holds: the other form of the second launch."""
    B, cap = 2, {32: 524288, 64: 262144}[r] * (2 if k == "int8" else 1)
    x = Cache([3, 5000], G, 1, r, 64, cap, 0, k, seed=3)
    need = tb.attn_weights_workspace(x.c, cap).numel()
    assert need > B * cap * G * 4
    _check(x, _queries(B, G, 1, r, 4), [0, 4990], 0.5, max_len=cap)


def test_long_context_and_many_splits():
    x = Cache([70001, 12345], 4, 1, 16, 64, 70016, 16, "bf16", seed=7)
    _check(x, _queries(2, 4, 2, 16, 5))


def test_peaked_and_flat_rows():
    """One token with all of the weight, tokens with equal weights, scores far below the maximum."""
    x = Cache([300, 300], 2, 1, 32, 64, 304, 0, "bf16", seed=8)
    x.c.k[1, 0, :300] = 0.5
    _check(x, _queries(2, 2, 1, 32, 6, size=12.0))
    _check(x, torch.zeros(2, 2, 1, 32, dtype=torch.bfloat16, device="cuda"))
    _check(x, _queries(2, 2, 1, 32, 7), scale=-0.3)


def test_decay_zero_reads_nothing():
    x = Cache([100], 2, 1, 32, 64, 112, 0, "bf16", seed=9)
    q, ws = _queries(1, 2, 1, 32, 8), tb.attn_weights_workspace(x.c, 100)
    a, b = torch.full_like(tb.slot_weights(x.c), float("nan")), tb.slot_weights(x.c)
    tb.tk_attn_weights(x.c, q, x.seq, 100, a, ws, x.seq, 0.0)
    tb.tk_attn_weights(x.c, q, x.seq, 100, b, ws)
    assert torch.equal(a[..., :100], b[..., :100]) and torch.isnan(a[..., 100:]).all()


def test_infinities_and_nans_stay_with_their_kv_head():
    x = Cache([200, 200], 4, 2, 32, 64, 208, 0, "bf16", seed=10)
    q = _queries(2, 4, 1, 32, 9)
    x.c.k[0, 0, 50, 3] = float("nan")
    x.c.k[1, 1, 60, 3] = float("inf")
    w = tb.slot_weights(x.c)
    tb.tk_attn_weights(x.c, q, x.seq, 200, w, tb.attn_weights_workspace(x.c, 200))
    ok = torch.isfinite(w[..., :200]).all(-1)
    assert not ok[0, 0] and ok[0, 1] and ok[1, 0]
    # a key that scores -inf has no weight, and the others have theirs
    y = Cache([40], 1, 1, 32, 64, 48, 0, "bf16", seed=11)
    qy = torch.ones(1, 1, 1, 32, dtype=torch.bfloat16, device="cuda")
    y.c.k[0, 0, 7, 0] = float("-inf")
    w = tb.slot_weights(y.c)
    tb.tk_attn_weights(y.c, qy, y.seq, 40, w, tb.attn_weights_workspace(y.c, 40))
    w = w[0, 0, :40].cpu()
    assert w[7] == 0 and torch.isfinite(w).all() and abs(float(w.sum()) - 1) < 1e-5


def test_bad_lengths_and_pages():
    x = Cache([64, 64], 2, 1, 32, 64, 64, 16, "bf16", seed=12)
    q, ws = _queries(2, 2, 1, 32, 10), tb.attn_weights_workspace(x.c, 48)
    w = tb.slot_weights(x.c)
    tb.tk_attn_weights(x.c, q, i32([-7, 64]), 48, w, ws)           # beyond the bound: 48 tokens
    assert tb.tk_get_device_error() == 1
    flat = w.view(-1).cpu().numpy()
    assert (flat[x.rows(0, 0)] == 0).all() and (flat[x.rows(1, 0)[:48]] > 0).all() and (flat[x.rows(1, 0)[48:]] == 0).all()
    x.c.page_table[0, 1] = 1 << 20
    w.zero_()
    tb.tk_attn_weights(x.c, q, x.seq, 64, w, tb.attn_weights_workspace(x.c, 64))
    assert tb.tk_get_device_error() == 1
    own = np.concatenate([x.rows(0, 0)[:16], x.rows(0, 0)[32:], x.rows(1, 0)])
    other = np.ones(w.numel(), bool)
    other[own] = False
    assert (w.view(-1).cpu().numpy()[other] == 0).all()            # nothing on the page that took its place


def test_the_same_bits_again_and_through_a_graph():
    x = Cache([3000, 777], 8, 2, 32, 64, 3008, 0, "int8", seed=13)
    q = _queries(2, 8, 1, 32, 11)
    s = torch.cuda.Stream()
    ws = tb.attn_weights_workspace(x.c, 3000)
    a, b = tb.slot_weights(x.c), tb.slot_weights(x.c)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        call = tb.prepare_attn_weights(x.c, q, x.seq, 3000, a, ws, x.seq, stream=s, graph=True)
        for _ in range(2):
            call()
    s.synchronize()
    for _ in range(3):
        tb.tk_attn_weights(x.c, q, x.seq, 3000, b, ws, x.seq)
    torch.cuda.synchronize()
    assert torch.equal(bits(a), bits(b)) and a.sum() > 0
    q = _queries(2, 8, 2, 32, 11)
    with pytest.raises(tb.TkError, match="TK_ERR_WORKSPACE"):
        tb.tk_attn_weights(x.c, q, x.seq, 3000, b, tb.attn_weights_workspace(x.c, 3000, 2)[:256])


def test_tiles_of_many_queries_behind_changing_lengths_and_keys():
    """Steps in a row, each with new lengths, keys and a new page, as with a wait between them."""
    def run(wait):
        x = Cache([700, 130], 8, 2, 64, 64, 1024, 16, "bf16", seed=15)
        keys, w, ws = x.c.k, tb.slot_weights(x.c), tb.attn_weights_workspace(x.c, 1024, 16)
        keys.nan_to_num_(0.25)
        q, seq, old = _queries(2, 8, 16, 64, 14), x.seq.clone(), x.seq.clone()
        for step in range(12):
            old.copy_(seq)
            seq.add_(16)
            keys.mul_(-1)
            x.c.page_table[:, 3:5] = x.c.page_table[:, 3:5].flip(1)
            if wait:
                torch.cuda.synchronize()
            tb.tk_attn_weights(x.c, q, seq, 1024, w, ws, old, 0.75)
            if wait:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        return w
    a, b = run(False), run(True)
    assert torch.equal(bits(a), bits(b)) and a.sum() > 0
