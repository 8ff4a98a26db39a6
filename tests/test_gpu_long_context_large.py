"""The operators over a long context at the ends of their ranges: caches whose offsets pass 32 bits,
several streams, graphs that share a workspace, refused devices, more units than one wave."""

import math

import numpy as np
import pytest
import torch

from _helpers import f64, parity, require_gpu
from _long_context import Cache, bits, i32
from oracle import attention as oa
from oracle import long_context as lc
from paper_2603_04427_gb300 import binding as tb

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean():
    require_gpu()
    tb.tk_get_device_error()
    yield
    assert tb.tk_get_device_error() == 0


def test_offsets_beyond_32_bits():
    """The last kv head of the last sequence starts 2^32 elements into the cache (8.6 GB of keys and of
    values): bounds, choice, decode, weights and eviction of its 300 tokens."""
    B, hq, hkv, r, dv, L = 3, 4, 2, 128, 128, 300
    cap = (2 ** 32 // 128 // 5 // 64 + 1) * 64          # row 5 cap is 2^32 / 128 and more
    c = tb.ThinKeyCache.allocate(B, hq, hkv, r, dv, capacity=cap)
    assert 5 * cap * r >= 2 ** 32
    g = torch.Generator(device="cuda").manual_seed(1)
    c.k[2, :, :L] = torch.randn(hkv, L, r, device="cuda", generator=g).to(torch.bfloat16)
    c.v[2, :, :L] = torch.randn(hkv, L, dv, device="cuda", generator=g).to(torch.bfloat16)
    k, v = f64(c.k[2, :, :L]), f64(c.v[2, :, :L])
    seq, q = i32([0, 0, L]), torch.randn(B, hq, r, device="cuda", generator=g).to(torch.bfloat16)
    qq = f64(q)[2]
    box = tb.block_bounds(c, 16)
    tb.tk_block_bounds(c, box, seq, max_new=512, block=16)
    sel = tb.BlockSelection.allocate(c, 7, 16, ids=True)
    tb.tk_block_select(c, q, box, seq, 512, sel)
    out = torch.empty(B, hq, dv, device="cuda")
    tb.tk_attn_decode_blocks(c, q, sel, out, tb.decode_blocks_workspace(c, sel))
    w = tb.slot_weights(c)
    tb.tk_attn_weights(c, q, seq, 512, w, tb.attn_weights_workspace(c, 512))
    for h in range(hkv):
        lo, hi = lc.block_bounds(k[h], 16)
        assert np.array_equal(f64(box[2, h, :19]), np.stack([lo, hi], 1)) and (box[2, h, 19:40] == 0).all()
        pick = lc.block_select(lc.block_scores(qq[2 * h:2 * h + 2], lo, hi), 7)
        assert sel.ids[2, h].tolist() == pick.tolist()
        t = np.concatenate([np.arange(16 * i, min(16 * i + 16, L)) for i in pick])
        parity(f64(out)[2, 2 * h:2 * h + 2], oa.attention_head(qq[2 * h:2 * h + 2], k[h, t], v[h, t], 1 / math.sqrt(r)))
        ref = lc.attn_weights(qq[2 * h:2 * h + 2, None], k[h], 1 / math.sqrt(r), 1)
        assert np.allclose(f64(w[2, h, :L]), ref, rtol=1e-3, atol=0) and (w[2, h, L:512] == 0).all()
    kept = torch.empty(B, hkv, 100, dtype=torch.int32, device="cuda")
    before = f64(w[2, :, :L])
    tb.tk_cache_evict(c, seq, 512, w, 100, 20, tb.cache_evict_workspace(c, 100), kept=kept)
    assert seq.tolist() == [0, 0, 100]
    for h in range(hkv):
        order = lc.evict(before[h], 100, 20)
        assert kept[2, h].tolist() == order.tolist()
        assert np.array_equal(f64(c.k[2, h, :100]), k[h, order]) and np.array_equal(f64(c.v[2, h, :100]), v[h, order])
        assert np.array_equal(f64(c.k[2, h, 100:L]), k[h, 100:])
    assert (c.k[1, 1, -64:] == 0).all() and (c.k[2, 0, L:400] == 0).all()


def _step(x, q, ws, stream, n=4):
    """Bounds, choice, decode, weights and eviction of one cache on a stream."""
    box, sel, out, w = ws["box"], ws["sel"], ws["out"], ws["w"]
    tb.tk_block_bounds(x.c, box, x.seq, stream=stream)
    tb.tk_block_select(x.c, q, box, x.seq, x.cap, sel, stream=stream)
    tb.tk_attn_decode_blocks(x.c, q, sel, out, ws["decode"], stream=stream)
    tb.tk_attn_weights(x.c, q, x.seq, x.cap, w, ws["weights"], stream=stream)
    tb.tk_cache_evict(x.c, x.seq, x.cap, w, 150, 20, ws["evict"], stream=stream)


def _spaces(x, n=4):
    sel = tb.BlockSelection.allocate(x.c, n)
    return dict(box=tb.block_bounds(x.c), sel=sel, out=torch.zeros(x.B, x.h_q, x.d_v, device="cuda"), w=tb.slot_weights(x.c),
                decode=tb.decode_blocks_workspace(x.c, sel), weights=tb.attn_weights_workspace(x.c, x.cap),
                evict=tb.cache_evict_workspace(x.c, 150))


def test_two_streams_at_once():
    """Two caches, each with workspaces of its own, on two streams, give what they give alone."""
    make = lambda s: Cache([300, 411, 17], 8, 2, 32, 64, 512, 32, "int8" if s else "bf16", seed=30 + s)  # noqa: E731
    q = [torch.randn(3, 8, 32, generator=torch.Generator().manual_seed(s)).to(torch.bfloat16).cuda() for s in range(2)]
    alone, both = [make(s) for s in range(2)], [make(s) for s in range(2)]
    wa, wb = [_spaces(x) for x in alone], [_spaces(x) for x in both]
    for s in range(2):
        for _ in range(3):
            _step(alone[s], q[s], wa[s], None)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for s in range(2):
            _step(both[s], q[s], wb[s], streams[s])
    torch.cuda.synchronize()
    for s in range(2):
        for a, b in ((alone[s].c.k, both[s].c.k), (alone[s].c.v, both[s].c.v), (alone[s].seq, both[s].seq),
                     (wa[s]["w"], wb[s]["w"]), (wa[s]["out"], wb[s]["out"]), (wa[s]["box"], wb[s]["box"])):
            assert torch.equal(bits(a), bits(b))


def test_graphs_that_share_workspaces_in_stream_order():
    """Calls of different shapes through one workspace each, recorded in two graphs and replayed in turn."""
    x = Cache([900, 33], 4, 2, 64, 64, 1024, 0, "bf16", seed=40)
    y = Cache([500, 200, 100], 8, 1, 64, 64, 512, 0, "bf16", seed=41)
    s = torch.cuda.Stream()
    n = 3
    qx, qy = (torch.randn(c.B, c.h_q, n, 64, generator=torch.Generator().manual_seed(5)).to(torch.bfloat16).cuda() for c in (x, y))
    ws = max((tb.attn_weights_workspace(c.c, c.cap, n) for c in (x, y)), key=torch.Tensor.numel)
    wx, wy = tb.slot_weights(x.c), tb.slot_weights(y.c)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        calls = [tb.prepare_attn_weights(x.c, qx, x.seq, 1024, wx, ws, stream=s, graph=True),
                 tb.prepare_attn_weights(y.c, qy, y.seq, 512, wy, ws, stream=s, graph=True)]
        for _ in range(3):
            wx.zero_()
            wy.zero_()
            for c in calls:
                c()
    s.synchronize()
    for c, q, w in ((x, qx, wx), (y, qy, wy)):
        ref = tb.slot_weights(c.c)
        tb.tk_attn_weights(c.c, q, c.seq, c.cap, ref, tb.attn_weights_workspace(c.c, c.cap, n))
        torch.cuda.synchronize()
        assert torch.equal(bits(w), bits(ref)) and float(ref.sum()) > 0


def test_more_sequences_than_a_wave():
    """2000 sequences: every launch has several waves of blocks."""
    B = 2000
    lens = [(13 * b) % 97 for b in range(B)]
    x = Cache(lens, 2, 1, 16, 64, 96, 0, "bf16", seed=50)
    x.lens = [min(n, 96) for n in lens]
    x.seq = i32(x.lens)
    q = torch.randn(B, 2, 16, generator=torch.Generator().manual_seed(6)).to(torch.bfloat16).cuda()
    w = tb.slot_weights(x.c)
    tb.tk_attn_weights(x.c, q, x.seq, 96, w, tb.attn_weights_workspace(x.c, 96))
    box = tb.block_bounds(x.c, 16)
    tb.tk_block_bounds(x.c, box, x.seq, block=16)
    sel = tb.BlockSelection.allocate(x.c, 3, 16, ids=True)
    tb.tk_block_select(x.c, q, box, x.seq, 96, sel)
    keys, before = x.keys64(), w.cpu().numpy().astype(np.float64).reshape(-1)
    kept = torch.empty(B, 1, 40, dtype=torch.int32, device="cuda")
    tb.tk_cache_evict(x.c, x.seq, 96, w, 40, 5, tb.cache_evict_workspace(x.c, 40), kept=kept)
    kept, ids, qq = kept.cpu().numpy(), sel.ids.cpu().numpy(), f64(q)
    for b in range(0, B, 7):
        rows = x.rows(b, 0)
        if len(rows):
            assert np.allclose(before[rows], lc.attn_weights(qq[b][:, None], keys[rows], 0.25, 1), rtol=1e-4, atol=1e-30)
        lo, hi = lc.block_bounds(keys[rows], 16)
        pick = lc.block_select(lc.block_scores(qq[b], lo, hi), 3)
        assert ids[b, 0, :len(pick)].tolist() == pick.tolist() and (ids[b, 0, len(pick):] == -1).all()
        order = lc.evict(before[rows], 40, 5)
        assert kept[b, 0, :len(order)].tolist() == order.tolist()
    assert x.seq.tolist() == [min(n, 40) for n in x.lens]


def test_empty_batch_is_a_no_op():
    c = tb.ThinKeyCache.allocate(0, 4, 2, 32, 64, capacity=64)
    seq, q = i32([]), torch.empty(0, 4, 32, dtype=torch.bfloat16, device="cuda")
    tb.tk_block_bounds(c, tb.block_bounds(c), seq)
    sel = tb.BlockSelection.allocate(c, 2)
    tb.tk_block_select(c, q, tb.block_bounds(c), seq, 64, sel)
    out = torch.empty(0, 4, 64, device="cuda")
    tb.tk_attn_decode_blocks(c, q, sel, out, tb.decode_blocks_workspace(c, sel))
    tb.tk_attn_weights(c, q, seq, 64, tb.slot_weights(c), tb.attn_weights_workspace(c, 64))
    tb.tk_cache_evict(c, seq, 64, tb.slot_weights(c), 8, 2, tb.cache_evict_workspace(c, 8))


def test_another_device_than_the_current_one_is_refused(monkeypatch):
    x = Cache([64], 2, 1, 32, 64, 64, 0, "bf16", seed=60)
    ws = _spaces(x)
    q = torch.zeros(1, 2, 32, dtype=torch.bfloat16, device="cuda")
    monkeypatch.setattr(tb, "_current_device", lambda: 1)
    for call in (lambda: tb.tk_block_bounds(x.c, ws["box"], x.seq),
                 lambda: tb.tk_block_select(x.c, q, ws["box"], x.seq, 64, ws["sel"]),
                 lambda: tb.tk_attn_decode_blocks(x.c, q, ws["sel"], ws["out"], ws["decode"]),
                 lambda: tb.tk_attn_weights(x.c, q, x.seq, 64, ws["w"], ws["weights"]),
                 lambda: tb.tk_cache_evict(x.c, x.seq, 64, ws["w"], 8, 2, ws["evict"]),
                 lambda: tb.attn_weights_workspace(x.c, 64), lambda: tb.decode_blocks_workspace(x.c, ws["sel"])):
        with pytest.raises(ValueError, match="current"):
            call()


def test_wrong_shapes_and_types_are_refused():
    x = Cache([64], 2, 1, 32, 64, 64, 16, "int8", seed=61)
    ws = _spaces(x)
    q = torch.zeros(1, 2, 32, dtype=torch.bfloat16, device="cuda")
    for call in (lambda: tb.tk_block_bounds(x.c, ws["box"].float(), x.seq),
                 lambda: tb.tk_block_bounds(x.c, ws["box"][1:], x.seq),
                 lambda: tb.tk_block_bounds(x.c, ws["box"], x.seq.long()),
                 lambda: tb.tk_block_bounds(x.c, ws["box"], x.seq, block=32),
                 lambda: tb.tk_block_select(x.c, q[..., :16], ws["box"], x.seq, 64, ws["sel"]),
                 lambda: tb.tk_block_select(x.c, q, ws["box"], x.seq, 64, ws["sel"], n_last=0),
                 lambda: tb.tk_attn_decode_blocks(x.c, q, ws["sel"], ws["out"][:, :1], ws["decode"]),
                 lambda: tb.tk_attn_decode_blocks(x.c, q.transpose(1, 2), ws["sel"], ws["out"], ws["decode"]),
                 lambda: tb.tk_attn_weights(x.c, q[:, :, None, None], x.seq, 64, ws["w"], ws["weights"]),
                 lambda: tb.tk_attn_weights(x.c, q, x.seq, 64, ws["w"].half(), ws["weights"]),
                 lambda: tb.tk_cache_evict(x.c, x.seq, 64, ws["w"], 8, 9, ws["evict"]),
                 lambda: tb.tk_cache_evict(x.c, x.seq, 64, ws["w"], 8, 2, ws["evict"], kept=i32([0])),
                 lambda: tb.tk_cache_evict(x.c, x.seq, 64, ws["w"], 8, 2, ws["evict"],
                                           pool=tb.PagePool.allocate(1, 4, 16, x.c.desc.num_pages))):
        with pytest.raises((ValueError, TypeError, tb.TkError)):
            call()


def test_many_queries_beyond_32_bit_offsets():
    """As above for the weights of 64 queries, whose key tiles come through a tensor map."""
    B, hq, hkv, r, L, n = 3, 4, 2, 128, 300, 64
    cap = (2 ** 32 // 128 // 5 // 64 + 1) * 64
    c = tb.ThinKeyCache.allocate(B, hq, hkv, r, 64, capacity=cap)
    g = torch.Generator(device="cuda").manual_seed(2)
    c.k[2, :, :L] = torch.randn(hkv, L, r, device="cuda", generator=g).to(torch.bfloat16)
    q = torch.randn(B, hq, n, r, device="cuda", generator=g).to(torch.bfloat16)
    w = tb.slot_weights(c)
    tb.tk_attn_weights(c, q, i32([0, 0, L]), 512, w, tb.attn_weights_workspace(c, 512, n))
    for h in range(hkv):
        ref = lc.attn_weights(f64(q)[2, 2 * h:2 * h + 2], f64(c.k[2, h, :L]), 1 / math.sqrt(r), n)
        assert np.allclose(f64(w[2, h, :L]), ref, rtol=1e-3, atol=0) and (w[2, h, L:512] == 0).all()
    assert (w[:2] == 0).all()


def test_many_queries_beside_prefills_on_another_stream():
    """Both hold tensor memory: calls that overlap give what they give alone."""
    x = Cache([2000, 1500, 900], 8, 2, 64, 64, 2048, 16, "bf16", seed=50)
    g = torch.Generator(device="cuda").manual_seed(3)
    qw = torch.randn(3, 8, 32, 64, device="cuda", generator=g).to(torch.bfloat16)
    q, k, v = (torch.randn(2, h, 1024, 64, device="cuda", generator=g).to(torch.bfloat16) for h in (8, 2, 2))
    ws, w = tb.attn_weights_workspace(x.c, 2048, 32), [tb.slot_weights(x.c) for _ in range(2)]
    out = [torch.empty(2, 8, 1024, 64, device="cuda") for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(2):                       # alone, then both streams at once
        for _ in range(20):
            tb.tk_attn_weights(x.c, qw, x.seq, 2048, w[i], ws, x.seq, 0.5, stream=streams[0])
            if i == 0:
                streams[0].synchronize()
            tb.tk_attn_prefill(q, k, v, out[i], stream=streams[1])
            if i == 0:
                streams[1].synchronize()
        torch.cuda.synchronize()
    assert torch.equal(bits(w[0]), bits(w[1])) and torch.equal(bits(out[0]), bits(out[1])) and w[0].sum() > 0
