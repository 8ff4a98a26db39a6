"""Bounds of key blocks, the choice of blocks and the decode over them, against the float64 oracle.

Bounds and choices have to be equal: bounds are values of the cache (or roundings that both sides
define), scores are compared in 64 bits.  The decode has the parity bar of the other decode tests."""

import math

import numpy as np
import pytest
import torch

from _helpers import f64, parity, parity_bf16, require_gpu
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


def _ref_bounds(x, block, old=None):
    """Rows [n] and bounds [n, 2, r] of the blocks that hold a token at old[b] .. lens[b] - 1."""
    keys = x.keys32()
    at, box = [], []
    for b in range(x.B):
        first = 0 if old is None else old[b] // block
        if old is not None and old[b] >= x.lens[b]:
            continue
        for g in range(x.h_kv):
            lo, hi = lc.block_bounds(keys[x.rows(b, g)], block, x.k != "bf16")
            rows = x.rows(b, g)[::block] // block
            at.append(rows[first:])
            box.append(np.stack([lo, hi], 1)[first:])
    return np.concatenate(at).astype(np.int64), np.concatenate(box)


def _check_bounds(x, block, old=None, max_new=None, stream=None):
    box = tb.block_bounds(x.c, block)
    box.fill_(7.0)
    tb.tk_block_bounds(x.c, box, x.seq, None if old is None else i32(old), max_new, block, stream=stream)
    torch.cuda.synchronize()
    at, ref = _ref_bounds(x, block, old)
    want = np.full((box.numel() // (2 * x.r), 2, x.r), 7.0)
    want[at] = ref
    assert np.array_equal(f64(box).reshape(want.shape), want)
    return box


@pytest.mark.parametrize("k,r,block,ps", [
    ("bf16", 16, 16, 0), ("bf16", 32, 64, 0), ("bf16", 64, 128, 0), ("bf16", 128, 256, 0), ("bf16", 128, 16, 16),
    ("bf16", 32, 64, 64), ("bf16", 16, 256, 256), ("int8", 16, 32, 0), ("int8", 32, 16, 16), ("int8", 64, 256, 0),
    ("int8", 128, 64, 64), ("int4", 32, 16, 0), ("int4", 64, 64, 64), ("int4", 128, 256, 256)])
def test_bounds(k, r, block, ps):
    lens = [0, 1, block - 1, block, block + 1, 5 * block + 3, 8 * block]
    x = Cache(lens, 6, 3, r, 64, 8 * block, ps, k, seed=r + block)
    _check_bounds(x, block)
    # the tokens of a step, of several, of none (old beyond the context too)
    _check_bounds(x, block, [0, 0, block - 2, block - 1, block, 2 * block + 5, 8 * block + 9], 4 * block)
    _check_bounds(x, block, [max(0, n - 1) for n in lens], 1)


def test_bounds_many_units_and_one_warp_of_blocks():
    """More blocks than the launch has warps, so that each takes several."""
    x = Cache([40000, 123, 39999], 4, 4, 32, 64, 40000 // 16 * 16 + 16, 0, "bf16", seed=5)
    _check_bounds(x, 16)


def test_bounds_of_infinities_and_nans():
    x = Cache([64, 40], 2, 2, 32, 64, 64, 0, "bf16", seed=1)
    x.c.k[0, 0, 3, 5] = float("inf")
    x.c.k[0, 0, 4, 6] = float("-inf")
    x.c.k[0, 1, 20, 7] = float("nan")
    x.c.k[1, 1, 39, 0] = float("nan")
    box = _check_bounds(x, 32)
    assert box[0, 0, 0, 1, 5] == math.inf and box[0, 0, 0, 0, 6] == -math.inf
    assert box[0, 1, 0, 0, 7] == -math.inf and box[0, 1, 0, 1, 7] == math.inf
    q = Cache([64], 1, 1, 32, 64, 64, 0, "int8", seed=2)
    q.c.k_scale[0, 0, 9] = float("nan")
    q.c.k_scale[0, 0, 40] = 3e38                # products beyond the largest number
    _check_bounds(q, 32)


def test_bounds_more_new_blocks_than_said():
    """Only as many blocks as max_new can touch are bounded, and the word is set."""
    x = Cache([256], 1, 1, 32, 64, 256, 0, "bf16", seed=3)
    box = tb.block_bounds(x.c, 32)
    tb.tk_block_bounds(x.c, box, x.seq, i32([0]), 33, 32)
    assert tb.tk_get_device_error() == 1
    at, ref = _ref_bounds(x, 32)
    got = f64(box).reshape(-1, 2, 32)
    assert np.array_equal(got[:2], ref[:2]) and (got[2:] == 0).all()


def test_bounds_bad_pages_and_lengths():
    x = Cache([60, 64], 2, 2, 32, 64, 64, 16, "bf16", seed=4)
    x.c.page_table[0, 1] = 99
    x.c.page_table[1, 0] = -5
    box = tb.block_bounds(x.c)
    box.fill_(7.0)
    tb.tk_block_bounds(x.c, box, x.seq)
    assert tb.tk_get_device_error() == 1
    want = np.full((box.shape[0] * 2, 2, 32), 7.0)
    at, ref = _ref_bounds(x, 16)
    bad = np.zeros(len(at), dtype=bool)
    for b, blk in ((0, 1), (1, 0)):
        for g in range(2):
            bad |= at == x.rows(b, g)[::16][blk] // 16
    want[at[~bad]] = ref[~bad]
    assert np.array_equal(f64(box).reshape(want.shape), want)
    for lens in ([-3, 64], [2**30, 64]):
        y = Cache([64, 64], 2, 2, 32, 64, 64, 0, "bf16", seed=4)
        tb.tk_block_bounds(y.c, tb.block_bounds(y.c, 16), i32(lens), block=16)
        assert tb.tk_get_device_error() == 1


# ------------------------------------------------------------------------------------ choice

def _boxes(n_rows, r, seed, spread=1.0):
    g = torch.Generator().manual_seed(seed)
    mid, half = spread * torch.randn(n_rows, r, generator=g), 0.5 + torch.rand(n_rows, r, generator=g)
    return torch.stack([mid - half, mid + half], 1).to(torch.bfloat16)


def _check_select(x, block, box, q, n, first=1, last=1, max_len=None, ids=True, stream=None):
    sel = tb.BlockSelection.allocate(x.c, n, block, ids=ids)
    tb.tk_block_select(x.c, q, box.view(tb._bounds_shape(x.c, block)), x.seq, max(x.lens) if max_len is None else max_len,
                       sel, first, last, stream=stream)
    torch.cuda.synchronize()
    flat, qq = f64(box).reshape(-1, 2, x.r), f64(q)
    G = x.h_q // x.h_kv
    table, lens = sel.table.cpu().numpy().reshape(x.B, x.h_kv, n), sel.lens.cpu().numpy().reshape(x.B, x.h_kv)
    for b in range(x.B):
        for g in range(x.h_kv):
            rows = x.rows(b, g)[::block] // block
            pick = lc.block_select(lc.block_scores(qq[b, g * G:(g + 1) * G], flat[rows, 0], flat[rows, 1]), n, first, last)
            pick = pick.astype(np.int64)
            pad = np.full(n - len(pick), -1)
            assert np.array_equal(table[b, g], np.concatenate([rows[pick] if len(pick) else pick, pad])), (b, g)
            if ids:
                assert np.array_equal(sel.ids[b, g].cpu().numpy(), np.concatenate([pick, pad]))
            L = x.lens[b]
            tail = 0 if L == 0 else L - (len(rows) - 1) * block
            assert lens[b, g] == (0 if L == 0 else (len(pick) - 1) * block + tail)
    return sel


def _queries(B, hq, r, seed):
    return torch.randn(B, hq, r, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).cuda()


@pytest.mark.parametrize("r,G,block,ps,n,first,last", [
    (16, 1, 16, 0, 3, 1, 1), (32, 4, 64, 64, 5, 1, 1), (64, 8, 32, 32, 9, 0, 2), (128, 2, 16, 16, 16, 3, 1),
    (32, 4, 16, 0, 1, 0, 1), (16, 8, 128, 128, 4, 2, 2), (128, 8, 64, 0, 200, 1, 1)])
def test_select(r, G, block, ps, n, first, last):
    lens = [0, 1, block, n * block, n * block + 1, 40 * block - 7, 40 * block]
    lens = [min(L, 40 * block) for L in lens]
    x = Cache(lens, 2 * G, 2, r, 64, 40 * block, ps, "bf16", seed=r + G)
    box = _boxes(x.rows_total // block, r, r + n).cuda()
    _check_select(x, block, box, _queries(x.B, x.h_q, r, n), n, first, last)


def test_select_long_contexts_and_clusters():
    """From 400 to 24576 blocks: one to eight blocks of threads for each kv head."""
    for blocks, batch, n in ((400, 3, 17), (1000, 2, 64), (5000, 1, 500), (24576, 1, 1000)):
        x = Cache([blocks * 16 - 5] + [blocks * 8] * (batch - 1), 4, 2, 16, 64, blocks * 16, 16, "bf16", seed=blocks)
        _check_select(x, 16, _boxes(x.rows_total // 16, 16, blocks).cuda(), _queries(batch, 4, 16, 3), n)


def test_select_equal_scores_take_the_lower_block():
    x = Cache([40 * 16] * 3, 4, 2, 32, 64, 40 * 16, 0, "bf16", seed=9)
    one = _boxes(1, 32, 4)
    box = one.expand(x.rows_total // 16, 2, 32).clone().cuda()            # every block the same
    _check_select(x, 16, box, _queries(3, 4, 32, 1), 7)
    box = _boxes(4, 32, 5)[torch.arange(x.rows_total // 16) % 4].cuda()   # four kinds of blocks
    _check_select(x, 16, box, _queries(3, 4, 32, 2), 13)
    _check_select(x, 16, _boxes(x.rows_total // 16, 32, 6).cuda(), torch.zeros(3, 4, 32, dtype=torch.bfloat16).cuda(), 5)
    _check_select(x, 16, torch.zeros_like(box), _queries(3, 4, 32, 2), 5)
    _check_select(x, 16, torch.full_like(box, 1e-39), _queries(3, 4, 32, 2), 5)


def test_select_decides_in_64_bits():
    """Scores that differ by 2^-40 of their size, in an order that 32 bits cannot see, many at the
    border; and few at it."""
    blocks, r = 64, 32
    x = Cache([blocks * 16], 1, 1, r, 64, blocks * 16, 0, "bf16", seed=11)
    q = torch.ones(1, 1, r, dtype=torch.bfloat16).cuda()
    for few in (False, True):
        box = torch.zeros(blocks, 2, r)
        box[:, :, 0] = 1024.0
        box[:, :, 1] = -1024.0 if few else 512.0
        box[:, 1, 2] = torch.randperm(blocks, generator=torch.Generator().manual_seed(3)).float() * 2.0 ** -30
        box[:, 0, 2] = box[:, 1, 2]
        if few:
            box[torch.arange(blocks) % 5 != 0, 1, 3] = 40.0
            box[7, 1, 3] = 0.0
        _check_select(x, 16, box.to(torch.bfloat16).cuda(), q, 20)


def test_select_infinities_and_nans():
    x = Cache([30 * 16, 25 * 16 + 3], 4, 2, 32, 64, 30 * 16, 0, "bf16", seed=12)
    box = _boxes(x.rows_total // 16, 32, 7)
    box[5, 0, 3] = float("-inf")
    box[9, 1, 3] = float("nan")
    box[40, 1, 0] = float("inf")
    box[77, 0, 31] = float("inf")
    _check_select(x, 16, box.cuda(), _queries(2, 4, 32, 8), 6)
    q = _queries(2, 4, 32, 9)
    q[0, 1, 4], q[1, 2, 0], q[1, 3, 1] = float("nan"), float("inf"), float("-inf")
    _check_select(x, 16, _boxes(x.rows_total // 16, 32, 8).cuda(), q, 6)
    # finite operands whose 32-bit products overflow
    _check_select(x, 16, (_boxes(x.rows_total // 16, 32, 9).float() * 1e38).to(torch.bfloat16).cuda(),
                  (_queries(2, 4, 32, 10).float() * 1e30).to(torch.bfloat16), 6)


def test_select_clamps_lengths_to_the_bound():
    x = Cache([20 * 16, 20 * 16], 2, 2, 32, 64, 20 * 16, 0, "bf16", seed=13)
    box = _boxes(x.rows_total // 16, 32, 9).cuda()
    x.seq = i32([-1, 999999])
    x.lens = [0, 10 * 16 + 4]
    _check_select(x, 16, box, _queries(2, 2, 32, 1), 4, max_len=10 * 16 + 4)
    assert tb.tk_get_device_error() == 1
    y = Cache([64], 2, 2, 32, 64, 64, 16, "bf16", seed=14)
    y.c.page_table[0, 2] = 1000
    sel = tb.BlockSelection.allocate(y.c, 2)
    tb.tk_block_select(y.c, _queries(1, 2, 32, 1), tb.block_bounds(y.c), y.seq, 64, sel)
    assert tb.tk_get_device_error() == 1
    assert sel.table.min() >= 0 and sel.table.max() < y.c.desc.num_pages * 2


# ------------------------------------------------------------------------------------ decode

def _ref_decode(x, q, pick, block):
    keys, vals = x.keys64(), x.values()
    G = x.h_q // x.h_kv
    out = np.zeros((x.B, x.h_q, x.d_v))
    for b in range(x.B):
        for g in range(x.h_kv):
            t = np.concatenate([np.arange(i * block, min((i + 1) * block, x.lens[b])) for i in pick[b][g]]) \
                if len(pick[b][g]) else np.zeros(0, dtype=int)
            if len(t):
                rows = x.rows(b, g)[t]
                out[b, g * G:(g + 1) * G] = oa.attention_head(q[b, g * G:(g + 1) * G], keys[rows], vals[rows],
                                                              1 / math.sqrt(x.r))
    return out


@pytest.mark.parametrize("k,r,dv,G,block,ps,out", [
    ("bf16", 16, 64, 1, 16, 0, "f32"), ("bf16", 32, 128, 4, 64, 64, "bf16"), ("int8", 64, 64, 8, 32, 32, "f32"),
    ("int4", 32, 128, 2, 128, 0, "f32"), ("bf16", 128, 128, 8, 256, 256, "bf16"), ("int8", 16, 128, 4, 16, 16, "f32")])
def test_bounds_choice_and_decode(k, r, dv, G, block, ps, out):
    """The three calls of a step, and the oracle's three steps on the same cache."""
    n = 6
    lens = [0, 1, block + 1, n * block, 30 * block - 9, 30 * block]
    x = Cache(lens, 3 * G, 3, r, dv, 30 * block, ps, k, seed=r + dv)
    box = tb.block_bounds(x.c, block)
    tb.tk_block_bounds(x.c, box, x.seq, block=block)
    q = _queries(x.B, x.h_q, r, 5)
    sel = _check_select(x, block, box, q, n)
    o = torch.full((x.B, x.h_q, dv), 9.0, device="cuda", dtype=torch.float32 if out == "f32" else torch.bfloat16)
    tb.tk_attn_decode_blocks(x.c, q, sel, o, tb.decode_blocks_workspace(x.c, sel))
    pick = [[[i for i in sel.ids[b, g].tolist() if i >= 0] for g in range(3)] for b in range(x.B)]
    (parity if out == "f32" else parity_bf16)(f64(o), _ref_decode(x, f64(q), pick, block))
    assert (f64(o)[0] == 0).all()


def test_decode_over_all_blocks_is_the_plain_decode():
    x = Cache([1000, 333, 64], 8, 2, 32, 128, 1024, 0, "bf16", seed=21)
    q = _queries(3, 8, 32, 6)
    sel = tb.BlockSelection.allocate(x.c, 16, 64)
    tb.tk_block_select(x.c, q, tb.block_bounds(x.c, 64), x.seq, 1024, sel)
    a, b = torch.empty(3, 8, 128, device="cuda"), torch.empty(3, 8, 128, device="cuda")
    tb.tk_attn_decode_blocks(x.c, q, sel, a, tb.decode_blocks_workspace(x.c, sel))
    tb.tk_attn_decode(x.c, q, x.seq, 1024, b, tb.decode_workspace(x.c.desc, 1024))
    parity(f64(a), f64(b))


def test_decode_with_a_table_of_the_callers_own():
    """Blocks in any order, the same block twice, a partly filled one at the end; a bad entry."""
    x = Cache([320], 2, 1, 32, 64, 320, 0, "bf16", seed=22)
    sel = tb.BlockSelection(32, i32([[7, 2, 2, 9]]), i32([3 * 32 + 5]))
    q, o = _queries(1, 2, 32, 7), torch.empty(1, 2, 64, device="cuda")
    ws = tb.decode_blocks_workspace(x.c, sel)
    tb.tk_attn_decode_blocks(x.c, q, sel, o, ws)
    rows = np.concatenate([np.arange(224, 256), np.arange(64, 96), np.arange(64, 96), np.arange(288, 293)])
    ref = oa.attention_head(f64(q)[0], x.keys64()[rows], x.values()[rows], 1 / math.sqrt(32))
    parity(f64(o)[0], ref)
    sel.table[0, 2] = 10           # begins the second 64 tokens
    tb.tk_attn_decode_blocks(x.c, q, sel, o, ws)
    assert tb.tk_get_device_error() == 1


def test_decode_of_more_sequences_than_one_launch_takes():
    """1024 / h_kv sequences a launch: 300 sequences of 4 kv heads are two."""
    B = 300
    x = Cache([(37 * b) % 160 for b in range(B)], 4, 4, 16, 64, 160, 0, "bf16", seed=23)
    q = _queries(B, 4, 16, 8)
    box = tb.block_bounds(x.c, 16)
    tb.tk_block_bounds(x.c, box, x.seq, block=16)
    sel = tb.BlockSelection.allocate(x.c, 3, 16, ids=True)
    tb.tk_block_select(x.c, q, box, x.seq, 160, sel)
    o, ws = torch.empty(B, 4, 64, device="cuda"), tb.decode_blocks_workspace(x.c, sel)
    for _ in range(2):
        tb.tk_attn_decode_blocks(x.c, q, sel, o, ws)
    ids = sel.ids.tolist()
    pick = [[[i for i in ids[b][g] if i >= 0] for g in range(4)] for b in range(B)]
    parity(f64(o), _ref_decode(x, f64(q), pick, 16))


def test_a_step_in_a_graph_and_on_another_stream():
    """Prepared calls, recorded and replayed with other lengths and queries, equal direct ones."""
    x = Cache([600, 1000], 8, 2, 32, 128, 1024, 64, "int8", seed=24)
    s = torch.cuda.Stream()
    box, q = tb.block_bounds(x.c), _queries(2, 8, 32, 9)
    sel, o = tb.BlockSelection.allocate(x.c, 5), torch.empty(2, 8, 128, device="cuda")
    old = torch.zeros(2, dtype=torch.int32, device="cuda")
    ws = tb.decode_blocks_workspace(x.c, sel)
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        calls = [tb.prepare_block_bounds(x.c, box, x.seq, old, stream=s, graph=True),
                 tb.prepare_block_select(x.c, q, box, x.seq, 1024, sel, stream=s, graph=True),
                 tb.prepare_attn_decode_blocks(x.c, q, sel, o, ws, stream=s, graph=True)]
    for lens in ([600, 1000], [100, 17], [320, 321]):
        with torch.cuda.stream(s):
            x.seq.copy_(i32(lens))
            q.copy_(_queries(2, 8, 32, lens[0]))
            for c in calls:
                c()
        s.synchronize()
        box2, sel2, o2 = tb.block_bounds(x.c), tb.BlockSelection.allocate(x.c, 5), torch.empty_like(o)
        box2.copy_(box)
        tb.tk_block_bounds(x.c, box2, x.seq)
        tb.tk_block_select(x.c, q, box2, x.seq, 1024, sel2)
        tb.tk_attn_decode_blocks(x.c, q, sel2, o2, tb.decode_blocks_workspace(x.c, sel2))
        torch.cuda.synchronize()
        assert torch.equal(bits(box), bits(box2)) and torch.equal(sel.table, sel2.table) and torch.equal(sel.lens, sel2.lens)
        assert torch.equal(bits(o), bits(o2))


def test_workspace_is_checked():
    x = Cache([64], 2, 1, 32, 64, 64, 0, "bf16", seed=25)
    sel = tb.BlockSelection.allocate(x.c, 2, 32)
    q, o = _queries(1, 2, 32, 1), torch.empty(1, 2, 64, device="cuda")
    with pytest.raises(tb.TkError, match="TK_ERR_WORKSPACE"):
        tb.tk_attn_decode_blocks(x.c, q, sel, o, torch.zeros(256, dtype=torch.uint8, device="cuda"))
