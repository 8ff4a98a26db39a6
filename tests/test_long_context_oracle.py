"""The oracle of the operators over a long context against closed forms, and what the entry points
refuse (checked on the host, before anything is launched)."""

import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import long_context as lc
from paper_2603_04427_gb300 import binding as tb
from paper_2603_04427_gb300 import build as tbuild


@pytest.fixture(scope="module")
def lib():
    tbuild.build()
    return tb.load_library()


# ------------------------------------------------------------------------------ oracle pins

def test_bf16_outward():
    x = np.array([1.0, 1.0 + 2 ** -9, -1.0 - 2 ** -9, 0.0, 2.0 ** -133, 1.5 * 2.0 ** -133, np.inf, -np.inf, 3.4e38])
    up, down = lc.bf16_outward(x, True), lc.bf16_outward(x, False)
    assert list(up[:6]) == [1.0, 1.0 + 2 ** -7, -1.0, 0.0, 2.0 ** -133, 2.0 ** -132]
    assert list(down[:6]) == [1.0, 1.0, -1.0 - 2 ** -7, 0.0, 2.0 ** -133, 2.0 ** -133]
    assert up[6] == np.inf and down[7] == -np.inf and up[8] == np.inf
    assert down[8] == (2 - 2.0 ** -7) * 2.0 ** 127
    r = np.random.default_rng(0).standard_normal(1000) * 10.0 ** np.random.default_rng(1).uniform(-30, 30, 1000)
    up, down = lc.bf16_outward(r, True), lc.bf16_outward(r, False)
    assert (down <= r).all() and (r <= up).all()
    t = torch.from_numpy(up).to(torch.bfloat16).double().numpy()
    assert (t == up).all()


def test_score_bounds_every_key():
    rng = np.random.default_rng(2)
    k, q = rng.standard_normal((100, 16)), rng.standard_normal((4, 16))
    lo, hi = lc.block_bounds(k, 32)
    s = lc.block_scores(q, lo, hi)
    assert len(s) == 4
    for j in range(4):
        assert s[j] >= (k[32 * j:32 * j + 32] @ q.T).max()
    # one key a block: the bound is the score
    lo, hi = lc.block_bounds(k, 1)
    assert np.allclose(lc.block_scores(q, lo, hi), (k @ q.T).max(1))


def test_select_ties_and_forced():
    s = np.array([1.0, 5.0, 5.0, 5.0, 0.0, 7.0, 2.0])
    assert list(lc.block_select(s, 4, 1, 1)) == [0, 1, 5, 6]
    assert list(lc.block_select(s, 3, 0, 1)) == [1, 5, 6]
    assert list(lc.block_select(s, 7, 1, 1)) == list(range(7))
    assert list(lc.block_select(s, 2, 1, 1)) == [0, 6]


def test_weights_sum_to_the_number_of_queries():
    rng = np.random.default_rng(3)
    w = lc.attn_weights(rng.standard_normal((4, 3, 16)), rng.standard_normal((50, 16)), 0.25, 3)
    assert math.isclose(w.sum(), 12.0)
    w = lc.attn_weights(np.zeros((1, 5, 8)), np.ones((2, 8)), 1.0, 5)     # three queries before the start
    assert np.allclose(w, [1.5, 0.5])


def test_evict_order():
    w = np.array([3.0, 0.0, 2.0, np.nan, 9.0, 1.0, 4.0, 0.5])
    # the last two stay; of the first six the three largest: 4, 0, 2
    assert list(lc.evict(w, 5, 2)) == [0, 4, 2, 6, 7]
    assert list(lc.evict(w, 8, 2)) == list(range(8))
    assert list(lc.evict(np.ones(6), 3, 0)) == [0, 1, 2]
    assert list(lc.evict(w, 3, 3)) == [5, 6, 7]


# --------------------------------------------------------------------------------- refusals

FAKE = ctypes.c_void_p(0x10000)
ODD16, ODD4 = ctypes.c_void_p(0x10008), ctypes.c_void_p(0x10002)
INV, UNS, WS = tb.TK_ERR_INVALID_ARG, tb.TK_ERR_UNSUPPORTED, tb.TK_ERR_WORKSPACE


def _desc(**kw):
    d = dict(batch=2, h_q=8, h_kv=2, r=32, d_v=128, capacity=256, page_size=0, num_pages=0,
             max_pages_per_seq=0, k_dtype=tb.TK_BF16)
    d.update(kw)
    return tb.tk_cache_desc(**d)


PAGED = dict(capacity=0, page_size=64, num_pages=8, max_pages_per_seq=4)


def _call(fn, order, base, kw):
    a = dict(base, **kw)
    d = a.pop("desc", _desc())
    return fn(ctypes.byref(d), *(a[n] for n in order))


BOUNDS = ["block", "k", "ks", "pt", "old", "seq", "max_new", "bounds", "stream"]
BOUNDS0 = dict(block=64, k=FAKE, ks=None, pt=None, old=None, seq=FAKE, max_new=1, bounds=FAKE, stream=None)


@pytest.mark.parametrize("kw,status,msg", [
    (dict(desc=_desc(r=48)), UNS, "r=48"),
    (dict(block=48), UNS, "block=48"), (dict(block=8), UNS, "block=8"), (dict(block=512), UNS, "block=512"),
    (dict(desc=_desc(**PAGED), pt=FAKE, block=32), INV, "page size"),
    (dict(desc=_desc(capacity=80)), INV, "multiple of block"),
    (dict(max_new=-1), INV, "max_new"), (dict(k=None), INV, "k_cache"), (dict(seq=None), INV, "seq_lens"),
    (dict(bounds=None), INV, "bounds"), (dict(bounds=ODD16), INV, "aligned"), (dict(seq=ODD4), INV, "aligned"),
    (dict(old=ODD4), INV, "aligned"), (dict(desc=_desc(k_dtype=tb.TK_I8)), INV, "k_scale"),
    (dict(desc=_desc(**PAGED)), INV, "page_table"),
    (dict(max_new=0, k=None, seq=None), tb.TK_OK, ""), (dict(desc=_desc(batch=0), k=None), tb.TK_OK, ""),
])
def test_block_bounds_refusals(lib, kw, status, msg):
    assert _call(lib.tk_block_bounds, BOUNDS, BOUNDS0, kw) == status
    assert status == tb.TK_OK or msg in tb.tk_last_error()


SELECT = ["block", "q", "bounds", "pt", "seq", "max_len", "n", "first", "last", "table", "lens", "ids", "stream"]
SELECT0 = dict(block=64, q=FAKE, bounds=FAKE, pt=None, seq=FAKE, max_len=256, n=4, first=1, last=1, table=FAKE,
               lens=FAKE, ids=None, stream=None)


@pytest.mark.parametrize("kw,status,msg", [
    (dict(n=0, first=0), INV, "n_select"), (dict(first=-1), INV, "n_first"), (dict(last=0), INV, "n_last"),
    (dict(n=3, first=2, last=2), INV, "n_first + n_last"), (dict(first=2**31 - 1, last=2**31 - 1), INV, "n_first"),
    (dict(n=2**23), INV, "n_select"), (dict(max_len=-1), INV, "max_seq_len"), (dict(q=None), INV, "q /"),
    (dict(bounds=ODD16), INV, "aligned"), (dict(table=ODD4), INV, "aligned"), (dict(lens=None), INV, "lens"),
    (dict(block=24), UNS, "block=24"), (dict(desc=_desc(**PAGED)), INV, "page_table"),
    (dict(desc=_desc(capacity=2**20), block=16, max_len=2**20), UNS, "blocks"),
    (dict(desc=_desc(batch=0), q=None), tb.TK_OK, ""),
])
def test_block_select_refusals(lib, kw, status, msg):
    assert _call(lib.tk_block_select, SELECT, SELECT0, kw) == status
    assert status == tb.TK_OK or msg in tb.tk_last_error()


DECODE = ["block", "q", "k", "v", "ks", "table", "lens", "n", "out", "out_dtype", "scale", "ws", "bytes", "stream"]
DECODE0 = dict(block=64, q=FAKE, k=FAKE, v=FAKE, ks=None, table=FAKE, lens=FAKE, n=4, out=FAKE,
               out_dtype=tb.TK_F32, scale=0.1, ws=FAKE, bytes=1 << 30, stream=None)


@pytest.mark.parametrize("kw,status,msg", [
    (dict(n=0), INV, "n_select"), (dict(n=2**23), INV, "n_select"), (dict(block=7), UNS, "block"),
    (dict(out_dtype=5), UNS, "out_dtype"), (dict(scale=float("nan")), INV, "scale"), (dict(q=None), INV, "q /"),
    (dict(table=None), INV, "table"), (dict(lens=ODD4), INV, "aligned"), (dict(q=ODD16), INV, "aligned"),
    (dict(k=None), INV, "k_cache"), (dict(desc=_desc(h_q=2048, h_kv=2048)), UNS, "h_kv"),
    (dict(desc=_desc(k_dtype=tb.TK_I4)), INV, "k_scale"), (dict(desc=_desc(batch=0), q=None), tb.TK_OK, ""),
    (dict(desc=_desc(batch=4096, capacity=2**20)), UNS, "rows"),
])
def test_attn_decode_blocks_refusals(lib, kw, status, msg):
    assert _call(lib.tk_attn_decode_blocks, DECODE, DECODE0, kw) == status
    assert status == tb.TK_OK or msg in tb.tk_last_error()
    assert lib.tk_decode_blocks_workspace_size(ctypes.byref(_desc()), 64, 0) == 0
    assert lib.tk_decode_blocks_workspace_size(ctypes.byref(_desc()), 48, 4) == 0


WEIGHTS = ["q", "n_q", "k", "ks", "pt", "old", "seq", "max_len", "scale", "decay", "w", "ws", "bytes", "stream"]
WEIGHTS0 = dict(q=FAKE, n_q=1, k=FAKE, ks=None, pt=None, old=None, seq=FAKE, max_len=256, scale=0.1, decay=1.0,
                w=FAKE, ws=FAKE, bytes=1 << 30, stream=None)


@pytest.mark.parametrize("kw,status,msg", [
    (dict(scale=float("inf")), INV, "scale"), (dict(decay=float("nan")), INV, "decay"), (dict(n_q=0), INV, "n_q"),
    (dict(max_len=-1), INV, "max_seq_len"), (dict(k=None), INV, "k_cache"), (dict(w=None), INV, "weights"),
    (dict(w=ODD16), INV, "aligned"), (dict(old=ODD4), INV, "aligned"), (dict(n_q=129), UNS, "n_q"),
    (dict(desc=_desc(k_dtype=tb.TK_I8)), INV, "k_scale"), (dict(desc=_desc(**PAGED)), INV, "page_table"),
    (dict(desc=_desc(batch=0), q=None), tb.TK_OK, ""),
])
def test_attn_weights_refusals(lib, kw, status, msg):
    assert _call(lib.tk_attn_weights, WEIGHTS, WEIGHTS0, kw) == status
    assert status == tb.TK_OK or msg in tb.tk_last_error()


EVICT = ["k", "v", "ks", "pt", "seq", "max_len", "w", "keep", "recent", "w_out", "seq_out", "kept", "free", "count",
         "ws", "bytes", "stream"]
EVICT0 = dict(k=FAKE, v=FAKE, ks=None, pt=None, seq=FAKE, max_len=256, w=FAKE, keep=64, recent=16, w_out=FAKE,
              seq_out=FAKE, kept=None, free=None, count=None, ws=FAKE, bytes=1 << 30, stream=None)


@pytest.mark.parametrize("kw,status,msg", [
    (dict(keep=0, recent=0), INV, "n_keep"), (dict(keep=2**27), INV, "n_keep"), (dict(recent=-1), INV, "n_recent"),
    (dict(recent=65), INV, "n_recent"), (dict(max_len=-1), INV, "max_seq_len"), (dict(v=None), INV, "v_cache"),
    (dict(w_out=None), INV, "weights_out"), (dict(seq_out=None), INV, "seq_lens_out"), (dict(w=ODD16), INV, "aligned"),
    (dict(kept=ODD4), INV, "aligned"), (dict(free=FAKE), INV, "free_count"),
    (dict(free=FAKE, count=FAKE), INV, "contiguous"), (dict(ws=None), WS, "workspace"),
    (dict(ws=ODD16), WS, "workspace"), (dict(bytes=100), WS, "needed"),
    (dict(desc=_desc(**PAGED)), INV, "page_table"), (dict(desc=_desc(batch=0), k=None), tb.TK_OK, ""),
])
def test_cache_evict_refusals(lib, kw, status, msg):
    assert _call(lib.tk_cache_evict, EVICT, EVICT0, kw) == status
    assert status == tb.TK_OK or msg in tb.tk_last_error()
    assert lib.tk_cache_evict_workspace_size(ctypes.byref(_desc()), 0) == 0
    assert lib.tk_cache_evict_workspace_size(ctypes.byref(_desc()), 64) >= 4 * 64 * 2 * 4


def test_binding_refuses_host_tensors_and_wrong_shapes():
    cache = tb.ThinKeyCache.allocate(2, 4, 2, 32, 64, capacity=128, device="cpu")
    box = tb.block_bounds(cache, 32)
    assert box.shape == (2, 2, 4, 2, 32)
    assert tb.slot_weights(cache).shape == (2, 2, 128)
    lens = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        tb.tk_block_bounds(cache, box, lens, block=32)
    with pytest.raises(ValueError, match="CUDA"):
        tb.tk_attn_weights(cache, torch.zeros(2, 4, 32, dtype=torch.bfloat16), lens, 128, tb.slot_weights(cache), lens)
    with pytest.raises(ValueError, match="CUDA"):
        tb.tk_cache_evict(cache, lens, 128, tb.slot_weights(cache), 64, 8, lens)
    for block in (8, 48, 256):
        with pytest.raises(ValueError, match="block"):
            tb.block_bounds(cache, block)
    sel = tb.BlockSelection.allocate(cache, 3, block=32, ids=True)
    assert sel.table.shape == (4, 3) and sel.ids.shape == (2, 2, 3)
    paged = tb.ThinKeyCache.allocate(2, 4, 2, 32, 64, page_size=16, num_pages=5,
                                     page_table=torch.zeros(2, 2), device="cpu")
    assert tb.block_bounds(paged).shape == (5, 2, 2, 32)
    with pytest.raises(ValueError, match="block"):
        tb.block_bounds(paged, 32)
