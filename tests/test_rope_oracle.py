"""Pins of oracle/rope.py and the host side of the norm + rotation and page-table entry points."""

import ctypes
import math

import numpy as np
import pytest

from oracle import rope
from paper_2603_04427_gb300 import binding as tb
from paper_2603_04427_gb300 import build as tbuild


@pytest.fixture(scope="module")
def lib():
    tbuild.build()
    return tb.load_library()


def test_rotation_is_a_complex_product():
    rng = np.random.default_rng(0)
    y = rng.standard_normal((2, 3, 5, 16))
    theta = rng.uniform(-4, 4, (2, 5, 4))
    got = rope.rotate(y, theta, 8, "pair")
    z = (y[..., 0:8:2] + 1j * y[..., 1:8:2]) * np.exp(1j * theta)[:, None]
    assert np.allclose(got[..., 0:8:2] + 1j * got[..., 1:8:2], z, atol=1e-14)
    assert np.array_equal(got[..., 8:], y[..., 8:])
    half = rope.rotate(y, theta, 8, "half")
    z = (y[..., :4] + 1j * y[..., 4:8]) * np.exp(1j * theta)[:, None]
    assert np.allclose(half[..., :4] + 1j * half[..., 4:8], z, atol=1e-14)


def test_rotated_scores_depend_on_the_distance_alone():
    rng = np.random.default_rng(1)
    f, ax = [1.0, 0.1, 0.01, 0.001], [0] * 4
    q, k = rng.standard_normal((2, 1, 1, 1, 8))
    score = [float((rope.rotate(q, rope.angles([[[i + 7]]], f, ax), 8, "half")
                    * rope.rotate(k, rope.angles([[[i]]], f, ax), 8, "half")).sum()) for i in (0, 3, 100)]
    assert np.allclose(score, score[0], atol=1e-12)


@pytest.mark.parametrize("layout", ["half", "pair"])
@pytest.mark.parametrize("norm", [True, False])
def test_oracle_gradient_against_differences(layout, norm):
    rng = np.random.default_rng(2)
    x = rng.standard_normal((2, 2, 3, 16))
    w = 1 + 0.3 * rng.standard_normal(16)
    theta = rng.uniform(-3, 3, (2, 3, 4))
    dy = rng.standard_normal(x.shape)
    f = lambda x, w: float((rope.norm_rope(x, w, theta, 8, layout, norm, 1e-3) * dy).sum())  # noqa: E731
    dx, dw, _, _ = rope.norm_rope_backward(x, w, dy, theta, 8, layout, norm, 1e-3)
    h = 1e-5
    for idx in [(0, 0, 0, 0), (1, 1, 2, 5), (0, 1, 1, 12), (1, 0, 0, 15)]:
        e = np.zeros_like(x)
        e[idx] = h
        assert abs((f(x + e, w) - f(x - e, w)) / (2 * h) - dx[idx]) < 1e-8
    if norm:
        for i in (0, 7, 9):
            e = np.zeros_like(w)
            e[i] = h
            assert abs((f(x, w + e) - f(x, w - e)) / (2 * h) - dw[i]) < 1e-8


def test_block_table_oracle_by_hand():
    """Two sequences share a pool of 4 pages of 16; one finishes, its page is popped first."""
    table = np.array([[2, -1, -1], [0, -1, -1], [-1, -1, -1]])
    got = rope.block_tables([5, 16, 0], [-1, 1, 40], table, np.array([1, 3, 0, 0]), 2, 16, 41, 0)
    # stack after the push: 1 3 2; sequence 1 pops 2, sequence 2 needs 3 pages of the 2 left
    assert got["page_table"].tolist() == [[2, -1, -1], [0, 2, -1], [-1, -1, -1]]
    assert got["free_count"] == 2 and got["free_pages"][:2].tolist() == [1, 3]
    assert got["seq_lens"].tolist() == [0, 17, 0] and got["refused"] == 1
    assert got["offsets"].tolist() == [0, 0, 1, 1]
    assert got["slots"][:2].tolist() == [32, -1] and got["positions"][:2].tolist() == [16, 0]


def test_rope_plan():
    p = tb.rope_plan(32, rot_dim=16, axes=(4, 2, 2), layout="pair", base=100.0, w_offset=1.0)
    assert (p.r, p.rot_dim, p.layout, p.n_axes, p.norm, p.w_offset) == (32, 16, 1, 3, 1, 1.0)
    assert list(p.pair_axis[:8]) == [0, 0, 0, 0, 1, 1, 2, 2]
    assert np.allclose(p.inv_freq[:8], [1, 100 ** -0.25, 0.1, 100 ** -0.75, 1, 0.1, 1, 0.1])
    assert tb.rope_plan(64).n_axes == 1 and tb.rope_plan(64).inv_freq[31] == pytest.approx(10000 ** (-31 / 32))
    with pytest.raises(ValueError):
        tb.rope_plan(32, axes=(4, 4))
    with pytest.raises(ValueError):
        tb.rope_plan(32, layout="diagonal")
    with pytest.raises(ValueError):
        tb.rope_plan(32, inv_freq=[1.0] * 15)
    with pytest.raises(ValueError):
        tb.rope_plan(32, pair_axis=[4] * 16)


FAKE = 0x10000  # never dereferenced: validation fails first


def _h(n=4, dtype=tb.TK_BF16, sb=65536, st=1024, sh=32, data=FAKE):
    return tb.tk_heads(data, n, dtype, sb, st, sh)


def _plan(**kw):
    p = tb.rope_plan(32)
    for k, v in kw.items():
        if k in ("inv_freq", "pair_axis"):
            getattr(p, k)[3] = v
        else:
            setattr(p, k, v)
    return p


def _forward(lib, plan=None, q=None, qo=None, k=None, ko=None, v=None, vo=None, batch=2, seq=3, dv=128,
             wq=None, w_dtype=tb.TK_F32, pos=FAKE, sa=0, sb=3):
    r = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
    plan = tb.rope_plan(32) if plan is None else plan
    q = _h() if q is None else q
    qo = _h(data=0x20000) if qo is None else qo
    return lib.tk_qk_norm_rope(ctypes.byref(plan), batch, seq, dv, r(q), r(k), r(v), wq, None, w_dtype, pos,
                               sa, sb, r(qo), r(ko), r(vo), None)


@pytest.mark.parametrize("kw,status,msg", [
    (dict(r=48), tb.TK_ERR_UNSUPPORTED, "r=48"),
    (dict(rot_dim=40), tb.TK_ERR_INVALID_ARG, "rot_dim"),
    (dict(rot_dim=-8), tb.TK_ERR_INVALID_ARG, "rot_dim"),
    (dict(rot_dim=12), tb.TK_ERR_UNSUPPORTED, "rot_dim"),
    (dict(layout=2), tb.TK_ERR_INVALID_ARG, "layout"),
    (dict(n_axes=0), tb.TK_ERR_INVALID_ARG, "n_axes"),
    (dict(n_axes=5), tb.TK_ERR_INVALID_ARG, "n_axes"),
    (dict(eps=0.0), tb.TK_ERR_INVALID_ARG, "eps"),
    (dict(eps=math.nan), tb.TK_ERR_INVALID_ARG, "eps"),
    (dict(w_offset=math.inf), tb.TK_ERR_INVALID_ARG, "w_offset"),
    (dict(inv_freq=math.nan), tb.TK_ERR_INVALID_ARG, "inv_freq[3]"),
    (dict(inv_freq=4.5), tb.TK_ERR_INVALID_ARG, "inv_freq[3]"),
    (dict(pair_axis=1), tb.TK_ERR_INVALID_ARG, "pair_axis[3]"),
])
def test_descriptor_refusals(lib, kw, status, msg):
    p = _plan(**kw)
    assert _forward(lib, plan=p) == status and msg in tb.tk_last_error()
    h, o = _h(), _h(data=0x20000)
    args = (None, None, tb.TK_F32, FAKE, 0, 3)
    assert lib.tk_qk_norm_rope_backward(ctypes.byref(p), 2, 3, 128, ctypes.byref(h), None, *args,
                                        ctypes.byref(h), None, None, ctypes.byref(o), None, None, None, None,
                                        None, 0, None) == status
    assert lib.tk_qk_norm_rope_workspace_size(ctypes.byref(p)) == 0


@pytest.mark.parametrize("kw,status,msg", [
    (dict(q=_h(data=None)), tb.TK_ERR_INVALID_ARG, "q: data is NULL"),
    (dict(q=_h(data=0x10008)), tb.TK_ERR_INVALID_ARG, "q must be 16-byte aligned"),
    (dict(q=_h(n=0), qo=_h(n=0)), tb.TK_ERR_INVALID_ARG, "n_heads"),
    (dict(q=_h(n=5)), tb.TK_ERR_INVALID_ARG, "heads"),
    (dict(q=_h(dtype=tb.TK_I8)), tb.TK_ERR_UNSUPPORTED, "dtype"),
    (dict(q=_h(st=1020)), tb.TK_ERR_INVALID_ARG, "stride"),
    (dict(q=_h(sh=-32)), tb.TK_ERR_INVALID_ARG, "stride"),
    (dict(q=_h(dtype=tb.TK_F32, st=1022)), tb.TK_ERR_INVALID_ARG, "stride"),
    (dict(qo=_h(sb=0)), tb.TK_ERR_INVALID_ARG, "overlap"),
    (dict(qo=_h(sh=24)), tb.TK_ERR_INVALID_ARG, "overlap"),
    (dict(qo=_h(st=96)), tb.TK_ERR_INVALID_ARG, "overlap"),
    (dict(k=_h()), tb.TK_ERR_INVALID_ARG, "k and its counterpart"),
    (dict(k=_h(dtype=tb.TK_F32), ko=_h(data=0x30000)), tb.TK_ERR_INVALID_ARG, "dtype"),
    (dict(k=_h(), ko=_h(dtype=tb.TK_F32, data=0x30000)), tb.TK_ERR_INVALID_ARG, "dtype"),
    (dict(v=_h(sh=128), vo=_h(sh=128), dv=96), tb.TK_ERR_UNSUPPORTED, "d_v"),
    (dict(pos=None), tb.TK_ERR_INVALID_ARG, "positions"),
    (dict(pos=0x10002), tb.TK_ERR_INVALID_ARG, "positions"),
    (dict(sb=-1), tb.TK_ERR_INVALID_ARG, "stride"),
    (dict(batch=-1), tb.TK_ERR_INVALID_ARG, "batch"),
    (dict(batch=1 << 16, seq=1 << 15), tb.TK_ERR_UNSUPPORTED, "2^31"),
    (dict(wq=0x10004), tb.TK_ERR_INVALID_ARG, "weights"),
    (dict(w_dtype=tb.TK_I8), tb.TK_ERR_UNSUPPORTED, "w_dtype"),
])
def test_forward_refusals(lib, kw, status, msg):
    assert _forward(lib, **kw) == status
    assert msg in tb.tk_last_error()


def test_empty_forward_and_strides_of_single_dimensions(lib):
    assert _forward(lib, batch=0) == tb.TK_OK
    assert _forward(lib, seq=0, pos=None) == tb.TK_OK
    # one head, one token, one sequence: their strides are not looked at (positions refuse the call later)
    odd = _h(n=1, sb=3, st=5, sh=7)
    assert _forward(lib, q=odd, qo=odd, batch=1, seq=1, pos=None) == tb.TK_ERR_INVALID_ARG
    assert "positions" in tb.tk_last_error()


def test_append_refusals(lib):
    r = ctypes.byref
    desc = tb.tk_cache_desc(2, 4, 2, 32, 128, 256, 0, 0, 0, tb.TK_BF16)
    plan = tb.rope_plan(32)
    q, k, v, o = _h(4), _h(2), _h(2, sh=128), _h(4, data=0x20000)

    def call(desc=desc, plan=plan, q=q, k=k, v=v, o=o, slots=FAKE, kc=FAKE, ks=None):
        ref = lambda x: None if x is None else r(x)  # noqa: E731
        return lib.tk_qk_norm_rope_append(r(desc), r(plan), 2, 3, ref(q), ref(k), ref(v), None, None, tb.TK_F32,
                                          FAKE, 0, 3, slots, ref(o), kc, FAKE, ks, None)

    for kw, st, msg in [
            (dict(plan=tb.rope_plan(64)), tb.TK_ERR_INVALID_ARG, "cache r=32"),
            (dict(k=None), tb.TK_ERR_INVALID_ARG, "k or v"),
            (dict(q=None), tb.TK_ERR_INVALID_ARG, "counterpart"),
            (dict(k=_h(4)), tb.TK_ERR_INVALID_ARG, "heads"),
            (dict(o=_h(4, dtype=tb.TK_F32)), tb.TK_ERR_UNSUPPORTED, "TK_BF16"),
            (dict(slots=None), tb.TK_ERR_INVALID_ARG, "slots"),
            (dict(kc=None), tb.TK_ERR_INVALID_ARG, "k_cache"),
            (dict(desc=tb.tk_cache_desc(2, 4, 2, 32, 128, 256, 0, 0, 0, tb.TK_I8)), tb.TK_ERR_INVALID_ARG, "k_scale"),
            (dict(desc=tb.tk_cache_desc(2, 4, 2, 32, 128, 250, 0, 0, 0, tb.TK_BF16)), tb.TK_ERR_INVALID_ARG, "capacity"),
            (dict(desc=tb.tk_cache_desc(2, 4, 2, 32, 128, 0, 256, 1 << 23, 8, tb.TK_BF16)), tb.TK_ERR_UNSUPPORTED, "slots")]:
        assert call(**kw) == st, msg
        assert msg in tb.tk_last_error()


def test_backward_refusals(lib):
    r = ctypes.byref
    plan = tb.rope_plan(32)
    h, o, f = _h(), _h(data=0x20000), _h(dtype=tb.TK_F32)
    w = ctypes.c_void_p(FAKE)

    def call(plan=plan, q=h, g=f, d=o, gk=None, dk=None, dwq=None, dwk=None, ws=None, wsb=0, batch=2):
        ref = lambda x: None if x is None else r(x)  # noqa: E731
        return lib.tk_qk_norm_rope_backward(r(plan), batch, 3, 128, ref(q), None, None, None, tb.TK_F32, FAKE, 0, 3,
                                            ref(g), ref(gk), None, ref(d), ref(dk), None, dwq, dwk, ws, wsb, None)

    for kw, st, msg in [
            (dict(q=None), tb.TK_ERR_INVALID_ARG, "counterpart"),
            (dict(g=None), tb.TK_ERR_INVALID_ARG, "counterpart"),
            (dict(g=None, d=None, q=None), tb.TK_ERR_INVALID_ARG, "all NULL"),
            (dict(d=_h(sb=0, data=0x20000)), tb.TK_ERR_INVALID_ARG, "overlap"),
            (dict(d=_h(dtype=tb.TK_F32)), tb.TK_ERR_INVALID_ARG, "dtype"),
            (dict(dwk=w), tb.TK_ERR_INVALID_ARG, "weight gradient"),
            (dict(plan=tb.rope_plan(32, norm=False), dwq=w), tb.TK_ERR_INVALID_ARG, "weight gradient")]:
        assert call(**kw) == st, msg
        assert msg in tb.tk_last_error()
    assert call(batch=0) == tb.TK_OK


def test_block_table_refusals(lib):
    base = dict(batch=4, ps=64, pages=10, mp=8, lens=FAKE, new=FAKE, table=FAKE, free=FAKE, count=FAKE, per=0,
                rows=16, slots=FAKE, pos=FAKE, off=FAKE, lens_out=FAKE, count_out=FAKE, refused=FAKE, ws=FAKE)

    def call(**kw):
        return lib.tk_block_tables(*{**base, **kw}.values(), None)

    for kw, st, msg in [
            (dict(batch=-1), tb.TK_ERR_INVALID_ARG, "batch"),
            (dict(batch=4097), tb.TK_ERR_UNSUPPORTED, "4096"),
            (dict(ps=48), tb.TK_ERR_UNSUPPORTED, "page_size"),
            (dict(pages=0), tb.TK_ERR_INVALID_ARG, "num_pages"),
            (dict(mp=0), tb.TK_ERR_INVALID_ARG, "max_pages"),
            (dict(pages=1 << 25), tb.TK_ERR_UNSUPPORTED, "2^30"),
            (dict(per=3), tb.TK_ERR_INVALID_ARG, "rows=16"),
            (dict(rows=-1), tb.TK_ERR_INVALID_ARG, "rows"),
            (dict(batch=0), tb.TK_ERR_INVALID_ARG, "empty batch"),
            (dict(lens=None), tb.TK_ERR_INVALID_ARG, "seq_lens"),
            (dict(table=None), tb.TK_ERR_INVALID_ARG, "page_table"),
            (dict(count=None), tb.TK_ERR_INVALID_ARG, "free_count"),
            (dict(ws=None), tb.TK_ERR_INVALID_ARG, "workspace"),
            (dict(slots=None), tb.TK_ERR_INVALID_ARG, "slots"),
            (dict(slots=0x10004), tb.TK_ERR_INVALID_ARG, "16-byte"),
            (dict(off=0x10002), tb.TK_ERR_INVALID_ARG, "4-byte")]:
        assert call(**kw) == st, msg
        assert msg in tb.tk_last_error()


def test_binding_refusals():
    import torch
    cpu = torch.device("cpu")
    x = torch.zeros(2, 4, 3, 32, dtype=torch.bfloat16)
    with pytest.raises(ValueError):                      # not on a GPU
        tb._heads(x, "q", (2, 4, 3, 32), cpu)
    with pytest.raises(TypeError):
        tb._heads(x.half(), "q", (2, 4, 3, 32), cpu)
    plan = tb.rope_plan(32, axes=(8, 8))
    with pytest.raises(TypeError):
        tb._positions(plan, torch.zeros(2, 3, dtype=torch.int64), 2, 3, cpu)
    with pytest.raises(ValueError):
        tb._positions(plan, torch.zeros(3, 2, 3, dtype=torch.int32), 2, 3, cpu)
    assert tb._positions(plan, torch.zeros(2, 3, dtype=torch.int32), 2, 3, cpu)[1:] == (0, 3)
    with pytest.raises(ValueError):
        tb._positions(plan, torch.zeros(2, 6, dtype=torch.int32)[:, ::2], 2, 3, cpu)
    with pytest.raises(TypeError):
        tb._weights(plan, torch.zeros(32), torch.zeros(32, dtype=torch.bfloat16), cpu)


def test_binding_refuses_host_tensors():
    """Every entry point raises before a host pointer could reach a kernel."""
    import torch
    x = torch.zeros(2, 4, 3, 32, dtype=torch.bfloat16)
    pos = torch.zeros(2, 3, dtype=torch.int32)
    plan = tb.rope_plan(32)
    with pytest.raises(ValueError):
        tb.tk_qk_norm_rope(plan, x, None, None, pos, x.clone(), None, None)
    with pytest.raises(ValueError):
        tb.tk_qk_norm_rope_backward(plan, x, None, pos, x, None, None, x.clone(), None, None)
    cache = tb.ThinKeyCache.allocate(2, 4, 4, 32, 64, capacity=16, device="cpu")
    with pytest.raises(ValueError):
        tb.tk_qk_norm_rope_append(cache, plan, x, x, torch.zeros(2, 4, 3, 64, dtype=torch.bfloat16), pos, pos, x.clone())
    pool = tb.PagePool.allocate(2, 4, 16, 8, device="cpu")
    with pytest.raises(ValueError):
        tb.tk_block_tables(pool, torch.ones(2, dtype=torch.int32), pos.view(-1).clone(), pos.view(-1).clone())


def test_binding_layouts_match_the_header():
    import struct
    assert ctypes.sizeof(tb.tk_heads) == struct.calcsize("Piiqqq") == 40
    assert ctypes.sizeof(tb.tk_rope_desc) == 5 * 4 + 2 * 4 + 64 * 4 + 64
