"""Per-head norm + rotation on the GPU against the fp64 oracle: forward, backward, into the cache.

Tolerances.  cos and sin carry at most 2^-19 each (include/tk.h), so a rotated pair is off by at
most 2 * 2^-19 times the row's largest |y|; the norm adds fewer than 16 roundings of 2^-24.  An
fp32 result is therefore within 5e-6 of the row's largest |y|, a bf16 one within half a bf16 unit
(at most 2^-8 |y|) more.
Gradients: the same relative error on each of the two terms of dx and on each term of dw, doubled
for the products' own roundings: 1e-5 times the sum of the terms' magnitudes.
"""

import numpy as np
import pytest
import torch

from _helpers import bf16_ulp, f64, parity, require_gpu
from oracle import attention as oa
from oracle import cache as oc
from oracle import rope
from paper_2603_04427_gb300 import binding as tb
from paper_2603_04427_gb300 import inputs

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
EPS = 1e-5


def _within(got, ref, scale, dtype, rel=5e-6, what=""):
    bound = rel * scale + (bf16_ulp(ref) / 2 if dtype == BF else 0.0) + 1e-37
    got = f64(got)
    assert np.all(np.isfinite(got)), what
    worst = np.max(np.abs(got - ref) / bound)
    assert worst <= 1.0, f"{what}: error at {worst:.2f} of its bound"


def _rowmax(y):
    return np.abs(y).max(axis=-1, keepdims=True)


def _inputs(B, S, hq, hkv, r, dv, dtype, seed, gap=0):
    """q, k, v [B, H, S, w] as slices of one packed projection with `gap` spare elements a row."""
    g = torch.Generator().manual_seed(seed)
    width = (hq + hkv) * r + hkv * dv + gap
    packed = (torch.randn(B, S, width, generator=g) * torch.exp(torch.randn(B, S, 1, generator=g))).to(dtype).cuda()
    q, k, v, _ = packed.split([hq * r, hkv * r, hkv * dv, gap], dim=-1)
    return packed, (q.view(B, S, hq, r).transpose(1, 2), k.view(B, S, hkv, r).transpose(1, 2),
                    v.view(B, S, hkv, dv).transpose(1, 2))


def _positions(B, S, axes, seed, top=131072):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-5, top, (axes, B, S), generator=g, dtype=torch.int32).cuda()


def _theta(plan, pos):
    n = plan.rot_dim // 2
    return rope.angles(pos.cpu().numpy(), list(plan.inv_freq[:n]), list(plan.pair_axis[:n]))


def _weights(r, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return (1 + 0.3 * torch.randn(2, r, generator=g)).to(dtype).cuda()


CASES = [
    # B, S, hq, hkv, r, dv, rot, layout, axes, norm, x, out, gap
    (1, 1, 1, 1, 16, 64, 16, "half", 1, True, BF, BF, 0),
    (1, 1, 8, 2, 128, 128, 128, "pair", 2, True, F32, F32, 0),
    (2, 37, 12, 12, 16, 64, 8, "half", 1, True, BF, F32, 8),
    (3, 5, 6, 3, 32, 128, 32, "half", 1, True, BF, BF, 16),
    (2, 65, 32, 8, 32, 128, 32, "pair", 3, True, BF, BF, 0),
    (1, 129, 5, 1, 64, 64, 24, "half", 2, True, F32, BF, 4),
    (2, 33, 4, 4, 64, 128, 64, "pair", 4, False, F32, F32, 0),
    (1, 300, 16, 2, 128, 64, 64, "half", 1, True, BF, BF, 24),
    (2, 31, 3, 3, 32, 64, 0, "half", 1, True, BF, F32, 0),
    (1, 7, 9, 9, 128, 128, 96, "pair", 1, False, BF, BF, 8),
    (1, 4099, 8, 8, 32, 128, 32, "half", 1, True, BF, BF, 0),
]


def _plan(r, rot, layout, axes, norm, w_offset=0.0):
    pairs = rot // 2
    # axes interleaved over the pairs, frequencies of the pairs' own
    return tb.rope_plan(r, rot_dim=rot, layout=layout, norm=norm, eps=EPS, w_offset=w_offset,
                        inv_freq=[10000.0 ** (-j / max(1, pairs)) for j in range(pairs)],
                        pair_axis=[j % axes for j in range(pairs)])


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c))
def test_forward(case):
    require_gpu()
    B, S, hq, hkv, r, dv, rot, layout, axes, norm, xt, ot, gap = case
    plan = _plan(r, rot, layout, axes, norm, w_offset=1.0 if S % 2 else 0.0)
    _, (q, k, v) = _inputs(B, S, hq, hkv, r, dv, xt, seed=S, gap=gap)
    pos = _positions(B, S, plan.n_axes, seed=S + 1)
    w = _weights(r, BF if S % 3 else F32, seed=S + 2)
    outs = [torch.full((B, h, S, n), 7.0, dtype=ot, device="cuda") for h, n in ((hq, r), (hkv, r), (hkv, dv))]
    tb.tk_qk_norm_rope(plan, q, k, v, pos, *outs, q_weight=w[0], k_weight=w[1])
    assert tb.tk_get_device_error() == 0
    theta = _theta(plan, pos)
    for x, got, wt, what in ((q, outs[0], w[0], "q"), (k, outs[1], w[1], "k")):
        ref = rope.norm_rope(f64(x), f64(wt) + plan.w_offset, theta, rot, layout, norm, EPS)
        # a turned pair mixes its elements: the bound goes by the row's largest value
        _within(got, ref, _rowmax(ref), ot, what=what)
    assert torch.equal(outs[2], v.to(ot))


def test_forward_layouts_parts_and_broadcasts():
    """Token-major outputs between sentinels, single tensors, shared and expanded positions, in place."""
    require_gpu()
    B, S, hq, hkv, r, dv = 2, 21, 6, 2, 32, 64
    plan = _plan(r, 32, "half", 2, True)
    packed, (q, k, v) = _inputs(B, S, hq, hkv, r, dv, BF, seed=3, gap=8)
    row = torch.arange(S, dtype=torch.int32, device="cuda")
    pos = torch.stack([row, 3 * row])[:, None].expand(2, B, S)          # batch stride 0
    full = [torch.empty(B, h, S, n, dtype=BF, device="cuda") for h, n in ((hq, r), (hkv, r), (hkv, dv))]
    tb.tk_qk_norm_rope(plan, q, k, v, pos, *full)
    dense = [torch.empty_like(t) for t in full]
    tb.tk_qk_norm_rope(plan, q.contiguous(), k.contiguous(), v.contiguous(), pos.contiguous(), *dense)
    for a, b in zip(full, dense):
        assert torch.equal(a, b)
    # each tensor alone, written token-major into a wider buffer
    for i, x in enumerate((q, k, v)):
        H, n = x.shape[1], x.shape[3]
        buf = torch.full((B, S, H * n + 16), 7.0, dtype=BF, device="cuda")
        out = buf[..., 8:8 + H * n].view(B, S, H, n).transpose(1, 2)
        ins, outs = [None] * 3, [None] * 3
        ins[i], outs[i] = x, out
        tb.tk_qk_norm_rope(plan, *ins, pos, *outs)
        assert torch.equal(out, full[i])
        assert bool((buf[..., :8] == 7).all()) and bool((buf[..., 8 + H * n:] == 7).all())
    # positions [B, S] stand for every axis
    same = tb.tk_qk_norm_rope(plan, q, None, None, row.expand(B, S), torch.empty_like(full[0]), None, None)[0]
    both = tb.tk_qk_norm_rope(plan, q, None, None, torch.stack([row, row])[:, None].expand(2, B, S),
                              torch.empty_like(full[0]), None, None)[0]
    assert torch.equal(same, both)
    # in place
    tb.tk_qk_norm_rope(plan, q, k, v, pos, q, k, v)
    for a, b in zip((q, k, v), full):
        assert torch.equal(a, b)
    assert tb.tk_get_device_error() == 0


def test_forward_angles_over_the_whole_position_range():
    """fp32 rotation of unit pairs: cos and sin themselves, within 2^-19 at any position."""
    require_gpu()
    pos = torch.tensor([0, 1, -1, 511, 4096, 131071, 999_983, -(1 << 20) - 1, (1 << 24) - 1, 1 << 24, -(1 << 24)],
                       dtype=torch.int32, device="cuda")[None]
    freq = [4.0, 3.999, 1.0, 0.7498942, 0.31622776, 0.1, 1e-3, 1e-4]
    plan = tb.rope_plan(16, inv_freq=freq, norm=False)
    S = pos.shape[1]
    x = torch.zeros(1, 1, S, 16, device="cuda")
    x[..., :8] = 1.0
    got = f64(tb.tk_qk_norm_rope(plan, x, None, None, pos, torch.empty_like(x), None, None)[0])
    theta = _theta(plan, pos[None])
    assert np.abs(got[0, 0, :, :8] - np.cos(theta[0])).max() <= 2.0 ** -19
    assert np.abs(got[0, 0, :, 8:] - np.sin(theta[0])).max() <= 2.0 ** -19
    assert tb.tk_get_device_error() == 0
    far = torch.tensor([[(1 << 24) + 1, -(2 ** 31)]], dtype=torch.int32, device="cuda")
    tb.tk_qk_norm_rope(plan, x[:, :, :2], None, None, far, torch.empty_like(x[:, :, :2]), None, None)
    assert tb.tk_get_device_error() == 1 and tb.tk_get_device_error() == 0


@pytest.mark.parametrize("xt", [BF, F32])
def test_forward_special_rows_stay_in_their_row(xt):
    require_gpu()
    B, S, H, r = 1, 19, 5, 32
    plan = _plan(r, 16, "half", 1, True)
    off = _plan(r, 16, "half", 1, False)
    _, (q, _, _) = _inputs(B, S, H, H, r, 64, xt, seed=8)
    q = q.contiguous()
    pos = _positions(B, S, 1, seed=9)
    clean = tb.tk_qk_norm_rope(plan, q, None, None, pos, torch.empty_like(q), None, None)[0]
    bad = q.clone()
    bad[0, 1, 3, 5] = float("nan")
    bad[0, 2, 4, 20] = float("inf")      # not rotated
    bad[0, 0, 0] = 0.0
    got = tb.tk_qk_norm_rope(plan, bad, None, None, pos, torch.empty_like(q), None, None)[0]
    assert bool(got[0, 1, 3].isnan().all()) and bool((got[0, 0, 0] == 0).all())
    keep = torch.ones(B, H, S, dtype=torch.bool, device="cuda")
    keep[0, 1, 3] = keep[0, 2, 4] = keep[0, 0, 0] = False
    assert torch.equal(got[keep], clean[keep])
    # without the norm an infinity outside rot_dim changes nothing but itself
    a = tb.tk_qk_norm_rope(off, q, None, None, pos, torch.empty_like(q), None, None)[0]
    b = tb.tk_qk_norm_rope(off, bad, None, None, pos, torch.empty_like(q), None, None)[0]
    assert b[0, 2, 4, 20].item() == float("inf")
    a[0, 2, 4, 20] = b[0, 2, 4, 20]
    assert torch.equal(a[0, 2], b[0, 2])
    assert tb.tk_get_device_error() == 0


BACKWARD = [
    # B, S, hq, hkv, r, dv, rot, layout, axes, norm, x, dy, gap
    (1, 1, 1, 1, 16, 64, 16, "half", 1, True, BF, F32, 0),
    (2, 37, 12, 12, 16, 64, 8, "half", 1, True, BF, F32, 8),
    (3, 5, 6, 3, 32, 128, 32, "pair", 2, True, BF, BF, 16),
    (1, 129, 5, 1, 64, 64, 24, "half", 2, True, F32, F32, 4),
    (2, 33, 4, 4, 64, 128, 64, "pair", 3, False, F32, BF, 0),
    (1, 300, 16, 2, 128, 64, 64, "half", 1, True, F32, F32, 0),
    (2, 1025, 32, 8, 32, 128, 32, "half", 1, True, BF, F32, 0),
    (1, 7, 9, 9, 128, 128, 128, "pair", 1, True, BF, BF, 8),
]


@pytest.mark.parametrize("case", BACKWARD, ids=lambda c: "-".join(str(x).replace("torch.", "") for x in c))
def test_backward(case):
    require_gpu()
    B, S, hq, hkv, r, dv, rot, layout, axes, norm, xt, gt, gap = case
    plan = _plan(r, rot, layout, axes, norm, w_offset=1.0 if S % 2 else 0.0)
    packed, (q, k, v) = _inputs(B, S, hq, hkv, r, dv, xt, seed=S, gap=gap)
    pos = _positions(B, S, plan.n_axes, seed=S + 1)
    w = _weights(r, F32 if S % 3 else BF, seed=S + 2)
    gen = torch.Generator().manual_seed(S + 3)
    gs = [torch.randn(B, h, S, n, generator=gen).to(gt).cuda() for h, n in ((hq, r), (hkv, r), (hkv, dv))]
    dpacked = torch.full_like(packed, 7.0)
    dq, dk, dvv, spare = dpacked.split([hq * r, hkv * r, hkv * dv, gap], dim=-1)
    ds = [t.view(B, S, h, n).transpose(1, 2) for t, h, n in ((dq, hq, r), (dk, hkv, r), (dvv, hkv, dv))]
    dw = [torch.full((r,), 7.0, device="cuda") for _ in range(2)] if norm else [None, None]
    ws = tb.qk_norm_rope_workspace(plan)

    def run():
        tb.tk_qk_norm_rope_backward(plan, q, k, pos, *gs, *ds, q_weight=w[0], k_weight=w[1], dq_weight=dw[0],
                                    dk_weight=dw[1], workspace=ws)
        assert tb.tk_get_device_error() == 0

    run()
    theta = _theta(plan, pos)
    for x, g, d, wt, dwt, what in ((q, gs[0], ds[0], w[0], dw[0], "q"), (k, gs[1], ds[1], w[1], dw[1], "k")):
        ref, rw, terms, size = rope.norm_rope_backward(f64(x), f64(wt) + plan.w_offset, f64(g), theta, rot, layout,
                                                       norm, EPS)
        _within(d, ref, size, xt, rel=1e-5, what="d" + what)
        if norm:
            assert np.all(np.abs(f64(dwt) - rw) <= 1e-5 * terms), what
    assert torch.equal(ds[2], gs[2].to(xt))
    assert bool((spare == 7).all())
    # the same call again on the same workspace: the same bits
    first, fw = dpacked.clone(), [None if t is None else t.clone() for t in dw]
    run()
    assert torch.equal(dpacked, first)
    for a, b in zip(dw, fw):
        assert a is None or torch.equal(a, b)


def test_backward_against_differences():
    """Directional derivatives of the fp64 forward along random directions of x and w."""
    require_gpu()
    B, S, H, r = 2, 11, 3, 32
    plan = _plan(r, 16, "pair", 2, True)
    g = torch.Generator().manual_seed(5)
    x, dx_dir, dy = (torch.randn(B, H, S, r, generator=g) for _ in range(3))
    w, dw_dir = 1 + 0.3 * torch.randn(r, generator=g), torch.randn(r, generator=g)
    pos = _positions(B, S, 2, seed=6)
    theta = _theta(plan, pos)
    f = lambda x, w: float((rope.norm_rope(x, w, theta, 16, "pair", True, EPS) * f64(dy)).sum())  # noqa: E731
    dx, dw = torch.empty(B, H, S, r, device="cuda"), torch.empty(r, device="cuda")
    tb.tk_qk_norm_rope_backward(plan, x.cuda(), None, pos, dy.cuda(), None, None, dx, None, None,
                                q_weight=w.cuda(), dq_weight=dw)
    h = 1e-5
    X, W, DX, DW = f64(x), f64(w), f64(dx_dir), f64(dw_dir)
    along_x = (f(X + h * DX, W) - f(X - h * DX, W)) / (2 * h)
    along_w = (f(X, W + h * DW) - f(X, W - h * DW)) / (2 * h)
    assert abs(along_x - (f64(dx) * DX).sum()) <= 1e-5 * np.abs(f64(dx) * DX).sum()
    assert abs(along_w - (f64(dw) * DW).sum()) <= 2e-5 * np.abs(f64(dw) * DW).sum() + 1e-5 * np.abs(f64(dy)).sum()


def test_backward_parts_and_empty_call():
    require_gpu()
    B, S, hq, hkv, r, dv = 2, 40, 4, 2, 64, 128
    plan = _plan(r, 64, "half", 1, True)
    _, (q, k, v) = _inputs(B, S, hq, hkv, r, dv, BF, seed=1)
    pos = _positions(B, S, 1, seed=2)
    gs = [torch.randn(B, h, S, n, device="cuda") for h, n in ((hq, r), (hkv, r), (hkv, dv))]
    full = [torch.empty(t.shape, dtype=BF, device="cuda") for t in gs]
    dw = [torch.empty(r, device="cuda") for _ in range(2)]
    tb.tk_qk_norm_rope_backward(plan, q, k, pos, *gs, *full, dq_weight=dw[0], dk_weight=dw[1])
    for i in range(3):
        ins, outs, xs = [None] * 3, [None] * 3, [None, None, None]
        ins[i], outs[i] = gs[i], torch.empty_like(full[i])
        if i < 2:
            xs[i] = (q, k)[i]
        one = torch.empty(r, device="cuda")
        kw = {("dq_weight", "dk_weight")[i]: one} if i < 2 else {}
        tb.tk_qk_norm_rope_backward(plan, xs[0], xs[1], pos, *ins, *outs, **kw)
        assert torch.equal(outs[i], full[i])
        if i < 2:   # another split of the same sum
            terms = f64(gs[i]).size ** 0.5
            assert np.abs(f64(one) - f64(dw[i])).max() <= 1e-5 * terms * 10
    z = torch.empty(B, hq, 0, r, device="cuda")
    tb.tk_qk_norm_rope_backward(plan, z.to(BF), None, None, z, None, None, z.to(BF), None, None, dq_weight=dw[0])
    assert bool((dw[0] == 0).all())
    assert tb.tk_get_device_error() == 0


def _cache(B, hq, hkv, r, dv, page, kfmt, tokens):
    kw = dict(k_int8=kfmt == "int8", k_int4=kfmt == "int4")
    if page:
        per = -(-tokens // page)
        table = torch.randperm(B * per, generator=torch.Generator().manual_seed(4)).to(torch.int32).view(B, per)
        c = tb.ThinKeyCache.allocate(B, hq, hkv, r, dv, page_size=page, num_pages=B * per, page_table=table, **kw)
    else:
        table = None
        c = tb.ThinKeyCache.allocate(B, hq, hkv, r, dv, capacity=(tokens + 15) // 16 * 16, **kw)
    for t in (c.k, c.v, c.k_scale):
        if t is not None:
            t.view(torch.uint8).fill_(7)
    return c, table


def _slots(c, table, lens, S):
    """Slots [B, S] of the positions lens[b] + t."""
    at = torch.tensor(lens)[:, None] + torch.arange(S)
    if table is None:
        s = torch.arange(len(lens))[:, None] * c.desc.capacity + at
    else:
        s = table.long().gather(1, at // c.desc.page_size) * c.desc.page_size + at % c.desc.page_size
    return s.to(torch.int32).cuda()


@pytest.mark.parametrize("page", [0, 16, 64])
@pytest.mark.parametrize("kfmt", ["bf16", "int8", "int4"])
@pytest.mark.parametrize("hq,hkv,r,dv,S,xt,layout", [
    (32, 8, 32, 128, 1, BF, "half"), (4, 2, 64, 64, 23, BF, "pair"), (8, 1, 128, 128, 5, F32, "half"),
    (12, 12, 16, 64, 9, BF, "half")])
def test_append_equals_norm_rope_then_append(page, kfmt, hq, hkv, r, dv, S, xt, layout):
    """bf16 keys and values: the two calls' bits.  Quantised keys: the codes and scales of the fp32 rotation."""
    require_gpu()
    if kfmt == "int4" and r < 32:
        pytest.skip("int4 keys need r >= 32")
    lens = [3, 0, 30]
    B = len(lens)
    plan = _plan(r, r // 2 if r > 16 else r, layout, 1, True)
    _, (q, k, v) = _inputs(B, S, hq, hkv, r, dv, xt, seed=r + S)
    w = _weights(r, F32, seed=1)
    a, table = _cache(B, hq, hkv, r, dv, page, kfmt, max(lens) + S)
    b, _ = _cache(B, hq, hkv, r, dv, page, kfmt, max(lens) + S)
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    pos = (seq[:, None] + torch.arange(S, device="cuda", dtype=torch.int32)).contiguous()
    slots = _slots(a, table, lens, S)
    q1 = torch.empty(B, hq, S, r, dtype=BF, device="cuda")
    tb.tk_qk_norm_rope_append(a, plan, q, k, v, pos, slots, q1, q_weight=w[0], k_weight=w[1])
    q2, k2 = torch.empty_like(q1), torch.empty(B, hkv, S, r, dtype=BF, device="cuda")
    v2 = torch.empty(B, hkv, S, dv, dtype=BF, device="cuda")
    tb.tk_qk_norm_rope(plan, q, k, v, pos, q2, k2, v2, q_weight=w[0], k_weight=w[1])
    tb.tk_kv_append(b, k2, v2, seq)
    assert tb.tk_get_device_error() == 0
    assert torch.equal(q1, q2)
    assert torch.equal(a.v.view(torch.int16), b.v.view(torch.int16))
    if kfmt == "bf16":
        assert torch.equal(a.k.view(torch.int16), b.k.view(torch.int16))
        return
    kf = torch.empty(B, hkv, S, r, device="cuda")
    tb.tk_qk_norm_rope(plan, None, k, None, pos, None, kf, None, k_weight=w[1])
    quant = oc.quantize_int8_per_token if kfmt == "int8" else oc.quantize_int4_per_token
    codes, scales = quant(kf.cpu().numpy())
    if kfmt == "int4":
        codes = oc.pack_int4(codes)
    rows = a.desc.page_size or a.desc.capacity
    ref_k, ref_s = b.k.cpu().numpy(), b.k_scale.cpu().numpy()
    ref_k.view(np.uint8)[:] = 7
    ref_s.view(np.uint8)[:] = 7
    sl = slots.cpu().numpy()
    for i in range(B):
        for t in range(S):
            ref_k[sl[i, t] // rows, :, sl[i, t] % rows] = codes[i, :, t]
            ref_s[sl[i, t] // rows, :, sl[i, t] % rows] = scales[i, :, t]
    assert np.array_equal(a.k.cpu().numpy(), ref_k)
    assert np.array_equal(a.k_scale.cpu().numpy().view(np.uint32), ref_s.view(np.uint32))


def test_append_skips_and_flags_slots():
    require_gpu()
    hq, hkv, r, dv, S = 4, 2, 32, 64, 6
    plan = _plan(r, 32, "half", 1, True)
    _, (q, k, v) = _inputs(1, S, hq, hkv, r, dv, BF, seed=2)
    pos = torch.arange(S, dtype=torch.int32, device="cuda")[None].contiguous()
    c, _ = _cache(1, hq, hkv, r, dv, 0, "bf16", 32)
    qo = torch.empty(1, hq, S, r, dtype=BF, device="cuda")
    ref = tb.tk_qk_norm_rope(plan, q, k, None, pos, torch.empty_like(qo),
                             torch.empty(1, hkv, S, r, dtype=BF, device="cuda"), None)
    slots = torch.tensor([5, -1, 0, 31, -7, 6], dtype=torch.int32, device="cuda")
    tb.tk_qk_norm_rope_append(c, plan, q, k, v, pos, slots, qo)
    assert tb.tk_get_device_error() == 0 and torch.equal(qo, ref[0])
    for t, s in ((0, 5), (2, 0), (3, 31), (5, 6)):
        assert torch.equal(c.k[0, :, s], ref[1][0, :, t]) and torch.equal(c.v[0, :, s], v[0, :, t])
    rest = [s for s in range(32) if s not in (5, 0, 31, 6)]
    assert bool((c.k[0, :, rest].view(torch.uint8) == 7).all()) and bool((c.v[0, :, rest].view(torch.uint8) == 7).all())
    before = c.k.clone()
    # keys and values alone; a slot beyond the cache is flagged and not written
    slots.copy_(torch.tensor([32, -1, -1, -1, -1, 2 ** 31 - 1]))
    tb.tk_qk_norm_rope_append(c, plan, None, k, v, pos, slots, None)
    assert tb.tk_get_device_error() == 1 and torch.equal(c.k.view(torch.int16), before.view(torch.int16))


def test_append_in_a_graph_on_another_stream():
    """The prepared call recorded once and replayed on new contents of the same buffers."""
    require_gpu()
    hq, hkv, r, dv, B = 8, 2, 64, 128, 5
    plan = _plan(r, 64, "half", 1, True)
    _, (q, k, v) = _inputs(B, 1, hq, hkv, r, dv, BF, seed=4)
    c, _ = _cache(B, hq, hkv, r, dv, 0, "bf16", 16)
    pos = torch.zeros(B, 1, dtype=torch.int32, device="cuda")
    slots = torch.arange(B, dtype=torch.int32, device="cuda") * 16
    qo = torch.empty(B, hq, 1, r, dtype=BF, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    call = tb.prepare_qk_norm_rope_append(c, plan, q, k, v, pos, slots, qo, stream=s, graph=True)
    with torch.cuda.stream(s):
        pos.fill_(9)
        slots += 9
        call()
    s.synchronize()
    ref = tb.tk_qk_norm_rope(plan, q, k, None, pos, torch.empty_like(qo),
                             torch.empty(B, hkv, 1, r, dtype=BF, device="cuda"), None)
    assert torch.equal(qo, ref[0]) and torch.equal(c.k[:, :, 9], ref[1][:, :, 0])
    assert tb.tk_get_device_error() == 0


def test_training_path_gradients():
    """Projection rows -> norm + rotation -> attention -> backward of both, against the fp64 oracle's chain."""
    require_gpu()
    B, S, hq, hkv, r, dv = 1, 130, 4, 2, 32, 64
    plan = _plan(r, 32, "half", 1, True)
    packed, (q, k, v) = _inputs(B, S, hq, hkv, r, dv, BF, seed=11)
    pos = torch.arange(S, dtype=torch.int32, device="cuda")[None].contiguous()
    w = _weights(r, F32, seed=12)
    qr, kr, vr = (torch.empty(B, h, S, n, dtype=BF, device="cuda") for h, n in ((hq, r), (hkv, r), (hkv, dv)))
    tb.tk_qk_norm_rope(plan, q, k, v, pos, qr, kr, vr, q_weight=w[0], k_weight=w[1])
    out, lse = torch.empty(B, hq, S, dv, dtype=BF, device="cuda"), torch.empty(B, hq, S, device="cuda")
    tb.tk_attn_forward(qr, kr, vr, out, lse)
    do = inputs.normal_bf16(out.shape, 13, device="cuda")
    gs = [torch.empty(t.shape, device="cuda") for t in (qr, kr, vr)]
    tb.tk_attn_backward(qr, kr, vr, out, do, lse, *gs)
    dpacked = torch.empty_like(packed)
    d = [t.view(B, S, h, n).transpose(1, 2) for t, h, n in zip(
        dpacked.split([hq * r, hkv * r, hkv * dv], dim=-1), (hq, hkv, hkv), (r, r, dv))]
    dw = [torch.empty(r, device="cuda") for _ in range(2)]
    tb.tk_qk_norm_rope_backward(plan, q, k, pos, *gs, *d, q_weight=w[0], k_weight=w[1], dq_weight=dw[0], dk_weight=dw[1])
    assert tb.tk_get_device_error() == 0
    theta = _theta(plan, pos[None])
    Q, K = (rope.norm_rope(f64(x), f64(wt), theta, 32, "half", True, EPS) for x, wt in ((q, w[0]), (k, w[1])))
    gq, gk, gv = oa.attention_backward(Q, K, f64(v), f64(do), 1 / np.sqrt(r))
    refs = [rope.norm_rope_backward(f64(x), f64(wt), g, theta, 32, "half", True, EPS)[0]
            for x, wt, g in ((q, w[0], gq), (k, w[1], gk))] + [gv]
    for got, ref, what in zip(d, refs, ("dq", "dk", "dv")):
        # the attention's own bar for gradients (bf16 P and dS), plus bf16 inputs and outputs here (2^-9 each)
        err = np.abs(f64(got) - ref)
        assert err.sum() <= 1.4e-2 * np.abs(ref).sum(), what


@pytest.mark.parametrize("kfmt", ["bf16", "int8"])
def test_serving_path(kfmt):
    """Requests of several lengths admitted, then decode steps: page tables, append and decode together."""
    require_gpu()
    B, hq, hkv, r, dv, ps = 4, 8, 2, 32, 64, 16
    plan = _plan(r, 32, "half", 1, True)
    w = _weights(r, F32, seed=21)
    pool = tb.PagePool.allocate(B, 8, ps, 20)
    c = tb.ThinKeyCache.allocate(B, hq, hkv, r, dv, page_size=ps, num_pages=20, page_table=pool.page_table,
                                 k_int8=kfmt == "int8")
    assert c.page_table.data_ptr() == pool.page_table.data_ptr()
    hist = [[] for _ in range(B)]
    for step, new in enumerate([[33, 1, 0, 47], [1, 1, 5, 1], [1, -1, 1, 1], [1, 20, 1, 1], [1, 1, 1, 1]]):
        rows = sum(max(n, 0) for n in new) + 3
        i32 = dict(dtype=torch.int32, device="cuda")
        slots, pos, offs = torch.empty(rows, **i32), torch.empty(rows, **i32), torch.empty(B + 1, **i32)
        refused = torch.empty(1, **i32)
        tb.tk_block_tables(pool, torch.tensor(new, **i32), slots, pos, offsets=offs, refused=refused)
        assert refused.item() == 0
        _, (q, k, v) = _inputs(1, rows, hq, hkv, r, dv, BF, seed=30 + step)
        qo = torch.empty(1, hq, rows, r, dtype=BF, device="cuda")
        tb.tk_qk_norm_rope_append(c, plan, q, k, v, pos[None], slots, qo, q_weight=w[0], k_weight=w[1])
        theta = _theta(plan, pos[None, None])
        kref = rope.norm_rope(f64(k), f64(w[1]), theta, 32, "half", True, EPS)
        o = offs.tolist()
        for b in range(B):
            if new[b] < 0:
                hist[b] = []
            hist[b] += [(kref[0, :, i], f64(v)[0, :, i]) for i in range(o[b], o[b + 1])]
        # decode the last token of every sequence that has one
        last = torch.tensor([max(0, o[b + 1] - 1) for b in range(B)], device="cuda")
        qd = qo[0][:, last].transpose(0, 1).contiguous()
        out = torch.empty(B, hq, dv, device="cuda")
        tb.tk_attn_decode(c, qd, pool.seq_lens, 128, out, tb.decode_workspace(c.desc, 128))
        assert tb.tk_get_device_error() == 0
        assert pool.seq_lens.tolist() == [len(h) for h in hist]
        for b in range(B):
            if not hist[b]:
                assert bool((out[b] == 0).all())
                continue
            K, V = (np.stack([h[j] for h in hist[b]], axis=1)[None] for j in (0, 1))
            ref = oa.attention_decode(f64(qd[b:b + 1]), K, V, [len(hist[b])], 1 / np.sqrt(r))
            # bf16 keys: 2^-9 of each key, scores of a few units; int8 keys: half a step, amax / 254
            parity(f64(out[b:b + 1]), ref, max_abs=2e-2 if kfmt == "bf16" else 6e-2,
                   mean_rel=5e-3 if kfmt == "bf16" else 2e-2, what=f"step {step} sequence {b}")


@pytest.mark.parametrize("kfmt", ["int8", "int4"])
def test_append_quantiser_over_all_magnitudes(kfmt):
    """Rows from denormals to near overflow, ties, zeros: codes and scales of the oracle's quantiser, bit for bit."""
    require_gpu()
    r, dv = 32, 64
    plan = tb.rope_plan(r, rot_dim=0, norm=False)          # rows pass through unchanged
    g = np.random.default_rng(6)
    mags = np.exp2(np.linspace(-148, 126, 400))
    x = (g.uniform(-1, 1, (400, r)) * mags[:, None]).astype(np.float32)
    top = 127 if kfmt == "int8" else 7
    x[::3] = np.round(x[::3] / np.abs(x[::3]).max(-1, keepdims=True) * 2 * top) / 2      # halves of a code
    x[::3, 0] = top
    x[5] = 0.0
    x[6] = -0.0
    x[7, 1:] = 0.0
    S = x.shape[0]
    k = torch.from_numpy(x)[None, None].cuda()
    v = torch.zeros(1, 1, S, dv, device="cuda")
    c, _ = _cache(1, 1, 1, r, dv, 0, kfmt, S)
    slots = torch.arange(S, dtype=torch.int32, device="cuda")
    tb.tk_qk_norm_rope_append(c, plan, None, k, v, None, slots, None)
    assert tb.tk_get_device_error() == 0
    codes, scales = (oc.quantize_int8_per_token if kfmt == "int8" else oc.quantize_int4_per_token)(x)
    codes = oc.pack_int4(codes) if kfmt == "int4" else codes
    assert np.array_equal(c.k_scale[0, 0, :S].cpu().numpy().view(np.uint32), scales.view(np.uint32))
    assert np.array_equal(c.k[0, 0, :S].cpu().numpy(), codes)


def test_append_of_infinite_keys_stays_in_its_row():
    require_gpu()
    r, dv, S = 32, 64, 9
    plan = tb.rope_plan(r, rot_dim=0, norm=False)
    x = torch.randn(1, 2, S, r, device="cuda")
    bad = x.clone()
    bad[0, 0, 4, 3] = float("inf")
    bad[0, 1, 2, 0] = float("nan")
    v = torch.randn(1, 2, S, dv, device="cuda")
    slots = torch.arange(S, dtype=torch.int32, device="cuda")
    caches = []
    for k in (x, bad):
        c, _ = _cache(1, 2, 2, r, dv, 0, "int8", S)
        tb.tk_qk_norm_rope_append(c, plan, None, k, v, None, slots, None)
        caches.append(c)
    a, b = caches
    keep = torch.ones(2, S, dtype=torch.bool, device="cuda")
    keep[0, 4] = keep[1, 2] = False
    assert torch.equal(a.k[0, :, :S][keep], b.k[0, :, :S][keep])
    assert torch.equal(a.k_scale[0, :, :S][keep], b.k_scale[0, :, :S][keep]) and torch.equal(a.v, b.v)


def test_broadcast_inputs_and_gradients_in_place():
    """One set of heads read for every sequence (stride 0); dq written over q, and over dq_out."""
    require_gpu()
    B, S, H, r = 3, 10, 4, 64
    plan = _plan(r, 64, "half", 1, True)
    one = torch.randn(1, H, S, r, device="cuda")
    pos = _positions(B, S, 1, seed=4)
    wide = one.expand(B, H, S, r)
    got = tb.tk_qk_norm_rope(plan, wide, None, None, pos, torch.empty(B, H, S, r, device="cuda"), None, None)[0]
    ref = tb.tk_qk_norm_rope(plan, wide.contiguous(), None, None, pos, torch.empty_like(got), None, None)[0]
    assert torch.equal(got, ref)
    heads = torch.randn(B, 1, S, r, device="cuda").expand(B, H, S, r)
    got = tb.tk_qk_norm_rope(plan, heads, None, None, pos, torch.empty_like(got), None, None)[0]
    assert all(torch.equal(got[:, 0], got[:, h]) for h in range(H))
    with pytest.raises(tb.TkError):          # a gradient cannot be written to shared rows
        tb.tk_qk_norm_rope_backward(plan, wide, None, pos, ref, None, None, wide, None, None)
    x, g = torch.randn(B, H, S, r, device="cuda"), torch.randn(B, H, S, r, device="cuda")
    dx = torch.empty_like(x)
    tb.tk_qk_norm_rope_backward(plan, x, None, pos, g, None, None, dx, None, None)
    over_x, over_g = x.clone(), g.clone()
    tb.tk_qk_norm_rope_backward(plan, over_x, None, pos, g, None, None, over_x, None, None)
    tb.tk_qk_norm_rope_backward(plan, x, None, pos, over_g, None, None, over_g, None, None)
    assert torch.equal(over_x, dx) and torch.equal(over_g, dx)
    assert tb.tk_get_device_error() == 0


def test_calls_on_another_stream():
    """Inputs made on one stream, the call and a workspace of its own on another."""
    require_gpu()
    B, S, H, r = 2, 700, 8, 64
    plan = _plan(r, 64, "half", 1, True)
    pos = _positions(B, S, 1, seed=4)
    x, g = torch.randn(B, H, S, r, device="cuda"), torch.randn(B, H, S, r, device="cuda")
    dx, dw = torch.empty_like(x), torch.empty(r, device="cuda")
    tb.tk_qk_norm_rope_backward(plan, x, None, pos, g, None, None, dx, None, None, dq_weight=dw)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(20):
        dx2, dw2 = torch.empty_like(x), torch.empty(r, device="cuda")
        s.wait_stream(torch.cuda.current_stream())
        tb.tk_qk_norm_rope_backward(plan, x, None, pos, g, None, None, dx2, None, None, dq_weight=dw2, stream=s)
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(dx, dx2) and torch.equal(dw, dw2)
    assert tb.tk_get_device_error() == 0
