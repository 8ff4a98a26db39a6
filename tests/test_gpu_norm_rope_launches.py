"""Norm + rotation at launch sizes of several waves against the fp64 oracle: blocks of tokens, runs of heads longer
than the rows a lane holds, several units a warp.  Sizes go by the SM count; tolerances are those of
tests/test_gpu_norm_rope.py."""

import numpy as np
import pytest
import torch

from _helpers import bf16_ulp, f64, require_gpu
from oracle import cache as oc
from oracle import rope
from paper_2603_04427_gb300 import binding as tb

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32
EPS = 1e-5


def _sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


def _tokens(waves, warps_per_sm, units_per_token):
    """An odd count of tokens that gives `waves` waves of units."""
    n = int(waves * _sms() * warps_per_sm / units_per_token) + 2
    return n + 1 - n % 2


def _tensors(n, heads, widths, dtype, seed):
    """Slices [1, H, n, w] of packed rows, with eight spare elements a row."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    sizes = [h * w for h, w in zip(heads, widths)]
    packed = torch.randn(1, n, sum(sizes) + 8, device="cuda", generator=g)
    packed = (packed * torch.exp(torch.randn(1, n, 1, device="cuda", generator=g))).to(dtype)
    parts = packed.split(sizes + [8], dim=-1)
    return packed, [t.view(1, n, h, w).transpose(1, 2) for t, h, w in zip(parts, heads, widths)]


def _plan(r, rot, layout, axes):
    pairs = rot // 2
    return tb.rope_plan(r, rot_dim=rot, layout=layout, eps=EPS,
                        inv_freq=[10000.0 ** (-j / pairs) for j in range(pairs)],
                        pair_axis=[j % axes for j in range(pairs)])


def _positions(n, axes, seed):
    g = torch.Generator().manual_seed(seed)
    pos = torch.randint(0, 131072, (axes, 1, n), generator=g, dtype=torch.int32).cuda()
    return pos


def _theta(plan, pos):
    m = plan.rot_dim // 2
    return rope.angles(pos.cpu().numpy(), list(plan.inv_freq[:m]), list(plan.pair_axis[:m]))


def _weights(r, seed):
    return (1 + 0.3 * torch.randn(2, r, generator=torch.Generator().manual_seed(seed))).cuda()


def _within(got, ref, scale, dtype, rel, what):
    bound = rel * scale + (bf16_ulp(ref) / 2 if dtype == BF else 0.0) + 1e-37
    got = f64(got)
    assert np.all(np.isfinite(got)), what
    worst = np.max(np.abs(got - ref) / bound)
    assert worst <= 1.0, f"{what}: error at {worst:.2f} of its bound"


def _runs(heads, most):
    return -(-heads // most)


@pytest.mark.parametrize("hq,hkv,r,dv,rot,layout,axes,xt,ot", [
    (12, 5, 32, 64, 32, "half", 1, BF, BF),      # runs of 6 + 6 and 5
    (7, 1, 64, 128, 64, "pair", 2, BF, F32),
    (32, 12, 16, 64, 16, "half", 1, BF, BF),
    (5, 7, 128, 64, 64, "half", 1, F32, BF),     # fp32 rows: four a lane, runs of 5 and 7
    (12, 7, 64, 128, 24, "pair", 3, F32, F32),
    (32, 8, 32, 128, 32, "half", 1, F32, F32),
])
def test_forward_of_several_waves(hq, hkv, r, dv, rot, layout, axes, xt, ot):
    require_gpu()
    units = (_runs(hq, 8) + _runs(hkv, 8)) * r / 256 + _runs(hkv, 8) * dv / 256
    n = _tokens(3.3, 20, units)
    plan = _plan(r, rot, layout, axes)
    _, (q, k, v) = _tensors(n, (hq, hkv, hkv), (r, r, dv), xt, seed=n)
    pos, w = _positions(n, axes, seed=1), _weights(r, seed=2)
    outs = [torch.full((1, h, n, m), 7.0, dtype=ot, device="cuda") for h, m in ((hq, r), (hkv, r), (hkv, dv))]
    tb.tk_qk_norm_rope(plan, q, k, v, pos, *outs, q_weight=w[0], k_weight=w[1])
    assert tb.tk_get_device_error() == 0
    theta = _theta(plan, pos)
    for x, got, wt, what in ((q, outs[0], w[0], "q"), (k, outs[1], w[1], "k")):
        ref = rope.norm_rope(f64(x), f64(wt), theta, rot, layout, True, EPS)
        _within(got, ref, np.abs(ref).max(axis=-1, keepdims=True), ot, 5e-6, what)
    assert torch.equal(outs[2], v.to(ot))


@pytest.mark.parametrize("kfmt", ["bf16", "int8", "int4"])
@pytest.mark.parametrize("hq,hkv,r,dv,page,layout,xt", [
    (12, 12, 32, 64, 0, "half", BF),             # bf16 rows: four a lane, runs of 6
    (7, 7, 64, 128, 64, "pair", BF),
    (10, 5, 128, 64, 16, "half", F32),           # fp32 rows: two a lane, runs of 5
    (32, 8, 32, 128, 0, "half", F32),
])
def test_append_of_several_waves(kfmt, hq, hkv, r, dv, page, layout, xt):
    """Two sequences' prompts; every eleventh token is not cached."""
    require_gpu()
    units = (_runs(hq, 8) + _runs(hkv, 8)) * r / 256 + _runs(hkv, 8) * dv / 256
    n = _tokens(2.2, 24, units)
    half = (n // 2 + 64) // 64 * 64
    plan = _plan(r, r, layout, 1)
    _, (q, k, v) = _tensors(n, (hq, hkv, hkv), (r, r, dv), xt, seed=n)
    w = _weights(r, seed=3)
    kw = dict(k_int8=kfmt == "int8", k_int4=kfmt == "int4")
    if page:
        pages = 2 * half // page
        c = tb.ThinKeyCache.allocate(2, hq, hkv, r, dv, page_size=page, num_pages=pages,
                                     page_table=torch.zeros(2, half // page, dtype=torch.int32), **kw)
        order = torch.randperm(pages, generator=torch.Generator().manual_seed(5))
        at = torch.arange(n)
        slots = order[at // page] * page + at % page
    else:
        c = tb.ThinKeyCache.allocate(2, hq, hkv, r, dv, capacity=half, **kw)
        slots = torch.arange(n)
    for t in (c.k, c.v, c.k_scale):
        if t is not None:
            t.view(torch.uint8).fill_(7)
    skipped = torch.arange(n) % 11 == 5
    slots = torch.where(skipped, -1, slots).to(torch.int32).cuda()
    pos = _positions(n, 1, seed=4)
    qo = torch.empty(1, hq, n, r, dtype=BF, device="cuda")
    tb.tk_qk_norm_rope_append(c, plan, q, k, v, pos, slots, qo, q_weight=w[0], k_weight=w[1])
    assert tb.tk_get_device_error() == 0
    theta = _theta(plan, pos)
    ref = rope.norm_rope(f64(q), f64(w[0]), theta, r, layout, True, EPS)
    _within(qo, ref, np.abs(ref).max(axis=-1, keepdims=True), BF, 5e-6, "q")
    rows = c.desc.page_size or c.desc.capacity
    there = slots[slots >= 0].long()
    block, off = there // rows, there % rows
    cached = ~skipped.cuda()
    # values, bit for bit; rows without a token are left alone
    assert torch.equal(c.v[block, :, off], v[0].transpose(0, 1)[cached].to(BF))
    free = torch.ones(c.v.shape[0], rows, dtype=torch.bool, device="cuda")
    free[block, off] = False
    for t in (c.k, c.v) + (() if c.k_scale is None else (c.k_scale,)):
        assert bool((t.transpose(1, 2)[free].contiguous().view(torch.uint8) == 7).all())
    if kfmt == "bf16":
        ref = rope.norm_rope(f64(k), f64(w[1]), theta, r, layout, True, EPS)[:, :, cached.cpu().numpy()]
        got = c.k[block, :, off].transpose(0, 1)[None]
        _within(got, ref, np.abs(ref).max(axis=-1, keepdims=True), BF, 5e-6, "k")
        return
    # codes and scales of the fp32 rotation, bit for bit
    kf = torch.empty(1, hkv, n, r, device="cuda")
    tb.tk_qk_norm_rope(plan, None, k, None, pos, None, kf, None, k_weight=w[1])
    codes, scales = (oc.quantize_int8_per_token if kfmt == "int8" else oc.quantize_int4_per_token)(
        kf[0].transpose(0, 1)[cached].cpu().numpy())
    codes = oc.pack_int4(codes) if kfmt == "int4" else codes
    assert np.array_equal(c.k[block, :, off].cpu().numpy(), codes)
    assert np.array_equal(c.k_scale[block, :, off].cpu().numpy().view(np.uint32), scales.view(np.uint32))


@pytest.mark.parametrize("hq,hkv,r,dv,rot,layout,axes,xt,gt", [
    (5, 3, 32, 64, 32, "half", 1, BF, F32),      # four rows a lane, runs of 3 + 2
    (7, 5, 64, 128, 64, "pair", 2, BF, BF),
    (5, 1, 128, 64, 64, "half", 1, F32, F32),    # two rows a lane, runs of 2 + 2 + 1
    (9, 4, 16, 64, 16, "half", 1, F32, BF),
])
def test_backward_of_several_units_a_warp(hq, hkv, r, dv, rot, layout, axes, xt, gt):
    require_gpu()
    rows = 2 if xt == F32 and gt == F32 else 4
    n = _tokens(3.3, 16, _runs(hkv, rows) * r / 256)      # of k; q has more
    plan = _plan(r, rot, layout, axes)
    packed, (q, k, v) = _tensors(n, (hq, hkv, hkv), (r, r, dv), xt, seed=n)
    pos, w = _positions(n, axes, seed=1), _weights(r, seed=2)
    gen = torch.Generator(device="cuda").manual_seed(3)
    gs = [torch.randn(1, h, n, m, device="cuda", generator=gen).to(gt) for h, m in ((hq, r), (hkv, r), (hkv, dv))]
    dpacked = torch.full_like(packed, 7.0)
    parts = dpacked.split([hq * r, hkv * r, hkv * dv, 8], dim=-1)
    ds = [t.view(1, n, h, m).transpose(1, 2) for t, h, m in zip(parts, (hq, hkv, hkv), (r, r, dv))]
    dw = [torch.full((r,), 7.0, device="cuda") for _ in range(2)]
    tb.tk_qk_norm_rope_backward(plan, q, k, pos, *gs, *ds, q_weight=w[0], k_weight=w[1], dq_weight=dw[0], dk_weight=dw[1])
    assert tb.tk_get_device_error() == 0
    theta = _theta(plan, pos)
    for x, g, d, wt, dwt, what in ((q, gs[0], ds[0], w[0], dw[0], "q"), (k, gs[1], ds[1], w[1], dw[1], "k")):
        ref, rw, terms, size = rope.norm_rope_backward(f64(x), f64(wt), f64(g), theta, rot, layout, True, EPS)
        _within(d, ref, size, xt, 1e-5, "d" + what)
        assert np.all(np.abs(f64(dwt) - rw) <= 1e-5 * terms), what
    assert torch.equal(ds[2], gs[2].to(xt))
    assert bool((parts[3] == 7).all())
