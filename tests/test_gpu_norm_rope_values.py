"""Norm + rotation on infinities and NaNs."""

import numpy as np
import pytest
import torch

from _helpers import f64, require_gpu
from oracle import rope
from paper_2603_04427_gb300 import binding as tb

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("xt,gt", [(BF, BF), (BF, F32), (F32, F32)])
@pytest.mark.parametrize("r,S,at", [(32, 19, (0, 18)), (32, 19, (3, 18)), (64, 9, (4, 8)), (128, 3, (3, 2)), (16, 16, (4, 7))])
def test_infinite_gradient_reaches_its_weight_alone(xt, gt, r, S, at):
    """One infinite incoming gradient, in the last token or the first row of a run of heads, whose row fills the
    places of rows that are not there: its weight's gradient is that infinity, the others are what they were."""
    require_gpu()
    H, c = 5, 6
    plan = tb.rope_plan(r, rot_dim=0, eps=1e-5)
    gen = torch.Generator().manual_seed(r + S)
    x, g = (torch.randn(1, H, S, r, generator=gen).cuda() for _ in range(2))
    x, g = x.to(xt), g.to(gt)
    h, t = at
    g[0, h, t, c] = float("inf")
    dx, dw = torch.empty_like(x), torch.empty(r, device="cuda")
    tb.tk_qk_norm_rope_backward(plan, x, None, None, g, None, None, dx, None, None, dq_weight=dw)
    assert tb.tk_get_device_error() == 0
    with np.errstate(invalid="ignore"):
        _, ref, terms, _ = rope.norm_rope_backward(f64(x), np.ones(r), f64(g), np.zeros((1, S, 0)), 0, "half", True, 1e-5)
    assert np.isinf(ref[c]) and dw[c].item() == ref[c]
    rest = np.arange(r) != c
    # the relative error of each term of dw: 1e-5 (tests/test_gpu_norm_rope.py)
    assert np.all(np.abs(f64(dw)[rest] - ref[rest]) <= 1e-5 * terms[rest])
    clean = torch.ones(H, S, dtype=torch.bool, device="cuda")
    clean[h, t] = False
    assert bool(dx[0][clean].isfinite().all())


@pytest.mark.parametrize("xt", [BF, F32])
@pytest.mark.parametrize("kfmt", ["int8", "int4"])
def test_codes_of_nan_and_infinite_rows_are_those_of_the_append(kfmt, xt):
    """Rows without any number, with NaNs between zeros or numbers, with infinities: codes and scales as
    tk_kv_append writes them for the same bf16 rows."""
    require_gpu()
    r, dv, S = 32, 64, 12
    nan, inf = float("nan"), float("inf")
    x = torch.randn(S, r, generator=torch.Generator().manual_seed(3))
    x[1] = nan
    x[3] = 0.0
    x[4] = 0.0
    x[4, ::2] = nan
    x[5, 7] = nan
    x[6, 9] = inf
    x[7] = -inf
    x[8, 1], x[8, 30] = nan, -inf
    x[9, :16] = nan
    x[10] = torch.tensor([nan, inf]).repeat(r // 2)
    k = x.to(BF)[None, None].expand(1, 2, S, r).contiguous().cuda()
    v = torch.randn(1, 2, S, dv, device="cuda").to(BF)
    caches = []
    for _ in range(2):
        c = tb.ThinKeyCache.allocate(1, 2, 2, r, dv, capacity=16, k_int8=kfmt == "int8", k_int4=kfmt == "int4")
        for t in (c.k, c.v, c.k_scale):
            t.view(torch.uint8).fill_(7)
        caches.append(c)
    a, b = caches
    plan = tb.rope_plan(r, rot_dim=0, norm=False)         # rows pass through unchanged
    slots = torch.arange(S, dtype=torch.int32, device="cuda")
    tb.tk_qk_norm_rope_append(a, plan, None, k.to(xt), v.to(xt), None, slots, None)
    tb.tk_kv_append(b, k, v, torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert tb.tk_get_device_error() == 0
    assert torch.equal(a.k_scale.view(torch.int32), b.k_scale.view(torch.int32))
    for t in range(S):
        assert torch.equal(a.k[:, :, t], b.k[:, :, t]), t
    assert bool((a.k[:, :, [1, 3, 4]] == 0).all())
    assert torch.equal(a.k, b.k) and torch.equal(a.v.view(torch.int16), b.v.view(torch.int16))
