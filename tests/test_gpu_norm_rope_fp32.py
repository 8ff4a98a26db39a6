"""Norm + rotation with 32-bit results against the fp64 oracle.

Tolerances.  cos and sin carry at most 2^-22 each (include/tk.h).  A turned pair a c - b s is off by twice that and by
three roundings (2^-24 each) of the row's largest |y| before the turn.  The norm: the mean of r <= 128 squares takes 3
roundings in a lane, 1 across its two halves, 4 across lanes, 1 for eps, of which the root keeps half; the root's own
arithmetic 3, two products 2: fewer than 10 in all.  Together (2 * 2^-22 + 13 * 2^-24) < 6 * 2^-22 of the row's largest.
Gradients: g is off by 2 * 2^-22 + 3 * 2^-24 as above, g u and g u x rho by 2 roundings more each, their mean by 8, rho
by 8 in each place it stands (twice in the second term), products by 3: below 2 * 2^-22 + 32 * 2^-24 = 10 * 2^-22 of the
terms' sizes; a term of dw by less than that.
"""

import numpy as np
import pytest
import torch

from _helpers import f64, require_gpu
from oracle import rope
from paper_2603_04427_gb300 import binding as tb

pytestmark = pytest.mark.gpu

F32, BF = torch.float32, torch.bfloat16
UNIT = 2.0 ** -22
EPS = 1e-5


@pytest.mark.parametrize("top", [64, 8192, 1 << 17, 1 << 20, 1 << 24])
def test_cos_and_sin(top):
    """Pairs (1, 0) turned: cos and sin themselves, over positions and frequencies."""
    require_gpu()
    g = np.random.default_rng(top)
    S = 20000
    pos = g.integers(-top, top + 1, S)
    pos[:4] = 0, top, -top, top - 1
    freq = np.float32(np.concatenate([10000.0 ** (-np.arange(32) / 32), g.uniform(-4, 4, 30), [4.0, -4.0]]))
    plan = tb.rope_plan(128, inv_freq=freq.tolist(), norm=False)
    x = torch.zeros(1, 1, S, 128, device="cuda")
    x[..., :64] = 1.0
    at = torch.tensor(pos, dtype=torch.int32, device="cuda")[None]
    got = f64(tb.tk_qk_norm_rope(plan, x, None, None, at, torch.empty_like(x), None, None)[0])[0, 0]
    assert tb.tk_get_device_error() == 0
    theta = pos[:, None] * freq[None].astype(np.float64)
    for what, a, b in (("cos", got[:, :64], np.cos(theta)), ("sin", got[:, 64:], np.sin(theta))):
        worst = np.abs(a - b).max()
        assert worst <= UNIT, f"{what}: 2^{np.log2(worst):.2f}"


def _case(B, S, H, r, rot, layout, axes, xt, seed):
    pairs = rot // 2
    plan = tb.rope_plan(r, rot_dim=rot, layout=layout, eps=EPS, inv_freq=[10000.0 ** (-j / max(1, pairs)) for j in range(pairs)],
                        pair_axis=[j % axes for j in range(pairs)])
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(B, H, S, r, generator=g) * torch.exp(torch.randn(B, H, S, 1, generator=g))).to(xt).cuda()
    w = (1 + 0.3 * torch.randn(r, generator=g)).cuda()
    pos = torch.randint(0, 131072, (axes, B, S), generator=g, dtype=torch.int32).cuda()
    theta = rope.angles(pos.cpu().numpy(), list(plan.inv_freq[:pairs]), list(plan.pair_axis[:pairs]))
    return plan, x, w, pos, theta


CASES = [(2, 37, 12, 16, 16, "half", 1), (1, 501, 5, 32, 32, "pair", 2), (3, 65, 8, 64, 24, "half", 3), (1, 1, 1, 128, 128, "half", 1),
         (2, 333, 8, 128, 64, "pair", 1), (1, 4097, 7, 32, 32, "half", 1)]


@pytest.mark.parametrize("xt", [F32, BF])
@pytest.mark.parametrize("B,S,H,r,rot,layout,axes", CASES)
def test_forward(B, S, H, r, rot, layout, axes, xt):
    require_gpu()
    plan, x, w, pos, theta = _case(B, S, H, r, rot, layout, axes, xt, seed=S)
    out = torch.empty(B, H, S, r, device="cuda")
    tb.tk_qk_norm_rope(plan, x, None, None, pos, out, None, None, q_weight=w)
    assert tb.tk_get_device_error() == 0
    y = rope.norm_rope(f64(x), f64(w), np.zeros_like(theta), rot, layout, True, EPS)
    ref = rope.rotate(y, theta, rot, layout)
    worst = (np.abs(f64(out) - ref) / np.abs(y).max(axis=-1, keepdims=True)).max()
    assert worst <= 6 * UNIT, f"{worst / UNIT:.2f} of 2^-22"


@pytest.mark.parametrize("gt", [F32, BF])
@pytest.mark.parametrize("B,S,H,r,rot,layout,axes", CASES)
def test_backward(B, S, H, r, rot, layout, axes, gt):
    require_gpu()
    plan, x, w, pos, theta = _case(B, S, H, r, rot, layout, axes, F32, seed=S)
    g = torch.randn(B, H, S, r, generator=torch.Generator().manual_seed(S + 1)).to(gt).cuda()
    dx, dw = torch.empty_like(x), torch.empty(r, device="cuda")
    tb.tk_qk_norm_rope_backward(plan, x, None, pos, g, None, None, dx, None, None, q_weight=w, dq_weight=dw)
    assert tb.tk_get_device_error() == 0
    ref, rw, terms, size = rope.norm_rope_backward(f64(x), f64(w), f64(g), theta, rot, layout, True, EPS)
    worst = (np.abs(f64(dx) - ref) / size).max()
    assert worst <= 10 * UNIT, f"{worst / UNIT:.2f} of 2^-22"
    # a term's g mixes the two elements of its pair: its size goes by the row's largest
    big = rope.rms(f64(x), EPS) * np.abs(f64(x)) * np.abs(f64(g)).max(axis=-1, keepdims=True)
    assert np.all(np.abs(f64(dw) - rw) <= 10 * UNIT * np.maximum(terms, big.sum(axis=(0, 1, 2))))


@pytest.mark.parametrize("xt,gt", [(BF, BF), (BF, F32), (F32, BF), (F32, F32)])
def test_cos_and_sin_in_weight_gradients(xt, gt):
    """One row of ones: dw is (cos, -sin) rho, in 32 bits for rows of any type.  rho = (1 + 2^-20)^(-1/2) is off by
    2^-25 + 2^-26, the product by 2^-25, the sums add zeros: with cos and sin below 1.5 * 2^-22."""
    require_gpu()
    r, eps = 128, 2.0 ** -20
    g = np.random.default_rng(4)
    freq = np.float32(np.concatenate([10000.0 ** (-np.arange(32) / 32), g.uniform(-4, 4, 32)]))
    plan = tb.rope_plan(r, inv_freq=freq.tolist(), eps=eps)
    x, dy = torch.ones(1, 1, 1, r, dtype=xt, device="cuda"), torch.zeros(1, 1, 1, r, dtype=gt, device="cuda")
    dy[..., :r // 2] = 1.0
    dx, ws = torch.empty_like(x), tb.qk_norm_rope_workspace(plan)
    for p in [0, 1, (1 << 24) - 1] + g.integers(-(1 << 17), 1 << 17, 200).tolist():
        at, dw = torch.tensor([[p]], dtype=torch.int32, device="cuda"), torch.empty(r, device="cuda")
        tb.tk_qk_norm_rope_backward(plan, x, None, at, dy, None, None, dx, None, None, dq_weight=dw, workspace=ws)
        theta = p * freq.astype(np.float64)
        ref = np.concatenate([np.cos(theta), -np.sin(theta)]) / np.sqrt(1 + eps)
        worst = np.abs(f64(dw) - ref).max()
        assert worst <= 1.5 * UNIT, f"position {p}: 2^{np.log2(worst):.2f}"
    assert tb.tk_get_device_error() == 0
