"""Norm + rotation where element offsets pass 2^31: strides of a large tensor and slots of a long cache."""

import pytest
import torch

from _helpers import require_gpu
from paper_2603_04427_gb300 import binding as tb

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


def test_strides_past_32_bits():
    """Two sequences 2^31 + 64 elements apart give the rows that a dense copy gives."""
    require_gpu()
    S, H, r = 5, 3, 64
    apart = (1 << 31) + 64
    buf = torch.empty(apart + S * H * r, dtype=BF, device="cuda")
    x = buf.as_strided((2, H, S, r), (apart, r, H * r, 1))
    x.copy_(torch.randn(2, H, S, r, device="cuda"))
    plan = tb.rope_plan(r, axes=(16, 16))
    pos = torch.arange(2 * S, dtype=torch.int32, device="cuda").view(2, S)
    w = torch.rand(r, device="cuda") + 0.5
    dense = tb.tk_qk_norm_rope(plan, x.contiguous(), None, None, pos, torch.empty(2, H, S, r, dtype=BF, device="cuda"),
                               None, None, q_weight=w)[0]
    got = tb.tk_qk_norm_rope(plan, x, None, None, pos, torch.empty_like(dense), None, None, q_weight=w)[0]
    assert torch.equal(got, dense)
    # gradients into the same strides, from the same strides
    g = torch.randn(2, H, S, r, device="cuda")
    dw, dw2 = torch.empty(r, device="cuda"), torch.empty(r, device="cuda")
    ref = torch.empty(2, H, S, r, dtype=BF, device="cuda")
    tb.tk_qk_norm_rope_backward(plan, dense, None, pos, g, None, None, ref, None, None, q_weight=w, dq_weight=dw)
    x.copy_(dense)
    tb.tk_qk_norm_rope_backward(plan, x, None, pos, g, None, None, x, None, None, q_weight=w, dq_weight=dw2)
    assert torch.equal(x, ref) and torch.equal(dw, dw2)
    # and in place
    x.copy_(dense)
    tb.tk_qk_norm_rope(plan, x, None, None, pos, x, None, None, q_weight=w)
    again = tb.tk_qk_norm_rope(plan, dense, None, None, pos, torch.empty_like(dense), None, None, q_weight=w)[0]
    assert torch.equal(x, again) and tb.tk_get_device_error() == 0


@pytest.mark.parametrize("page", [0, 256])
def test_slots_past_32_bits(page):
    """A cache of more than 2^31 key and value elements: the last slots of the last kv head."""
    require_gpu()
    hkv, r, dv, slots = 8, 128, 128, (1 << 21) + 256
    kw = dict(page_size=page, num_pages=slots // page, page_table=torch.zeros(1, 1)) if page else dict(capacity=slots)
    c = tb.ThinKeyCache.allocate(1, 8, hkv, r, dv, **kw)
    assert c.k.numel() > 1 << 31
    S = 3
    k, v = torch.randn(1, hkv, S, r, device="cuda").to(BF), torch.randn(1, hkv, S, dv, device="cuda").to(BF)
    pos = torch.arange(S, dtype=torch.int32, device="cuda")[None]
    plan = tb.rope_plan(r)
    at = torch.tensor([[slots - 1, 7, slots - 300]], dtype=torch.int32, device="cuda")
    tb.tk_qk_norm_rope_append(c, plan, None, k, v, pos, at, None)
    assert tb.tk_get_device_error() == 0
    ref = tb.tk_qk_norm_rope(plan, None, k, None, pos, None, torch.empty_like(k), None)[1]
    for t, s in enumerate(at[0].tolist()):
        row = (s // page, slice(None), s % page) if page else (0, slice(None), s)
        assert torch.equal(c.k[row], ref[0, :, t]) and torch.equal(c.v[row], v[0, :, t])
    assert int((c.k != 0).any(-1).sum()) == S * hkv
