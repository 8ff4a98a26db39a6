"""The example layer: serving equals one prefill of the same tokens, training matches the fp64 chain."""

import importlib.util
import os

import numpy as np
import pytest
import torch

from _helpers import f64, require_gpu
from oracle import attention as oa
from oracle import rope
from paper_2603_04427_gb300 import binding as tb

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "rope_layer.py")


def _example():
    spec = importlib.util.spec_from_file_location("rope_layer", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_example_runs():
    require_gpu()
    # one bf16 unit of P (2^-8) times values of a few units, averaged over the context
    assert _example().main() <= 2e-2


@pytest.mark.parametrize("k_int8", [False, True])
def test_serving_reuses_pages(k_int8):
    """Requests come and go through a pool that holds them only because pages are given back."""
    require_gpu()
    m = _example()
    layer = m.Layer(d_model=128, h_q=8, h_kv=2, r=32, d_v=64, seed=3)
    server = m.Server(layer, 3, max_len=128, num_pages=15, k_int8=k_int8)
    g = torch.Generator(device="cuda").manual_seed(1)
    new = lambda n: torch.randn(n, 128, device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
    held = [new(60), new(17), new(90)]                  # 4 + 2 + 6 pages
    server.admit(held)
    for round_ in range(6):
        x = new(3)
        got = server.decode(x).clone()
        held = [torch.cat([h, x[b:b + 1]]) for b, h in enumerate(held)]
        for b, h in enumerate(held):
            pos = torch.arange(h.shape[0], dtype=torch.int32, device="cuda")[None]
            q, k, v = layer.rotated((h @ layer.w)[None], pos)
            out = torch.empty(1, 8, h.shape[0], 64, device="cuda")
            tb.tk_attn_prefill(q, k, v, out)
            # bf16 keys: P in bf16 on either side; int8 keys: half a step of each key
            assert float((out[0, :, -1] - got[b]).abs().max()) <= (6e-2 if k_int8 else 2e-2)
        gone = round_ % 3
        server.finish([gone])
        held[gone] = new(80 if round_ % 2 else 33)
        server.admit([held[b] if b == gone else None for b in range(3)])
    assert tb.tk_get_device_error() == 0
    owned = sum(-(-h.shape[0] // 16) for h in held)
    assert server.pool.free_count.item() == 15 - owned
    with pytest.raises(RuntimeError):                   # a prompt that the pool does not hold
        server.finish([0])
        server.admit([new(128), None, None])
        server.admit([None, new(100), None])


def test_train_step_gradients():
    require_gpu()
    m = _example()
    layer = m.Layer(d_model=64, h_q=4, h_kv=2, r=32, d_v=64, seed=5)
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn(1, 70, 64, device="cuda", generator=g).to(torch.bfloat16)
    do = torch.randn(1, 4, 70, 64, device="cuda", generator=g).to(torch.bfloat16)
    _, d_packed, dwq, dwk = m.train_step(layer, x, do)
    q, k, v = (f64(t) for t in layer.heads(x @ layer.w))
    pairs = layer.plan.rot_dim // 2
    theta = rope.angles(np.arange(70)[None, None], list(layer.plan.inv_freq[:pairs]), [0] * pairs)
    Q, K = (rope.norm_rope(t, f64(w), theta, 32, "half") for t, w in ((q, layer.norm_q), (k, layer.norm_k)))
    gq, gk, gv = oa.attention_backward(Q, K, v, f64(do), 1 / np.sqrt(32))
    dq, wq, _, _ = rope.norm_rope_backward(q, f64(layer.norm_q), gq, theta, 32, "half")
    dk, wk, _, _ = rope.norm_rope_backward(k, f64(layer.norm_k), gk, theta, 32, "half")
    # the attention's bar for gradients (bf16 P and dS) plus bf16 inputs and outputs
    for got, ref in zip(layer.heads(d_packed), (dq, dk, gv)):
        assert np.abs(f64(got) - ref).sum() <= 1.4e-2 * np.abs(ref).sum()
    for got, ref in ((dwq, wq), (dwk, wk)):
        assert np.abs(f64(got) - ref).sum() <= 3e-2 * np.abs(ref).sum()
