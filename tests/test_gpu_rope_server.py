"""The example's server when requests do not fit or are finished."""

import importlib.util
import os

import pytest
import torch

from _helpers import require_gpu
from paper_2603_04427_gb300 import binding as tb

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "rope_layer.py")


def _server(batch, max_len, num_pages):
    spec = importlib.util.spec_from_file_location("rope_layer", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    layer = m.Layer(d_model=128, h_q=8, h_kv=2, r=32, d_v=64, seed=3)
    g = torch.Generator(device="cuda").manual_seed(1)
    new = lambda n: torch.randn(n, 128, device="cuda", generator=g).to(torch.bfloat16)  # noqa: E731
    return m.Server(layer, batch, max_len=max_len, num_pages=num_pages), new


def _state(server):
    return server.pool.seq_lens.tolist(), server.pool.free_count.item()


def _is_last_row_of_prefill(server, tokens, got):
    layer, n = server.layer, tokens.shape[0]
    q, k, v = layer.rotated((tokens @ layer.w)[None], torch.arange(n, dtype=torch.int32, device="cuda")[None])
    out = torch.empty(1, 8, n, 64, device="cuda")
    tb.tk_attn_prefill(q, k, v, out)
    # P in bf16 on either side (tests/test_gpu_rope_layer.py)
    assert float((out[0, :, -1] - got).abs().max()) <= 2e-2


@pytest.mark.parametrize("max_len,num_pages", [(64, 3), (64, 4), (32, 8)])
def test_decode_step_that_does_not_fit(max_len, num_pages):
    """No page left, a page for one of two, a full row of the page table: the step raises and changes nothing, and
    can be made once a request has finished."""
    require_gpu()
    server, new = _server(2, max_len, num_pages)
    held = [new(32), new(16)]                          # 2 + 1 full pages
    server.admit(held)
    before = _state(server)
    assert before == ([32, 16], num_pages - 3)
    x = new(2)
    for _ in range(2):
        with pytest.raises(RuntimeError):
            server.decode(x)
        assert _state(server) == before
    server.finish([0])
    got = server.decode(x)
    _is_last_row_of_prefill(server, torch.cat([held[1], x[1:]]), got[1])
    assert tb.tk_get_device_error() == 0


def test_finished_sequence_stays_empty():
    """Its place in the batch takes no tokens and no pages until a prompt is admitted to it."""
    require_gpu()
    server, new = _server(2, 64, 8)
    held = new(40)
    server.admit([new(20), held])
    server.finish([0])
    assert _state(server) == ([0, 40], 5)
    for i in range(3):
        x = new(2)
        held = torch.cat([held, x[1:]])
        got = server.decode(x)
        assert _state(server) == ([0, 41 + i], 5)
        assert bool((got[0] == 0).all())
        _is_last_row_of_prefill(server, held, got[1])
    prompt, x = new(5), new(2)
    server.admit([prompt, None])
    got = server.decode(x)
    _is_last_row_of_prefill(server, torch.cat([prompt, x[:1]]), got[0])
    assert _state(server)[0] == [6, 44] and tb.tk_get_device_error() == 0


def test_refused_prompts_change_nothing():
    """A call whose second prompt does not fit leaves the first one out too, and it can be admitted later."""
    require_gpu()
    server, new = _server(2, 64, 4)
    prompt = new(20)
    for _ in range(2):
        with pytest.raises(RuntimeError):
            server.admit([prompt, new(40)])            # 2 + 3 pages
        assert _state(server) == ([0, 0], 4)
    server.admit([prompt, None])
    assert _state(server) == ([20, 0], 2)
    x = new(2)
    got = server.decode(x)
    _is_last_row_of_prefill(server, torch.cat([prompt, x[:1]]), got[0])
    with pytest.raises(RuntimeError):                  # one more chunk than the row holds
        server.admit([new(50), None])
    assert _state(server)[0][0] == 21 and tb.tk_get_device_error() == 0
