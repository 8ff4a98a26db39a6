"""Weights that a BudgetServer (examples/long_context.py) starts prompts with, against the float64 oracle:
prompts shorter than the window of queries, first ones and ones that go on from cached tokens."""

import importlib.util
import math
import os

import numpy as np
import pytest
import torch

from _helpers import f64, require_gpu
from oracle import long_context as lc
from paper_2603_04427_gb300 import binding as tb

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    require_gpu()
    spec = importlib.util.spec_from_file_location("long_context", os.path.join(ROOT, "examples", "long_context.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    tb.tk_get_device_error()
    yield m
    assert tb.tk_get_device_error() == 0


@pytest.mark.parametrize("window", [8, 16])
def test_each_prompt_adds_its_own_queries(ex, window):
    layer = ex.Layer(d_model=128, h_q=8, h_kv=2, r=32, d_v=64, seed=3)
    s = ex.BudgetServer(layer, 4, 192, keep=180, recent=8, window=window)
    gen = torch.Generator(device="cuda").manual_seed(2)
    seen = [[] for _ in range(4)]
    want = [np.zeros((2, 0)) for _ in range(4)]
    for lens in ([40, 3, 17, None], [5, 30, None, 8], [1, 16, 2, 7], [None, 1, None, None]):
        new = [None if n is None else torch.randn(n, 128, device="cuda", generator=gen).to(torch.bfloat16) for n in lens]
        s.admit(new)
        keys = f64(s.cache.k)
        for b, x in enumerate(new):
            if x is None:
                continue
            seen[b].append(x)
            L, n = sum(len(t) for t in seen[b]), min(window, len(x))
            pos = torch.arange(L - n, L, dtype=torch.int32, device="cuda")
            q = f64(layer.rotated((x[-n:] @ layer.w)[None], pos[None])[0][0])
            want[b] = np.pad(want[b], ((0, 0), (0, L - want[b].shape[1])))
            for g in range(2):
                k = np.concatenate([keys[p, g] for p in s.pool.page_table[b, :-(-L // 16)].tolist()])[:L]
                want[b][g] += lc.attn_weights(q[4 * g:4 * g + 4], k, 1 / math.sqrt(32), n)
        for b in range(4):
            L = want[b].shape[1]
            got = np.zeros((2, 0)) if L == 0 else np.concatenate(
                [f64(s.weights[p]) for p in s.pool.page_table[b, :-(-L // 16)].tolist()], 1)[:, :L]
            # weights are within 1e-5 of themselves (test_gpu_attn_weights.py), at most four sums of them
            assert np.abs(got - want[b]).max(initial=0) <= 2e-5 * max(1.0, want[b].max(initial=0)), (lens, b)
