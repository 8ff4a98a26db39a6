"""Attention weights of scores far from zero, where a row's maximum is hundreds of log2 units and its
tokens differ by a few: the weights' error goes by the differences, not by the maximum.

Scores are whole numbers below 2^24, so every product and sum of them is exact.  What is left, with
D the largest distance of a score to its row's maximum in log2 units (below 10 here):
  the factor scale log2(e) is rounded twice (its constant and the product), 2^-23 of a distance;
  scale s - maximum is rounded once, 2^-24 D (the maximum's own rounding is common to a row's weights
    and their sum, and cancels);
  each in a weight and, averaged, in its sum: 2 ln2 (2^-23 + 2^-24) D;
  two exponentials of 2^-22, the join's too (2^-22 each time ranges meet, two levels);
  sums of positive terms: 2^-24 for each term that a thread adds in turn at most where they are all
    alike; a thread adds at most 16 of a step, then one a step (T steps), 5 levels of lanes and 4 of
    warps, ranges and row sums 10: (T + 35) 2^-24."""

import math

import numpy as np
import pytest
import torch

from _helpers import require_gpu
from paper_2603_04427_gb300 import binding as tb

pytestmark = pytest.mark.gpu

# scales with which 509 scale log2(e), rounded to 32 bits, is off by nearly half a unit
SCALES = [0.705, 0.7072, 0.7039]


@pytest.fixture(autouse=True)
def _clean():
    require_gpu()
    tb.tk_get_device_error()
    yield
    assert tb.tk_get_device_error() == 0


def _run(B, G, n_q, r, cap, L, scale):
    """Weights and expected weights of sequence 0, whose scores are 509 - (0 .. 8)."""
    desc = tb.tk_cache_desc(B, G, 1, r, 64, cap, 0, 0, 0, tb.TK_BF16)
    keys = torch.zeros(B, 1, cap, r, device="cuda", dtype=torch.bfloat16)
    gen = torch.Generator(device="cuda").manual_seed(L)
    less = torch.randint(0, 9, (L,), device="cuda", generator=gen)
    less[::7] = 0                                       # the maximum, in every range
    keys[0, 0, :L, 0] = 16
    keys[0, 0, :L, 3] = -(less + 3).to(keys.dtype)
    c = tb.ThinKeyCache(desc, keys, None, None, None)
    q = torch.zeros(B, G, n_q, r, device="cuda", dtype=torch.bfloat16)
    q[..., 0], q[..., 3] = 32.0, 1.0
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    lens[0] = L
    w = tb.slot_weights(c)
    tb.tk_attn_weights(c, q, lens, cap, w, tb.attn_weights_workspace(c, cap, n_q), scale=scale)
    torch.cuda.synchronize()
    x = -less.double().cpu().numpy() * float(np.float32(scale))
    e = np.exp(x)
    want = np.zeros(L)
    for i in range(n_q):
        last = L - n_q + i + 1
        if last > 0:
            want[:last] += G * e[:last] / e[:last].sum()
    return w[0, 0, :L].double().cpu().numpy(), want


def _tol(steps, scale):
    D = 8 * scale * math.log2(math.e)
    return 2 * math.log(2) * (2.0 ** -23 + 2.0 ** -24) * D + 4 * 2.0 ** -22 + (steps + 35) * 2.0 ** -24


@pytest.mark.parametrize("scale", SCALES)
@pytest.mark.parametrize("B,G,n_q,r,cap,L,steps", [
    (2, 8, 1, 32, 4096, 4096, 8),              # one query in one launch
    (304, 8, 1, 16, 65536, 65536, 128),        # with its scores kept: steps of 512 tokens
    (304, 4, 3, 32, 16384, 16381, 32),         # more on mma.sync
    (304, 8, 2, 64, 16384, 16000, 63),
    (152, 8, 16, 16, 16384, 16384, 64),        # on tcgen05: two groups in turn, tiles of 128 tokens
    (152, 8, 8, 64, 16384, 15999, 63)])
def test_sums_over_many_steps(B, G, n_q, r, cap, L, steps, scale):
    """One range holds a whole context: a thread's running sum goes through many steps, whose maximum is
    the same."""
    got, want = _run(B, G, n_q, r, cap, L, scale)
    err = np.abs(got / want - 1).max()
    assert err <= _tol(steps, scale), (err, _tol(steps, scale))


@pytest.mark.parametrize("scale", SCALES + [0.5, 0.9])
@pytest.mark.parametrize("G,n_q,r,L", [(8, 16, 16, 100), (8, 6, 64, 128), (4, 8, 128, 90), (8, 64, 32, 128)])
def test_tiles_of_many_queries_of_one_step(G, n_q, r, L, scale):
    """Products on tcgen05, every row in one step: what is left is how its maximum and sum are kept."""
    got, want = _run(1, G, n_q, r, 128, L, scale)
    err = np.abs(got / want - 1).max()
    assert err <= _tol(1, scale), (err, _tol(1, scale))


@pytest.mark.parametrize("n_q", [1, 3, 16])
@pytest.mark.parametrize("size", [1e2, 1e3, 1e4])
def test_scores_up_to_the_largest(n_q, size):
    """Random keys and queries of a size that gives scores of up to 6e8 log2 units (below 2^30): a row has
    nearly all of its weight on one token, and a sum of one."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    desc = tb.tk_cache_desc(1, 8, 1, 32, 64, 112, 0, 0, 0, tb.TK_BF16)
    keys = (size * torch.randn(1, 1, 112, 32, device="cuda", generator=gen)).to(torch.bfloat16)
    q = (size * torch.randn(1, 8, n_q, 32, device="cuda", generator=gen)).to(torch.bfloat16)
    c = tb.ThinKeyCache(desc, keys, None, None, None)
    w = tb.slot_weights(c)
    tb.tk_attn_weights(c, q, torch.tensor([100], dtype=torch.int32, device="cuda"), 100, w,
                       tb.attn_weights_workspace(c, 100, n_q))
    w = w[0, 0].double().cpu().numpy()
    x = np.abs((q[0].double() @ keys[0, 0, :100].double().T).cpu().numpy()).max() / math.sqrt(32) * math.log2(math.e)
    assert x < 2.0 ** 30 and (w >= 0).all() and (w[100:] == 0).all()
    # a row's weights are its terms over their own sum: two exponentials, the sums' levels and the
    # division, all of them positive
    assert abs(w.sum() / (8 * n_q) - 1) <= 4 * 2.0 ** -22 + 40 * 2.0 ** -24
