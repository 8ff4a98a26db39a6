"""Bounds of quantised keys against the exact products code * scale: the nearest bf16 numbers on the outer
side, also where a product rounded to 32 bits would be a bf16 number itself."""

import numpy as np
import pytest
import torch

from _helpers import f64, require_gpu
from _long_context import Cache
from oracle import long_context as lc
from paper_2603_04427_gb300 import binding as tb

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _clean():
    require_gpu()
    tb.tk_get_device_error()
    yield
    assert tb.tk_get_device_error() == 0


def _check(x, block):
    box = tb.block_bounds(x.c, block)
    tb.tk_block_bounds(x.c, box, x.seq, block=block)
    got, keys, rounded = f64(box).reshape(-1, 2, x.r), x.keys64(), x.keys32().astype(np.float64)
    inside = 0
    for b in range(x.B):
        for g in range(x.h_kv):
            rows = x.rows(b, g)
            if len(rows) == 0:
                continue
            at = rows[::block] // block
            want = np.stack(lc.block_bounds(keys[rows], block, True), 1)
            assert np.array_equal(got[at], want), (b, g)
            inside += (want != np.stack(lc.block_bounds(rounded[rows], block, True), 1)).sum()
            assert (got[rows // block, 0] <= keys[rows]).all() and (keys[rows] <= got[rows // block, 1]).all()
    return inside


def test_a_product_that_rounds_to_a_bf16_number():
    """-96 * 0x1.5d5554p-6 is -2.04687488; the fp32 number nearest to it is the bf16 number -2.046875."""
    x = Cache([16], 1, 1, 32, 64, 16, 0, "int8", seed=1)
    x.c.k.fill_(-96)
    x.c.k_scale.fill_(float.fromhex("0x1.5d5554p-6"))
    box = tb.block_bounds(x.c, 16)
    tb.tk_block_bounds(x.c, box, x.seq, block=16)
    assert (box[..., 0, :] == -2.046875).all() and (box[..., 1, :] == -2.03125).all()
    _check(x, 16)


@pytest.mark.parametrize("k,r,block,ps", [
    ("int8", 16, 32, 0), ("int8", 32, 16, 16), ("int8", 64, 256, 0), ("int8", 128, 64, 64), ("int4", 32, 16, 0),
    ("int4", 64, 64, 64), ("int4", 128, 256, 256)])
def test_bounds(k, r, block, ps):
    lens = [0, 1, block - 1, block, block + 1, 5 * block + 3, 8 * block]
    _check(Cache(lens, 6, 3, r, 64, 8 * block, ps, k, seed=r + block), block)


def test_many_bounds():
    """Blocks enough for products that 32 bits would bring inside."""
    assert sum(_check(Cache([8192] * 4, 2, 2, 64, 64, 8192, 0, "int8", seed=s), 16) for s in range(4)) > 0


def test_scales_at_the_ends_of_the_range():
    """Products beyond the largest number, and in the subnormal range, where products and bounds lose bits."""
    x = Cache([512], 1, 1, 32, 64, 512, 0, "int8", seed=5)
    with torch.no_grad():
        for i, s in enumerate((3e38, 1e37, 1e-36, 3e-38, 1e-39, 7e-43, 1.4e-45, 0.0)):
            x.c.k_scale[0, 0, 64 * i:64 * i + 64] = s
    _check(x, 16)
