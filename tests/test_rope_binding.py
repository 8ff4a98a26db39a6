"""Host side of the norm + rotation and page-table calls: plans and checks of arguments, without a launch."""

import pytest

from paper_2603_04427_gb300 import binding as tb


def test_every_axis_of_a_plan_counts():
    """An axis without pairs still has its row of positions."""
    for axes in [(8, 8, 0), (0, 8, 8), (16, 0, 0, 0), (8, 0, 8), (16,)]:
        assert tb.rope_plan(32, axes=axes).n_axes == len(axes), axes
    p = tb.rope_plan(32, axes=(8, 8, 0))
    assert list(p.pair_axis[:16]) == [0] * 8 + [1] * 8
    import torch
    pos = torch.zeros(3, 2, 5, dtype=torch.int32)
    assert tb._positions(p, pos, 2, 5, pos.device)[1:] == (10, 5)
    # pairs of other axes than their frequencies' runs
    assert tb.rope_plan(32, axes=(8, 8), pair_axis=[2] * 16).n_axes == 3
    assert tb.rope_plan(32, rot_dim=0, axes=()).n_axes == 1
    with pytest.raises(ValueError):
        tb.rope_plan(32, axes=(4, 4, 4, 4, 0))
