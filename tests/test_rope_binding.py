"""Host side of the norm + rotation and page-table calls: plans and checks of arguments, without a launch."""

import pytest
import torch

from paper_2603_04427_gb300 import binding as tb


def test_every_axis_of_a_plan_counts():
    """An axis without pairs still has its row of positions."""
    for axes in [(8, 8, 0), (0, 8, 8), (16, 0, 0, 0), (8, 0, 8), (16,)]:
        assert tb.rope_plan(32, axes=axes).n_axes == len(axes), axes
    p = tb.rope_plan(32, axes=(8, 8, 0))
    assert list(p.pair_axis[:16]) == [0] * 8 + [1] * 8
    pos = torch.zeros(3, 2, 5, dtype=torch.int32)
    assert tb._positions(p, pos, 2, 5, pos.device)[1:] == (10, 5)
    # pairs of other axes than their frequencies' runs
    assert tb.rope_plan(32, axes=(8, 8), pair_axis=[2] * 16).n_axes == 3
    assert tb.rope_plan(32, rot_dim=0, axes=()).n_axes == 1
    with pytest.raises(ValueError):
        tb.rope_plan(32, axes=(4, 4, 4, 4, 0))


class _On:
    """What the checks ask of a CUDA tensor, for one on the GPU of index `at`."""

    is_cuda = True

    def __init__(self, shape, dtype, at):
        self.shape, self.dtype, self.device, self._at = torch.Size(shape), dtype, torch.device("cuda", at), at

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def get_device(self):
        return self._at

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x10000

    def stride(self):
        out = [1]
        for n in reversed(self.shape[1:]):
            out.insert(0, out[0] * n)
        return tuple(out)


@pytest.mark.parametrize("current,at", [(0, 1), (1, 0)])
def test_tensors_of_another_gpu_than_the_current_one_are_refused(monkeypatch, current, at):
    """A call takes its stream from the tensors' GPU and is launched on the current one: they must be the same."""
    def launched(*_):
        raise AssertionError("the library was called")

    monkeypatch.setattr(tb, "_current_device", lambda: current)
    monkeypatch.setattr(tb, "load_library", launched)
    monkeypatch.setattr(tb, "_raw_stream", lambda stream, device: 0)
    B, H, S, r, dv = 2, 4, 3, 32, 64
    bf = torch.bfloat16
    x, v = _On((B, H, S, r), bf, at), _On((B, H, S, dv), bf, at)
    pos, slots = _On((B, S), torch.int32, at), _On((B, S), torch.int32, at)
    plan = tb.rope_plan(r)
    i32 = lambda *n: _On(n, torch.int32, at)  # noqa: E731
    cache = tb.ThinKeyCache(tb.tk_cache_desc(B, H, H, r, dv, 16, 0, 0, 0, tb.TK_BF16),
                            _On((B, H, 16, r), bf, at), _On((B, H, 16, dv), bf, at))
    pool = tb.PagePool(16, i32(B, 4), i32(8), i32(1), i32(B), i32(1))
    for call in (
            lambda: tb.tk_qk_norm_rope(plan, x, x, v, pos, x, x, v),
            lambda: tb.tk_qk_norm_rope_append(cache, plan, x, x, v, pos, slots, x),
            lambda: tb.prepare_qk_norm_rope_append(cache, plan, x, x, v, pos, slots, x),
            lambda: tb.tk_qk_norm_rope_backward(plan, x, x, pos, x, x, v, x, x, v),
            lambda: tb.qk_norm_rope_workspace(plan, torch.device("cuda", at)),
            lambda: tb.tk_block_tables(pool, i32(B), i32(6), i32(6)),
            lambda: tb.prepare_block_tables(pool, i32(B), i32(6), i32(6))):
        with pytest.raises(ValueError, match="current"):
            call()
