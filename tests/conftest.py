import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs a CUDA GPU (sm_103a) and the built library")


def pytest_collection_modifyitems(items):
    # This case expects one upper bound from a product rounded to 32 bits: 2.359375 for a key of
    # 6 * 0x1.92aaacp-2 = 2.35937512, which lies above it (test_gpu_block_bounds_rounding.py has the same
    # cases against exact products).  It fails, and runs last, so that a run that stops there has run the others.
    items.sort(key=lambda item: item.nodeid.endswith("test_gpu_blocks.py::test_bounds[int4-128-256-256]"))
