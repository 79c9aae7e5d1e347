import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def pytest_configure(config):
    config.addinivalue_line("markers", "gpu: needs an MI355X (gfx950) GPU and the built HIP library")


@pytest.fixture(scope="session")
def orc():
    """The CPU oracle (test infrastructure)."""
    from oracle import oracle as o
    o.lib()
    return o


def pytest_collection_modifyitems(items):
    for item in items:
        # Its caches are meant to lie one page behind the other (4096 bytes), but are given 2048 bytes apart: key i of
        # token t of head 1 of page p lies at byte 2 (4096 p + 1024 + 64 t + i) behind k_cache, and so does value i of
        # head 0, at 2048 + 2 (4096 p + 64 t + i).  Both are stored, so the call is refused.
        # (test_seq_overlaps.py has the call that was meant.)
        if item.nodeid.endswith("test_seq_ops.py::test_neighbours_are_no_overlap[base1-changes1]"):
            item.add_marker(pytest.mark.xfail(strict=True, reason="keys of head 1 and values of head 0 share their places"))
