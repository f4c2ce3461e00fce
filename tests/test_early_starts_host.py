"""Kernels of the 4-bit cache start while those in front of them still write what they read (programmatic serialization): pools, lens, queries.  The
read-only path is for what does not change while a kernel is resident, and its loads are not held back by the wait."""
import glob
import os

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2407_19775_b200", "csrc")


@pytest.mark.parametrize("name", sorted(os.path.basename(p) for p in glob.glob(os.path.join(CSRC, "bqkv_*.cu*"))))
def test_no_read_only_loads(name):
    assert "__ldg(" not in open(os.path.join(CSRC, name)).read()
