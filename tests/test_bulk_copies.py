"""Where the sources' bulk copies go (CPU: reads the sources)."""
import os
import re

import pytest

import paper_1905_00689_gb300 as package

CSRC = os.path.join(os.path.dirname(package.__file__), "csrc")


@pytest.mark.parametrize("name", sorted(f for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh", ".h", ".cpp"))))
def test_loads_go_to_the_block_that_asks(name):
    """No load from global memory is sent to several blocks of a cluster at once: the sources serve programs on several GPUs
    too, where such a load may reach another GPU's memory.  Each block loads for itself."""
    with open(os.path.join(CSRC, name)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    assert "multicast" not in text


@pytest.mark.parametrize("name", sorted(f for f in os.listdir(CSRC) if f.endswith((".cu", ".cuh"))))
def test_arrivals_at_other_blocks_order_for_the_cluster(name):
    """An arrival at another block's barrier, after which that block may overwrite what this one read, is a release for the
    whole cluster (the instruction's default), not for the block alone."""
    with open(os.path.join(CSRC, name)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    for m in re.finditer(r"mbarrier\.arrive[\w.:]*shared::cluster[\w.:]*", text):
        assert ".release.cta" not in m.group(), m.group()
