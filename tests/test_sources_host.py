"""CPU checks of the kernels' sources."""
import glob
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCES = sorted(f for e in ("*.cu", "*.cuh", "*.cc", "*.h")
                 for f in glob.glob(os.path.join(ROOT, "paper_2608_28003_gb300", "csrc", e)) +
                 glob.glob(os.path.join(ROOT, "include", e)))


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_no_bulk_copy_to_several_ctas(path):
    """The library runs as replicas on any number of GPUs, so no copy of it is a multicast to a cluster (commits of the
    tensor cores' work may arrive at several CTAs)."""
    text = re.sub(r'"\s*"', "", open(path).read())  # adjacent string literals are one
    assert not re.search(r'cp\.async\.bulk[^"]*\.multicast', text)


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_no_shuffle_among_whoever_is_active(path):
    """The lanes of a warp's exchange follow from a condition, never from which of them happen to run together."""
    assert "__activemask" not in open(path).read()
