"""What the shared-prefix attention and the prompt's calls promise that shows without a GPU: in their sources, and in what the binding refuses."""
import glob
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2509_15235_b200", "csrc")


def test_barriers_are_arrived_at_with_release():
    """The products that overwrite an accumulator start behind the arrivals of the threads that have read it: arrivals that order nothing
    (.relaxed) would leave that to the hardware."""
    sources = glob.glob(os.path.join(CSRC, "*.cu")) + glob.glob(os.path.join(CSRC, "*.cuh"))
    assert sources
    for path in sources:
        assert not re.search(r"mbarrier\.arrive[.\w]*\.relaxed", open(path).read()), path
