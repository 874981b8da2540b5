"""The committed counters are of the kernels as they are: bench.py takes none of other sources."""
import glob
import os
import re

import pytest

import bench

SUMMARIES = sorted(glob.glob(os.path.join(bench.ROOT, "profiles", "pmc_*.md")))


def test_there_are_summaries():
    assert SUMMARIES


@pytest.mark.parametrize("path", SUMMARIES, ids=os.path.basename)
def test_digest_is_that_of_the_sources(path):
    found = re.findall(r"kernel sources: (\w+)", open(path).read())
    assert found == [bench.source_digest()], "kernels changed: collect the counters again"
