"""bench.py reports recorded memory traffic only while the sources that the counters were taken of are the same:
every file of the kernels' folder that they are compiled from has to be among those it looks at (the public header
declares entry points and numbers of the interface)."""
import os
import re

import bench

CSRC = os.path.join(bench.ROOT, "paper_2609_36932_amd", "csrc")


def _included(name, seen):
    if name not in seen and name in os.listdir(CSRC):
        seen.add(name)
        for inc in re.findall(r'^#include "([^"]+)"', open(os.path.join(CSRC, name)).read(), re.M):
            _included(inc, seen)
    return seen


def test_every_source_of_the_measured_kernels_counts():
    assert {os.path.basename(f) for f in bench.KERNEL_SRCS} >= _included("lmhead.hip", set())
