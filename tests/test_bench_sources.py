"""The traffic record of bench.py goes with the source that the decode kernel is built from."""

import os
import re

import bench

CSRC = os.path.dirname(bench.KERNEL_SOURCES[0])


def test_kernel_sources_are_all_that_the_kernel_includes():
    """A record taken on other code than the kernel runs must not be accepted: cmc_attn.cu and every
    file of csrc that it includes, directly or not."""
    found, ahead = set(), ["cmc_attn.cu"]
    while ahead:
        name = ahead.pop()
        if name in found:
            continue
        found.add(name)
        with open(os.path.join(CSRC, name)) as f:
            ahead += [n for n in re.findall(r'^#include "([^"/]+)"', f.read(), flags=re.M)]
    assert {os.path.basename(p) for p in bench.KERNEL_SOURCES} == found
