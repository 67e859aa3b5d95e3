"""CPU: the sources by whose hash bench.py takes a kernel's committed counters for present ones are all that its device code
stands in."""
import os
import re

import pytest

import bench

CSRC = os.path.join("paper_2606_01839_amd", "csrc")


def _read(path):
    with open(os.path.join(bench.ROOT, path)) as f:
        return f.read()


def _device_headers(path, seen):
    for name in re.findall(r'#include "([^"]+)"', _read(path)):
        header = os.path.join(CSRC, name)
        if header not in seen and os.path.exists(os.path.join(bench.ROOT, header)):
            seen.add(header)
            _device_headers(header, seen)
    return {h for h in seen if "__device__" in _read(h)}


@pytest.mark.parametrize("group", list(bench.KERNEL_SOURCES))
def test_hash_covers_device_code(group):
    sources = bench.KERNEL_SOURCES[group]
    kernels = [s for s in sources if s.endswith(".hip")]
    assert kernels
    assert set().union(*(_device_headers(k, set()) for k in kernels)) <= set(sources)
