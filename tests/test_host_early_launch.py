"""Kernels that are launched while the one before them still runs read global memory by plain loads: read-only ones may be moved above
the wait for that kernel, or find a line that was cached before it."""
import glob
import os
import re

import pytest

from paper_2411_00288_b200 import build


def _kernels():
    """(file, name, text up to the closing brace) of every kernel in the sources."""
    for path in sorted(glob.glob(os.path.join(build.CSRC, "*.cu"))):
        with open(path) as f:
            text = f.read()
        for start in re.finditer(r"__global__", text):
            body = text[start.start():text.index("\n}\n", start.start())]
            yield os.path.basename(path), re.search(r"\b\w+_kernel(?=\()", body).group(0), body


WAITING = [k for k in _kernels() if "grid_dependency_wait()" in k[2]]


def test_the_kernels_are_found():
    assert len(WAITING) >= 20
    assert {f for f, _, _ in WAITING} >= {"forward.cu", "wgrad.cu", "optim.cu", "resnorm.cu", "mxfp4.cu"}


@pytest.mark.parametrize("file,name,body", WAITING, ids=[f"{f}:{n}" for f, n, _ in WAITING])
def test_no_read_only_load_behind_a_wait(file, name, body):
    assert "__ldg" not in body and "ld.global.nc" not in body
