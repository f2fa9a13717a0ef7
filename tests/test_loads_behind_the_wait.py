"""Kernels that are placed while the kernel in front of them is still writing (programmatic launch) read its results by ordinary loads.

A non-coherent load (__ldg, or what the compiler makes of a pointer to const __restrict__) promises that nobody writes the place while the
kernel lives, and a __restrict__ pointer that nobody writes it by another name: neither holds for a block table, a length, a count, a
token or a page that the kernel in front brings up to date, and both let a load be moved ahead of griddepcontrol.wait.
"""
import glob
import os
import re

import pytest

from paper_2509_25224_b200 import build

NO_PROMISES = re.compile(r"__restrict__|__ldg\b|ld\.global\.nc")


def kernels(path):
    """(what stands in front of the first kernel, [each kernel with what follows it])"""
    text = re.sub(r"//[^\n]*", "", open(path).read())
    head, *rest = text.split("__global__")
    return head, rest


def waits(kernel):
    return "griddepcontrol.wait" in kernel or re.search(r"\bbegin\(\);", kernel) is not None


@pytest.mark.parametrize("path", sorted(glob.glob(os.path.join(build.CSRC, "*.cu"))), ids=os.path.basename)
def test_kernels_that_wait_promise_nothing(path):
    head, rest = kernels(path)
    waiting = [k for k in rest if waits(k)]
    for k in waiting + ([head] if waiting else []):
        assert not NO_PROMISES.search(k), k[:200]


def test_headers_promise_nothing():
    for path in glob.glob(os.path.join(build.CSRC, "*.cuh")):
        assert not NO_PROMISES.search(re.sub(r"//[^\n]*", "", open(path).read())), path


def test_the_kernels_that_wait_are_found():
    found = {os.path.basename(p) for p in glob.glob(os.path.join(build.CSRC, "*.cu")) if any(waits(k) for k in kernels(p)[1])}
    assert found == {"amla_decode_few.cu", "amla_decode_fp4.cu", "amla_decode_pair.cu", "amla_decode_quad.cu", "amla_fp4.cu", "amla_pages.cu", "amla_plan_combine.cu"}
