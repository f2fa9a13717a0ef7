"""pages_reserve refuses lists that overlap where one row's answer would be another row's question (no GPU)."""
import ctypes

import pytest

from paper_2509_25224_b200 import binding, build

P, Z = ctypes.c_void_p, ctypes.c_void_p(0)
B, BLOCKS, WIDTH = 8, 100, 4
SEQLENS, NEW, GRANTED = 1 << 20, 1 << 21, 1 << 22       # (addresses that no call here gets to use)


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def reserve(lib, new=NEW, granted=GRANTED, size=0):
    # a workspace that is too small is refused too, so that what is in order otherwise launches nothing
    return lib.amla_pages_reserve(P(1 << 23), P(SEQLENS), P(1 << 24), P(new), B, BLOCKS, WIDTH, P(granted), P(1 << 25), size, Z)


@pytest.mark.parametrize("at", [-(B - 1), -1, 0, 1, B - 1])
def test_lists_that_overlap(lib, at):
    n = ctypes.c_size_t(0)
    assert lib.amla_pages_workspace_size(BLOCKS, B, ctypes.byref(n)) == 0
    assert reserve(lib, new=SEQLENS + 4 * at) == -1
    assert reserve(lib, granted=SEQLENS + 4 * at, size=n.value) == -1
    assert at == 0 or reserve(lib, granted=NEW + 4 * at, size=n.value) == -1


@pytest.mark.parametrize("at", [-B, B])
def test_lists_that_lie_side_by_side(lib, at):
    assert reserve(lib, new=SEQLENS + 4 * at) == -3
