"""A cache that runs full: who is served and who is not, on a GPU against the rule, one request at a time, in numpy."""
import numpy as np
import pytest
import torch

import _fp4_util as F
from paper_2509_25224_b200 import paging

pytestmark = pytest.mark.gpu


def reserve(table, lens, refs, new):
    """The rule of amla_pages_reserve: rows in order take the lowest free pages; a row that is refused takes none."""
    table, lens, refs, granted = table.copy(), lens.copy(), refs.copy(), []
    pool = [int(p) for p in np.flatnonzero(refs <= 0)]
    at = 0
    for b, then in enumerate(new):
        have, want = F.pages_of(lens[b]), F.pages_of(then)
        more = max(0, want - have)
        if then > table.shape[1] * F.PAGE or more > len(pool) - at:
            granted.append(0)
            continue
        for i in range(more):
            table[b, have + i] = pool[at + i]
            refs[pool[at + i]] = 1
        at += more
        lens[b] = max(lens[b], then)
        granted.append(1)
    return table, lens, refs, np.array(granted, np.int32)


def check(table, lens, refs, new):
    t, n, r = (torch.from_numpy(x.copy()).cuda() for x in (table, lens, refs))
    got = paging.pages_reserve(t, n, r, torch.from_numpy(np.array(new, np.int32)).cuda())
    want = reserve(table, lens, refs, new)
    for have, should in zip((t, n, r, got), want):
        assert np.array_equal(have.cpu().numpy(), should)
    return want[3]


def empty(rows, blocks, width, free):
    """Rows without pages, and a cache of which `free` pages, spread over it, are free."""
    refs = np.ones(blocks, np.int32)
    refs[np.random.default_rng(rows + blocks).permutation(blocks)[:free]] = 0
    return np.full((rows, width), -1, np.int32), np.zeros(rows, np.int32), refs


# (one launch, up to 8192 pages; and the launches of larger caches)
@pytest.mark.parametrize("blocks", [200, 8192, 8193, 30000])
def test_a_request_for_too_much_does_not_stand_in_the_way(blocks):
    table, lens, refs = empty(64, blocks, 110, 50)
    granted = check(table, lens, refs, [64 * 100] + [64] * 63)
    assert granted.tolist() == [0] + [1] * 50 + [0] * 13


@pytest.mark.parametrize("blocks", [200, 8193])
def test_the_last_pages_go_to_whom_they_suffice_for(blocks):
    table, lens, refs = empty(8, blocks, 20, 7)
    lens[3] = 64                                              # (its first page is one that is held)
    table[3, 0] = int(np.flatnonzero(refs)[0])
    assert check(table, lens, refs, [64 * 3, 64 * 5, 0, 64, 64 * 21, 64 * 4, 64 * 1, 65]).tolist() == [1, 0, 1, 1, 0, 1, 0, 0]
    assert check(table, lens, refs, [64 * 8] * 4 + [64 * 7, 1, 0, -5]).tolist() == [0, 0, 0, 1, 0, 0, 1, 1]
    assert check(table, lens, refs * 0 + 1, [1] * 8).tolist() == [0, 0, 0, 1, 0, 0, 0, 0]


# rows below, at and above what a block looks at in one go
@pytest.mark.parametrize("rows", [1, 31, 33, 64, 1023, 1024, 1025, 2500])
@pytest.mark.parametrize("blocks", [8192, 20000])
def test_rows_of_all_sizes_over_a_cache_that_runs_full(rows, blocks):
    rng = np.random.default_rng(rows)
    table, lens, refs = empty(rows, blocks, 64, blocks // 3)
    new = np.minimum(64 * 64 + 40, (rng.pareto(0.7, rows) * 64 * blocks / 30 / rows).astype(np.int64))
    granted = check(table, lens, refs, new)
    assert rows < 31 or 0 < granted.sum() < rows
