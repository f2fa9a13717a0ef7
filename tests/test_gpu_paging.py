"""Copying, forking, freeing, reserving and compacting pages on a GPU against the same, one request at a time, in numpy."""
import numpy as np
import pytest
import torch

import _fp4_util as F
from paper_2509_25224_b200 import paging

pytestmark = pytest.mark.gpu

SHAPES = {"bf16": ((64, 576), torch.bfloat16), "e4m3": ((64, 576), torch.uint8), "fp4": ((F.PAGE_BYTES,), torch.uint8), "16 bytes": ((16,), torch.uint8), "1040 bytes": ((260,), torch.int32)}


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def filled(blocks, fmt, seed):
    shape, dtype = SHAPES[fmt]
    size = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(0, 256, (blocks, size), generator=gen, device="cuda", dtype=torch.uint8).view(dtype).view(blocks, *shape)


def raw(cache):
    return cache.view(cache.shape[0], -1).view(torch.uint8)


def books(rows, blocks, width, seed, fill=0.7, shared=0):
    """Random rows over random pages, the first `shared` pages of even rows the same; (table, lens, refs)."""
    rng = np.random.default_rng(seed)
    place = list(rng.permutation(blocks)[: int(blocks * fill)])
    common = [place.pop() for _ in range(shared)]
    table, lens, refs = np.full((rows, width), -1, np.int32), np.zeros(rows, np.int32), np.zeros(blocks, np.int32)
    for r in range(rows):
        pages = list(common) if r % 2 == 0 else []
        more = int(rng.integers(0, max(1, min(width - len(pages) - 1, 2 * len(place) // max(1, rows - r)) + 1)))
        more = min(more, len(place), width - len(pages))
        pages += [place.pop() for _ in range(more)]
        table[r, : len(pages)] = pages
        np.add.at(refs, pages, 1)
        if pages:
            # rows that share pages hold them full
            lens[r] = 64 * (len(pages) - 1) + (int(rng.integers(1, 65)) if more else 64)
    return table, lens, refs


class Both:
    """The operators under test and the plain form, side by side; a page's content is the index of its original."""

    def __init__(self, table, lens, refs, fmt="fp4", seed=9):
        self.original = filled(len(refs), fmt, seed)
        self.cache, self.table, self.lens, self.refs = self.original.clone(), dev(table), dev(lens), dev(refs)
        self.plain = F.Books(table, lens, refs, np.arange(len(refs)))

    def same(self):
        assert np.array_equal(self.table.cpu().numpy(), self.plain.table)
        assert np.array_equal(self.lens.cpu().numpy(), self.plain.lens)
        assert np.array_equal(self.refs.cpu().numpy(), self.plain.refs)
        assert torch.equal(raw(self.cache), raw(self.original)[dev(self.plain.cache).long()])

    def free(self, rows):
        paging.pages_free(self.table, self.lens, self.refs, dev(np.array(rows, np.int32)))
        self.plain.free(rows)
        self.same()

    def fork(self, parents, children):
        got = paging.pages_fork(self.cache, self.table, self.lens, self.refs, dev(np.array(parents, np.int32)), dev(np.array(children, np.int32)))
        want = self.plain.fork(parents, children)
        assert np.array_equal(got.cpu().numpy(), want)
        self.same()
        return want

    def reserve(self, new):
        got = paging.pages_reserve(self.table, self.lens, self.refs, dev(np.array(new, np.int32)))
        want = self.plain.reserve(new)
        assert np.array_equal(got.cpu().numpy(), want)
        self.same()
        return want

    def compact(self):
        got = paging.pages_compact(self.cache, self.table, self.lens, self.refs)
        assert got.item() == self.plain.compact()
        self.same()


@pytest.mark.parametrize("fmt", list(SHAPES))
@pytest.mark.parametrize("blocks,pairs", [(2, 1), (64, 30), (500, 250)])
def test_copy(fmt, blocks, pairs):
    cache = filled(blocks, fmt, 1)
    before = raw(cache).clone()
    place = np.random.default_rng(2).permutation(blocks).astype(np.int32)
    src, dst = place[:pairs].copy(), place[pairs: 2 * pairs].copy()
    want = before.clone()
    want[dev(dst).long()] = before[dev(src).long()]
    if pairs > 4:                                            # pairs that are not in the cache are left out
        want[int(dst[1])], want[int(dst[2])] = before[int(dst[1])], before[int(dst[2])]
        src[1], src[2] = -1, blocks
        src, dst = np.append(src, np.int32(0)), np.append(dst, np.int32(blocks))
    paging.pages_copy(cache, dev(src), dev(dst))
    assert torch.equal(raw(cache), want)


@pytest.mark.parametrize("rows,blocks,width,shared", [(1, 1, 1, 0), (6, 40, 9, 2), (100, 700, 12, 3), (40, 8192, 200, 10), (40, 8193, 200, 10), (300, 30000, 130, 1), (1500, 9000, 6, 0)])
@pytest.mark.parametrize("fmt", ["16 bytes", "fp4"])
def test_steps_of_a_serving_loop(rows, blocks, width, shared, fmt):
    rng = np.random.default_rng(rows)
    b = Both(*books(rows, blocks, width, rows + 1, shared=shared), fmt)
    for step in range(3):
        lost = rng.permutation(rows)[: rows // 2]
        kept = np.setdiff1d(np.arange(rows), lost)
        b.free(lost)
        if len(lost):
            b.fork(rng.choice(kept, len(lost)), lost)
        b.reserve(b.plain.lens + rng.integers(0, 130, rows).astype(np.int32))
        b.compact()


def test_a_row_that_is_listed_twice_is_freed_once_and_strangers_are_skipped():
    b = Both(*books(6, 40, 9, 4, shared=2))
    b.free([2, 4, 2, -1, 6, 4])
    b.free([])
    b.free([0, 1, 2, 3, 4, 5])
    assert (b.refs == 0).all() and (b.table == -1).all()


def test_forks_of_one_parent_strangers_and_forks_onto_oneself():
    table, lens, refs = books(8, 60, 9, 5, shared=2)
    lens[0] = 64 * (F.pages_of(lens[0]) - 1) + 17             # its last page is copied for every child
    lens[2] = 64 * F.pages_of(lens[2])                        # all of its pages are shared
    b = Both(table, lens, refs, "bf16")
    b.free([1, 3, 5, 7])
    assert list(b.fork([0, 0, 2, 2, -1, 0, 8, 4], [1, 3, 5, 7, 0, 8, 6, 4])) == [1, 1, 1, 1, 0, 0, 0, 0]


def test_an_empty_parent_makes_empty_children():
    b = Both(*books(4, 30, 6, 6))
    b.free([0, 1, 2])
    b.fork([0, 0], [1, 2])
    assert b.lens[1].item() == 0


@pytest.mark.parametrize("left", [0, 1, 3])
def test_forks_and_rows_that_find_no_page(left):
    table, lens, refs = books(10, 50, 9, 7, fill=1.0)
    lens[:5] = np.maximum(64 * (np.array([F.pages_of(n) for n in lens[:5]]) - 1), 0) + np.where(lens[:5] > 0, 9, 0)
    b = Both(table, lens, refs)
    b.free([5, 6, 7, 8, 9])
    free = np.flatnonzero(b.plain.refs <= 0)
    hold = free[left:]                                        # all but `left` free pages are held from outside the table
    b.plain.refs[hold] = 1
    b.refs[dev(hold).long()] = 1
    b.fork([0, 1, 2, 3, 4], [5, 6, 7, 8, 9])
    b.reserve(b.plain.lens + np.array([1, 60, 200, 0, 64, 1, 1, 64, 128, 1], np.int32))
    b.reserve(np.array([64 * 9 + 1] * 10, np.int32))          # more than the table has room for
    b.reserve(np.array([-7, 0] * 5, np.int32))                # shorter: as they were


def test_a_full_an_empty_and_a_compact_cache():
    b = Both(*books(5, 20, 8, 8, fill=1.0))
    b.compact()
    b.free([0, 1, 2, 3, 4])
    b.refs.zero_()
    b.plain.refs[:] = 0
    b.compact()
    b.reserve([70, 0, 300, 1, 64])
    b.compact()


def test_books_in_views_that_begin_anywhere():
    table, lens, refs = books(6, 100, 9, 11, shared=1)
    b = Both(table, lens, refs)
    for name in ("table", "lens", "refs"):
        t = getattr(b, name)
        room = torch.full((t.numel() + 3,), 77, dtype=torch.int32, device="cuda")
        room[3:] = t.flatten()
        setattr(b, name, room[3:].view(t.shape))
    b.free([1, 2])
    b.fork([0, 4], [1, 2])
    b.reserve(b.plain.lens + 65)
    b.compact()


def test_a_step_is_replayed_from_a_graph_and_runs_on_another_stream():
    table, lens, refs = books(12, 200, 9, 12, shared=2)
    b = Both(table, lens, refs)
    ws = torch.empty(paging.workspace_size(200, 12), dtype=torch.uint8, device="cuda")
    lost, parents = dev(np.array([1, 3], np.int32)), dev(np.array([0, 2], np.int32))
    served, granted, live = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (2, 12, 1))
    new = torch.zeros(12, dtype=torch.int32, device="cuda")

    def step():
        paging.pages_free(b.table, b.lens, b.refs, lost)
        paging.pages_fork(b.cache, b.table, b.lens, b.refs, parents, lost, served, ws)
        torch.add(b.lens, 1, out=new)
        paging.pages_reserve(b.table, b.lens, b.refs, new, granted, ws)
        paging.pages_compact(b.cache, b.table, b.lens, b.refs, live, ws)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()                                                # outside a capture first
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            step()
        for _ in range(4):
            g.replay()
    s.synchronize()
    for _ in range(5):
        b.plain.free([1, 3])
        b.plain.fork([0, 2], [1, 3])
        b.plain.reserve(b.plain.lens + 1)
        b.plain.compact()
    b.same()
