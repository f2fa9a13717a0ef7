"""What the 4-bit cache's and the pages' entries refuse, without a device: the C ABI by its codes, the Python side by ValueError; and that
the plain forms which the GPU tests hold them to are what they should be."""
import ctypes
import math

import numpy as np
import pytest
import torch

import _fp4_util as F
from paper_2509_25224_b200 import binding, build, paging
from test_binding import fake  # noqa: F401  (a fixture: a library that records the calls)

P, Z = ctypes.c_void_p, ctypes.c_void_p(0)
OK, BAD, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def at(k):
    """An address (that no call here gets to use)."""
    return P(1 << 20 | k)


def decode_fp4(lib, q=at(0), cache=at(0), kv_scale=1.0, table=at(0), lens=at(0), scale=0.1, B=1, Sq=1, H=16, blocks=4, width=4, out=at(0), lse=at(0), ws=at(0), size=0):
    return lib.amla_mla_decode_fp4(q, cache, kv_scale, table, lens, scale, B, Sq, H, blocks, width, out, lse, ws, size, Z)


@pytest.mark.parametrize("bad", [dict(q=Z), dict(cache=Z), dict(table=Z), dict(lens=Z), dict(out=Z), dict(lse=Z), dict(ws=Z), dict(q=at(8)), dict(cache=at(8)), dict(out=at(2)), dict(table=at(2)),
                                 dict(lens=at(1)), dict(lse=at(2)), dict(ws=at(16)), dict(B=0), dict(Sq=0), dict(H=0), dict(blocks=0), dict(width=0), dict(scale=math.nan),
                                 dict(kv_scale=0.0), dict(kv_scale=-1.0), dict(kv_scale=math.nan), dict(kv_scale=math.inf), dict(kv_scale=1e-38), dict(kv_scale=1e38)])
def test_decode_refuses(lib, bad):
    assert decode_fp4(lib, **bad) == BAD


@pytest.mark.parametrize("bad", [dict(Sq=9), dict(H=129), dict(width=1 << 25), dict(B=1 << 25)])
def test_decode_does_not_cover(lib, bad):
    assert decode_fp4(lib, **bad) == UNSUPPORTED
    n = ctypes.c_size_t(0)
    shape = dict(B=1, Sq=1, H=16, width=4) | bad
    assert lib.amla_mla_decode_fp4_workspace_size(shape["B"], shape["Sq"], shape["H"], shape["width"], 0, ctypes.byref(n)) == UNSUPPORTED


def tokens(lib, entry, rows=at(0), stride=576, n=3, starts=at(0), cache=at(0), kv_scale=1.0, table=at(0), lens=at(0), B=2, blocks=4, width=4):
    if entry == "store":
        return lib.amla_cache_store_fp4(rows, stride, n, starts, cache, kv_scale, table, lens, B, blocks, width, Z)
    return lib.amla_cache_load_fp4(cache, kv_scale, table, lens, starts, B, blocks, width, rows, stride, n, Z)


@pytest.mark.parametrize("entry", ["store", "load"])
@pytest.mark.parametrize("bad", [dict(rows=Z), dict(starts=Z), dict(cache=Z), dict(table=Z), dict(lens=Z), dict(rows=at(1)), dict(cache=at(4)), dict(starts=at(2)), dict(table=at(2)), dict(lens=at(2)),
                                 dict(n=-1), dict(stride=575), dict(stride=-576), dict(B=0), dict(blocks=0), dict(width=0), dict(kv_scale=0.0), dict(kv_scale=math.nan)])
def test_tokens_refuse(lib, entry, bad):
    assert tokens(lib, entry, **bad) == BAD
    assert tokens(lib, entry, n=0, rows=Z) == OK              # nothing to do, nothing launched


def test_pages_refuse(lib):
    c, page = at(0), 20736
    assert lib.amla_pages_copy(c, page, 4, Z, Z, 0, Z) == OK
    for args in [(Z, page, 4, c, c, 1), (at(8), page, 4, c, c, 1), (c, 0, 4, c, c, 1), (c, 24, 4, c, c, 1), (c, page, 0, c, c, 1), (c, page, 4, Z, c, 1), (c, page, 4, c, Z, 1), (c, page, 4, c, c, -1),
                 (c, page, 4, at(2), c, 1)]:
        assert lib.amla_pages_copy(*args, Z) == BAD
    assert lib.amla_pages_copy(c, page, (1 << 28) + 1, c, c, 1, Z) == UNSUPPORTED
    assert lib.amla_pages_free(c, c, c, Z, 0, 2, 4, 4, Z) == OK
    for args in [(Z, c, c, c, 1, 2, 4, 4), (c, Z, c, c, 1, 2, 4, 4), (c, c, Z, c, 1, 2, 4, 4), (c, c, c, Z, 1, 2, 4, 4), (c, c, c, c, -1, 2, 4, 4), (c, c, c, c, 1, 0, 4, 4), (c, c, c, c, 1, 2, 0, 4),
                 (c, c, c, c, 1, 2, 4, 0), (c, c, c, at(1), 1, 2, 4, 4), (at(2), c, c, c, 1, 2, 4, 4)]:
        assert lib.amla_pages_free(*args, Z) == BAD
    n = ctypes.c_size_t(0)
    assert lib.amla_pages_workspace_size(100, 3, ctypes.byref(n)) == OK and n.value > 0
    assert lib.amla_pages_workspace_size(0, 3, ctypes.byref(n)) == BAD
    assert lib.amla_pages_workspace_size(100, 0, ctypes.byref(n)) == BAD
    assert lib.amla_pages_workspace_size(100, 3, None) == BAD
    assert lib.amla_pages_workspace_size((1 << 28) + 1, 3, ctypes.byref(n)) == UNSUPPORTED
    lib.amla_pages_workspace_size(4, 2, ctypes.byref(n))
    size, d = n.value, at(256)
    fork = lambda cache=c, refs=c, parents=c, children=c, k=1, served=c, ws=c, ws_size=size: lib.amla_pages_fork(cache, page, c, c, refs, parents, children, k, 2, 4, 4, served, ws, ws_size, Z)  # noqa: E731
    assert fork(k=0, ws=Z, ws_size=0) == OK
    for bad in [dict(cache=Z), dict(refs=Z), dict(parents=Z), dict(children=Z), dict(k=3), dict(k=-1), dict(served=at(2)), dict(ws=Z), dict(ws=at(16))]:
        assert fork(**bad) == BAD
    assert fork(ws_size=size - 1) == WORKSPACE
    reserve = lambda new=d, refs=c, granted=c, ws=c, ws_size=size: lib.amla_pages_reserve(c, c, refs, new, 2, 4, 4, granted, ws, ws_size, Z)  # noqa: E731
    for bad in [dict(new=Z), dict(new=c), dict(new=at(258)), dict(refs=Z), dict(granted=at(1)), dict(ws=Z)]:
        assert reserve(**bad) == BAD
    assert reserve(ws_size=size - 1) == WORKSPACE
    compact = lambda cache=c, refs=c, live=c, ws=c, ws_size=size: lib.amla_pages_compact(cache, page, c, c, refs, 2, 4, 4, live, ws, ws_size, Z)  # noqa: E731
    for bad in [dict(cache=Z), dict(cache=at(8)), dict(refs=Z), dict(live=at(2)), dict(ws=Z), dict(ws=at(8))]:
        assert compact(**bad) == BAD
    assert compact(ws_size=size - 1) == WORKSPACE


def test_host_tensors_never_reach_a_kernel(fake):  # noqa: F811
    i = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    cache, rows = torch.zeros((4, F.PAGE_BYTES), dtype=torch.uint8), torch.zeros((3, 576), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        binding.mla_decode_fp4(torch.zeros((1, 1, 16, 576), dtype=torch.bfloat16), cache, 1.0, i(1, 4), i(1), 0.1, torch.empty((1, 1, 16, 512), dtype=torch.bfloat16),
                               torch.empty((1, 1, 16)), torch.empty(1 << 20, dtype=torch.uint8))
    for call in [lambda: paging.cache_store_fp4(rows, i(3), cache, 1.0, i(2, 4), i(2)), lambda: paging.cache_load_fp4(cache, 1.0, i(2, 4), i(2), i(3), rows),
                 lambda: paging.pages_copy(cache, i(1), i(1)), lambda: paging.pages_free(i(2, 4), i(2), i(4), i(1)),
                 lambda: paging.pages_fork(cache, i(2, 4), i(2), i(4), i(1), i(1)), lambda: paging.pages_reserve(i(2, 4), i(2), i(4), i(2)),
                 lambda: paging.pages_compact(cache, i(2, 4), i(2), i(4))]:
        with pytest.raises(ValueError):
            call()
    assert fake.calls == []


def test_the_plain_quantiser_is_nearest_with_ties_to_even():
    assert F.E4M3[126] == 448.0 and F.E4M3[1] == 2.0 ** -9 and (np.diff(F.E4M3) > 0).all()
    x = np.zeros(576)
    x[:16] = [6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.76, -1.24, 0.0, 0.26, -5.0, -5.01, 6.0]
    c, s = F.quantise(x, 1.0)
    v = F.values(c, s)
    assert list(v[:16]) == [6.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 0.0, -1.0, -1.0, 0.0, 0.5, -4.0, -6.0, 6.0] and (v[16:] == 0).all()
    rng = np.random.default_rng(1)
    x = rng.standard_normal((50, 576))
    c, s = F.quantise(x, 0.25)
    v = F.values(c, s) * 0.25
    top = np.abs(x).reshape(50, 36, 16).max(-1).repeat(16, -1)
    # half of E2M1's widest gap (2 of 6), and the scale's own rounding (1/16) of the largest
    assert (np.abs(v - x) <= top * (1 / 6 + 1 / 16)).all()


def test_the_quotient_that_the_kernel_corrects_is_the_true_one_at_every_tie():
    # fl(x * fl(1 / step)) with one correction by the remainder, for every E4M3 scale and every midpoint of E2M1: FP32 in numpy, the
    # fused remainder (exact here: x has at most seven bits, y 24, step 4) in FP64
    f = np.float32
    step = F.E4M3[1:][:, None].astype(f)
    for mid in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0):
        x = f(mid) * step
        inv = f(1) / step
        y = x * inv
        rest = (x.astype(np.float64) - y.astype(np.float64) * step.astype(np.float64)).astype(f)
        fixed = (rest.astype(np.float64) * inv.astype(np.float64) + y.astype(np.float64)).astype(f)
        assert (fixed == f(mid)).all()


def test_plain_books_by_hand():
    table = np.array([[3, 1, -1], [3, 4, -1], [-1, -1, -1]], np.int32)
    b = F.Books(table, np.array([100, 128, 0], np.int32), np.array([0, 1, 0, 2, 1, 0], np.int32), np.arange(6))
    assert list(b.fork([0], [2])) == [1] and list(b.table[2]) == [3, 0, -1] and list(b.refs) == [1, 1, 0, 3, 1, 0] and b.cache[0] == 1
    b.free([0])
    assert list(b.refs) == [1, 0, 0, 2, 1, 0]
    assert list(b.reserve([1, 129, 128])) == [1, 1, 1] and b.table[0, 0] == 1 and b.table[1, 2] == 2
    b.free([0, 2])
    assert b.compact() == 3 and list(b.table[1]) == [0, 1, 2] and list(b.refs) == [1, 1, 1, 0, 0, 0] and list(b.cache[:3]) == [3, 4, 2]
