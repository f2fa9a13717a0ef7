"""The 4-bit cache and its pages at their limits on a GPU: caches of more than 2^32 bytes, lengths that no table holds, and what the Python calls refuse."""
import numpy as np
import pytest
import torch

import _fp4_util as F
from paper_2509_25224_b200 import binding, paging
from paper_2509_25224_b200.binding import AmlaError

from tests.test_gpu_lengths_from_device import late  # noqa: F401
from test_gpu_fp4 import bf16, compare, dev, expected, run, SCALE, tokens, workload

pytestmark = pytest.mark.gpu

FAR = 2 ** 32 // F.PAGE_BYTES + 5000                     # a page whose bytes begin beyond 2^32


@pytest.fixture(scope="module")
def far_cache():
    cache = torch.empty((FAR + 16, F.PAGE_BYTES), dtype=torch.uint8, device="cuda")
    yield cache
    del cache
    torch.cuda.empty_cache()


@pytest.mark.parametrize("H", [16, 128])
def test_decode_reads_pages_beyond_32_bits(far_cache, H):
    q, cache, table, lens = workload([300, 129], 1, H)
    used = cache.shape[0]
    far_cache[FAR: FAR + used] = dev(cache)
    out, lse = torch.empty((2, 1, H, 512), dtype=torch.bfloat16, device="cuda"), torch.empty((2, 1, H), device="cuda")
    binding.mla_decode_fp4(bf16(q), far_cache, 0.25, dev(np.where(table >= 0, table + FAR, -1).astype(np.int32)), dev(lens), SCALE, out, lse)
    compare(out.double().cpu().numpy(), lse.double().cpu().numpy(), *expected(q, cache, table, lens, 0.25))


def test_tokens_and_copies_beyond_32_bits(far_cache):
    x = bf16(tokens(100, 8))
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    near = torch.zeros((2, F.PAGE_BYTES), dtype=torch.uint8, device="cuda")
    far_cache[FAR: FAR + 4] = 0
    paging.cache_store_fp4(x, i(0, 100), near, 0.5, i(0, 1).view(1, 2), i(100))
    paging.cache_store_fp4(x, i(0, 100), far_cache, 0.5, i(FAR, FAR + 1).view(1, 2), i(100))
    assert torch.equal(far_cache[FAR: FAR + 2], near)
    paging.pages_copy(far_cache, i(FAR, FAR + 1), i(FAR + 2, 7))
    assert torch.equal(far_cache[FAR + 2], near[0]) and torch.equal(far_cache[7], near[1])
    back = torch.empty((100, F.D), dtype=torch.bfloat16, device="cuda")
    paging.cache_load_fp4(far_cache, 0.5, i(FAR + 2, 7).view(1, 2), i(100), i(0, 100), back)
    assert torch.equal(back, paging.cache_load_fp4(near, 0.5, i(0, 1).view(1, 2), i(100), i(0, 100), torch.empty_like(back)))


def test_fork_reserve_and_compact_beyond_32_bits(far_cache):
    # everything in front is held by nobody but counted: the free pages are the last ones
    blocks = far_cache.shape[0]
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    table, lens, refs = i(FAR, -1, -1, -1).view(2, 2), i(40, 0), torch.ones(blocks, dtype=torch.int32, device="cuda")
    refs[FAR + 1: FAR + 3] = 0
    far_cache[FAR] = torch.arange(F.PAGE_BYTES, device="cuda") % 251
    assert int(paging.pages_fork(far_cache, table, lens, refs, i(0), i(1))[0]) == 1
    assert table[1].tolist() == [FAR + 1, -1] and torch.equal(far_cache[FAR + 1], far_cache[FAR])
    assert paging.pages_reserve(table, lens, refs, i(40, 100)).tolist() == [1, 1] and table[1].tolist() == [FAR + 1, FAR + 2]
    refs[:FAR] = 0
    refs[FAR + 3:] = 0
    assert int(paging.pages_compact(far_cache, table, lens, refs)) == 3
    assert table.tolist() == [[0, -1], [1, 2]] and refs[:4].tolist() == [1, 1, 1, 0] and int(refs.sum()) == 3
    assert torch.equal(far_cache[0], far_cache[FAR]) and torch.equal(far_cache[1], far_cache[FAR])


@pytest.mark.parametrize("H", [16, 64])
def test_lengths_that_no_table_holds_are_cut_to_it(H):
    q, cache, table, lens = workload([256, 5, 70], 1, H, spare=0)
    table = table[:, :4].copy()                           # (a row of four pages, all of them used)
    wrong = np.array([100000, -3, 70], np.int32)
    out, lse = run(q, cache, table, wrong, 0.25)
    compare(out, lse, *expected(q, cache, table, np.array([256, 0, 70], np.int32), 0.25))


# (the kernel for 16 rows, for 64 with the lengths on chip, with more than 512 items, with one item a row block of more than 64 rows)
@pytest.mark.parametrize("B,Sq,H,longest", [(5, 1, 16, 900), (150, 1, 16, 200), (6, 1, 64, 900), (6, 2, 128, 900), (520, 1, 16, 100), (300, 1, 128, 150)])
def test_lengths_written_directly_in_front_of_the_call(late, B, Sq, H, longest):  # noqa: F811
    q, cache, table, full = workload([longest] * B, Sq, H)
    q, cache, table = bf16(q), dev(cache), dev(table)
    rng = np.random.default_rng(B + H)
    one = rng.integers(0, longest + 1, B).astype(np.int32)
    lens = [dev(x) for x in (one, np.minimum(one + 1, longest), full)]
    garbage = dev(rng.integers(-2**31, 2**31 - 1, B, dtype=np.int64).astype(np.int32))
    seqlens = torch.empty(B, dtype=torch.int32, device="cuda")
    ws = torch.empty(binding.fp4_workspace_size(B, Sq, H, table.shape[1], 0), dtype=torch.uint8, device="cuda")

    def decode():
        return binding.mla_decode_fp4(q, cache, 0.25, table, seqlens, SCALE, workspace=ws)

    want = []
    for x in lens:
        seqlens.copy_(x)
        torch.cuda.synchronize()
        want.append(decode())
        torch.cuda.synchronize()
    stream = torch.cuda.current_stream().cuda_stream
    for delay in (0, 1000, 4000, 16000, 30000):
        for x, (o, l) in zip(lens, want):
            seqlens.copy_(garbage)
            assert late(x.data_ptr(), seqlens.data_ptr(), B, delay, stream) == 0
            out, lse = decode()
            binding.check_status(ws)
            assert torch.equal(out.view(torch.int16), o.view(torch.int16)) and torch.equal(lse, l)


def test_refusals_of_tensors():
    i = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")  # noqa: E731
    z = lambda dtype, *shape: torch.zeros(shape, dtype=dtype, device="cuda")  # noqa: E731
    b, u = torch.bfloat16, torch.uint8
    cache, q, rows = z(u, 4, F.PAGE_BYTES), z(b, 2, 1, 16, 576), z(b, 3, 576)
    decode = lambda q=q, cache=cache, table=i(2, 4), lens=i(2), **more: binding.mla_decode_fp4(q, cache, 1.0, table, lens, 0.1, **more)  # noqa: E731
    for bad in [dict(q=q.float()), dict(q=q[..., :575]), dict(q=z(b, 16, 1, 2, 576).transpose(0, 2)), dict(cache=z(u, 4, 64, 576)), dict(cache=cache.view(torch.int8)), dict(cache=z(u, 8, F.PAGE_BYTES)[::2]),
                dict(table=i(3, 4)), dict(table=i(2, 8)[:, ::2]), dict(table=i(2, 4).long()), dict(lens=i(3)), dict(lens=i(2).cpu()), dict(out=z(b, 2, 1, 16, 576)), dict(out=z(torch.float32, 2, 1, 16, 512)),
                dict(lse=z(b, 2, 1, 16))]:
        with pytest.raises(ValueError):
            decode(**bad)
    with pytest.raises(AmlaError):
        decode(workspace=z(u, 256))
    store = lambda kv=rows, starts=i(3), cache=cache, table=i(2, 4), lens=i(2), scale=1.0: paging.cache_store_fp4(kv, starts, cache, scale, table, lens)  # noqa: E731
    load = lambda kv=rows, starts=i(3), cache=cache, table=i(2, 4), lens=i(2), scale=1.0: paging.cache_load_fp4(cache, scale, table, lens, starts, kv)  # noqa: E731
    for call in (store, load):
        for bad in [dict(kv=rows.float()), dict(kv=z(b, 3, 512)), dict(kv=z(b, 576, 3).t()), dict(kv=z(b, 1, 576).expand(3, 576)), dict(kv=rows.cpu()), dict(starts=i(2)), dict(starts=i(3).long()),
                    dict(cache=z(u, 4, F.PAGE_BYTES + 16)), dict(cache=z(b, 4, 64, 576)), dict(table=i(3, 4)), dict(table=i(8)), dict(lens=i(1))]:
            with pytest.raises(ValueError):
                call(**bad)
        for scale in (0.0, -1.0, float("nan"), float("inf"), 1e-38):
            with pytest.raises(AmlaError):
                call(scale=scale)
    for src, dst in [(i(2), i(3)), (i(2).long(), i(2)), (i(2, 2), i(2, 2)), (i(2).cpu(), i(2))]:
        with pytest.raises(ValueError):
            paging.pages_copy(cache, src, dst)
    for odd in (cache[:, :-1], z(u, 8, F.PAGE_BYTES)[::2], z(u, 16)):
        with pytest.raises(ValueError):
            paging.pages_copy(odd, i(1), i(1))
    with pytest.raises(AmlaError):
        paging.pages_copy(z(u, 4, 24), i(1), i(1))       # pages are whole pieces of 16 bytes
    with pytest.raises(ValueError):
        paging.pages_free(i(2, 4), i(2), i(4), i(1, 1))
    fork = lambda cache=cache, table=i(2, 4), lens=i(2), refs=i(4), parents=i(1), children=i(1), **more: paging.pages_fork(cache, table, lens, refs, parents, children, **more)  # noqa: E731
    for bad in [dict(refs=i(5)), dict(lens=i(3)), dict(table=i(8)), dict(children=i(2)), dict(parents=i(1).long()), dict(served=i(2)), dict(workspace=z(u, 4096).cpu())]:
        with pytest.raises(ValueError):
            fork(**bad)
    with pytest.raises(AmlaError):
        fork(workspace=z(u, 256))
    with pytest.raises(AmlaError):
        fork(parents=i(3), children=i(3))                 # more forks than rows
    for bad in [dict(new=i(3)), dict(new=i(2).long()), dict(granted=i(3))]:
        with pytest.raises(ValueError):
            paging.pages_reserve(i(2, 4), i(2), i(4), bad.get("new", i(2)), bad.get("granted"))
    same = i(2)
    with pytest.raises(AmlaError):
        paging.pages_reserve(i(2, 4), same, i(4), same)
    with pytest.raises(ValueError):
        paging.pages_compact(cache, i(2, 4), i(2), i(4), live=i(2))
