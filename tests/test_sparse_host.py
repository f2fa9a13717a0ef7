"""What the entries for tokens into any cache, means, scores, selection and sparse decode refuse, without a device: the C ABI by its codes, the Python side by
ValueError; that their kernels read behind the wait and promise nothing; and that the plain forms which the GPU tests hold them to are what they should be."""
import ctypes
import math
import os
import re

import numpy as np
import pytest
import torch

import _fp4_util as F
import _sparse_util as S
from paper_2509_25224_b200 import binding, build, long_context, paging, sparse
from test_binding import fake  # noqa: F401  (a fixture: a library that records the calls)

P, Z = ctypes.c_void_p, ctypes.c_void_p(0)
OK, BAD, UNSUPPORTED, WORKSPACE, CUDA = 0, -1, -2, -3, -4


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.lib()


def at(k):
    """An address (that no call here gets to use)."""
    return P(1 << 20 | k)


def append(lib, fmt=0, kv=at(0), stride=576, n=3, starts=at(0), cache=at(0), kv_scale=1.0, table=at(0), lens=at(0), B=2, blocks=4, width=4, cos_sin=at(0), n_pos=100, positions=Z, weight=at(0), f32=0,
           eps=1e-6, interleaved=0, q_pe=at(0), qpt=64, qph=64, q=at(0), qt=9216, qh=576, H=16):
    return lib.amla_cache_append(fmt, kv, stride, n, starts, cache, kv_scale, table, lens, B, blocks, width, cos_sin, n_pos, positions, weight, f32, eps, interleaved, q_pe, qpt, qph, q, qt, qh, H, Z)


@pytest.mark.parametrize("bad", [dict(fmt=3), dict(fmt=-1), dict(kv=Z), dict(starts=Z), dict(cache=Z), dict(table=Z), dict(lens=Z), dict(cos_sin=Z), dict(q_pe=Z), dict(q=Z), dict(kv=at(1)), dict(cache=at(8)),
                                 dict(starts=at(2)), dict(table=at(2)), dict(lens=at(1)), dict(cos_sin=at(8)), dict(positions=at(2)), dict(weight=at(1)), dict(weight=at(2), f32=1), dict(q_pe=at(1)), dict(q=at(1)),
                                 dict(n=-1), dict(stride=575), dict(B=0), dict(blocks=0), dict(width=0), dict(n_pos=0), dict(eps=-1e-9), dict(eps=math.nan), dict(qpt=-1), dict(qph=-64), dict(qt=575),
                                 dict(qh=64), dict(H=-1), dict(fmt=1, kv_scale=0.0), dict(fmt=1, kv_scale=math.nan), dict(fmt=2, kv_scale=-1.0), dict(fmt=2, kv_scale=math.inf), dict(fmt=1, kv_scale=1e-38)])
def test_append_refuses(lib, bad):
    assert append(lib, **bad) == BAD


def test_append_of_nothing_and_of_too_many_heads(lib):
    assert append(lib, n=0, kv=Z, q=Z, q_pe=Z, H=0) == OK
    assert append(lib, H=1025) == UNSUPPORTED
    assert append(lib, fmt=0, kv_scale=math.nan, n=0) == OK              # not used by bf16


def means(lib, fmt=0, cache=at(0), kv_scale=1.0, table=at(0), lens=at(0), starts=at(0), n=3, B=2, blocks=4, width=4, out=at(0)):
    return lib.amla_page_means(fmt, cache, kv_scale, table, lens, starts, n, B, blocks, width, out, Z)


@pytest.mark.parametrize("bad", [dict(fmt=3), dict(cache=Z), dict(table=Z), dict(lens=Z), dict(starts=Z), dict(out=Z), dict(out=at(8)), dict(cache=at(8)), dict(n=-1), dict(B=0), dict(blocks=0), dict(width=0),
                                 dict(fmt=2, kv_scale=0.0)])
def test_means_refuse(lib, bad):
    assert means(lib, **bad) == BAD
    assert means(lib, n=0) == OK


def scores(lib, q=at(0), m=at(0), table=at(0), lens=at(0), scale=0.1, B=1, Sq=1, H=16, blocks=4, width=4, out=at(0), ws=at(0), size=1 << 20):
    return lib.amla_page_scores(q, m, table, lens, scale, B, Sq, H, blocks, width, out, ws, size, Z)


@pytest.mark.parametrize("bad", [dict(q=Z), dict(m=Z), dict(table=Z), dict(lens=Z), dict(out=Z), dict(ws=Z), dict(q=at(8)), dict(m=at(8)), dict(out=at(2)), dict(table=at(2)), dict(lens=at(2)), dict(ws=at(16)),
                                 dict(B=0), dict(Sq=0), dict(H=0), dict(blocks=0), dict(width=0), dict(scale=math.nan)])
def test_scores_refuse(lib, bad):
    assert scores(lib, **bad) == BAD


def test_scores_do_not_cover(lib):
    n = ctypes.c_size_t(0)
    assert scores(lib, size=0) == WORKSPACE
    for bad in [dict(Sq=9), dict(H=129), dict(B=1 << 14, width=(1 << 14) + 1)]:
        assert scores(lib, **bad) == UNSUPPORTED
        shape = dict(B=1, Sq=1, H=16, width=4) | bad
        assert lib.amla_page_scores_workspace_size(shape["B"], shape["Sq"], shape["H"], shape["width"], 0, ctypes.byref(n)) == UNSUPPORTED
    assert lib.amla_page_scores_workspace_size(1, 1, 16, 4, 0, None) == BAD
    assert lib.amla_page_scores_workspace_size(1, 1, 16, 4, -1, ctypes.byref(n)) == BAD
    assert lib.amla_page_scores_workspace_size(4, 8, 128, 5000, 0, ctypes.byref(n)) == OK and 0 < n.value <= 4096


def select(lib, s=1 << 20, table=1 << 24, lens=1 << 25, B=2, Sq=1, width=100, keep=8, sink=1, recent=1, out=1 << 26, out_lens=1 << 27, chosen=1 << 28):
    return lib.amla_pages_select(P(s), P(table), P(lens), B, Sq, width, keep, sink, recent, P(out), P(out_lens), P(chosen), Z)


@pytest.mark.parametrize("bad", [dict(s=0), dict(table=0), dict(lens=0), dict(out=0), dict(out_lens=0), dict(s=2), dict(table=2), dict(out=2), dict(chosen=(1 << 28) + 2), dict(keep=0), dict(keep=-1), dict(sink=-1), dict(recent=0),
                                 dict(sink=4, recent=5), dict(sink=2 ** 31 - 1, recent=2 ** 31 - 1), dict(B=0), dict(Sq=0), dict(width=0),
                                 # answers over questions, and over one another
                                 dict(out=(1 << 24) + 796), dict(out=(1 << 24) - 60), dict(out_lens=(1 << 25) + 4), dict(chosen=1 << 20), dict(chosen=(1 << 26) + 60), dict(out_lens=1 << 28), dict(out=(1 << 20) + 796)])
def test_selection_refuses(lib, bad):
    assert select(lib, **bad) == BAD


def test_selection_does_not_cover(lib):
    for bad in [dict(Sq=9), dict(B=(1 << 23) + 1, width=1), dict(B=1 << 14, width=(1 << 14) + 1), dict(keep=1 << 25)]:
        assert select(lib, **bad) == UNSUPPORTED


def decode(lib, fmt=0, q=at(0), cache=at(0), kv_scale=1.0, m=at(0), table=at(0), lens=at(0), scale=0.1, B=1, Sq=1, H=16, blocks=4, width=40, keep=8, sink=1, recent=1, out=at(0), lse=at(0), ws=at(0), size=0):
    return lib.amla_mla_decode_sparse(fmt, q, cache, kv_scale, m, table, lens, scale, B, Sq, H, blocks, width, keep, sink, recent, out, lse, ws, size, Z)


@pytest.mark.parametrize("bad", [dict(fmt=3), dict(q=Z), dict(cache=Z), dict(m=Z), dict(table=Z), dict(lens=Z), dict(out=Z), dict(lse=Z), dict(ws=Z), dict(q=at(8)), dict(cache=at(8)), dict(m=at(8)), dict(out=at(8)),
                                 dict(lse=at(2)), dict(table=at(2)), dict(ws=at(16)), dict(B=0), dict(Sq=0), dict(H=0), dict(blocks=0), dict(width=0), dict(keep=0), dict(sink=-1), dict(recent=0), dict(sink=4, recent=5),
                                 dict(scale=math.nan), dict(fmt=1, kv_scale=0.0), dict(fmt=2, kv_scale=math.nan), dict(fmt=1, kv_scale=-2.0)])
def test_sparse_decode_refuses(lib, bad):
    assert decode(lib, **bad) == BAD


@pytest.mark.parametrize("bad", [dict(Sq=9), dict(H=129), dict(width=1 << 25), dict(keep=1 << 25), dict(B=(1 << 23) + 1, width=9)])
def test_sparse_decode_does_not_cover(lib, bad):
    assert decode(lib, **bad) == UNSUPPORTED
    shape, n = dict(B=1, Sq=1, H=16, width=40, keep=8) | bad, ctypes.c_size_t(0)
    assert lib.amla_mla_decode_sparse_workspace_size(shape["B"], shape["Sq"], shape["H"], shape["width"], shape["keep"], 0, ctypes.byref(n)) == UNSUPPORTED
    assert lib.amla_mla_decode_sparse_workspace_size(1, 1, 16, 40, 8, 0, None) == BAD
    assert lib.amla_mla_decode_sparse_workspace_size(1, 1, 16, 40, 0, 0, ctypes.byref(n)) == BAD
    assert lib.amla_sparse_check_status(Z, Z) == BAD


def test_host_tensors_never_reach_a_kernel(fake):  # noqa: F811
    i = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    b = lambda *shape: torch.zeros(shape, dtype=torch.bfloat16)  # noqa: E731
    cache, q = b(4, 64, 576), b(2, 1, 16, 576)
    for call in [lambda: paging.cache_append(b(3, 576), i(3), cache, 1.0, i(2, 4), i(2), torch.zeros(9, 64)), lambda: paging.page_means(cache, 1.0, i(2, 4), i(2), i(3), 3, b(4, 576)),
                 lambda: sparse.page_scores(q, b(4, 576), i(2, 4), i(2), 0.1), lambda: sparse.pages_select(torch.zeros(2, 1, 4), i(2, 4), i(2), 2),
                 lambda: sparse.mla_decode_sparse(q, cache, 1.0, b(4, 576), i(2, 4), i(2), 0.1, 2)]:
        with pytest.raises(ValueError):
            call()
    assert fake.calls == []


class Standin:
    """A tensor that says it is on a GPU, for what the Python side asks of one."""

    def __init__(self, shape, dtype, on=0, contiguous=True, stride=None):
        self.shape, self.dtype, self._on, self._contiguous = torch.Size(shape), dtype, on, contiguous
        self.device = torch.device("cuda", on)
        steps = [1]
        for n in reversed(shape[1:]):
            steps.append(steps[-1] * n)
        self._stride = tuple(reversed(steps)) if stride is None else stride

    def get_device(self):
        return self._on

    def is_contiguous(self):
        return self._contiguous

    def data_ptr(self):
        return 1 << 20

    def numel(self):
        return self.shape.numel()

    def dim(self):
        return len(self.shape)

    def stride(self, axis=None):
        return self._stride if axis is None else self._stride[axis]

    def element_size(self):
        return 1

    def new_empty(self, *shape, dtype=None):
        return Standin(shape[0] if isinstance(shape[0], tuple) else shape, self.dtype if dtype is None else dtype, self._on)


B16, I32, U8, F32 = torch.bfloat16, torch.int32, torch.uint8, torch.float32


@pytest.fixture
def on_gpu(fake, monkeypatch):  # noqa: F811
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    return fake


def append_args(**changed):
    a = dict(kv=Standin((5, 576), B16), starts=Standin((3,), I32), cache=Standin((4, 64, 576), B16), kv_scale=1.0, block_table=Standin((2, 6), I32), seqlens=Standin((2,), I32), cos_sin=Standin((50, 64), F32),
             positions=Standin((5,), I32), norm_weight=Standin((512,), B16), q_pe=Standin((5, 16, 64), B16), q=Standin((5, 16, 576), B16))
    a.update(changed)
    return a


def test_append_marshals(on_gpu):
    paging.cache_append(**append_args(kv=Standin((5, 576), B16, stride=(600, 1)), q_pe=Standin((5, 16, 64), B16, stride=(6144, 192, 1)), q=Standin((5, 16, 576), B16, stride=(576, 5 * 576, 1))))
    (name, args), = on_gpu.calls
    assert name == "amla_cache_append" and len(args) == 27
    assert args[0] == 0 and args[2:4] == (600, 5) and args[9:12] == (2, 4, 6) and args[13] == 50 and args[16] == 0 and args[20:22] == (6144, 192) and args[23:26] == (576, 2880, 16)
    for cache, fmt in ((Standin((4, 64, 576), U8), 1), (Standin((4, F.PAGE_BYTES), U8), 2)):
        paging.cache_append(**append_args(cache=cache, positions=None, norm_weight=None, q_pe=None, q=None))
        assert on_gpu.calls[-1][1][0] == fmt and on_gpu.calls[-1][1][14:16] == (0, 0) and on_gpu.calls[-1][1][19:26] == (0,) * 7
    # an axis of one entry has no stride that matters
    paging.cache_append(**append_args(kv=Standin((1, 576), B16, stride=(3, 1)), starts=Standin((3,), I32), positions=None, q_pe=Standin((1, 1, 64), B16, stride=(1, 1, 1)), q=Standin((1, 1, 576), B16, stride=(7, 9, 1))))
    assert len(on_gpu.calls) == 4


@pytest.mark.parametrize("changed", [
    dict(kv=Standin((5, 576), F32)), dict(kv=Standin((5, 512), B16)), dict(kv=Standin((5, 1, 576), B16)), dict(kv=Standin((5, 576), B16, on=1)), dict(kv=Standin((5, 576), B16, stride=(575, 1))),
    dict(kv=Standin((5, 576), B16, stride=(1152, 2))), dict(starts=Standin((2,), I32)), dict(starts=Standin((3,), torch.int64)), dict(starts=Standin((3,), I32, contiguous=False)), dict(cache=Standin((4, 64, 576), F32)),
    dict(cache=Standin((4, 32, 576), B16)), dict(cache=Standin((4, 20735), U8)), dict(cache=Standin((4, 64, 576), B16, contiguous=False)), dict(block_table=Standin((3, 6), I32)), dict(block_table=Standin((2, 6), I32, on=1)),
    dict(seqlens=Standin((3,), I32)), dict(seqlens=Standin((2,), F32)), dict(cos_sin=Standin((50, 32), F32)), dict(cos_sin=Standin((50, 64), B16)), dict(cos_sin=Standin((50, 64), F32, contiguous=False)),
    dict(positions=Standin((4,), I32)), dict(positions=Standin((5,), torch.int64)), dict(norm_weight=Standin((576,), B16)), dict(norm_weight=Standin((512,), torch.float16)), dict(norm_weight=Standin((512,), F32, on=1)),
    dict(q=None), dict(q_pe=None), dict(q=Standin((5, 16, 512), B16)), dict(q=Standin((5, 8, 576), B16)), dict(q_pe=Standin((4, 16, 64), B16)), dict(q_pe=Standin((5, 16, 64), F32)), dict(q=Standin((5, 16, 576), B16, on=1)),
    dict(q=Standin((5, 16, 576), B16, stride=(576, 0, 1))), dict(q=Standin((5, 16, 576), B16, stride=(64, 5 * 576, 1))), dict(q=Standin((5, 16, 576), B16, stride=(9216 * 2, 1152, 2)))])
def test_append_refuses_tensors(on_gpu, changed):
    with pytest.raises(ValueError):
        paging.cache_append(**append_args(**changed))
    assert on_gpu.calls == []


def sparse_args(**changed):
    a = dict(q=Standin((2, 1, 16, 576), B16), kv_cache=Standin((9, 64, 576), B16), kv_scale=1.0, means=Standin((9, 576), B16), block_table=Standin((2, 40), I32), seqlens=Standin((2,), I32), softmax_scale=0.1, keep=8,
             out=Standin((2, 1, 16, 512), B16), lse=Standin((2, 1, 16), F32), workspace=Standin((1 << 20,), U8))
    a.update(changed)
    return a


@pytest.mark.parametrize("changed", [
    dict(q=Standin((2, 1, 16, 576), F32)), dict(q=Standin((2, 1, 16, 512), B16)), dict(q=Standin((2, 16, 576), B16)), dict(q=Standin((2, 1, 16, 576), B16, contiguous=False)), dict(kv_cache=Standin((9, 64, 576), F32)),
    dict(kv_cache=Standin((9, 64, 576), B16, on=1)), dict(kv_cache=Standin((9, 64, 576), B16, contiguous=False)), dict(means=Standin((8, 576), B16)), dict(means=Standin((9, 576), F32)), dict(means=Standin((9, 576), B16, on=1)),
    dict(block_table=Standin((3, 40), I32)), dict(block_table=Standin((2, 40), torch.int64)), dict(seqlens=Standin((1,), I32)), dict(seqlens=Standin((2,), I32, on=1)), dict(out=Standin((2, 1, 16, 576), B16)),
    dict(out=Standin((2, 1, 16, 512), F32)), dict(lse=Standin((2, 16), F32)), dict(lse=Standin((2, 1, 16), F32, on=1)), dict(workspace=Standin((1 << 20,), U8, on=1)), dict(workspace=Standin((1 << 20,), U8, contiguous=False))])
def test_sparse_decode_refuses_tensors(on_gpu, changed):
    with pytest.raises(ValueError):
        sparse.mla_decode_sparse(**sparse_args(**changed))
    assert on_gpu.calls == []


def test_sparse_decode_marshals(on_gpu):
    sparse.mla_decode_sparse(**sparse_args())
    sparse.mla_decode_sparse(**sparse_args(kv_cache=Standin((9, F.PAGE_BYTES), U8), means=None))
    (a, x), (b, y) = on_gpu.calls
    assert a == b == "amla_mla_decode_sparse" and x[0] == 0 and y[0] == 2 and y[4] == 0 and x[8:16] == (2, 1, 16, 9, 40, 8, 1, 1) and x[19] == 1 << 20


@pytest.mark.parametrize("changed", [dict(scores=Standin((2, 1, 40), B16)), dict(scores=Standin((2, 40), F32)), dict(scores=Standin((2, 1, 40), F32, contiguous=False)), dict(block_table=Standin((2, 41), I32)),
                                     dict(seqlens=Standin((3,), I32)), dict(keep=0), dict(table=Standin((2, 7), I32)), dict(lens=Standin((1,), I32)), dict(chosen=Standin((2, 8), F32)), dict(lens=Standin((2,), I32, on=1))])
def test_selection_refuses_tensors(on_gpu, changed):
    args = dict(scores=Standin((2, 1, 40), F32), block_table=Standin((2, 40), I32), seqlens=Standin((2,), I32), keep=8) | changed
    with pytest.raises(ValueError):
        sparse.pages_select(**args)
    assert on_gpu.calls == []


def test_means_refuse_tensors(on_gpu):
    good = dict(cache=Standin((9, 64, 576), U8), kv_scale=1.0, block_table=Standin((2, 4), I32), seqlens=Standin((2,), I32), starts=Standin((3,), I32), n_tokens=5, means=Standin((9, 576), B16))
    paging.page_means(**good)
    assert len(on_gpu.calls) == 1
    for changed in [dict(means=Standin((8, 576), B16)), dict(means=Standin((9, 512), B16)), dict(means=Standin((9, 576), F32)), dict(means=Standin((9, 576), B16, on=1)), dict(starts=Standin((2,), I32)), dict(cache=Standin((9, 64, 512), U8))]:
        with pytest.raises(ValueError):
            paging.page_means(**(good | changed))
    assert len(on_gpu.calls) == 1


# ------------------------------------------------------------------------------------------------ the sources

@pytest.mark.parametrize("name,kernels", [("amla_append.cu", 2), ("amla_select.cu", 2)])
def test_kernels_read_behind_the_wait_and_promise_nothing(name, kernels):
    """They are placed while the kernel in front of them is still writing: no non-coherent load of what it brings up to date, and no load at all ahead of the wait."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, name)).read())
    assert not re.search(r"__restrict__|__ldg\b|ld\.global\.nc", text)
    found = text.split("__global__")[1:]
    assert len(found) == kernels
    for k in found:
        body = k[k.index("{"):]
        front = body[:body.index("behind_the_kernel_in_front();")]
        for pointer in ("p.seqlens[", "p.block_table[", "p.scores[", "p.tokens", "p.kv", "p.q", "p.means", "tokens.", "cache,"):
            assert pointer not in front, (name, pointer)


def test_a_scoring_kernel_that_gives_up_waits_for_its_products_and_its_peers():
    text = re.sub(r"//[^\n]*", "", open(os.path.join(build.CSRC, "amla_select.cu")).read())
    kernel = text[text.index("page_scores_kernel(const ScoreParams p, int blocks, int longest_first, const SelectParams select)"):text.index("pages_select_kernel(const SelectParams p)")]
    role = kernel[kernel.index("wid == kMmaWarp) {\n    if (elect_one())"):kernel.index("    const int quarter")]
    assert re.search(r"if \(!ok\) \{\s*mma_commit\(bar\(X_GIVE_UP\)\);\s*mbar_wait\(bar\(X_GIVE_UP\), 0\);", role)
    assert "cp_async_wait_all();" in kernel[:kernel.index("wid == kMmaWarp) {\n    if (elect_one())")]
    # all blocks of a cluster meet at the end, whether the block goes on to select or not
    last = kernel[kernel.rindex("tmem_dealloc("):]
    assert re.search(r"if \(select\.table == nullptr\) \{\s*cluster_arrive_relaxed\(\);\s*cluster_wait\(\);\s*return;\s*\}", last) and re.search(r"cluster_arrive\(\);\s*cluster_wait\(\);", last)
    # between the barrier behind which tensor memory is allocated and the end nobody returns
    assert "return;" not in kernel[kernel.index("tmem_alloc("):kernel.rindex("tmem_dealloc(")].replace("return s;", "")


# ------------------------------------------------------------------------------------------------ the plain forms

def test_the_plain_forms_by_hand():
    assert S.places(np.array([1, 3, 3, 7]), np.array([5, 9, 2]), np.array([[0, 1], [2, 3], [7, -1]]), 5) == [(1, 0, 3, 0), (2, 0, 4, 0), (5, 2, 0, None), (6, 2, 1, None)]
    x = np.arange(64.0)
    turn = np.concatenate([np.zeros(32), np.ones(32)])                              # by a quarter
    y, _ = S.rotate(x, turn, False)
    assert y[0] == -32 and y[32] == 0 and y[5] == -37 and y[37] == 5
    y, _ = S.rotate(x, turn, True)
    assert y[0] == -1 and y[1] == 0 and y[10] == -11 and y[11] == 10
    k, _ = S.key(np.ones(576) * 3.0, np.concatenate([np.ones(32), np.zeros(32)]), np.full(512, 2.0), 0.0, False)
    assert np.allclose(k[:512], 2.0) and (k[512:] == 3.0).all()
    assert S.rounded(1.0 + 2.0 ** -8, S.BF16) == 1.0 and S.rounded(-1.0 - 3 * 2.0 ** -8, S.BF16) == -1.0 - 2.0 ** -6 and S.rounded(1e9, F.E4M3) == 448.0
    assert S.select(np.array([[[5.0, 1.0, 9.0, 9.0, np.nan, 2.0, 7.0]]]), [64 * 6 + 3], 4, 1, 1, 1, 7) == [([0, 2, 3, 6], 64 * 3 + 3)]
    assert S.select(np.zeros((1, 2, 3)), [1], 2, 0, 1, 2, 3) == [([], 0), ([0], 1)]
    s, _ = S.scores(np.zeros((1, 1, 3, 576)), np.zeros((4, 576)), np.array([[3, 1, 0]]), [129], 1.0)
    assert s.tolist() == [[[1.5, 1.5, 0.0]]]


# ------------------------------------------------------------------------------------------------ the example

@pytest.mark.parametrize("bad", [dict(sequences=0), dict(heads=0), dict(prompt=0), dict(steps=0), dict(cache="fp8"), dict(keep=5), dict(recent=0), dict(sink=-1), dict(prompt=300), dict(needles=-1)])
def test_the_example_refuses(bad):
    with pytest.raises(ValueError):
        long_context.serve(**bad)


def result():
    """Two sequences of two pages and a key, one head: the second page of the first and the first of the second are left out and have a hundredth of the attention."""
    gen = torch.Generator().manual_seed(1)
    cache = torch.randn((7, 64, 576), generator=gen).bfloat16()
    out, lse = torch.randn((2, 1, 1, 512), generator=gen).bfloat16(), torch.zeros((2, 1, 1))
    i = lambda x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    return dict(cache=cache, kv_scale=1.0, format="bf16", means=cache.float().mean(1).bfloat16(), table=i([[0, 1, 2], [3, 4, 5]]), lens=i([129, 129]), out=out, lse=lse - 0.01005, whole=(out.clone(), lse),
                chosen=i([[0, 2], [1, 2]]), planted=torch.tensor([[0], [1]]), failed=0, prompt=100, steps=29)


def test_a_sound_run_has_no_faults():
    assert long_context.faults(result()) == []


@pytest.mark.parametrize("change", [lambda r: r.update(failed=1), lambda r: r["lens"].__setitem__(0, 128), lambda r: r["chosen"].__setitem__((1, 0), 0), lambda r: r["lse"].__setitem__((0, 0, 0), -1.0),
                                    lambda r: r["lse"].__setitem__((0, 0, 0), 0.1), lambda r: r["out"].__setitem__((0, 0, 0, 3), 9.0), lambda r: r["means"].__setitem__((4, 7), 1.0)])
def test_faults_are_found(change):
    r = result()
    change(r)
    assert len(long_context.faults(r)) == 1
