"""Calls of scores, selection and sparse decode that other tests do not make: the first one of a process in a capture, tables too wide for one launch, pages that were moved."""
import subprocess
import sys

import numpy as np
import pytest
import torch

import _sparse_util as S
from conftest import ROOT
from paper_2509_25224_b200 import binding, paging, sparse
from test_gpu_sparse import SCALE, dev, dev_bf16, workload

pytestmark = pytest.mark.gpu

FIRST = """
import torch
from paper_2509_25224_b200 import paging, sparse
B, H, W, keep = 3, 32, %d, 4
gen = torch.Generator(device="cuda").manual_seed(1)
normal = lambda *shape: torch.randn(shape, generator=gen, device="cuda")
cache, q, kv = normal(B * 40, 64, 576).bfloat16(), normal(B, 1, H, 576).bfloat16(), normal(B, 576).bfloat16()
table = torch.full((B, W), -1, dtype=torch.int32, device="cuda")
n = min(W, 40)
table[:, :n] = torch.randperm(B * 40, generator=gen, device="cuda").int().view(B, 40)[:, :n]
lens = torch.tensor([64 * n - 70, 640, 1], dtype=torch.int32, device="cuda")
starts = torch.arange(B + 1, dtype=torch.int32, device="cuda")
cs = normal(64 * n, 64)
means = cache.float().mean(1).bfloat16()
old = cache.clone()
def calls():
    paging.cache_append(kv, starts, cache, 1.0, table, lens, cs, norm_weight=cs[0, :1].expand(512).contiguous(), q_pe=q.view(B, H, 576)[..., 512:], q=out_q)
    paging.page_means(cache, 1.0, table, lens, starts, B, means)
    scores = sparse.page_scores(q, means, table, lens, 0.07)
    return (out_q, cache, means, scores, *sparse.pages_select(scores, table, lens, keep), *sparse.mla_decode_sparse(q, cache, 1.0, means, table, lens, 0.07, keep))
out_q = torch.zeros(B, H, 576, dtype=torch.bfloat16, device="cuda")
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    results = calls()
graph.replay()
torch.cuda.synchronize()
first = [r.clone() for r in results]
cache.copy_(old)
out_q.zero_()
again = calls()
print(all(torch.equal(a, b) for a, b in zip(first, again)), bool(first[-2].any()))
"""


@pytest.mark.parametrize("W", [40, 4200, 25000])
def test_the_first_calls_of_a_process_are_recorded(W):
    r = subprocess.run([sys.executable, "-c", FIRST % W], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    assert r.stdout.split() == ["True", "True"]


@pytest.mark.parametrize("width", [24576, 24577, 30000])
@pytest.mark.parametrize("Sq,H", [(1, 128), (3, 50)])
def test_sparse_decode_in_tables_of_more_pages_than_one_launch_selects_among(width, Sq, H):
    keep = 6
    q, cache, values, kv_scale, means, table, lens = workload("bf16", [3000, 0, 64 * 5, 64 * 6 + 1, 64 * 30], Sq, H, width=width)
    q, table, lens = dev_bf16(q), dev(table), dev(lens)
    B = 5
    out, lse = sparse.mla_decode_sparse(q, cache, kv_scale, means, table, lens, SCALE, keep, 1, 2)
    scores = sparse.page_scores(q, means, table, lens, SCALE)
    sub, sub_lens, chosen = sparse.pages_select(scores, table, lens, keep, 1, 2)
    o, l = binding.mla_decode(q.view(B * Sq, 1, H, 576), cache, sub, sub_lens, SCALE)
    assert torch.equal(o.view_as(out), out) and torch.equal(l.view_as(lse), lse)
    for r, (pages, n) in enumerate(S.select(scores.cpu().numpy(), lens.tolist(), keep, 1, 2, Sq, width)):
        assert chosen[r].tolist() == pages + [-1] * (keep - len(pages)) and int(sub_lens[r]) == n


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "fp4"])
def test_pages_that_were_moved_get_their_means_again(fmt):
    """Compaction moves pages and leaves their means behind: summarised with all tokens, the same pages are chosen and the attention has the same bits."""
    keep = 5
    q, cache, values, kv_scale, means, table, lens = workload(fmt, [3000, 700, 64 * 9], 1, 40)
    cache = torch.cat([cache, torch.zeros_like(cache)])                                 # (half of the pages are free)
    blocks, B = cache.shape[0], len(lens)
    place = np.random.default_rng(2).permutation(blocks).astype(np.int32)              # where the pages lie
    moved = torch.empty_like(cache)
    moved[dev(place).long()] = cache
    table_d, lens_d, q_d = dev(np.where(table >= 0, place[np.maximum(table, 0)], -1).astype(np.int32)), dev(lens), dev_bf16(q)
    refs = torch.bincount(table_d[table_d >= 0].long(), minlength=blocks).int()
    starts = dev(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32))

    def attend():
        # (a page that was not full when it was moved has no mean, and is not asked for one)
        means = torch.full((blocks, 576), float("nan"), dtype=torch.bfloat16, device="cuda")
        paging.page_means(moved, kv_scale, table_d, lens_d, starts, int(lens.sum()), means)
        scores = sparse.page_scores(q_d, means, table_d, lens_d, SCALE)
        return scores, sparse.pages_select(scores, table_d, lens_d, keep)[2], *sparse.mla_decode_sparse(q_d, moved, kv_scale, means, table_d, lens_d, SCALE, keep)

    before = [x.clone() for x in attend()]
    assert not any(torch.isnan(x.float()).any() for x in before)
    old = table_d.clone()
    live = paging.pages_compact(moved, table_d, lens_d, refs)
    assert int(live) == sum(S.pages_of(n) for n in lens) and not torch.equal(old, table_d)
    assert all(torch.equal(a, b) for a, b in zip(before, attend()))
