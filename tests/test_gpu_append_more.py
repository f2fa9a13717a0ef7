"""Tokens into a cache and means of pages at the limits of what numbers and counts can be."""
import numpy as np
import pytest
import torch

import _sparse_util as S
from paper_2509_25224_b200 import paging
from test_gpu_append import FORMATS, batch, check, dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("weight", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("size", [2.0 ** -133, 2.0 ** -131, 2.0 ** -129, 2.0 ** -128, 2.0 ** -127, 2.0 ** -126, 2.0 ** -64, 2.0 ** -62])
def test_norm_of_the_smallest_latents(size, fmt, weight):
    """Without eps the norm of any numbers but zeros is of ordinary size; that of the smallest has a factor beyond FP32's range (2^132.5)."""
    def kv(n):
        rng = np.random.default_rng(2)
        bits = S.bf16(rng.standard_normal((n, 576)))
        smallest = 2.0 ** -133                                       # bf16's: all numbers here are multiples of it
        x = np.maximum(1, np.round(rng.uniform(1, 2, (n, 512)) * size / smallest)) * smallest * rng.choice([-1.0, 1.0], (n, 512))
        x[1, 5:] = 0.0                                               # five numbers beside zeros
        bits[:, :512] = S.bf16(x)
        return bits
    check(fmt, [3, 2], [5, 66], weight=weight, eps=0.0, kv=kv)


@pytest.mark.parametrize("bound", [65, 2 ** 31 - 64, 2 ** 31 - 63, 2 ** 31 - 1])
def test_means_with_a_bound_far_above_the_tokens(bound):
    """n_tokens bounds the tokens: any number that is large enough will do."""
    starts, lens, table, blocks = batch([64, 1], [64, 128])
    cache, means = torch.ones((blocks, 64, 576), dtype=torch.bfloat16, device="cuda"), torch.zeros((blocks, 576), dtype=torch.bfloat16, device="cuda")
    paging.page_means(cache, 1.0, dev(table), dev(lens), dev(starts), bound, means)
    assert means[:, 0].nonzero().flatten().tolist() == sorted([int(table[0, 0]), int(table[1, 1])])
