"""Decode on 4-bit caches whose values, or averages of them, are small or of any size: an output is as exact against its own size as any other,
in calls that split their sequences and merge them as in those that do not."""
import numpy as np
import pytest
import torch

import _fp4_util as F
from oracle import reference as R
from paper_2509_25224_b200 import binding
from test_gpu_fp4 import SCALE, bf16, dev

pytestmark = pytest.mark.gpu

# Relative L2 error of a row: the output's rounding to bf16 (evenly spread over half a step of 2^-7 either way: 2^-8 / sqrt(3) = 2.3e-3 of a value at most, on
# average 1.5e-3), P~ and a partial in half precision (2^-12 each at most, 2.4e-4) and FP32 sums (below 1e-4) add up to less than 2.9e-3.
TOL = 3e-3


def decode(q, cache, table, lens, kv_scale, rows):
    """The rows (b, token, head) of a call, and of the FP64 oracle in units of kv_scale."""
    B, Sq, H, _ = q.shape
    ws = torch.full((binding.fp4_workspace_size(B, Sq, H, table.shape[1], 0),), 0xFF, dtype=torch.uint8, device="cuda")
    out, lse = binding.mla_decode_fp4(bf16(q), dev(cache), kv_scale, dev(table), dev(lens), SCALE / kv_scale, workspace=ws)
    binding.check_status(ws)
    at = torch.from_numpy(rows).long().cuda()
    out, lse = (x[at[:, 0], at[:, 1], at[:, 2]].double().cpu().numpy() for x in (out, lse))
    v = F.values(*F.unpack(cache))
    want, want_lse = R.decode_rows(q, F.bf16_bits(v), np.maximum(table, 0), lens, SCALE, rows)
    return out / kv_scale, lse, want, want_lse


def check(q, cache, table, lens, kv_scale):
    B, Sq, H, _ = q.shape
    rng = np.random.default_rng(B * H)
    rows = np.stack([rng.integers(0, n, 48) for n in (B, Sq, H)], 1).astype(np.int32)
    rows[:2] = [[0, 0, 0], [B - 1, Sq - 1, H - 1]]
    out, lse, want, want_lse = decode(q, cache, table, lens, kv_scale, rows)
    error = np.linalg.norm(out - want, axis=-1) / np.linalg.norm(want, axis=-1)
    assert error.max() <= TOL, error.max()
    assert np.abs(lse - want_lse).max() <= 1e-3


def few_halves(n, every, seed):
    """A cache of n keys of which one element in `every` is +-0.5 with the smallest scale (2^-10) and the others are zero."""
    rng = np.random.default_rng(seed)
    pages = F.pages_of(n)
    nibbles = np.where(rng.integers(0, every, (pages * 64, F.D)) == 0, 1 + 8 * rng.integers(0, 2, (pages * 64, F.D)), 0).astype(np.uint8)
    codes = nibbles[:, 0::2] | (nibbles[:, 1::2] << 4)
    return F.pack(codes.reshape(pages, 64, F.CODE_ROW), np.ones((pages, 64, F.SCALE_ROW), np.uint8))


def queries(B, Sq, H, seed):
    f = np.random.default_rng(seed).standard_normal((B, Sq, H, F.D)).astype(np.float32)
    return (f.view(np.uint32) >> 16).astype(np.uint16)


# every SM gets some 16 000 keys of the same pages, so that a partial is an average of thousands of values of which few are not zero
@pytest.mark.parametrize("B,H", [(99, 1), (99, 32), (99, 64), (50, 128)])
def test_averages_far_below_the_smallest_value(B, H):
    n = 24000
    cache = few_halves(n, 64, B + H)
    table = np.tile(np.random.default_rng(H).permutation(cache.shape[0]).astype(np.int32), (B, 1))
    check(queries(B, 1, H, 3), cache, table, np.full(B, n, np.int32), 1.0)


@pytest.mark.parametrize("kv_scale", [2.0 ** -100, 2.0 ** -60, 0.3, 1.7, 2.0 ** 60, 1.9 * 2.0 ** 99, 2.0 ** 100])
@pytest.mark.parametrize("lens,H", [([20011], 16), ([9000, 1], 64), ([64, 5], 16)])
def test_outputs_of_any_size_split_or_not(lens, H, kv_scale):
    rng = np.random.default_rng(H + lens[0])
    pages = [F.pages_of(n) for n in lens]
    table = np.full((len(lens), max(pages)), -1, np.int32)
    place = rng.permutation(sum(pages)).astype(np.int32)
    for b, k in enumerate(pages):
        table[b, :k] = place[sum(pages[:b]): sum(pages[:b]) + k]
    x = rng.standard_normal((sum(pages) * 64, F.D))
    c, s = F.quantise(x, 0.25)
    check(queries(len(lens), 1, H, 4), F.pack(c.reshape(-1, 64, F.CODE_ROW), s.reshape(-1, 64, F.SCALE_ROW)), table, np.array(lens, np.int32), kv_scale)
