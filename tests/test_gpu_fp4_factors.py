"""Tokens into a 4-bit cache, and decode from it, with factors of any size and the latents that such factors are for."""
import numpy as np
import pytest
import torch

import _fp4_util as F
from _gpu_util import TOL_LSE, TOL_REL_L2
from oracle import reference as R
from paper_2509_25224_b200 import binding, paging
from test_gpu_fp4 import SCALE, bf16, dev, sequences, tokens

pytestmark = pytest.mark.gpu


def bits_of(x):
    """FP32 numbers to bf16 bit patterns, to nearest with ties to even."""
    b = np.asarray(x, np.float32).view(np.uint32)
    return ((b + 0x7FFF + ((b >> 16) & 1)) >> 16).astype(np.uint16)


def stored(bits, kv_scale, n):
    """(codes, scales) of the first n keys of a sequence that holds these tokens."""
    table, lens, starts, blocks = sequences([0], [n])
    cache = torch.zeros((blocks, F.PAGE_BYTES), dtype=torch.uint8, device="cuda")
    paging.cache_store_fp4(bf16(bits), dev(starts), cache, kv_scale, dev(table), dev(lens))
    codes, scales = F.unpack(cache.cpu().numpy()[table[0, : F.pages_of(n)]])
    back = paging.cache_load_fp4(cache, kv_scale, dev(table), dev(lens), dev(starts), torch.empty((n, F.D), dtype=torch.bfloat16, device="cuda"))
    return codes.reshape(-1, F.CODE_ROW)[:n], scales.reshape(-1, F.SCALE_ROW)[:n], back.double().cpu().numpy()


@pytest.mark.parametrize("power", [-100, -30, 20, 30, 100])
@pytest.mark.parametrize("spread", [False, True])
def test_powers_of_two_to_the_bit(power, spread):
    # a power of two in the latents and in the factor changes no bit of codes and scales
    n, factor = 130, 2.0 ** power
    x = F.bf16_values(tokens(n, 6, spread)) * factor
    keep = np.abs(x) < 2.0 ** 127
    bits = bits_of(np.where(keep, x, 0.0))
    codes, scales, back = stored(bits, factor, n)
    c, s = F.quantise(F.bf16_values(bits), factor)
    assert np.array_equal(codes, c) and np.array_equal(scales, s)
    assert (scales > 0).mean() > 0.4 and (F.values(codes, scales) != 0).mean() > 0.3      # (it is a test of something)
    assert np.array_equal(back, F.values(c, s) * factor)


# FP32: 6 kv_scale, top / that and e4m3 kv_scale are rounded once each (2^-24 of them), a quotient once more: so a number is rounded to the other
# neighbour only where it lies within 2^-22 of a midpoint.
NEAR = 2.0 ** -22


def near_midpoint(v, grid):
    mid = (grid[1:] + grid[:-1]) / 2
    i = np.clip(np.searchsorted(mid, v), 1, len(mid) - 1)
    return (np.abs(v - mid[i]) <= NEAR * mid[i]) | (np.abs(v - mid[i - 1]) <= NEAR * mid[i - 1])


@pytest.mark.parametrize("kv_scale", [0.3, 1.7, 1 / 3, 0.037, 5.1e7, 3.3e-9])
@pytest.mark.parametrize("spread", [False, True])
def test_other_factors_are_the_definition(kv_scale, spread):
    n, factor = 260, float(np.float32(kv_scale))
    bits = bits_of(F.bf16_values(tokens(n, 7, spread)) * factor * 4)
    x = F.bf16_values(bits)
    codes, scales, back = stored(bits, kv_scale, n)
    c, s = F.quantise(x, factor)
    g = x.reshape(n, F.SCALE_ROW, F.GROUP) / factor
    unsure = near_midpoint(np.minimum(np.abs(g).max(-1) / 6.0, 448.0), F.E4M3)
    assert unsure.mean() < 0.1                                 # (6 / 3 is a power of two: ties are common there)
    assert np.array_equal(scales[~unsure], s[~unsure])
    assert (np.abs(scales.astype(int) - s) <= 1).all()
    # elements against the scale that was taken
    step = F.E4M3[scales][..., None]
    q = np.where(step > 0, np.abs(g) / np.where(step > 0, step, 1.0), 0.0)
    want = F.nearest(np.minimum(q, 6.0), F.E2M1) + 8 * np.signbit(g)
    nibbles = np.stack([codes & 15, codes >> 4], -1).reshape(g.shape)
    tie = near_midpoint(q, F.E2M1)
    assert tie.mean() < 0.02 and np.array_equal(nibbles[~tie], want[~tie]) and (np.abs((nibbles & 7).astype(int) - (want & 7)) <= 1).all()
    assert (scales > 0).mean() > 0.4 and ((nibbles & 7) > 0).mean() > 0.3
    # what is read back: the value times the factor, rounded to FP32 and then to bf16
    assert np.array_equal(back, F.bf16_values(bits_of(F.values(codes, scales).astype(np.float32) * np.float32(kv_scale))))


@pytest.mark.parametrize("kv_scale", [2.0 ** -20, 0.3, 2.0 ** 20, 1.7e9])
@pytest.mark.parametrize("H", [16, 128])
def test_stored_latents_of_any_size_are_attended_to(kv_scale, H):
    n, factor = 700, float(np.float32(kv_scale))
    rng = np.random.default_rng(H)
    bits = bits_of(rng.standard_normal((n, F.D)) * factor * 4)
    table, lens, starts, blocks = sequences([0], [n])
    cache = torch.zeros((blocks, F.PAGE_BYTES), dtype=torch.uint8, device="cuda")
    paging.cache_store_fp4(bf16(bits), dev(starts), cache, kv_scale, dev(table), dev(lens))
    q = bits_of(rng.standard_normal((1, 1, H, F.D)))
    out, lse = binding.mla_decode_fp4(bf16(q), cache, kv_scale, dev(table), dev(lens), SCALE / (4 * factor))
    v = F.values(*F.unpack(cache.cpu().numpy()))
    want, want_lse = R.decode(q, F.bf16_bits(v), np.maximum(table, 0), lens, SCALE / 4)
    got = out.double().cpu().numpy() / factor
    assert np.linalg.norm(want) > 1.0
    assert np.linalg.norm(got - want) <= TOL_REL_L2 * np.linalg.norm(want)
    assert np.abs(lse.double().cpu().numpy() - want_lse).max() <= TOL_LSE


def test_zeros_keep_their_sign():
    # in groups of zeros, and beside numbers
    x = np.zeros((4, F.D), np.float32)
    x[:, ::2] = -0.0
    x[1, 5], x[2, :16] = 3.0, 1.0
    x[2, 1::2] = -0.0
    codes, scales, _ = stored(bits_of(x), 0.25, 4)
    c, s = F.quantise(x.astype(np.float64), 0.25)
    assert np.array_equal(scales, s) and np.array_equal(codes, c) and (c == 8).any()
