"""The 4-bit cache on a GPU: decode against the FP64 oracle, tokens in and out against their definition in 64 bits."""
import numpy as np
import pytest
import torch

import _fp4_util as F
from _gpu_util import compare
from oracle import reference as R
from paper_2509_25224_b200 import binding, paging

pytestmark = pytest.mark.gpu

SCALE = 1.0 / np.sqrt(192.0)


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def bf16(bits):
    return dev(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16)


def workload(lens, Sq, H, seed=5, kv_scale=0.25, spare=3, rising=False):
    """q bits, 4-bit cache, table, lengths: N(0, 1) latents in randomly placed pages; what no sequence holds is all ones (scales NaN)."""
    rng = np.random.default_rng(seed)
    pages = [F.pages_of(n) for n in lens]
    blocks, width = sum(pages) + spare, max(max(pages), 1) + 1
    cache = np.full((blocks, F.PAGE_BYTES), 0xFF, np.uint8)
    codes, scales = F.unpack(cache)
    place = rng.permutation(blocks)[:sum(pages)]
    table = np.full((len(lens), width), -1, np.int32)
    q = rng.standard_normal((len(lens), Sq, H, F.D))
    at = 0
    for b, n in enumerate(lens):
        x = rng.standard_normal((n, F.D))
        if rising and n:
            q[b, ..., 512] = 4.0
            x[:, 512] = (-30.0 + 60.0 * (32 * np.arange(n) // n) / 31.0) / (4.0 * SCALE)
        c, s = F.quantise(x, kv_scale)
        for i in range(pages[b]):
            k = min(64, n - 64 * i)
            table[b, i] = place[at]
            codes[place[at], :k] = c[64 * i: 64 * i + k]
            scales[place[at], :k] = s[64 * i: 64 * i + k]
            at += 1
    f = q.astype(np.float32)
    q_bits = ((f.view(np.uint32) + 0x7FFF + ((f.view(np.uint32) >> 16) & 1)) >> 16).astype(np.uint16)
    return q_bits, F.pack(codes, scales), table, np.array(lens, np.int32)


def expected(q, cache, table, lens, kv_scale, scale=SCALE):
    """The FP64 oracle on what the cache stands for (numbers that bf16 holds); rows beyond the lengths zeroed."""
    codes, scales = F.unpack(cache)
    v = F.values(codes, scales)
    v[np.isnan(v)] = 0.0
    o, l = R.decode(q, F.bf16_bits(v), np.maximum(table, 0), lens, scale * kv_scale)
    return o * kv_scale, l


def run(q, cache, table, lens, kv_scale, scale=SCALE):
    B, Sq, H, _ = q.shape
    out = torch.full((B, Sq, H, 512), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((B, Sq, H), float("nan"), device="cuda")
    ws = torch.full((binding.fp4_workspace_size(B, Sq, H, table.shape[1], 0),), 0xFF, dtype=torch.uint8, device="cuda")
    binding.mla_decode_fp4(bf16(q), dev(cache), kv_scale, dev(table), dev(lens), scale, out, lse, ws)
    binding.check_status(ws)
    return out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)


def check(lens, Sq, H, kv_scale=0.25, **more):
    w = workload(lens, Sq, H, kv_scale=kv_scale, **more)
    out, lse = run(*w, kv_scale)
    ref_out, ref_lse = expected(*w, kv_scale)
    # outputs are averages of N(0, 1) numbers: the tolerances of the bf16 decode call
    return compare(out, lse, ref_out, ref_lse)


@pytest.mark.parametrize("H", [1, 16, 17, 32, 33, 64, 65, 128])
@pytest.mark.parametrize("lens", [[1], [2, 63, 64, 65], [127, 128, 129, 0, 191, 192, 193], [1000, 3, 0, 257, 64]])
def test_decode_lengths_and_heads(lens, H):
    check(lens, 1, H)


@pytest.mark.parametrize("Sq,H", [(2, 16), (2, 128), (3, 50), (5, 100), (8, 17), (8, 128), (4, 16), (8, 1)])
def test_decode_several_query_tokens(Sq, H):
    check([300, 1, 0, 2, 64, 7, 129], Sq, H)


@pytest.mark.parametrize("Sq,H", [(1, 16), (1, 128), (2, 128), (2, 32)])
def test_decode_rescales_along_long_sequences(Sq, H):
    check([5000, 700, 4096], Sq, H, rising=True)


@pytest.mark.parametrize("H", [16, 40, 128])
def test_decode_splits_one_sequence_over_all_sms(H):
    check([20011], 1, H)


@pytest.mark.parametrize("B,H", [(200, 16), (300, 128), (600, 64), (2100, 4), (1100, 128)])
def test_decode_many_short_sequences(B, H):
    # around the schedules that are kept on chip (512 items), worked out by every block (2048), and by a launch of their own
    lens = [int(n) for n in np.random.default_rng(B).integers(0, 150, B)]
    check(lens, 1, H)


@pytest.mark.parametrize("H", [16, 32, 64, 128])
def test_decode_units_of_many_tiles_behind_one_another(H):
    # every part gets several units, of one tile to dozens: whoever runs ahead of whom at their ends has to come out right
    lens = [int(n) for n in np.random.default_rng(H).integers(0, 1500, 260)]
    check(lens, 1, H)


@pytest.mark.parametrize("kv_scale", [1.0, 2.0 ** -20, 2.0 ** 20, 0.3])
def test_decode_with_other_factors(kv_scale):
    w = workload([500, 77], 1, 128, kv_scale=kv_scale)
    scale = SCALE
    out, lse = run(*w, kv_scale, scale)
    ref_out, ref_lse = expected(*w, kv_scale, scale)
    compare(out, lse, ref_out, ref_lse)


@pytest.mark.parametrize("gain", [0.0, 2.0 ** -130, 2.0 ** -100, 2.0 ** 20, 2.0 ** 100])
def test_decode_of_any_magnitude_of_q(gain):
    # logits of the same size whatever Q's: the softmax scale undoes the gain (as far as FP32 holds it); a row is the oracle's row
    q, cache, table, lens = workload([300, 64], 1, 20)
    qv = F.bf16_values(q) * gain
    f = qv.astype(np.float32)
    bits = (f.view(np.uint32) >> 16).astype(np.uint16)
    scale = SCALE / gain if 2.0 ** -101 < gain < 2.0 ** 60 else SCALE if gain < 1 else SCALE / gain
    out, lse = run(bits, cache, table, lens, 0.25, scale)
    ref_out, ref_lse = expected(bits, cache, table, lens, 0.25, scale)
    compare(out, lse, ref_out, ref_lse)


def test_decode_with_a_negative_scale():
    w = workload([700, 65, 1], 2, 64)
    out, lse = run(*w, 0.25, -SCALE)
    compare(out, lse, *expected(*w, 0.25, -SCALE))


@pytest.mark.parametrize("H", [16, 64, 128])
def test_what_is_not_a_number_stays_with_the_rows_that_see_it(H):
    q, cache, table, lens = workload([200, 200, 200], 2, H)
    q = q.copy()
    q[0, 0, 3, 100] = 0x7FC0                                  # NaN in one row of Q
    codes, scales = F.unpack(cache)
    scales = scales.copy()
    scales[table[1, 3], 199 - 192, 2] = 0x7F                  # NaN in the last key of sequence 1: seen by its last token alone
    cache = F.pack(codes, scales)
    out, lse = run(q, cache, table, lens, 0.25)
    ref_out, ref_lse = expected(q, cache, table, lens, 0.25)
    bad = np.zeros(lse.shape, bool)
    bad[0, 0, 3] = True
    bad[1, 1, :] = True
    assert np.isnan(lse[bad]).all() and np.isnan(out[bad]).all()
    compare(out[~bad], lse[~bad], ref_out[~bad], ref_lse[~bad])


@pytest.mark.parametrize("beyond", [0, 100000, None])
@pytest.mark.parametrize("H", [16, 128])
def test_pages_outside_the_cache_are_pages_of_zeros(H, beyond):
    q, cache, table, lens = workload([300, 64, 130], 1, H)
    zeros = np.concatenate([cache, np.zeros((1, F.PAGE_BYTES), np.uint8)])
    bad, ref = table.copy(), table.copy()
    for b, n in enumerate(lens):
        bad[b, 0:F.pages_of(n):2] = -1 if beyond is None else cache.shape[0] + beyond
        ref[b, 0:F.pages_of(n):2] = cache.shape[0]
    out, lse = run(q, cache, bad, lens, 0.25)
    compare(out, lse, *expected(q, zeros, ref, lens, 0.25))


def test_decode_reruns_are_bit_identical_on_another_stream():
    w = workload([3000, 65, 900, 0], 1, 128)
    q, cache, table, lens = bf16(w[0]), dev(w[1]), dev(w[2]), dev(w[3])
    first = binding.mla_decode_fp4(q, cache, 0.25, table, lens, SCALE)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        again = [binding.mla_decode_fp4(q, cache, 0.25, table, lens, SCALE) for _ in range(5)]
    s.synchronize()
    for o, l in again:
        assert torch.equal(o.view(torch.int16), first[0].view(torch.int16)) and torch.equal(l, first[1])


# ------------------------------------------------------------------------------------------ tokens in and out

def tokens(n, seed, spread=False):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n, F.D))
    if spread:                                                # every exponent that bf16 has, ties, zeros, groups of one value
        x = x * 2.0 ** rng.integers(-30, 12, (n, F.D // 16)).repeat(16, 1)
        x[::3, 16:32] = 0.0
        x[1::3, 32:48] = 1.5 * 2.0 ** rng.integers(-8, 4, (len(x[1::3]), 1))
        x[2::3, 48:64] = rng.integers(-24, 25, (len(x[2::3]), 16)) / 4.0     # quotients that are ties
    f = x.astype(np.float32)
    bits = ((f.view(np.uint32) + 0x7FFF + ((f.view(np.uint32) >> 16) & 1)) >> 16).astype(np.uint16)
    return bits


def sequences(before, new, seed=3, spare=2):
    rng = np.random.default_rng(seed)
    lens = [a + b for a, b in zip(before, new)]
    pages = [F.pages_of(n) for n in lens]
    blocks = sum(pages) + spare
    place = rng.permutation(blocks)
    table = np.full((len(lens), max(max(pages), 1) + 1), -1, np.int32)
    at = 0
    for b, k in enumerate(pages):
        table[b, :k] = place[at: at + k]
        at += k
    return table, np.array(lens, np.int32), np.concatenate([[0], np.cumsum(new)]).astype(np.int32), blocks


@pytest.mark.parametrize("kv_scale", [1.0, 0.25, 2.0 ** 30])
@pytest.mark.parametrize("before,new", [([0], [1]), ([0, 63, 64, 65, 5], [1, 1, 1, 1, 1]), ([0, 100, 0, 7, 64], [70, 0, 3, 129, 64]), ([1000], [500])])
@pytest.mark.parametrize("spread", [False, True])
def test_store_and_load_are_the_definition_to_the_bit(before, new, kv_scale, spread):
    # ties included: with bf16 tokens and a power of two as factor there is one right answer for every bit
    table, lens, starts, blocks = sequences(before, new)
    x = tokens(int(starts[-1]), 1, spread)
    cache = torch.full((blocks, F.PAGE_BYTES), 0xA5, dtype=torch.uint8, device="cuda")
    paging.cache_store_fp4(bf16(x), dev(starts), cache, kv_scale, dev(table), dev(lens))
    c, s = F.quantise(F.bf16_values(x), kv_scale)
    codes, scales = (y.copy() for y in F.unpack(np.full((blocks, F.PAGE_BYTES), 0xA5, np.uint8)))
    for b in range(len(lens)):
        for i in range(starts[b], starts[b + 1]):
            at = lens[b] - starts[b + 1] + i
            codes[table[b, at // 64], at % 64] = c[i]
            scales[table[b, at // 64], at % 64] = s[i]
    got = cache.cpu().numpy()
    assert np.array_equal(F.unpack(got)[1], scales)
    want = F.pack(codes, scales)
    # (the sign of a zero whose group is all zeros is the element's)
    assert np.array_equal(got, want)
    back = torch.full((int(starts[-1]) + 2, F.D), 7.0, dtype=torch.bfloat16, device="cuda")
    paging.cache_load_fp4(cache, kv_scale, dev(table), dev(lens), dev(starts), back[:-2])
    v = F.values(c, s) * kv_scale
    assert np.array_equal(back[:-2].double().cpu().numpy(), v)
    assert (back[-2:] == 7.0).all()


@pytest.mark.parametrize("offset,width", [(0, 640), (8, 600), (3, 579), (1, 577)])
def test_tokens_may_be_slices_of_wider_rows(offset, width):
    table, lens, starts, blocks = sequences([10, 60], [5, 9])
    wide = np.zeros((14, width), np.uint16)
    x = tokens(14, 2)
    wide[:, offset: offset + F.D] = x
    rows = bf16(wide)[:, offset: offset + F.D]
    one, two = (torch.zeros((blocks, F.PAGE_BYTES), dtype=torch.uint8, device="cuda") for _ in range(2))
    paging.cache_store_fp4(rows, dev(starts), one, 0.5, dev(table), dev(lens))
    paging.cache_store_fp4(bf16(x), dev(starts), two, 0.5, dev(table), dev(lens))
    assert torch.equal(one, two)
    out = torch.full((14, width), 7.0, dtype=torch.bfloat16, device="cuda")
    paging.cache_load_fp4(one, 0.5, dev(table), dev(lens), dev(starts), out[:, offset: offset + F.D])
    assert torch.equal(out[:, offset: offset + F.D], paging.cache_load_fp4(one, 0.5, dev(table), dev(lens), dev(starts), torch.empty((14, F.D), dtype=torch.bfloat16, device="cuda")))
    assert (out[:, :offset] == 7.0).all() and (out[:, offset + F.D:] == 7.0).all()


def test_tokens_without_a_place_are_left_out():
    table, lens, starts, blocks = sequences([0, 30], [64, 70])
    bad = table.copy()
    bad[0, 0], bad[1, 1] = blocks, -5
    starts = np.array([1, 64, 134 + 8], np.int32)              # token 0 belongs to nobody; sequence 1 has eight more than its length gives places to
    lens = np.array([63, 70], np.int32)
    x = tokens(150, 4)
    cache = torch.full((blocks, F.PAGE_BYTES), 0xA5, dtype=torch.uint8, device="cuda")
    paging.cache_store_fp4(bf16(x), dev(starts), cache, 1.0, dev(bad), dev(lens))
    got = cache.cpu().numpy()
    codes, scales = (y.copy() for y in F.unpack(np.full((blocks, F.PAGE_BYTES), 0xA5, np.uint8)))
    c, s = F.quantise(F.bf16_values(x), 1.0)
    codes[bad[1, 0], :] = c[142 - 70: 142 - 6]
    scales[bad[1, 0], :] = s[142 - 70: 142 - 6]
    assert np.array_equal(got, F.pack(codes, scales))
    out = torch.full((150, F.D), 7.0, dtype=torch.bfloat16, device="cuda")
    paging.cache_load_fp4(cache, 1.0, dev(bad), dev(lens), dev(starts), out)
    want = np.zeros((150, F.D))
    want[142 - 70: 142 - 6] = F.values(c, s)[142 - 70: 142 - 6]
    assert np.array_equal(out.double().cpu().numpy(), want)


def test_tokens_that_are_not_numbers():
    table, lens, starts, blocks = sequences([0], [4])
    x = tokens(4, 5)
    x[0, 20], x[1, 40], x[2, 60], x[3, 0:16] = 0x7FC0, 0x7F80, 0xFF80, 0x7F7F
    cache = torch.zeros((blocks, F.PAGE_BYTES), dtype=torch.uint8, device="cuda")
    paging.cache_store_fp4(bf16(x), dev(starts), cache, 0.5, dev(table), dev(lens))
    out = paging.cache_load_fp4(cache, 0.5, dev(table), dev(lens), dev(starts), torch.empty((4, F.D), dtype=torch.bfloat16, device="cuda")).double().cpu().numpy()
    assert np.isnan(out[0, 16:32]).all() and np.isfinite(out[0, :16]).all() and np.isfinite(out[0, 32:]).all()
    assert out[1, 40] == 1344.0 and out[2, 60] == -1344.0 and (out[3, :16] == 1344.0).all()
    assert np.isfinite(out[1:]).all()


def test_no_tokens_is_no_work():
    table, lens, starts, blocks = sequences([5], [0])
    cache = torch.full((blocks, F.PAGE_BYTES), 0xA5, dtype=torch.uint8, device="cuda")
    none = torch.empty((0, F.D), dtype=torch.bfloat16, device="cuda")
    paging.cache_store_fp4(none, dev(starts), cache, 1.0, dev(table), dev(lens))
    assert paging.cache_load_fp4(cache, 1.0, dev(table), dev(lens), dev(starts), none).shape == (0, F.D)
    assert (cache == 0xA5).all()
