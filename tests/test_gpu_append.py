"""Tokens into a cache of any format with norm and rotation, and the means of the pages that they fill, against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import _fp4_util as F
import _sparse_util as S
from paper_2509_25224_b200 import paging

pytestmark = pytest.mark.gpu

FORMATS = ["bf16", "e4m3", "fp4"]


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def dev_bf16(bits):
    return dev(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16)


def poisoned(fmt, blocks):
    if fmt == "fp4":
        return torch.full((blocks, F.PAGE_BYTES), 0xFF, dtype=torch.uint8, device="cuda")
    if fmt == "e4m3":
        return torch.full((blocks, 64, 576), 0xFF, dtype=torch.uint8, device="cuda")
    return torch.full((blocks, 64, 576), -1, dtype=torch.int16, device="cuda").view(torch.bfloat16)


def raw(cache):
    return cache.contiguous().view(torch.uint8).cpu().numpy()


def angles(n, seed=3):
    a = np.random.default_rng(seed).uniform(-100, 100, (n, 32))
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


def batch(news, lens, spare=2, seed=1, width=None):
    """starts, lengths, table of sequences with scattered pages"""
    rng = np.random.default_rng(seed)
    count = [S.pages_of(max(0, n)) for n in lens]
    blocks, width = sum(count) + spare, max(max(count), 1) + 1 if width is None else width
    place, table, at = rng.permutation(blocks), np.full((len(lens), width), -1, np.int32), 0
    for b, c in enumerate(count):
        table[b, :min(c, width)] = place[at:at + c][:width]
        at += c
    return np.concatenate([[0], np.cumsum(news)]).astype(np.int32), np.array(lens, np.int32), table, blocks


def check(fmt, news, lens, H=0, interleaved=False, weight="bf16", eps=1e-6, kv_scale=None, shift=0, seed=1, positions=None, table_rows=None, kv=None, width=None, spoil=None, in_place=False,
          heads_first=False, q_shift=0, first=0):
    """Appends and compares all of the cache and of the queries.  shift: bf16 elements by which rows begin off 16 bytes; first: rows in front of the first sequence's."""
    rng = np.random.default_rng(seed)
    starts, lens, table, blocks = batch(news, lens, seed=seed, width=width)
    starts = starts + first
    if spoil is not None:
        spoil(table, blocks)
    n = int(starts[-1]) + 2                                                # (two that are nobody's)
    kv_scale = {"bf16": 1.0, "e4m3": 1 / 48, "fp4": 0.3}[fmt] if kv_scale is None else kv_scale
    wide = np.zeros((n, 576 + 16), np.uint16)
    wide[:, shift:shift + 576] = S.bf16(2.0 * rng.standard_normal((n, 576))) if kv is None else kv(n)
    kv_d = dev_bf16(wide)[:, shift:shift + 576]
    x = S.values(wide[:, shift:shift + 576])
    rows = max(int(max(lens.max(), 1)), 1) if table_rows is None else table_rows
    cs = angles(rows)
    w = w_d = None
    if weight == "bf16":
        bits = S.bf16(1.0 + 0.3 * rng.standard_normal(512))
        w, w_d = S.values(bits), dev_bf16(bits)
    elif weight == "f32":
        w = (1.0 + 0.3 * rng.standard_normal(512)).astype(np.float32)
        w, w_d = w.astype(np.float64), dev(w)
    cache = poisoned(fmt, blocks)
    before = raw(cache)
    q_pe = q = None
    if H:
        src = S.bf16(rng.standard_normal((n, H, 192)))
        old = S.bf16(rng.standard_normal((n, H, 576)))
        q_store = torch.zeros(n * H * 576 + 8, dtype=torch.bfloat16, device="cuda")
        q = q_store[q_shift:q_shift + n * H * 576].view((H, n, 576) if heads_first else (n, H, 576))
        q = q.transpose(0, 1) if heads_first else q
        q.copy_(dev_bf16(old))
        if in_place:
            q_pe, src = q[..., 512:], old[..., 512:]
        else:
            q_pe, src = dev_bf16(src)[..., 128:], src[..., 128:]
    pos = None if positions is None else dev(np.asarray(positions(n), np.int32))
    paging.cache_append(kv_d, dev(starts), cache, kv_scale, dev(table), dev(lens), dev(cs), pos, w_d, eps, interleaved, q_pe, q)
    got = raw(cache)
    at_of = np.full(n, -1, np.int64)
    stored = set()
    for token, b, at, page in S.places(starts, lens, table, blocks):
        at_of[token] = at
        position = at if positions is None else int(positions(n)[token])
        if page is None or not 0 <= position < rows:
            continue
        row = at % 64
        stored.add((page, row))
        y, err = S.key(x[token], cs[position].astype(np.float64), w, eps, interleaved)
        if fmt == "bf16":
            v = S.values(got[page, row].view(np.uint16))
            assert S.between(v, y, err, S.BF16).all(), (token, np.flatnonzero(~S.between(v, y, err, S.BF16))[:8])
        elif fmt == "e4m3":
            v = F.e4m3(got[page, row])
            fits = S.between(v, y / kv_scale, err / kv_scale + abs(y / kv_scale) * 2.0 ** -23, F.E4M3)
            assert fits.all(), (token, np.flatnonzero(~fits)[:8])
        else:
            codes, scales = F.unpack(got[page:page + 1])
            assert S.groups_fit(codes[0, row], scales[0, row], y, err, kv_scale).all(), token
    # nothing else has changed
    if fmt == "fp4":
        codes, scales = (z.copy() for z in F.unpack(got))
        for page, row in stored:
            codes[page, row] = scales[page, row] = 0xFF
        assert (codes == 0xFF).all() and (scales == 0xFF).all()
    else:
        for page, row in stored:
            got[page, row] = before[page, row]
        assert (got == before).all()
    if H:
        out = q.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)
        assert (out[..., :512] == old[..., :512]).all()
        for token in range(n):
            position = at_of[token] if positions is None else int(positions(n)[token])
            if not 0 <= position < rows:
                assert (out[token] == old[token]).all()
                continue
            y, size = S.rotate(S.values(src[token]), cs[position].astype(np.float64), interleaved)
            assert S.between(S.values(out[token, :, 512:]), y, size * 2.0 ** -23, S.BF16).all()
    return stored


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("weight", [None, "bf16", "f32"])
def test_formats_pairs_and_weights(fmt, interleaved, weight):
    assert len(check(fmt, [1, 1, 3, 0, 70], [1, 64, 65, 9, 100], H=5, interleaved=interleaved, weight=weight)) == 75


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("H", [0, 1, 16, 31, 32, 33, 128])
def test_heads(fmt, H):
    check(fmt, [1] * 9, [5, 64, 1, 128, 129, 77, 200, 63, 2], H=H, interleaved=H == 31)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("shift", [1, 2, 4, 8])
def test_rows_off_16_bytes(fmt, shift):
    check(fmt, [1, 5, 2], [30, 70, 2], H=7, shift=shift)


@pytest.mark.parametrize("more", [dict(in_place=True), dict(in_place=True, interleaved=True), dict(heads_first=True), dict(heads_first=True, in_place=True), dict(q_shift=1), dict(q_shift=4, in_place=True)])
@pytest.mark.parametrize("H", [3, 64])
def test_layouts_of_queries(H, more):
    check("bf16", [1, 4, 2], [30, 70, 2], H=H, **more)


@pytest.mark.parametrize("B", [1, 2, 31, 32, 33, 64, 65, 1000, 1025, 1100])
def test_many_sequences(B):
    rng = np.random.default_rng(B)
    news = rng.integers(0, 3, B)
    check("e4m3", list(news), list(news + rng.integers(0, 90, B)), H=1)


def test_tokens_without_a_place_or_a_position():
    # more new tokens than the sequence has keys; a length of zero; a table that is too narrow; pages outside the cache; rows in front of the first sequence's
    assert len(check("bf16", [5, 3, 2], [3, 0, 2], H=2)) == 5
    assert len(check("bf16", [5, 3, 2], [3, 0, 2], H=2, first=4)) == 5
    # (positions 197 .. 199 and 126 .. 129, 97 .. 99 and 126 .. 129, of which the table has room for those below 128)
    assert len(check("fp4", [3, 4], [200, 130], H=2, width=2)) == 2
    assert len(check("e4m3", [3, 4], [100, 130], H=2, width=2)) == 5

    def spoil(table, blocks):
        table[0, 0], table[1, 1], table[2, 0] = -1, blocks, -7
    assert len(check("bf16", [2, 66, 1], [2, 66, 1], H=2, spoil=spoil)) == 64
    # positions beyond the table of angles
    assert len(check("bf16", [8, 2], [8, 70], H=2, table_rows=6)) == 6
    assert len(check("fp4", [8, 2], [8, 70], H=2, table_rows=70)) == 10


def test_positions_of_their_own():
    check("bf16", [3, 70, 2], [10, 75, 2], H=4, table_rows=50, positions=lambda n: [(7 * i) % 50 for i in range(n)])
    check("e4m3", [3, 7, 2], [10, 9, 2], H=40, table_rows=50, positions=lambda n: [(-1, 49, 50, 0, -2 ** 31, 2 ** 31 - 1)[i % 6] for i in range(n)])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("size,eps", [(1.0, 0.0), (2.0 ** -60, 0.0), (2.0 ** -60, 1e-6), (2.0 ** -75, 0.0), (2.0 ** 60, 1e-6), (2.0 ** 66, 0.0), (2.0 ** -10, 1e-5)])
def test_sizes_of_latents(fmt, size, eps):
    def kv(n):
        x = np.random.default_rng(2).standard_normal((n, 576))
        x[:, :512] *= size
        return S.bf16(x)
    check(fmt, [3, 2], [5, 66], weight="f32", eps=eps, kv=kv)


@pytest.mark.parametrize("fmt", FORMATS)
def test_zeros_keep_their_sign_and_need_no_scale(fmt):
    def kv(n):
        x = np.zeros((n, 576))
        x[:, 1::2] = -0.0
        return S.bf16(x)
    check(fmt, [3], [3], kv=kv)
    starts, lens, table, blocks = batch([2], [2])
    cache = poisoned(fmt, blocks)
    cs = np.concatenate([np.ones((2, 32)), np.zeros((2, 32))], 1).astype(np.float32)
    paging.cache_append(dev_bf16(kv(2)), dev(starts), cache, 1.0, dev(table), dev(lens), dev(cs))
    got = raw(cache)[table[0, 0]]
    if fmt == "fp4":
        assert (F.unpack(got[None])[0][0, :2, :256] == 0x80).all()
    else:
        sign = got[:2].view(np.uint16) >> 15 if fmt == "bf16" else got[:2] >> 7
        assert (sign[:, :512] == [0, 1] * 256).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_what_is_not_a_number(fmt):
    """A NaN in the latent makes the token's latent NaN (its norm is), one in the position part its pair; infinities of the position part saturate (8 and 4 bits)."""
    starts, lens, table, blocks = batch([4], [4])
    x = np.ones((4, 576))
    bits = S.bf16(x)
    bits[0, 5], bits[1, 512 + 3], bits[2, 512 + 3], bits[3, 512 + 40] = 0x7FC0, 0x7FC0, 0x7F80, 0xFF80
    cs = np.concatenate([np.ones((4, 32)), np.zeros((4, 32))], 1).astype(np.float32)
    cs[:, 32:] = 0.5                                                                     # (a zero times an infinity would be NaN)
    cs[:, 32 + 3], cs[:, 32 + 8] = 0.5, 0.5
    cache = poisoned(fmt, blocks)
    cache.view(torch.uint8).zero_()
    paging.cache_append(dev_bf16(bits), dev(starts), cache, 0.5, dev(table), dev(lens), dev(cs), norm_weight=torch.ones(512, device="cuda"))
    page = int(table[0, 0])
    if fmt == "fp4":
        out = torch.empty((4, 576), dtype=torch.bfloat16, device="cuda")
        v = paging.cache_load_fp4(cache, 0.5, dev(table), dev(lens), dev(starts), out).float().cpu().numpy()
        group = lambda *columns: sorted({16 * (c // 16) + i for c in columns for i in range(16)})  # noqa: E731
    else:
        v = S.values(raw(cache)[page, :4].view(np.uint16)) if fmt == "bf16" else F.e4m3(raw(cache)[page, :4]) * 0.5
        group = lambda *columns: sorted(columns)  # noqa: E731
    nan = [list(np.flatnonzero(np.isnan(r))) for r in v]
    assert nan[0] == list(range(512)) and nan[1] == group(512 + 3, 512 + 35) and nan[2] == [] and nan[3] == []
    top = {"bf16": np.inf, "e4m3": 224.0, "fp4": 1344.0}[fmt]
    assert v[2, 512 + 3] == top and v[2, 512 + 35] == top and v[3, 512 + 8] == top and v[3, 512 + 40] == -top


@pytest.mark.parametrize("size", [2.0 ** -90, 2.0 ** 90])
@pytest.mark.parametrize("fmt", ["e4m3", "fp4"])
def test_factors_of_every_size(fmt, size):
    def kv(n):
        return S.bf16(np.random.default_rng(2).standard_normal((n, 576)) * size)
    check(fmt, [3, 2], [5, 66], weight=None, kv=kv, kv_scale=size / 3)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt", FORMATS)
def test_weights_off_16_bytes_give_the_same_bits(fmt, dtype):
    starts, lens, table, blocks = batch([5, 3], [7, 66])
    kv, cs = torch.randn(8, 576, device="cuda").bfloat16(), dev(angles(70))
    room = torch.rand(513, device="cuda").to(dtype)
    a, b = poisoned(fmt, blocks), poisoned(fmt, blocks)
    paging.cache_append(kv, dev(starts), a, 0.25, dev(table), dev(lens), cs, norm_weight=room[1:])
    paging.cache_append(kv, dev(starts), b, 0.25, dev(table), dev(lens), cs, norm_weight=room[1:].clone())
    assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)) and not torch.equal(a.view(torch.uint8), poisoned(fmt, blocks).view(torch.uint8))


def test_no_tokens_and_no_heads():
    starts, lens, table, blocks = batch([0, 0], [7, 66])
    cache, cs = poisoned("bf16", blocks), dev(angles(70))
    empty = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    paging.cache_append(empty(0, 576), dev(starts), cache, 1.0, dev(table), dev(lens), cs, q_pe=empty(0, 16, 64), q=empty(0, 16, 576))
    paging.page_means(cache, 1.0, dev(table), dev(lens), dev(starts), 0, empty(blocks, 576))
    assert bool((cache.view(torch.int16) == -1).all())
    paging.cache_append(torch.ones(2, 576, dtype=torch.bfloat16, device="cuda"), dev(np.array([0, 1, 2], np.int32)), cache, 1.0, dev(table), dev(lens), cs, q_pe=empty(2, 0, 64), q=empty(2, 0, 576))
    assert int((cache.view(torch.int16) != -1).sum()) == 2 * 576


def test_as_the_store_without_norm_and_rotation():
    starts, lens, table, blocks = batch([100, 3, 40], [130, 3, 41])
    kv = dev_bf16(S.bf16(np.random.default_rng(4).standard_normal((143, 576))))
    cs = torch.cat([torch.ones(200, 32), torch.zeros(200, 32)], 1).cuda()
    a, b = poisoned("fp4", blocks), poisoned("fp4", blocks)
    paging.cache_append(kv, dev(starts), a, 0.25, dev(table), dev(lens), cs)
    paging.cache_store_fp4(kv, dev(starts), b, 0.25, dev(table), dev(lens))
    assert torch.equal(a, b)


def test_a_captured_call_on_another_stream_reads_what_is_there_when_it_is_replayed():
    starts, lens, table, blocks = batch([1] * 40, [70] * 40)
    lens[:] = 5
    kv, cs = torch.randn(40, 576, device="cuda").bfloat16(), dev(angles(70))
    q = torch.randn(40, 64, 576, device="cuda").bfloat16()
    starts, lens, table = dev(starts), dev(lens), dev(table)
    caches = [poisoned("bf16", blocks) for _ in range(3)]
    q_out = [torch.zeros_like(q) for _ in range(2)]
    weight = torch.rand(512, device="cuda")
    call = lambda c, o: paging.cache_append(kv, starts, c, 1.0, table, lens, cs, norm_weight=weight, q_pe=q[..., 512:], q=o)  # noqa: E731
    means = torch.zeros((blocks, 576), dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        lens.add_(1)
        kv.mul_(-1)
        call(caches[0], q_out[0])
        paging.page_means(caches[0], 1.0, table, lens, starts, 40, means)
    kv0 = kv.clone()
    for _ in range(62):
        graph.replay()
    torch.cuda.synchronize()
    assert int(lens[0]) == 67 and torch.equal(kv, kv0)
    full = table[:, 0].long()
    keys = caches[0][full].double()
    # (of positions 5 on; what was there before is NaN)
    assert torch.isnan(means[full].float()).all() and torch.isnan(keys[:, :5]).all() and not torch.isnan(keys[:, 5:]).any()
    call(caches[1], q_out[1])
    # the last of the replays wrote the same token at the same place
    assert torch.equal(caches[0][table[:, 1].long(), 2], caches[1][table[:, 1].long(), 2]) and torch.equal(q_out[0], q_out[1])


@pytest.mark.parametrize("fmt", FORMATS)
def test_pages_beyond_32_bits(fmt):
    blocks = {"bf16": 62000, "e4m3": 120000, "fp4": 215000}[fmt]                      # 4.4 GB
    cache = torch.empty((blocks, F.PAGE_BYTES) if fmt == "fp4" else (blocks, 64, 576), dtype=torch.bfloat16 if fmt == "bf16" else torch.uint8, device="cuda")
    table = dev(np.array([[blocks - 1]], np.int32))
    kv, cs = torch.randn(64, 576, device="cuda").bfloat16(), dev(angles(64))
    starts, lens = dev(np.array([0, 64], np.int32)), dev(np.array([64], np.int32))
    means = torch.zeros((blocks, 576), dtype=torch.bfloat16, device="cuda")
    paging.cache_append(kv, starts, cache, 0.25, table, lens, cs)
    paging.page_means(cache, 0.25, table, lens, starts, 64, means)
    one, mean = cache[-1:].clone(), torch.zeros((1, 576), dtype=torch.bfloat16, device="cuda")
    cache[-1].view(torch.uint8).zero_()
    paging.cache_append(kv, starts, one, 0.25, torch.zeros_like(table), lens, cs)
    paging.page_means(one, 0.25, torch.zeros_like(table), lens, starts, 64, mean)
    paging.cache_append(kv, starts, cache, 0.25, table, lens, cs)
    assert torch.equal(cache[-1], one[0]) and torch.equal(means[-1], mean[0]) and bool(mean.any()) and not bool(means[:-1].any())


# ------------------------------------------------------------------------------------------------ means

def keys_of(fmt, cache, kv_scale):
    if fmt == "bf16":
        return S.values(cache.view(np.uint16))
    if fmt == "e4m3":
        return F.e4m3(cache) * kv_scale
    return F.values(*F.unpack(cache)) * kv_scale


def random_cache(fmt, blocks, seed=0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((blocks, 64, 576))
    if fmt == "bf16":
        return S.bf16(x).view(np.uint8).reshape(blocks, 64, 1152)
    if fmt == "e4m3":
        return F.nearest(np.minimum(abs(x) * 48, 448), F.E4M3).astype(np.uint8) + (128 * (x < 0)).astype(np.uint8)
    return F.pack(*F.quantise(x, 0.3))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("news,lens", [([64], [64]), ([1], [63]), ([1, 1, 1], [64, 65, 128]), ([200, 0, 64, 1, 63], [300, 64, 127, 320, 63]), ([1] * 90, [64] * 90), ([5] * 300, list(range(60, 360))),
                                       ([10000, 9000], [10050, 9000])])
def test_means(fmt, news, lens):
    starts, lens, table, blocks = batch(news, lens)
    host = random_cache(fmt, blocks)
    cache = dev(host)
    cache = cache.view(torch.bfloat16).view(blocks, 64, 576) if fmt == "bf16" else cache
    kv_scale = {"bf16": 1.0, "e4m3": 1 / 48, "fp4": 0.3}[fmt]
    means = torch.full((blocks, 576), -1, dtype=torch.int16, device="cuda").view(torch.bfloat16)
    paging.page_means(cache, kv_scale, dev(table), dev(lens), dev(starts), int(starts[-1]), means)
    got = means.view(torch.int16).cpu().numpy().view(np.uint16)
    full = [page for _, _, at, page in S.places(starts, lens, table, blocks) if at % 64 == 63]
    keys = keys_of(fmt, host[full].reshape((len(full), -1)) if fmt == "fp4" else host[full], kv_scale) if full else np.zeros((0, 64, 576))
    mean = keys.mean(1)
    # 64 numbers (exact ones) added up in FP32, a factor: 66 roundings of at most the sum of their magnitudes
    assert S.between(S.values(got[full]), mean, abs(keys).mean(1) * 66 * 2.0 ** -24, S.BF16).all()
    others = np.ones(blocks, bool)
    others[full] = False
    assert (got[others] == 0xFFFF).all() and len(full) == sum(n // 64 - (n - k) // 64 for n, k in zip(lens, news))


def test_means_of_pages_outside_the_cache_are_left_out():
    starts, lens, table, blocks = batch([64, 64, 64], [64, 64, 64])
    table[0, 0], table[1, 0] = -1, blocks
    means = torch.zeros((blocks, 576), dtype=torch.bfloat16, device="cuda")
    paging.page_means(torch.ones((blocks, 64, 576), dtype=torch.bfloat16, device="cuda"), 1.0, dev(table), dev(lens), dev(starts), 192, means)
    assert means.sum(1).nonzero().flatten().tolist() == [int(table[2, 0])] and bool((means[int(table[2, 0])] == 1).all())
    # fewer tokens than the starts count out: the others are not looked at
    means.zero_()
    paging.page_means(torch.ones((blocks, 64, 576), dtype=torch.bfloat16, device="cuda"), 1.0, dev(table), dev(lens), dev(starts), 128, means)
    assert not bool(means.any())
