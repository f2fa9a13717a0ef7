"""Scores of pages, their selection, and decode on what is selected, against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import _fp4_util as F
import _sparse_util as S
from _gpu_util import compare
from oracle import reference as R
from paper_2509_25224_b200 import binding, paging, sparse

pytestmark = pytest.mark.gpu

SCALE = 1.0 / np.sqrt(192.0)
FORMATS = ["bf16", "e4m3", "fp4"]


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def dev_bf16(bits):
    return dev(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16)


def scattered(lens, seed=0, width=None, spare=2):
    rng = np.random.default_rng(seed)
    count = [S.pages_of(max(0, n)) for n in lens]
    width = max(max(count), 1) if width is None else width
    count = [min(c, width) for c in count]
    blocks = sum(count) + spare
    table = np.full((len(lens), width), -1, np.int32)
    place, at = rng.permutation(blocks), 0
    for b, c in enumerate(count):
        table[b, :c] = place[at:at + c]
        at += c
    return table, blocks


# ------------------------------------------------------------------------------------------------ scores

def check_scores(lens, Sq, H, scale=SCALE, size=0.5, width=None, spoil=None, seed=0):
    rng = np.random.default_rng(seed)
    table, blocks = scattered(lens, seed, width)
    lens = np.array(lens, np.int32)
    if spoil is not None:
        spoil(table, blocks)
    q, means = S.bf16(rng.standard_normal((len(lens), Sq, H, 576))), S.bf16(size * rng.standard_normal((blocks, 576)))
    W = table.shape[1]
    scores = torch.full((len(lens), Sq, W), float("nan"), device="cuda")
    ws = torch.full((sparse.scores_workspace_size(len(lens), Sq, H, W),), 0xFF, dtype=torch.uint8, device="cuda")
    got = sparse.page_scores(dev_bf16(q), dev_bf16(means), dev(table), dev(lens), scale, scores, ws)
    binding.check_status(ws)
    assert got is scores
    got = got.double().cpu().numpy()
    want, bound = S.scores(S.values(q), S.values(means), table, lens, scale)
    assert (np.abs(got - want) <= bound[..., None] * want).all(), np.abs(got - want).max()
    assert ((got == 0) >= (want == 0)).all()
    # all of the heads' attention is given out
    some = want.sum(-1) > 0
    assert (np.abs(got.sum(-1) - H) <= 2 * bound * H)[some].all() and not got[~some].any()
    # errors add up at random: far below the bound (an FP32 product of the same numbers is 6e-8 off; this is held to a hundredth of what a bf16 rounding would leave)
    if want.any():
        assert np.linalg.norm(got - want) <= 1e-5 * max(1.0, size * scale / (0.5 * SCALE)) * np.linalg.norm(want)


@pytest.mark.parametrize("H", [1, 5, 16, 17, 64, 100, 127, 128])
@pytest.mark.parametrize("lens", [[65], [0, 1, 63, 64, 65, 128, 129], [64 * 63, 64 * 64, 64 * 64 + 1, 64 * 65 + 1], [8192, 8193, 8256, 8257, 700], [20000, 3, 900]])
def test_scores_lengths_and_heads(lens, H):
    check_scores(lens, 1, H)


@pytest.mark.parametrize("Sq,H", [(2, 16), (2, 128), (3, 43), (5, 77), (8, 16), (8, 17), (8, 128)])
def test_scores_several_query_tokens(Sq, H):
    check_scores([0, 1, Sq, 60 + Sq, 63 + Sq, 64 + Sq, 65, 64 * 128 + 2, 64 * 129 + 3, 5000], Sq, H)


@pytest.mark.parametrize("width", [1, 2, 31, 33, 129, 1000])
def test_scores_in_tables_of_every_width(width):
    check_scores([min(n, 64 * width) for n in (64 * width, 64 * width - 1, 100, 64 * width - 63)], 2, 20, width=width)


def test_lengths_beyond_the_table_count_as_its_width():
    check_scores([64 * 10 + 7, 2 ** 31 - 1, 64 * 10], 1, 16, width=10)


def test_scores_where_pages_are_outside_the_cache():
    def spoil(table, blocks):
        table[0, 0], table[0, 5], table[1, 3], table[1, 70] = -1, blocks, 2 ** 31 - 1, -2 ** 31
    check_scores([2000, 64 * 90, 100], 2, 30, spoil=spoil)


@pytest.mark.parametrize("size,scale", [(4.0, SCALE), (0.5, -SCALE), (0.5, 0.0), (30.0, SCALE), (2.0 ** -20, 2.0 ** 16)])
def test_scores_of_other_sizes(size, scale):
    check_scores([3000, 700], 1, 64, scale=scale, size=size)


def test_means_beyond_32_bits():
    blocks, W = 3_900_000, 20                            # 4.5 GB of means
    means = torch.empty((blocks, 576), dtype=torch.bfloat16, device="cuda")
    few = torch.randn(W, 576, device="cuda").bfloat16()
    means[-W:] = few
    means[:W].zero_()
    q, lens = torch.randn(1, 1, 64, 576, device="cuda").bfloat16(), torch.tensor([64 * W], dtype=torch.int32, device="cuda")
    table = torch.arange(W, dtype=torch.int32, device="cuda").view(1, W)
    want = sparse.page_scores(q, few, table, lens, SCALE)
    assert torch.equal(sparse.page_scores(q, means, table + (blocks - W), lens, SCALE), want) and float(want.sum()) > 63


def test_queries_beyond_32_bits():
    B = 30000                                            # 4.4 GB of queries
    q = torch.zeros(B, 1, 128, 576, dtype=torch.bfloat16, device="cuda")
    few, means = torch.randn(1, 1, 128, 576, device="cuda").bfloat16(), torch.randn(4, 576, device="cuda").bfloat16()
    q[-1] = few[0]
    table, lens = torch.arange(4, dtype=torch.int32, device="cuda").expand(B, 4).contiguous(), torch.full((B,), 250, dtype=torch.int32, device="cuda")
    got = sparse.page_scores(q, means, table, lens, SCALE)
    want = sparse.page_scores(few, means, table[:1], lens[:1], SCALE)
    assert torch.equal(got[-1], want[0]) and torch.allclose(got[:-1, :, :3], torch.full_like(got[:-1, :, :3], 128 / 3), rtol=1e-6) and not got[..., 3].any()


def test_scores_many_sequences():
    rng = np.random.default_rng(5)
    check_scores([int(n) for n in rng.integers(0, 2000, 300)], 1, 24)


def test_scores_of_a_long_context():
    check_scores([400000, 130000], 2, 16)


@pytest.mark.parametrize("B,Sq,H", [(24, 1, 16), (12, 2, 128), (40, 1, 5), (3, 8, 128)])
def test_scores_of_more_clusters_than_fit_at_once(B, Sq, H):
    # (the longest sequences come first then: several of one length, some of none, the longest last)
    rng = np.random.default_rng(B)
    lens = [int(n) for n in rng.choice([0, 1, 65, 4000, 4000, 30000, 30000, 64 * 900], B - 1)] + [64 * 2150 + 9]
    check_scores(lens, Sq, H)


def test_scores_twice_are_the_same_bits():
    q, means = torch.randn(4, 2, 128, 576, device="cuda").bfloat16(), torch.randn(4000, 576, device="cuda").bfloat16()
    table, lens = torch.randperm(4000, device="cuda").int().view(4, 1000), torch.tensor([64000, 5, 30000, 63000], dtype=torch.int32, device="cuda")
    a = sparse.page_scores(q, means, table, lens, 0.1)
    for _ in range(5):
        assert torch.equal(a, sparse.page_scores(q, means, table, lens, 0.1))


def test_scores_and_answers_at_any_address():
    """Views that begin at 4 bytes, with something in front and behind that stays as it was."""
    table, blocks = scattered([1000, 900, 64 * 31])
    lens, W, keep = dev(np.array([1000, 900, 64 * 31], np.int32)), table.shape[1], 5
    table = dev(table)
    q, means = torch.randn(3, 1, 40, 576, device="cuda").bfloat16(), torch.randn(blocks, 576, device="cuda").bfloat16()
    want = sparse.page_scores(q, means, table, lens, SCALE)
    room = torch.full((3 * W + 2,), 7.0, device="cuda")
    got = sparse.page_scores(q, means, table, lens, SCALE, room[1:-1].view(3, 1, W))
    assert torch.equal(got, want) and float(room[0]) == float(room[-1]) == 7.0
    a, b, c = sparse.pages_select(want, table, lens, keep)
    rooms = [torch.full((n + 2,), 77, dtype=torch.int32, device="cuda") for n in (3 * keep, 3, 3 * keep)]
    x, y, z = sparse.pages_select(got, table, lens, keep, table=rooms[0][1:-1].view(3, keep), lens=rooms[1][1:-1], chosen=rooms[2][1:-1].view(3, keep))
    assert torch.equal(a, x) and torch.equal(b, y) and torch.equal(c, z) and all(int(r[0]) == int(r[-1]) == 77 for r in rooms)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_row_that_is_not_a_number_spoils_its_own_token_only(bad):
    table, blocks = scattered([1000, 900])
    q = torch.randn(2, 2, 16, 576, device="cuda").bfloat16()
    means = torch.randn(blocks, 576, device="cuda").bfloat16()
    args = (means, dev(table), dev(np.array([1000, 900], np.int32)), SCALE)
    good = sparse.page_scores(q, *args)
    q[1, 0, 7, 100] = bad
    got = sparse.page_scores(q, *args)
    same = [(0, 0), (0, 1), (1, 1)]
    assert all(torch.equal(got[i], good[i]) for i in same)
    assert torch.isnan(got[1, 0, :14]).all() and not got[1, 0, 14:].any()


def test_a_mean_that_is_not_a_number_spoils_the_tokens_that_have_it_in_front():
    table, blocks = scattered([1000, 900])
    q, means = torch.randn(2, 2, 16, 576, device="cuda").bfloat16(), torch.randn(blocks, 576, device="cuda").bfloat16()
    args = (q, means, dev(table), dev(np.array([1000, 900], np.int32)), SCALE)
    good = sparse.page_scores(*args)
    means[int(table[0, 15])] = float("nan")              # the page of the first sequence's last tokens: not scored
    means[int(table[1, 3]), 5] = float("inf")
    got = sparse.page_scores(*args)
    assert torch.equal(got[0], good[0]) and torch.isnan(got[1, :, :14]).all() and not got[1, :, 14:].any()


def test_the_wait_status_is_reset():
    table, blocks = scattered([500])
    lens = dev(np.array([500], np.int32))
    q, means = torch.randn(1, 1, 16, 576, device="cuda").bfloat16(), torch.randn(blocks, 576, device="cuda").bfloat16()
    ws = torch.full((sparse.scores_workspace_size(1, 1, 16, 8),), 0xFF, dtype=torch.uint8, device="cuda")
    sparse.page_scores(q, means, dev(table), lens, SCALE, workspace=ws)
    binding.check_status(ws)
    for keep in (3, 8):                  # with and without scoring
        ws = torch.full((sparse.sparse_workspace_size(1, 1, 16, 8, keep),), 0xFF, dtype=torch.uint8, device="cuda")
        sparse.mla_decode_sparse(q, torch.zeros((blocks, 64, 576), dtype=torch.bfloat16, device="cuda"), 1.0, means, dev(table), lens, SCALE, keep, workspace=ws)
        sparse.check_status(ws)


# ------------------------------------------------------------------------------------------------ selection

def check_select(scores, lens, keep, sink, recent, table=None, seed=0):
    B, Sq, W = scores.shape
    lens = np.array(lens, np.int32)
    table = np.random.default_rng(seed).integers(0, 2 ** 31 - 1, (B, W)).astype(np.int32) if table is None else table
    out = [torch.full((B * Sq, keep), 77, dtype=torch.int32, device="cuda"), torch.full((B * Sq,), 77, dtype=torch.int32, device="cuda"), torch.full((B * Sq, keep), 77, dtype=torch.int32, device="cuda")]
    sparse.pages_select(dev(scores.astype(np.float32)), dev(table), dev(lens), keep, sink, recent, *out)
    got = [o.cpu().numpy() for o in out]
    want = S.select(scores.astype(np.float32), lens, keep, sink, recent, Sq, W)
    for r, (pages, n) in enumerate(want):
        assert got[2][r].tolist() == pages + [-1] * (keep - len(pages)), r
        assert got[0][r].tolist() == [int(table[r // Sq, p]) for p in pages] + [-1] * (keep - len(pages))
        assert got[1][r] == n


@pytest.mark.parametrize("keep,sink,recent", [(1, 0, 1), (2, 1, 1), (3, 0, 1), (5, 2, 3), (8, 1, 2), (33, 1, 2), (64, 4, 4), (1000, 1, 1)])
@pytest.mark.parametrize("Sq", [1, 2, 8])
def test_selection(keep, sink, recent, Sq):
    rng = np.random.default_rng(keep)
    W = 70
    lens = [0, 1, Sq, 64, 65, 64 * keep, 64 * keep + 1, 64 * W, 64 * W - 5, 64 * 33 + Sq - 1, 64 * 33, 64 * 2 ** 24]
    lens = [min(n, 64 * W) for n in lens[:-1]] + lens[-1:]
    check_select(rng.standard_normal((len(lens), Sq, W)) ** 2, lens, keep, sink, recent)


@pytest.mark.parametrize("kind", ["equal", "few", "zeros", "signs", "infinite", "nan", "all nan", "close", "tiny"])
@pytest.mark.parametrize("W,keep", [(100, 7), (513, 100), (1500, 33)])
def test_selection_among_scores_that_are_alike(kind, W, keep):
    rng = np.random.default_rng(W)
    s = {"equal": lambda: np.full((3, 2, W), 0.3), "few": lambda: rng.integers(0, 4, (3, 2, W)) / 4.0, "zeros": lambda: np.where(rng.random((3, 2, W)) < 0.5, 0.0, -0.0),
         "signs": lambda: rng.standard_normal((3, 2, W)), "infinite": lambda: rng.choice([np.inf, -np.inf, 0.0, 1.0], (3, 2, W)),
         "nan": lambda: np.where(rng.random((3, 2, W)) < 0.9, np.nan, rng.choice([-np.inf, -3.0, 5.0], (3, 2, W))), "all nan": lambda: np.full((3, 2, W), np.nan),
         "close": lambda: (1.0 + rng.integers(0, 300, (3, 2, W)) * 2.0 ** -23), "tiny": lambda: rng.integers(0, 50, (3, 2, W)) * 2.0 ** -149}[kind]()
    check_select(s, [64 * W, 64 * (W // 2) + 9, 64 * W - 64], keep, 1, 2)


@pytest.mark.parametrize("W,keep", [(511, 40), (512, 40), (2047, 300), (4096, 1), (16384, 512), (40000, 2000)])
def test_selection_of_long_contexts(W, keep):
    rng = np.random.default_rng(W)
    check_select(np.exp(3 * rng.standard_normal((2, 1, W))), [64 * W - 30, 64 * (W - 1)], keep, 0, 1)


def test_selection_goes_by_no_score_of_other_pages():
    s = np.random.default_rng(1).random((1, 1, 50))
    poisoned = s.copy()
    poisoned[..., :2], poisoned[..., 37:] = np.nan, np.inf
    for x in (s, poisoned):
        check_select(x, [64 * 39 + 1], 9, 2, 3)


def test_selection_of_many_rows():
    rng = np.random.default_rng(3)
    check_select(rng.random((700, 2, 40)), [int(n) for n in rng.integers(0, 64 * 40, 700)], 12, 1, 1)


# ------------------------------------------------------------------------------------------------ attention

def pages_with(fmt, x):
    """N(0, 1)-like keys [blocks, 64, 576] as pages, and the float64 numbers they stand for without their factor."""
    if fmt == "bf16":
        bits = S.bf16(x)
        return dev_bf16(bits), S.values(bits), 1.0
    if fmt == "e4m3":
        codes = F.nearest(np.minimum(abs(x) * 64, 448), F.E4M3).astype(np.uint8) + (128 * (x < 0)).astype(np.uint8)
        return dev(codes), F.e4m3(codes), 1 / 64
    codes, scales = F.quantise(x, 0.25)
    return dev(F.pack(codes, scales)), F.values(codes, scales), 0.25


def workload(fmt, lens, Sq, H, seed=0, width=None):
    rng = np.random.default_rng(seed)
    table, blocks = scattered(lens, seed, width)
    x = rng.standard_normal((blocks, 64, 576)) + 0.7 * rng.standard_normal((blocks, 1, 576))
    cache, values, kv_scale = pages_with(fmt, x)
    means = dev_bf16(S.bf16(values.mean(1) * kv_scale))
    q = S.bf16(rng.standard_normal((len(lens), Sq, H, 576)))
    return q, cache, values, kv_scale, means, table, np.array(lens, np.int32)


def check_sparse(fmt, lens, Sq, H, keep, sink=1, recent=1, seed=0, width=None):
    q, cache, values, kv_scale, means, table, lens = workload(fmt, lens, Sq, H, seed, width)
    B, W = table.shape
    q_d, table_d, lens_d = dev_bf16(q), dev(table), dev(lens)
    out = torch.full((B, Sq, H, 512), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((B, Sq, H), float("nan"), device="cuda")
    ws = torch.full((sparse.sparse_workspace_size(B, Sq, H, W, keep),), 0xFF, dtype=torch.uint8, device="cuda")
    sparse.mla_decode_sparse(q_d, cache, kv_scale, means, table_d, lens_d, SCALE, keep, sink, recent, out, lse, ws)
    sparse.check_status(ws)
    # one call is what its three parts are, to the bit
    scores = sparse.page_scores(q_d, means, table_d, lens_d, SCALE)
    sub, sub_lens, chosen = sparse.pages_select(scores, table_d, lens_d, keep, sink, recent)
    rows = q_d.view(B * Sq, 1, H, 576)
    if fmt == "bf16":
        o, l = binding.mla_decode(rows, cache, sub, sub_lens, SCALE)
    elif fmt == "e4m3":
        o, l = binding.mla_decode_fp8(rows, cache, kv_scale, sub, sub_lens, SCALE)
    else:
        o, l = binding.mla_decode_fp4(rows, cache, kv_scale, sub, sub_lens, SCALE)
    assert torch.equal(o.view_as(out), out) and torch.equal(l.view_as(lse), lse)
    # the selection is that of the scores, the attention that of the selection
    for r, (pages, n) in enumerate(S.select(scores.cpu().numpy(), lens, keep, sink, recent, Sq, W)):
        assert chosen[r].tolist() == pages + [-1] * (keep - len(pages)) and int(sub_lens[r]) == n
    bits = F.bf16_bits(values)
    ro, rl = R.decode(q.reshape(B * Sq, 1, H, 576), bits, np.maximum(sub.cpu().numpy(), 0), sub_lens.cpu().numpy(), SCALE * kv_scale)
    compare(out.double().cpu().numpy().reshape(B * Sq, 1, H, 512), lse.double().cpu().numpy().reshape(B * Sq, 1, H), ro * kv_scale, rl)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("Sq,H", [(1, 16), (1, 128), (2, 128), (3, 33), (8, 16)])
def test_sparse_decode(fmt, Sq, H):
    check_sparse(fmt, [2000, 0, 1, 64, 300, 64 * 20, 64 * 20 + 1, 700], Sq, H, 6, 1, 2)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("keep,sink,recent", [(1, 0, 1), (2, 0, 1), (12, 4, 8), (31, 0, 1), (32, 1, 1), (40, 1, 1)])
def test_sparse_decode_keeps_few_and_all(fmt, keep, sink, recent):
    check_sparse(fmt, [2000, 500], 2, 20, keep, sink, recent)


def test_sparse_decode_of_many_sequences():
    rng = np.random.default_rng(8)
    check_sparse("bf16", [int(n) for n in rng.integers(0, 900, 150)], 1, 16, 4)
    check_sparse("e4m3", [int(n) for n in rng.integers(0, 900, 150)], 1, 128, 4)


@pytest.mark.parametrize("Sq,H", [(1, 128), (2, 64), (3, 100), (8, 16)])
def test_sequences_that_keep_all_beside_some_that_do_not(Sq, H):
    # (at 5 pages and some, the first tokens keep all and the last do not)
    check_sparse("bf16", [320, 321, 319 + Sq, 2000, 0, 63, 320 + Sq // 2, 1], Sq, H, 5, 1, 1, width=700)


def test_where_no_page_is_left_out_the_means_are_not_read():
    q, cache, values, kv_scale, means, table, lens = workload("bf16", [500, 512, 3], 1, 64)
    args = (dev(table), dev(lens), SCALE)
    out, lse = sparse.mla_decode_sparse(dev_bf16(q), cache, 1.0, None, *args, table.shape[1])
    o, l = binding.mla_decode(dev_bf16(q), cache, *args)
    assert torch.equal(o, out) and torch.equal(l, lse)


def test_captured_graphs_that_share_a_workspace_and_lengths_that_grow():
    B, H, W, keep = 6, 32, 40, 5
    table = torch.randperm(B * W, device="cuda").int().view(B, W)
    cache = torch.randn(B * W, 64, 576, device="cuda").bfloat16()
    means = cache.float().mean(1).bfloat16()
    q = torch.randn(B, 1, H, 576, device="cuda").bfloat16()
    lens = torch.tensor([1000, 64 * 40 - 30, 64, 0, 100, 700], dtype=torch.int32, device="cuda")
    ws = torch.empty(sparse.sparse_workspace_size(B, 1, H, W, keep), dtype=torch.uint8, device="cuda")
    outs = [torch.empty(B, 1, H, 512, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lses = [torch.empty(B, 1, H, device="cuda") for _ in range(2)]
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            lens.add_(1)
            sparse.mla_decode_sparse(q, cache, 1.0, means, table, lens, SCALE, keep + i - 1, 1, 1, outs[i], lses[i], ws)
        graphs.append(g)
    for step in range(24):
        graphs[step % 2].replay()
        o, l = sparse.mla_decode_sparse(q, cache, 1.0, means, table, lens, SCALE, keep + step % 2 - 1)
        assert torch.equal(o, outs[step % 2]) and torch.equal(l, lses[step % 2]), step


def test_another_stream():
    q, cache, values, kv_scale, means, table, lens = workload("fp4", [3000, 1500], 2, 64)
    args = (dev_bf16(q), cache, kv_scale, means, dev(table), dev(lens), SCALE, 9, 1, 2)
    want = sparse.mla_decode_sparse(*args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = sparse.mla_decode_sparse(*args)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_two_threads_at_once():
    import threading
    work = [workload("bf16", [3000, 1500, 9000], 2, 64, seed=1), workload("fp4", [64 * 300, 77, 5000], 1, 128, seed=2)]
    args = [(dev_bf16(q), cache, kv_scale, means, dev(table), dev(lens), SCALE, 9, 1, 2) for q, cache, _, kv_scale, means, table, lens in work]
    want = [sparse.mla_decode_sparse(*a) for a in args]
    torch.cuda.synchronize()
    wrong = []

    def call(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(200):
                out, lse = sparse.mla_decode_sparse(*args[i])
                if not (torch.equal(out, want[i][0]) and torch.equal(lse, want[i][1])):
                    wrong.append(i)

    threads = [threading.Thread(target=call, args=(i,)) for i in (0, 1)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert wrong == []


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_serving_step_together(fmt):
    """A prompt in chunks, then steps of one and two tokens: what is scored and attended to is what was put in, and shared pages serve both their sequences."""
    rng = np.random.default_rng(6)
    B, W, H, keep = 3, 12, 16, 4
    blocks = B * W + 1
    table = dev(rng.permutation(blocks)[:B * W].reshape(B, W).astype(np.int32))
    kv_scale = {"bf16": 1.0, "e4m3": 1 / 64, "fp4": 0.25}[fmt]
    cache = torch.zeros((blocks, F.PAGE_BYTES) if fmt == "fp4" else (blocks, 64, 576), dtype=torch.bfloat16 if fmt == "bf16" else torch.uint8, device="cuda")
    means = torch.zeros((blocks, 576), dtype=torch.bfloat16, device="cuda")
    a = rng.uniform(-3, 3, (W * 64, 32))
    cs = dev(np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32))
    weight = torch.ones(512, device="cuda")
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    for news in ([200, 0, 64], [100, 130, 1], [1, 1, 1], [2, 2, 2], [2, 2, 2], [60, 200, 62], [1, 1, 1]):
        n = sum(news)
        starts = dev(np.concatenate([[0], np.cumsum(news)]).astype(np.int32))
        kv = torch.randn(n, 576, device="cuda").bfloat16()
        q, q_pe = torch.randn(n, H, 576, device="cuda").bfloat16(), torch.randn(n, H, 64, device="cuda").bfloat16()
        lens += dev(np.array(news, np.int32))
        paging.cache_append(kv, starts, cache, kv_scale, table, lens, cs, norm_weight=weight, q_pe=q_pe, q=q)
        paging.page_means(cache, kv_scale, table, lens, starts, n, means)
        if min(news) != max(news):
            continue
        Sq = news[0]
        out, lse = sparse.mla_decode_sparse(q.view(B, Sq, H, 576), cache, kv_scale, means, table, lens, SCALE, keep)
        raw = cache.view(torch.int16).cpu().numpy().view(np.uint16) if fmt == "bf16" else cache.cpu().numpy()
        values = S.values(raw) if fmt == "bf16" else F.e4m3(raw) if fmt == "e4m3" else F.values(*F.unpack(raw))
        n_host, t_host = lens.cpu().numpy(), table.cpu().numpy()
        for b in range(B):
            full = n_host[b] // 64
            want = values[t_host[b, :full]].mean(1) * kv_scale
            got = S.values(means[table[b, :full].long()].view(torch.int16).cpu().numpy().view(np.uint16))
            assert (abs(got - want) <= abs(want) * 2.0 ** -8 + 1e-6).all()
        scores = sparse.page_scores(q.view(B, Sq, H, 576), means, table, lens, SCALE)
        sub, sub_lens, _ = sparse.pages_select(scores, table, lens, keep)
        ro, rl = R.decode(q.view(torch.int16).cpu().numpy().view(np.uint16).reshape(B * Sq, 1, H, 576), F.bf16_bits(values), np.maximum(sub.cpu().numpy(), 0), sub_lens.cpu().numpy(), SCALE * kv_scale)
        compare(out.double().cpu().numpy().reshape(B * Sq, 1, H, 512), lse.double().cpu().numpy().reshape(B * Sq, 1, H), ro * kv_scale, rl)
